// Tree step on fp32 CUDA cores: the hybrid layer over a tree of up to 64 drafted tokens (Section 4.1's generation with both
// hidden states kept; fp32 storage, NATSL_FORCE_SIMT, and four softmax heads per linear head).
//
// Along the path of a node the recurrence of Section 4.3 unrolls as in a chunk of the chunkwise form, with "ancestor" in the
// place of "earlier": with D_ij the decay on the path from j (exclusive) to i and D_i the one from the context,
//   u_i = beta_i (v_i - D_i k_i S0 - sum_{j above i, folded} D_ij (k_i.k_j) u_j)
//   o_la_i = scale_la (D_i q_i S0 + sum_{j above or i, folded} D_ij (q_i.k_j) u_j),
// so the state is read once and never written, and the tokens' own products form two T x T tables.  Sums over ancestors
// run over the set bits of the node's ancestor word: a sibling's infinity or NaN cannot reach a node through 0 * inf.
//
// Bound by the fp32 pipes; tree_common.cuh has the cut into CTAs and the join.
#include <algorithm>
#include "tree_common.cuh"

namespace natsl {
namespace {

using namespace tree;

constexpr int kKeys = 32;                         // keys per tile: one per lane
constexpr int kThreads = 128, kWarps = kThreads / 32;
using SimtSums = Sums<4, kMaxNodes>;
using SimtNodes = Nodes<4, kMaxNodes>;

constexpr int kHead = sizeof(SimtSums) / 4;           // floats; then acc [T][D + 4], then what one of the two parts needs:
__host__ __device__ inline int acc_floats(int T, int D) { return T * (D + 4); }
// the tree's part: o_la, o_tree, u (own columns); q, k; two tables and the probabilities of the columns' softmax heads
__host__ __device__ inline int tree_floats(int T, int D, int G, int cluster) {
    const int cols = D / cluster, heads = cols * G > D ? cols * G / D : 1;
    return 3 * T * cols + 2 * T * (D + 4) + (2 + heads) * T * T;
}
__host__ __device__ inline int cache_floats(int TT, int D, int G) {
    return TT * (D + 4) + kKeys * (D + 4) + kKeys * D + G * TT * kKeys + 3 * G * TT + G * kKeys;
}

// The CTA's share of the cache.  Lane = key for the logits (a warp owns whole rows of a tile, so maximum and sum are shuffles), thread =
// column for the products with V (RC rows of accumulators).
template <typename ST, int D, int TT>
__device__ void cache_part(const Args &a, SimtSums *sums, float *out_acc, float *sm, int b, int h, int n_nodes, const Share &c) {
    constexpr int RC = TT * D / 128, P = D + 4;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.G, ds = D / G;
    const int bh = b * a.H + h;
    float *sq = sm, *sk = sq + TT * P, *sv = sk + kKeys * P, *sp = sv + kKeys * D, *s_m = sp + G * TT * kKeys,
          *s_z = s_m + G * TT, *s_f = s_z + G * TT, *s_rk = s_f + G * TT;
    for (int i = tid; i < TT * D; i += kThreads) {
        const int t = i / D, x = i - t * D;
        sq[t * P + x] = t < n_nodes ? to_f32(reinterpret_cast<const ST *>(a.q)[(((size_t)b * a.T + t) * a.H + h) * D + x]) : 0.f;
    }
    for (int i = tid; i < G * TT; i += kThreads) { s_m[i] = -INFINITY; s_z[i] = 0.f; }
    __syncthreads();
    for (int i = tid; i < G * TT; i += kThreads) {   // logits in base-2 units: scale and the row's RMS factor on q
        const int g = i / TT, t = i - g * TT;
        float *row = sq + t * P + g * ds, f = a.scale_sm * kLog2e;
        if (a.norm_eps >= 0.f) {
            float s = 0.f;
            for (int x = 0; x < ds; ++x) s = fmaf(row[x], row[x], s);
            f *= rsqrtf(s / ds + a.norm_eps);
        }
        for (int x = 0; x < ds; ++x) row[x] *= f;
    }
    const int col = tid % D, r0 = tid / D * RC, gc = col / ds;
    float acc[RC];
#pragma unroll
    for (int r = 0; r < RC; ++r) acc[r] = 0.f;
    const ST *kc = reinterpret_cast<const ST *>(a.k_cache) + (size_t)bh * a.cap * D;
    const ST *vc = reinterpret_cast<const ST *>(a.v_cache) + (size_t)bh * a.cap * D;
    const int to = c.to;
    for (int j0 = c.from; j0 < to; j0 += kKeys) {
        __syncthreads();                          // (the tile before has been read)
        for (int i = tid; i < kKeys * D / 4; i += kThreads) {
            const int j = i / (D / 4), x = (i - j * (D / 4)) * 4;
            const bool in = j0 + j < to;          // rows past the end count as zeros: what lies there may be anything
            const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
            *reinterpret_cast<float4 *>(sk + j * P + x) = in ? load4(kc + (size_t)(j0 + j) * D + x) : zero;
            *reinterpret_cast<float4 *>(sv + j * D + x) = in ? load4(vc + (size_t)(j0 + j) * D + x) : zero;
        }
        __syncthreads();
        if (a.norm_eps >= 0.f) {
            for (int i = tid; i < G * kKeys; i += kThreads) {
                const float *row = sk + (i % kKeys) * P + i / kKeys * ds;
                float s = 0.f;
                for (int x = 0; x < ds; ++x) s = fmaf(row[x], row[x], s);
                s_rk[i] = rsqrtf(s / ds + a.norm_eps);
            }
            __syncthreads();
        }
        const bool seen = j0 + lane < to;
        for (int t = warp * 4; t < TT; t += kWarps * 4) {
            if (t >= n_nodes) break;
            for (int g = 0; g < G; ++g) {
                float s[4] = {0.f, 0.f, 0.f, 0.f};
                for (int x = g * ds; x < (g + 1) * ds; x += 4) {
                    const float4 kk = *reinterpret_cast<const float4 *>(sk + lane * P + x);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float4 qq = *reinterpret_cast<const float4 *>(sq + (t + r) * P + x);
                        s[r] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[r]))));
                    }
                }
                const float f = a.norm_eps >= 0.f ? s_rk[g * kKeys + lane] : 1.f;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int at = g * TT + t + r;
                    const float x = seen ? s[r] * f : -INFINITY, m0 = s_m[at], m1 = fmaxf(m0, warp_max(x));
                    const float mu = m1 == -INFINITY ? 0.f : m1;
                    const float p = tc::ex2_ftz(x - mu), e = tc::ex2_ftz(m0 - mu), z = warp_sum(p);
                    sp[at * kKeys + lane] = p;
                    __syncwarp();
                    if (lane == 0) { s_m[at] = m1; s_f[at] = e; s_z[at] = fmaf(s_z[at], e, z); }
                    __syncwarp();
                }
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RC; ++r)
            if (r0 + r < n_nodes) acc[r] *= s_f[gc * TT + r0 + r];
        for (int j = 0; j < kKeys; j += 4) {
            float vv[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) vv[x] = sv[(j + x) * D + col];
#pragma unroll
            for (int r = 0; r < RC; ++r) {
                if (r0 + r >= n_nodes) break;
                const float4 p = *reinterpret_cast<const float4 *>(sp + (gc * TT + r0 + r) * kKeys + j);
                acc[r] = fmaf(p.x, vv[0], fmaf(p.y, vv[1], fmaf(p.z, vv[2], fmaf(p.w, vv[3], acc[r]))));
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < G * TT; i += kThreads) {
        const int g = i / TT, t = i - g * TT;
        sums->cache_m[g][t] = s_m[i];
        sums->cache_z[g][t] = s_z[i];
    }
#pragma unroll
    for (int r = 0; r < RC; ++r)
        if (r0 + r < n_nodes) out_acc[(r0 + r) * P + col] = acc[r];
}

// The tree's own part, for the columns c0 .. c0 + D / cluster - 1.
template <typename ST, int D>
__device__ void tree_part(const Args &a, SimtSums *sums, float *sm, SimtNodes *nd, int b, int h, int n, int rank) {
    constexpr int P = D + 4;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.G, ds = D / G, T = a.T, cols = D / a.cluster, c0 = rank * cols;
    const int g0 = c0 / ds, heads = (c0 + cols - 1) / ds - g0 + 1;       // softmax heads that these columns belong to
    float *so = sm, *st = so + T * cols, *su = st + T * cols, *sq = su + T * cols, *sk = sq + T * P, *sa = sk + T * P, *sb = sa + T * T,
          *sp = sb + T * T;
    const ST *v = reinterpret_cast<const ST *>(a.v) + ((size_t)b * T * a.H + h) * D + c0;      // row t: v + t H D
    for (int i = tid; i < n * D; i += kThreads) {
        const int t = i / D, x = i - t * D;
        const size_t at = (((size_t)b * T + t) * a.H + h) * D + x;
        sq[t * P + x] = to_f32(reinterpret_cast<const ST *>(a.q)[at]);
        sk[t * P + x] = to_f32(reinterpret_cast<const ST *>(a.k)[at]);
    }
    read_nodes(a, b, h, n, tid, nd, [] { __syncthreads(); });
    __syncthreads();
    for (int t = warp; t < n; t += kWarps) {      // the rows' norms: lanes of a softmax head's columns together
        float xq = 0.f, xk = 0.f;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            const float y = sq[t * P + lane * (D / 32) + x], z = sk[t * P + lane * (D / 32) + x];
            xq = fmaf(y, y, xq);
            xk = fmaf(z, z, xk);
        }
        const int ls = 32 / G;
        for (int s = ls / 2; s > 0; s >>= 1) {
            xq += __shfl_xor_sync(0xffffffffu, xq, s);
            xk += __shfl_xor_sync(0xffffffffu, xk, s);
        }
        const bool nrm = a.norm_eps >= 0.f;
        if (lane % ls == 0) {
            nd->rq_sm[lane / ls][t] = nrm ? rsqrtf(xq / ds + a.norm_eps) : 1.f;
            nd->rk_sm[lane / ls][t] = nrm ? rsqrtf(xk / ds + a.norm_eps) : 1.f;
        }
        for (int s = ls; s < 32; s <<= 1) {
            xq += __shfl_xor_sync(0xffffffffu, xq, s);
            xk += __shfl_xor_sync(0xffffffffu, xk, s);
        }
        if (lane == 0) {
            nd->rq_la[t] = nrm ? rsqrtf(xq + a.norm_eps) : 1.f;
            nd->rk_la[t] = nrm ? rsqrtf(xk + a.norm_eps) : 1.f;
        }
    }
    __syncthreads();
    // k S0 and q S0: thread = column and a group of rows, four rows at a time
    const int col = tid % cols, side = tid / cols, sides = kThreads / cols;
    const float *S = a.state + ((size_t)b * a.H + h) * D * D + c0 + col;
    for (int t0 = side * 4; t0 < n; t0 += 4 * sides) {
        float ak[4], aq[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) ak[r] = aq[r] = 0.f;
#pragma unroll 4
        for (int x = 0; x < D; x += 4) {
            const float s0 = S[(size_t)x * D], s1 = S[(size_t)(x + 1) * D], s2 = S[(size_t)(x + 2) * D], s3 = S[(size_t)(x + 3) * D];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int t = min(t0 + r, n - 1);
                const float4 kk = *reinterpret_cast<const float4 *>(sk + t * P + x), qq = *reinterpret_cast<const float4 *>(sq + t * P + x);
                ak[r] = fmaf(kk.x, s0, fmaf(kk.y, s1, fmaf(kk.z, s2, fmaf(kk.w, s3, ak[r]))));
                aq[r] = fmaf(qq.x, s0, fmaf(qq.y, s1, fmaf(qq.z, s2, fmaf(qq.w, s3, aq[r]))));
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int t = t0 + r;
            if (t >= n) break;
            su[t * cols + col] = nd->beta[t] * (to_f32(v[(size_t)t * a.H * D + col]) - nd->whole[t] * nd->rk_la[t] * ak[r]);
            so[t * cols + col] = a.scale_la * nd->whole[t] * nd->rq_la[t] * aq[r];
        }
    }
    // the tables, where j is above i or i itself
    for (int i = tid; i < n * n; i += kThreads) {
        const int t = i / n, j = i - t * n;
        if (j > t || !((nd->above[t] | 1ull << t) >> j & 1)) continue;
        float kk = 0.f, qk = 0.f;
        for (int g = 0; g < G; ++g) {
            float qg = 0.f;
            for (int x = g * ds; x < (g + 1) * ds; x += 4) {
                const float4 y = *reinterpret_cast<const float4 *>(sk + j * P + x), q4 = *reinterpret_cast<const float4 *>(sq + t * P + x),
                             k4 = *reinterpret_cast<const float4 *>(sk + t * P + x);
                qg = fmaf(q4.x, y.x, fmaf(q4.y, y.y, fmaf(q4.z, y.z, fmaf(q4.w, y.w, qg))));
                kk = fmaf(k4.x, y.x, fmaf(k4.y, y.y, fmaf(k4.z, y.z, fmaf(k4.w, y.w, kk))));
            }
            if (g >= g0 && g < g0 + heads) sp[((g - g0) * T + t) * T + j] = a.scale_sm * kLog2e * nd->rq_sm[g][t] * nd->rk_sm[g][j] * qg;
            qk += qg;
        }
        const float dec = decay_of(nd, t, j);
        sa[t * T + j] = nd->beta[t] * dec * nd->rk_la[t] * nd->rk_la[j] * kk;
        sb[t * T + j] = a.scale_la * dec * nd->rq_la[t] * nd->rk_la[j] * qk;
    }
    __syncthreads();
    for (int i = tid; i < heads * n; i += kThreads) {  // the softmax over the kept nodes of the path
        const int g = i / n, t = i - g * n;
        float m = -INFINITY, z = 0.f;
        const unsigned long long seen = (nd->above[t] | 1ull << t) & nd->keep;
        float *row = sp + (g * T + t) * T;
        for (unsigned long long w = seen; w; w &= w - 1) m = fmaxf(m, row[__ffsll(w) - 1]);
        const float mu = m == -INFINITY ? 0.f : m;      // (every logit -inf or NaN)
        for (unsigned long long w = seen; w; w &= w - 1) {
            const int j = __ffsll(w) - 1;
            z += row[j] = tc::ex2_ftz(row[j] - mu);
        }
        sums->tree_m[g0 + g][t] = m;
        sums->tree_z[g0 + g][t] = z;
    }
    __syncthreads();
    // up the tree node by node; a column's thread needs no other column
    if (tid < cols) {
        const int gc = (c0 + col) / ds - g0;
        for (int t = 0; t < n; ++t) {
            float u = su[t * cols + col], o = so[t * cols + col], s = 0.f;
            for (unsigned long long w = nd->above[t]; w; w &= w - 1) {
                const int j = __ffsll(w) - 1;
                if (nd->fold >> j & 1) {
                    const float x = su[j * cols + col];
                    u = fmaf(-sa[t * T + j], x, u);
                    o = fmaf(sb[t * T + j], x, o);
                }
                if (nd->keep >> j & 1) s = fmaf(sp[(gc * T + t) * T + j], to_f32(v[(size_t)j * a.H * D + col]), s);
            }
            if (nd->fold >> t & 1) o = fmaf(sb[t * T + t], u, o);
            else u = 0.f;
            if (nd->keep >> t & 1) s = fmaf(sp[(gc * T + t) * T + t], to_f32(v[(size_t)t * a.H * D + col]), s);
            su[t * cols + col] = u;
            so[t * cols + col] = o;
            st[t * cols + col] = s;
            if (a.u) a.u[(((size_t)b * T + t) * a.H + h) * D + c0 + col] = u;
        }
    }
}

template <typename ST, int D, int TT>
__global__ void __launch_bounds__(kThreads) tree_simt_kernel(Args a) {
    extern __shared__ __align__(16) float dyn[];
    __shared__ SimtNodes nodes;
    const int bh = blockIdx.x / a.cluster, rank = blockIdx.x - bh * a.cluster, b = bh / a.H, h = bh - b * a.H, n = nodes_of(a, b);
    SimtSums *sums = reinterpret_cast<SimtSums *>(dyn);
    float *acc = dyn + kHead, *work = acc + acc_floats(a.T, D);
    cache_part<ST, D, TT>(a, sums, acc, work, b, h, n, share_of(a.cache_len[bh], a.cap, a.cluster, rank));
    __syncthreads();
    tree_part<ST, D>(a, sums, work, &nodes, b, h, n, rank);
    join_rows<ST, D>(a, b, h, n, rank, sums, acc, D + 4, work, work + a.T * (D / a.cluster));
}

template <typename ST, int D, int TT>
cudaError_t launch(const Args &a, int BH, cudaStream_t st) {
    const auto bytes = [](int T, int G, int cluster) {
        return 4 * (kHead + acc_floats(T, D) + std::max(tree_floats(T, D, G, cluster), cache_floats(TT, D, G)));
    };
    cudaError_t e = allow_smem(tree_simt_kernel<ST, D, TT>, bytes(TT, D / 32, 2));
    if (e != cudaSuccess) return e;
    return launch_clusters(tree_simt_kernel<ST, D, TT>, a, BH, kThreads, bytes(a.T, a.G, a.cluster), st);
}
template <typename ST, int D>
cudaError_t by_rows(const Args &a, int BH, cudaStream_t st) {
    if (a.T <= 4) return launch<ST, D, 4>(a, BH, st);
    if (a.T <= 16) return launch<ST, D, 16>(a, BH, st);
    return launch<ST, D, 64>(a, BH, st);
}

}  // namespace

size_t tree_workspace_bytes() { return 256; }

cudaError_t launch_tree_step(const TreeCall &c, Shape s, HeadGroups hg, bool tensor_cores, cudaStream_t st) {
    const int BH = s.B * s.H;
    // CTAs per pair: as many as one resident set (one CTA per multiprocessor beyond 32 nodes, else two) has for each
    const int resident = s.L > 32 ? 148 : 2 * 148, cluster = BH * 8 <= resident ? 8 : BH * 4 <= resident ? 4 : 2;
    const Args a{c.q, c.k, c.v, c.g, c.beta, c.route, c.parent, c.n_nodes, c.w, c.state, c.k_cache, c.v_cache, c.cache_len,
                 c.out, c.u, c.lse, (int32_t *)c.ws, s.H, s.L, c.cap, hg.G, cluster, c.scale_la, c.scale_sm, c.eps, hg.norm_eps};
    if (tensor_cores && hg.G <= 2) return launch_tree_tc(a, BH, s.d, st);
    if (s.bf16) return s.d == 128 ? by_rows<__nv_bfloat16, 128>(a, BH, st) : by_rows<__nv_bfloat16, 64>(a, BH, st);
    return s.d == 128 ? by_rows<float, 128>(a, BH, st) : by_rows<float, 64>(a, BH, st);
}

}  // namespace natsl
