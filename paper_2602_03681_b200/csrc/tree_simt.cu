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
// Bound by latencies for few nodes, by the fp32 pipes for many; tree_common.cuh has the cut into CTAs and the join.  The two
// halves of a CTA, four warps each, read the cache and compute the tree's own part side by side where shared memory holds
// both parts' data, else one after the other.
#include <algorithm>
#include "tree_common.cuh"

namespace natsl {
namespace {

using namespace tree;

constexpr int kKeys = 32;                         // keys per tile: one per lane
constexpr int kThreads = 256, kHalf = 128, kWarps = kHalf / 32;
using SimtSums = Sums<4, kMaxNodes>;
using SimtNodes = Nodes<4, kMaxNodes>;

constexpr int kHead = sizeof(SimtSums) / 4;       // floats; then acc [T][D + 4], then what the two parts need:
__host__ __device__ inline int acc_floats(int T, int D) { return T * (D + 4); }
// the tree's part: o_la, o_tree, u, v (own columns); q, k; the state's columns, then two tables and the probabilities
__host__ __device__ inline int tree_floats(int T, int D, int cluster) {
    const int cols = D / cluster, tables = 3 * T * T;
    return 4 * T * cols + 2 * T * (D + 4) + ((tables > D * cols ? tables : D * cols) + 3) / 4 * 4;
}
__host__ __device__ inline int cache_floats(int TT, int D, int G) {
    return TT * (D + 4) + kKeys * (D + 4) + kKeys * D + G * TT * kKeys + 4 * G * TT + G * kKeys;
}

// 16 bytes global -> shared past the registers
__device__ __forceinline__ void cp_async16(void *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}

// The CTA's share of the cache.  Lane = key for the logits (a warp owns whole rows of a tile, so maximum and sum are shuffles),
// thread = column for the products with V (RC rows of accumulators).
template <typename ST, int D, int TT>
__device__ void cache_part(const Args &a, SimtSums *sums, float *out_acc, float *sm, int b, int h, int n_nodes, const Share &c) {
    constexpr int RC = TT * D / 128, P = D + 4;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, G = a.G, ds = D / G;
    const int bh = b * a.H + h;
    auto sync = [] { tc::named_barrier_sync(1, kHalf); };
    float *sq = sm, *sk = sq + TT * P, *sv = sk + kKeys * P, *sp = sv + kKeys * D, *s_m = sp + G * TT * kKeys,
          *s_z = s_m + G * TT, *s_f = s_z + G * TT, *s_rq = s_f + G * TT, *s_rk = s_rq + G * TT;
    const bool norm = a.norm_eps >= 0.f;
    const float to_base2 = a.scale_sm * kLog2e, scale = norm ? 1.f : to_base2;      // (on q, or on q's factors)
#pragma unroll 4
    for (int i = tid; i < TT * D / 4; i += kHalf) {
        const int t = i / (D / 4), x = (i - t * (D / 4)) * 4;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        if (t < n_nodes) y = load4(reinterpret_cast<const ST *>(a.q) + (((size_t)b * a.T + t) * a.H + h) * D + x);
        *reinterpret_cast<float4 *>(sq + t * P + x) = make_float4(y.x * scale, y.y * scale, y.z * scale, y.w * scale);
    }
    for (int i = tid; i < G * TT; i += kHalf) { s_m[i] = -INFINITY; s_z[i] = 0.f; }
    auto factor = [&](const float *row) {         // of a row's slice: RMS
        float s = 0.f;
        for (int x = 0; x < ds; x += 4) {
            const float4 y = *reinterpret_cast<const float4 *>(row + x);
            s = fmaf(y.x, y.x, fmaf(y.y, y.y, fmaf(y.z, y.z, fmaf(y.w, y.w, s))));
        }
        return s;
    };
    if (norm) {
        sync();
        for (int i = tid; i < G * TT; i += kHalf)
            s_rq[i] = to_base2 * rsqrtf(factor(sq + i % TT * P + i / TT * ds) / ds + a.norm_eps);
    }
    const int col = tid % D, r0 = tid / D * RC, gc = col / ds;
    float acc[RC];
#pragma unroll
    for (int r = 0; r < RC; ++r) acc[r] = 0.f;
    const ST *kc = reinterpret_cast<const ST *>(a.k_cache) + (size_t)bh * a.cap * D;
    const ST *vc = reinterpret_cast<const ST *>(a.v_cache) + (size_t)bh * a.cap * D;
    const int to = c.to;
    for (int j0 = c.from; j0 < to; j0 += kKeys) {
        sync();                                   // (the tile before has been read)
#pragma unroll 4
        for (int i = tid; i < kKeys * D / 4; i += kHalf) {
            const int j = i / (D / 4), x = (i - j * (D / 4)) * 4;
            const bool in = j0 + j < to;          // rows past the end count as zeros: what lies there may be anything
            float4 yk = make_float4(0.f, 0.f, 0.f, 0.f), yv = yk;
            if (in) {
                yk = load4(kc + (size_t)(j0 + j) * D + x);
                yv = load4(vc + (size_t)(j0 + j) * D + x);
            }
            *reinterpret_cast<float4 *>(sk + j * P + x) = yk;
            *reinterpret_cast<float4 *>(sv + j * D + x) = yv;
        }
        sync();
        if (norm) {
            for (int i = tid; i < G * kKeys; i += kHalf)
                s_rk[i] = rsqrtf(factor(sk + (i % kKeys) * P + i / kKeys * ds) / ds + a.norm_eps);
            sync();
        }
        const bool seen = j0 + lane < to;
        for (int t = warp * 4; t < TT; t += kWarps * 4) {
            if (t >= n_nodes) break;
            for (int g = 0; g < G; ++g) {
                float s[4] = {0.f, 0.f, 0.f, 0.f}, top[4];
                for (int x = g * ds; x < (g + 1) * ds; x += 4) {
                    const float4 kk = *reinterpret_cast<const float4 *>(sk + lane * P + x);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float4 qq = *reinterpret_cast<const float4 *>(sq + (t + r) * P + x);
                        s[r] = fmaf(qq.x, kk.x, fmaf(qq.y, kk.y, fmaf(qq.z, kk.z, fmaf(qq.w, kk.w, s[r]))));
                    }
                }
                const float rk = norm ? s_rk[g * kKeys + lane] : 1.f;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float f = norm ? rk * s_rq[g * TT + t + r] : 1.f;
                    s[r] = seen ? s[r] * f : -INFINITY;
                    top[r] = warp_max(s[r]);
                }
                const float m0 = s_m[g * TT + t + (lane & 3)];       // (lane r looks after row r's running values)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float m1 = fmaxf(__shfl_sync(0xffffffffu, m0, r), top[r]), mu = m1 == -INFINITY ? 0.f : m1;
                    s[r] = tc::ex2_ftz(s[r] - mu);
                    sp[(g * TT + t + r) * kKeys + lane] = s[r];
                    top[r] = m1;
                    s[r] = warp_sum(s[r]);
                }
                const float m1 = lane == 0 ? top[0] : lane == 1 ? top[1] : lane == 2 ? top[2] : top[3];
                const float z1 = lane == 0 ? s[0] : lane == 1 ? s[1] : lane == 2 ? s[2] : s[3];
                if (lane < 4) {
                    const int at = g * TT + t + lane;
                    const float e = tc::ex2_ftz(m0 - (m1 == -INFINITY ? 0.f : m1));
                    s_m[at] = m1;
                    s_f[at] = e;
                    s_z[at] = fmaf(s_z[at], e, z1);
                }
                __syncwarp();
            }
        }
        sync();
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
    sync();
    for (int i = tid; i < G * TT; i += kHalf) {
        const int g = i / TT, t = i - g * TT;
        sums->cache_m[g][t] = s_m[i];
        sums->cache_z[g][t] = s_z[i];
    }
#pragma unroll
    for (int r = 0; r < RC; ++r)
        if (r0 + r < n_nodes) out_acc[(r0 + r) * P + col] = acc[r];
}

// The tree's own part, for the columns c0 .. c0 + D / cluster - 1, which belong to one softmax head.
template <typename ST, int D>
__device__ void tree_part(const Args &a, SimtSums *sums, float *sm, SimtNodes *nd, int b, int h, int n, int rank, const NodeRow &node) {
    constexpr int P = D + 4;
    const int tid = threadIdx.x - kHalf, warp = tid >> 5, lane = tid & 31, G = a.G, ds = D / G, T = a.T, cols = D / a.cluster, c0 = rank * cols;
    const int gc = c0 / ds;
    auto sync = [] { tc::named_barrier_sync(2, kHalf); };
    float *so = sm, *st = so + T * cols, *su = st + T * cols, *sv = su + T * cols, *sq = sv + T * cols, *sk = sq + T * P, *sa = sk + T * P,
          *sb = sa + T * T, *sp = sb + T * T, *ss = sa;       // (ss: the state's columns, until the tables take their place)
    const float *S = a.state + ((size_t)b * a.H + h) * D * D + c0;
    for (int i = tid; i < D * cols / 4; i += kHalf) {
        const int x = i / (cols / 4), y = (i - x * (cols / 4)) * 4;
        cp_async16(ss + x * cols + y, S + (size_t)x * D + y);
    }
#pragma unroll 4
    for (int i = tid; i < n * D / 4; i += kHalf) {
        const int t = i / (D / 4), x = (i - t * (D / 4)) * 4;
        const size_t at = (((size_t)b * T + t) * a.H + h) * D + x;
        const float4 q4 = load4(reinterpret_cast<const ST *>(a.q) + at), k4 = load4(reinterpret_cast<const ST *>(a.k) + at);
        *reinterpret_cast<float4 *>(sq + t * P + x) = q4;
        *reinterpret_cast<float4 *>(sk + t * P + x) = k4;
    }
    for (int i = tid; i < n * cols / 4; i += kHalf) {
        const int t = i / (cols / 4), x = (i - t * (cols / 4)) * 4;
        *reinterpret_cast<float4 *>(sv + t * cols + x) = load4(reinterpret_cast<const ST *>(a.v) + (((size_t)b * T + t) * a.H + h) * D + c0 + x);
    }
    walk_nodes(a, b, h, n, tid, node, nd, sync);
    const bool norm = a.norm_eps >= 0.f;
    for (int t = warp; t < n; t += kWarps) {      // the rows' norms: lanes of a softmax head's columns together
        float xq = 0.f, xk = 0.f;
        if (norm) {
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
            if (lane % ls == 0) {
                nd->rq_sm[lane / ls][t] = rsqrtf(xq / ds + a.norm_eps);
                nd->rk_sm[lane / ls][t] = rsqrtf(xk / ds + a.norm_eps);
            }
            for (int s = ls; s < 32; s <<= 1) {
                xq += __shfl_xor_sync(0xffffffffu, xq, s);
                xk += __shfl_xor_sync(0xffffffffu, xk, s);
            }
        } else if (lane < G) {
            nd->rq_sm[lane][t] = nd->rk_sm[lane][t] = 1.f;
        }
        if (lane == 0) {
            nd->rq_la[t] = norm ? rsqrtf(xq + a.norm_eps) : 1.f;
            nd->rk_la[t] = norm ? rsqrtf(xk + a.norm_eps) : 1.f;
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    sync();
    // k S0 and q S0: thread = column and a group of rows, two rows at a time
    const int col = tid % cols, side = tid / cols, sides = kHalf / cols;
    for (int t0 = side * 2; t0 < n; t0 += 2 * sides) {
        float ak[2] = {0.f, 0.f}, aq[2] = {0.f, 0.f};
#pragma unroll 4
        for (int x = 0; x < D; x += 4) {
            const float s0 = ss[x * cols + col], s1 = ss[(x + 1) * cols + col], s2 = ss[(x + 2) * cols + col], s3 = ss[(x + 3) * cols + col];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = min(t0 + r, n - 1);
                const float4 kk = *reinterpret_cast<const float4 *>(sk + t * P + x), qq = *reinterpret_cast<const float4 *>(sq + t * P + x);
                ak[r] = fmaf(kk.x, s0, fmaf(kk.y, s1, fmaf(kk.z, s2, fmaf(kk.w, s3, ak[r]))));
                aq[r] = fmaf(qq.x, s0, fmaf(qq.y, s1, fmaf(qq.z, s2, fmaf(qq.w, s3, aq[r]))));
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = t0 + r;
            if (t >= n) break;
            su[t * cols + col] = nd->beta[t] * (sv[t * cols + col] - nd->whole[t] * nd->rk_la[t] * ak[r]);
            so[t * cols + col] = a.scale_la * nd->whole[t] * nd->rq_la[t] * aq[r];
        }
    }
    sync();
    // the tables, where j is above i or i itself
    for (int i = tid; i < n * n; i += kHalf) {
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
            if (g == gc) sp[t * T + j] = a.scale_sm * kLog2e * nd->rq_sm[g][t] * nd->rk_sm[g][j] * qg;
            qk += qg;
        }
        const float decay = decay_between(nd->total[t], nd->wipes[t], nd->total[j], nd->wipes[j]);
        sa[t * T + j] = nd->beta[t] * decay * nd->rk_la[t] * nd->rk_la[j] * kk;
        sb[t * T + j] = a.scale_la * decay * nd->rq_la[t] * nd->rk_la[j] * qk;
    }
    sync();
    for (int t = tid; t < n; t += kHalf) {        // the softmax over the kept nodes of the path
        float m = -INFINITY, z = 0.f;
        const unsigned long long seen = (nd->above[t] | 1ull << t) & nd->keep;
        float *row = sp + t * T;
        for (unsigned long long w = seen; w; w &= w - 1) m = fmaxf(m, row[__ffsll(w) - 1]);
        const float mu = m == -INFINITY ? 0.f : m;      // (every logit -inf or NaN)
        for (unsigned long long w = seen; w; w &= w - 1) {
            const int j = __ffsll(w) - 1;
            z += row[j] = tc::ex2_ftz(row[j] - mu);
        }
        sums->tree_m[gc][t] = m;
        sums->tree_z[gc][t] = z;
    }
    // up the tree node by node; a column's thread needs no other column
    const unsigned long long fold = nd->fold, keep = nd->keep;
    if (tid < cols)
        for (int t = 0; t < n; ++t) {
            float u = su[t * cols + tid], o = so[t * cols + tid];
            for (unsigned long long w = nd->above[t] & fold; w; w &= w - 1) {
                const int j = __ffsll(w) - 1;
                const float x = su[j * cols + tid];
                u = fmaf(-sa[t * T + j], x, u);
                o = fmaf(sb[t * T + j], x, o);
            }
            if (fold >> t & 1) o = fmaf(sb[t * T + t], u, o);
            else u = 0.f;
            su[t * cols + tid] = u;
            so[t * cols + tid] = o;
        }
    sync();
    for (int i = tid; i < n * cols; i += kHalf) {
        const int t = i / cols, x = i - t * cols;
        float s = 0.f;
        for (unsigned long long w = (nd->above[t] | 1ull << t) & keep; w; w &= w - 1) {
            const int j = __ffsll(w) - 1;
            s = fmaf(sp[t * T + j], sv[j * cols + x], s);
        }
        st[i] = s;
        if (a.u) a.u[(((size_t)b * T + t) * a.H + h) * D + c0 + x] = su[i];
    }
}

// beside: the two parts' data lie beside one another.
template <typename ST, int D, int TT>
__global__ void __launch_bounds__(kThreads, 1) tree_simt_kernel(Args a, bool beside) {
    extern __shared__ __align__(16) float dyn[];
    __shared__ SimtNodes nodes;
    tc::grid_dependency_wait();
    tc::launch_dependents();
    const int bh = blockIdx.x / a.cluster, rank = blockIdx.x - bh * a.cluster, b = bh / a.H, h = bh - b * a.H, tid = threadIdx.x;
    const NodeRow node = load_node(a, b, h, tid >= kHalf ? tid - kHalf : a.T);
    const int n = nodes_of(a, b);
    SimtSums *sums = reinterpret_cast<SimtSums *>(dyn);
    float *acc = dyn + kHead, *work = acc + acc_floats(a.T, D), *cache_work = beside ? work + tree_floats(a.T, D, a.cluster) : work;
    if (tid < kHalf) cache_part<ST, D, TT>(a, sums, acc, cache_work, b, h, n, share_of(a.cache_len[bh], a.cap, a.cluster, rank));
    if (!beside) __syncthreads();
    if (tid >= kHalf) tree_part<ST, D>(a, sums, work, &nodes, b, h, n, rank, node);
    join_rows<ST, D>(a, b, h, n, rank, sums, acc, D + 4, work, work + a.T * (D / a.cluster));
}

template <typename ST, int D, int TT>
cudaError_t launch(const Args &a, int BH, cudaStream_t st) {
    constexpr int kMost = 226 * 1024 - (int)sizeof(SimtNodes);
    const int fixed = kHead + acc_floats(a.T, D), tree = tree_floats(a.T, D, a.cluster), cache = cache_floats(TT, D, a.G);
    const bool beside = 4 * (fixed + tree + cache) <= kMost;
    const int bytes = 4 * (fixed + (beside ? tree + cache : std::max(tree, cache)));
    cudaError_t e = allow_smem(tree_simt_kernel<ST, D, TT>, kMost);
    if (e != cudaSuccess) return e;
    return launch_clusters(tree_simt_kernel<ST, D, TT>, BH * a.cluster, a.cluster, kThreads, bytes, st, a, beside);
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
    // CTAs per pair: as many as can be resident for all pairs at once.  A cluster lies within one of the GPU's groups of 16 to 18
    // multiprocessors, so 148 of them hold 15 clusters of eight or 33 of four, twice that where a multiprocessor holds two CTAs
    // (tensor cores, up to 32 nodes).  Pairs over 1638 keys of 128 columns, eight / four: 64 nodes of 16 pairs 31 / 19 us, of 8 17 /
    // 18.5; 16 nodes of 28 pairs 11.3 / 12.3, 32 of 32 17.9 / 16.0; four / two: 64 nodes of 33 pairs 20 / 25, of 48 37 / 26; 16 nodes
    // of 60 15 / 17, of 71 17.1 / 17.3.  The CUDA-core kernel has one CTA per multiprocessor throughout: fp32 pairs over 1024 keys,
    // eight / four: 2 nodes of 20 pairs 28 / 25, 16 of 20 55 / 50, 32 of 28 101 / 93; four / two: 2 nodes of 40 47 / 44, 16 of 64 105 /
    // 102, 32 of 40 184 / 179.  With four softmax heads of 32 columns four at least: a CTA's columns belong to one of them.
    const bool on_tensor_cores = tensor_cores && hg.G <= 2;
    const int per = on_tensor_cores && s.L <= 32 ? 2 : 1, cluster = BH <= 14 * per ? 8 : BH <= 33 * per || hg.G == 4 ? 4 : 2;
    const Args a{c.q, c.k, c.v, c.g, c.beta, c.route, c.parent, c.n_nodes, c.w, c.state, c.k_cache, c.v_cache, c.cache_len,
                 c.out, c.u, c.lse, (int32_t *)c.ws, s.H, s.L, c.cap, hg.G, cluster, c.scale_la, c.scale_sm, c.eps, hg.norm_eps};
    if (on_tensor_cores) return launch_tree_tc(a, BH, s.d, st);
    if (s.bf16) return s.d == 128 ? by_rows<__nv_bfloat16, 128>(a, BH, st) : by_rows<__nv_bfloat16, 64>(a, BH, st);
    return s.d == 128 ? by_rows<float, 128>(a, BH, st) : by_rows<float, 64>(a, BH, st);
}

}  // namespace natsl
