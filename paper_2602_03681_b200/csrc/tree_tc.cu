// Tree step on the tensor cores (bf16 storage): the hybrid layer over a tree of up to 64 drafted tokens.  The mathematics is
// tree_simt.cu's; here the products are warp-level MMAs: a tree has 1 to 64 query rows, far below a tcgen05 tile of 128, and
// the call is bound by reading the retained K/V once.
//
// Cache items stream K/V tiles of 64 keys through a ring of asynchronous copies.  The four warps share the tile by keys (and,
// beyond 32 nodes, by two halves of the rows), each with its own running maximum and sum, so that a key's row leaves shared
// memory once (twice) whatever the number of nodes; the warps' results meet at the end of the item.  A running maximum moves
// only when a logit exceeds it by 2^8.  Probabilities meet V rounded to bf16 (2^-8 of themselves, V's own precision); their
// sum is taken before the rounding.
//
// The tree item multiplies q and k with the fp32 state as three bf16 terms that together hold all of its 24 bits, so that
// u, which goes into the state at the commit, is as exact as on CUDA cores.
#include <algorithm>
#include "tree_common.cuh"

namespace natsl {
namespace {

using namespace tree;
using tc::ldmatrix_x4;
using tc::ldmatrix_x4_trans;

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// 16 bytes global -> shared past the registers; `in` false: zeros.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ float2 bf2(uint32_t x) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); }

// R: 16-row tiles that hold the tree's nodes (1, 2, 4).
template <int D, int R> struct Layout {
    static constexpr int kRows = 16 * R;                     // nodes, padded
    static constexpr int kMt = R < 2 ? R : 2;                // row tiles per warp
    static constexpr int kRowGroups = R / kMt, kKeyGroups = 4 / kRowGroups, kWarpKeys = kTileKeys / kKeyGroups;
    static constexpr int kRowBytes = D * 2, kTileBytes = kTileKeys * kRowBytes;
    static constexpr int kStages = D == 128 ? 3 : 4;
    static constexpr int kRing = kStages * 2 * kTileBytes;
    static constexpr int kAccPitch = D + 4;
    static constexpr int kMerge = kKeyGroups * kRows * kAccPitch * 4;
    // tree item
    static constexpr int kPitch = kRowBytes + 16;            // (an odd number of 16-byte pieces: eight rows, eight banks)
    static constexpr int oV = 0, oQ = oV + kRows * kPitch, oK = oQ + kRows * kPitch;
    static constexpr int oA = oQ, oP = oA + kRows * kRows * 4;   // over q and k, once their products are in registers
    static constexpr int kTables = kRows * kRows * (4 + 2 * 2), kOperands = 2 * kRows * kPitch;   // (two softmax heads at most)
    static constexpr int oB = oQ + (kTables > kOperands ? kTables : kOperands), oU = oB + kRows * kRows * 4;
    static constexpr int kTree = oU + kRows * D * 4;
    static constexpr int kTotal = kRing > kMerge ? (kRing > kTree ? kRing : kTree) : (kMerge > kTree ? kMerge : kTree);
};

template <int D, int G, bool kNorm, int R>
__device__ void cache_item(const Args &a, uint8_t *sm, int b, int h, int part, int n_nodes, const Cut &c) {
    using L = Layout<D, R>;
    constexpr int ds = D / G, kMt = L::kMt, kNt = L::kWarpKeys / 8, kKs = ds / 16;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, c4 = lane & 3;
    const int rg = warp / L::kKeyGroups, kg = warp - rg * L::kKeyGroups, r0 = rg * 16 * kMt;
    const int bh = b * a.H + h;
    const uint32_t ring = tc::smem_u32(sm);

    // copies: thread = 16-byte piece of every eighth (sixteenth) row of a tile
    constexpr int kPieces = L::kRowBytes / 16, kStep = kThreads / kPieces;
    const int piece = tid % kPieces, row0 = tid / kPieces;
    const uint8_t *kc = reinterpret_cast<const uint8_t *>(a.k_cache) + (size_t)bh * a.cap * L::kRowBytes + piece * 16;
    const uint8_t *vc = reinterpret_cast<const uint8_t *>(a.v_cache) + (size_t)bh * a.cap * L::kRowBytes + piece * 16;
    const uint32_t dst0 = row0 * L::kRowBytes + ((piece ^ (row0 & 7)) << 4);
    const int t_begin = part * c.tpp, t_end = min((c.n + kTileKeys - 1) / kTileKeys, t_begin + c.tpp);
    auto fetch = [&](int t) {
        if (t < t_end) {
            const uint32_t at = ring + (t - t_begin) % L::kStages * 2 * L::kTileBytes + dst0;
#pragma unroll
            for (int i = 0; i < kTileKeys / kStep; ++i) {
                const int j = t * kTileKeys + row0 + i * kStep;
                const bool in = j < c.n;          // rows past the end count as zeros: what lies there may be anything
                const size_t off = (size_t)(in ? j : 0) * L::kRowBytes;
                cp_async16(at + i * kStep * L::kRowBytes, kc + off, in);
                cp_async16(at + L::kTileBytes + i * kStep * L::kRowBytes, vc + off, in);
            }
        }
        cp_async_commit();
    };
    for (int i = 0; i < L::kStages - 1; ++i) fetch(t_begin + i);

    // q as A fragments, and each row's factor to base-2 logits
    uint32_t qf[kMt][D / 16][4];
    float f[kMt][2][kNorm ? G : 1];
#pragma unroll
    for (int m = 0; m < kMt; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = r0 + m * 16 + r * 8 + g4;
            const uint32_t *row = reinterpret_cast<const uint32_t *>(a.q) + (((size_t)b * a.T + min(t, n_nodes - 1)) * a.H + h) * (D / 2);
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
#pragma unroll
                for (int x = 0; x < 2; ++x) qf[m][k][r + 2 * x] = t < n_nodes ? __ldg(row + k * 8 + x * 4 + c4) : 0u;
            if (kNorm) {
#pragma unroll
                for (int s = 0; s < G; ++s) {
                    float ss = 0.f;
#pragma unroll
                    for (int k = s * kKs; k < (s + 1) * kKs; ++k)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const float2 y = bf2(qf[m][k][r + 2 * x]);
                            ss = fmaf(y.x, y.x, fmaf(y.y, y.y, ss));
                        }
                    ss += __shfl_xor_sync(0xffffffffu, ss, 1);
                    ss += __shfl_xor_sync(0xffffffffu, ss, 2);
                    f[m][r][s] = a.scale_sm * kLog2e * rsqrtf(ss / ds + a.norm_eps);
                }
            } else {
                f[m][r][0] = a.scale_sm * kLog2e;
            }
        }
    float o[kMt][D / 8][4], mx[G][kMt][2], z[G][kMt][2];
#pragma unroll
    for (int m = 0; m < kMt; ++m) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) o[m][i][x] = 0.f;
#pragma unroll
        for (int s = 0; s < G; ++s)
#pragma unroll
            for (int r = 0; r < 2; ++r) { mx[s][m][r] = -INFINITY; z[s][m][r] = 0.f; }
    }
    const int key0 = kg * L::kWarpKeys;
    for (int t = t_begin; t < t_end; ++t) {
        cp_async_wait<L::kStages - 2>();
        __syncthreads();                          // tile t is there, and every warp is done with tile t - 1 ...
        fetch(t + L::kStages - 1);                // ... whose place this one takes
        const int left = c.n - t * kTileKeys - key0;      // of the warp's keys
        if (left <= 0) continue;
        const uint32_t kt = ring + (t - t_begin) % L::kStages * 2 * L::kTileBytes, vt = kt + L::kTileBytes;
#pragma unroll
        for (int s = 0; s < G; ++s) {
            float x[kMt][kNt][4], kk[kNt];
#pragma unroll
            for (int i = 0; i < kNt; ++i) {
                kk[i] = 0.f;
#pragma unroll
                for (int m = 0; m < kMt; ++m)
#pragma unroll
                    for (int y = 0; y < 4; ++y) x[m][i][y] = 0.f;
            }
#pragma unroll
            for (int i = 0; i < kNt; i += 2) {
                const int row = key0 + i * 8 + (lane & 7) + (lane >> 4) * 8;
#pragma unroll
                for (int k = s * kKs; k < (s + 1) * kKs; ++k) {
                    uint32_t bf[4];
                    ldmatrix_x4(kt + row * L::kRowBytes + (((2 * k + ((lane >> 3) & 1)) ^ (row & 7)) << 4), bf);
#pragma unroll
                    for (int m = 0; m < kMt; ++m) {
                        mma_bf16(x[m][i], qf[m][k], bf[0], bf[1]);
                        mma_bf16(x[m][i + 1], qf[m][k], bf[2], bf[3]);
                    }
                    if (kNorm) {                  // the key's sum of squares rides along
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const float2 w = bf2(bf[y]);
                            kk[i + y / 2] = fmaf(w.x, w.x, fmaf(w.y, w.y, kk[i + y / 2]));
                        }
                    }
                }
            }
            // logits; a lane's columns of tile i are keys 2 c4, 2 c4 + 1, its sum of squares belongs to key g4
#pragma unroll
            for (int i = 0; i < kNt; ++i) {
                float w0 = 1.f, w1 = 1.f;
                if (kNorm) {
                    kk[i] += __shfl_xor_sync(0xffffffffu, kk[i], 1);
                    kk[i] += __shfl_xor_sync(0xffffffffu, kk[i], 2);
                    const float w = rsqrtf(fmaf(kk[i], 1.f / ds, a.norm_eps));
                    w0 = __shfl_sync(0xffffffffu, w, c4 * 8);
                    w1 = __shfl_sync(0xffffffffu, w, c4 * 8 + 4);
                }
                const bool in0 = i * 8 + 2 * c4 < left, in1 = i * 8 + 2 * c4 + 1 < left;
#pragma unroll
                for (int m = 0; m < kMt; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float fr = f[m][r][kNorm ? s : 0];
                        x[m][i][2 * r] = in0 ? x[m][i][2 * r] * (fr * w0) : -INFINITY;
                        x[m][i][2 * r + 1] = in1 ? x[m][i][2 * r + 1] * (fr * w1) : -INFINITY;
                    }
            }
            bool raise = false;
            float top[kMt][2];
#pragma unroll
            for (int m = 0; m < kMt; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float y = x[m][0][2 * r];
#pragma unroll
                    for (int i = 0; i < kNt; ++i) y = tc::max3(y, x[m][i][2 * r], x[m][i][2 * r + 1]);
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 1));
                    top[m][r] = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 2));
                    raise |= top[m][r] > mx[s][m][r] + 8.f;
                }
            if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                for (int m = 0; m < kMt; ++m)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float m1 = fmaxf(mx[s][m][r], top[m][r]);
                        const float e = mx[s][m][r] == m1 ? 1.f : tc::ex2_ftz(mx[s][m][r] - m1);
                        mx[s][m][r] = m1;
                        z[s][m][r] *= e;
#pragma unroll
                        for (int i = s * ds / 8; i < (s + 1) * ds / 8; ++i) {
                            o[m][i][2 * r] *= e;
                            o[m][i][2 * r + 1] *= e;
                        }
                    }
            }
            uint32_t pf[kMt][kNt / 2][4];
#pragma unroll
            for (int m = 0; m < kMt; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float mu = mx[s][m][r] == -INFINITY ? 0.f : mx[s][m][r];
#pragma unroll
                    for (int i = 0; i < kNt; ++i) {
                        const float p0 = tc::ex2_ftz(x[m][i][2 * r] - mu), p1 = tc::ex2_ftz(x[m][i][2 * r + 1] - mu);
                        z[s][m][r] += p0 + p1;
                        pf[m][i / 2][(i & 1) * 2 + r] = tc::pack_bf162(p0, p1);
                    }
                }
#pragma unroll
            for (int i = 0; i < kNt / 2; ++i) {
                const int row = key0 + i * 16 + (lane & 15);
#pragma unroll
                for (int n = s * ds / 16; n < (s + 1) * ds / 16; ++n) {
                    uint32_t bf[4];
                    ldmatrix_x4_trans(vt + row * L::kRowBytes + (((2 * n + (lane >> 4)) ^ (row & 7)) << 4), bf);
#pragma unroll
                    for (int m = 0; m < kMt; ++m) {
                        mma_bf16(o[m][2 * n], pf[m][i], bf[0], bf[1]);
                        mma_bf16(o[m][2 * n + 1], pf[m][i], bf[2], bf[3]);
                    }
                }
            }
        }
    }
    // the key groups' results -> one partial result
    __shared__ float s_m[G][L::kKeyGroups][L::kRows], s_z[G][L::kKeyGroups][L::kRows];
    cp_async_wait<0>();
    __syncthreads();
    float *acc = reinterpret_cast<float *>(sm);
#pragma unroll
    for (int m = 0; m < kMt; ++m)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = r0 + m * 16 + r * 8 + g4;
            float *to = acc + (kg * L::kRows + t) * L::kAccPitch + 2 * c4;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2 *>(to + 8 * i) = make_float2(o[m][i][2 * r], o[m][i][2 * r + 1]);
#pragma unroll
            for (int s = 0; s < G; ++s) {
                float y = z[s][m][r];
                y += __shfl_xor_sync(0xffffffffu, y, 1);
                y += __shfl_xor_sync(0xffffffffu, y, 2);
                if (c4 == 0) { s_m[s][kg][t] = mx[s][m][r]; s_z[s][kg][t] = y; }
            }
        }
    __syncthreads();
    float *pp = reinterpret_cast<float *>(a.ws + off_pairs((size_t)gridDim.x / (a.parts + 1))) +
                (size_t)bh * pair_floats(a.T, D, a.parts) + (size_t)a.T * D + part * part_floats(a.T, D);
    for (int i = tid; i < n_nodes * (D / 4); i += kThreads) {
        const int t = i / (D / 4), x = (i - t * (D / 4)) * 4, s = x / ds;
        float M = -INFINITY, e[L::kKeyGroups];
#pragma unroll
        for (int k = 0; k < L::kKeyGroups; ++k) M = fmaxf(M, s_m[s][k][t]);
        const float mu = M == -INFINITY ? 0.f : M;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        float Z = 0.f;
#pragma unroll
        for (int k = 0; k < L::kKeyGroups; ++k) {
            e[k] = tc::ex2_ftz(s_m[s][k][t] - mu);
            const float4 w = *reinterpret_cast<const float4 *>(acc + (k * L::kRows + t) * L::kAccPitch + x);
            Z = fmaf(s_z[s][k][t], e[k], Z);
            y.x = fmaf(w.x, e[k], y.x); y.y = fmaf(w.y, e[k], y.y);
            y.z = fmaf(w.z, e[k], y.z); y.w = fmaf(w.w, e[k], y.w);
        }
        *reinterpret_cast<float4 *>(pp + 8 * a.T + (size_t)t * D + x) = y;
        if (x % ds == 0) { pp[s * a.T + t] = M; pp[(4 + s) * a.T + t] = Z; }
    }
}

// x as three bf16 terms, pairwise packed: what two rounded terms leave over is exact in the third.
__device__ __forceinline__ void split3(float x0, float x1, uint32_t (&t)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        t[i] = tc::pack_bf162(x0, x1);
        const float2 y = bf2(t[i]);
        x0 -= y.x;
        x1 -= y.y;
    }
}

template <int D, int G, bool kNorm, int R>
__device__ void tree_item(const Args &a, uint8_t *sm, Nodes *nd, int b, int h, int n) {
    using L = Layout<D, R>;
    constexpr int ds = D / G, kRows = L::kRows, kCols = D / 4, kNs = kCols / 8;    // kCols: the state's columns per warp
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, c4 = lane & 3, T = a.T;
    const int bh = b * a.H + h;
    float *sa = reinterpret_cast<float *>(sm + L::oA), *sb = reinterpret_cast<float *>(sm + L::oB), *su = reinterpret_cast<float *>(sm + L::oU);
    __half *sp = reinterpret_cast<__half *>(sm + L::oP);
    float *base = reinterpret_cast<float *>(a.ws + off_pairs((size_t)gridDim.x / (a.parts + 1))) +
                  (size_t)bh * pair_floats(T, D, a.parts);
    float *own = base + (size_t)T * D + a.parts * part_floats(T, D);

    constexpr int kPieces = L::kRowBytes / 16;
    for (int i = tid; i < kRows * kPieces; i += kThreads) {
        const int t = i / kPieces, c = i - t * kPieces;
        const size_t at = (((size_t)b * T + min(t, max(n - 1, 0))) * a.H + h) * kPieces + c;
        const uint4 zero = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(sm + L::oQ + t * L::kPitch + c * 16) = t < n ? reinterpret_cast<const uint4 *>(a.q)[at] : zero;
        *reinterpret_cast<uint4 *>(sm + L::oK + t * L::kPitch + c * 16) = t < n ? reinterpret_cast<const uint4 *>(a.k)[at] : zero;
        *reinterpret_cast<uint4 *>(sm + L::oV + t * L::kPitch + c * 16) = t < n ? reinterpret_cast<const uint4 *>(a.v)[at] : zero;
    }
    read_nodes(a, b, h, n, nd, sb, kRows);
    __syncthreads();
    if (tid < 2 * kRows) {                        // a row's norms, thread = row of q or k
        const int t = tid % kRows;
        const bool is_k = tid >= kRows;
        const uint8_t *row = sm + (is_k ? L::oK : L::oQ) + t * L::kPitch;
        float all = 0.f;
#pragma unroll
        for (int s = 0; s < G; ++s) {
            float ss = 0.f;
            if (kNorm)
                for (int c = s * kPieces / G; c < (s + 1) * kPieces / G; ++c) {
                    const uint4 y = *reinterpret_cast<const uint4 *>(row + c * 16);
                    const float2 y0 = bf2(y.x), y1 = bf2(y.y), y2 = bf2(y.z), y3 = bf2(y.w);
                    ss += y0.x * y0.x + y0.y * y0.y + y1.x * y1.x + y1.y * y1.y + y2.x * y2.x + y2.y * y2.y + y3.x * y3.x + y3.y * y3.y;
                }
            (is_k ? nd->rk_sm : nd->rq_sm)[s][t] = kNorm ? rsqrtf(ss / ds + a.norm_eps) : 1.f;
            all += ss;
        }
        (is_k ? nd->rk_la : nd->rq_la)[t] = kNorm ? rsqrtf(all + a.norm_eps) : 1.f;
    }
    __syncthreads();
    const uint32_t q_at = tc::smem_u32(sm + L::oQ), k_at = tc::smem_u32(sm + L::oK);
    {
        // k S0 and q S0.  A warp has kCols columns; the lane that holds column j of a B fragment loads kNs neighbouring columns,
        // one for each of the warp's column tiles, so that a lane's results are 2 kNs neighbouring columns of a row.
        float acc[2 * R][kNs][4];
#pragma unroll
        for (int m = 0; m < 2 * R; ++m)
#pragma unroll
            for (int i = 0; i < kNs; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[m][i][x] = 0.f;
        const float *S = a.state + (size_t)bh * D * D + warp * kCols + g4 * kNs;
        float s[2][4][kNs];                       // rows 2 c4, + 1, + 8, + 9 of a step of 16
        auto load = [&](int k, float (&y)[4][kNs]) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float *row = S + (size_t)(16 * k + 2 * c4 + (i & 1) + (i >> 1) * 8) * D;
                if constexpr (kNs == 4) {
                    const float4 v = __ldg(reinterpret_cast<const float4 *>(row));
                    y[i][0] = v.x; y[i][1] = v.y; y[i][2] = v.z; y[i][3] = v.w;
                } else {
                    const float2 v = __ldg(reinterpret_cast<const float2 *>(row));
                    y[i][0] = v.x; y[i][1] = v.y;
                }
            }
        };
        load(0, s[0]);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            if (k + 1 < D / 16) load(k + 1, s[(k + 1) & 1]);
            uint32_t b0[kNs][3], b1[kNs][3];
#pragma unroll
            for (int i = 0; i < kNs; ++i) {
                split3(s[k & 1][0][i], s[k & 1][1][i], b0[i]);
                split3(s[k & 1][2][i], s[k & 1][3][i], b1[i]);
            }
#pragma unroll
            for (int m = 0; m < 2 * R; ++m) {
                uint32_t af[4];
                ldmatrix_x4((m < R ? k_at : q_at) + ((m % R) * 16 + (lane & 15)) * L::kPitch + (2 * k + (lane >> 4)) * 16, af);
#pragma unroll
                for (int i = 0; i < kNs; ++i)
#pragma unroll
                    for (int x = 2; x >= 0; --x) mma_bf16(acc[m][i], af, b0[i][x], b1[i][x]);
            }
        }
        const int col = warp * kCols + 2 * kNs * c4;
#pragma unroll
        for (int m = 0; m < 2 * R; ++m)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = (m % R) * 16 + r * 8 + g4;
                const float fk = nd->whole[t] * nd->rk_la[t], fq = a.scale_la * nd->whole[t] * nd->rq_la[t], bt = nd->beta[t];
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < kNs; i += 2) {
                        const int at = col + x * kNs + i;
                        if (m < R) {
                            const float2 v = bf2(*reinterpret_cast<const uint32_t *>(sm + L::oV + t * L::kPitch + at * 2));
                            *reinterpret_cast<float2 *>(su + t * D + at) =
                                make_float2(bt * (v.x - fk * acc[m][i][2 * r + x]), bt * (v.y - fk * acc[m][i + 1][2 * r + x]));
                        } else if (t < n) {
                            *reinterpret_cast<float2 *>(base + (size_t)t * D + at) =
                                make_float2(fq * acc[m][i][2 * r + x], fq * acc[m][i + 1][2 * r + x]);
                        }
                    }
            }
    }
    {
        // the tables: warp = 16 rows, all columns
        constexpr int kNt = 2 * R;
        float kk[kNt][4], qk[G][kNt][4];
#pragma unroll
        for (int i = 0; i < kNt; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                kk[i][x] = 0.f;
#pragma unroll
                for (int s = 0; s < G; ++s) qk[s][i][x] = 0.f;
            }
        if (warp < R) {
#pragma unroll
            for (int k = 0; k < D / 16; k += 2) {
                uint32_t ak[2][4], aq[2][4];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t off = (warp * 16 + (lane & 15)) * L::kPitch + (2 * (k + y) + (lane >> 4)) * 16;
                    ldmatrix_x4(k_at + off, ak[y]);
                    ldmatrix_x4(q_at + off, aq[y]);
                }
#pragma unroll
                for (int i = 0; i < kNt; ++i) {
                    uint32_t bf[4];
                    ldmatrix_x4(k_at + (i * 8 + (lane & 7)) * L::kPitch + (2 * k + (lane >> 3)) * 16, bf);
                    mma_bf16(kk[i], ak[0], bf[0], bf[1]);
                    mma_bf16(kk[i], ak[1], bf[2], bf[3]);
                    mma_bf16(qk[k * 16 / ds][i], aq[0], bf[0], bf[1]);
                    mma_bf16(qk[k * 16 / ds][i], aq[1], bf[2], bf[3]);
                }
            }
        }
        __syncthreads();                          // q and k have been read: the tables take their place
        if (warp < R) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int t = warp * 16 + r * 8 + g4;
                const unsigned long long path = t < n ? nd->above[t] | 1ull << t : 0ull, seen = path & nd->keep;
                const float bt = nd->beta[t] * nd->rk_la[t], fq = a.scale_la * nd->rq_la[t];
#pragma unroll
                for (int i = 0; i < kNt; ++i)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int j = i * 8 + 2 * c4 + x;
                        if (!(path >> j & 1)) continue;
                        float q = qk[0][i][2 * r + x];
#pragma unroll
                        for (int s = 1; s < G; ++s) q += qk[s][i][2 * r + x];
                        const float w = sb[t * kRows + j] * nd->rk_la[j];      // (the decay)
                        sa[t * kRows + j] = bt * w * kk[i][2 * r + x];
                        sb[t * kRows + j] = fq * w * q;
                    }
#pragma unroll
                for (int s = 0; s < G; ++s) {
                    const float f = a.scale_sm * kLog2e * nd->rq_sm[s][t];
                    float m = -INFINITY, z = 0.f;
#pragma unroll
                    for (int i = 0; i < kNt; ++i)
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const int j = i * 8 + 2 * c4 + x;
                            float &y = qk[s][i][2 * r + x];
                            y = seen >> j & 1 ? y * f * nd->rk_sm[s][j] : -INFINITY;
                            m = fmaxf(m, y);
                        }
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
                    const float mu = m == -INFINITY ? 0.f : m;
#pragma unroll
                    for (int i = 0; i < kNt; ++i) {
                        const float p0 = tc::ex2_ftz(qk[s][i][2 * r] - mu), p1 = tc::ex2_ftz(qk[s][i][2 * r + 1] - mu);
                        z += p0 + p1;
                        // (fp16: 2^-11 of a probability, finer than the bf16 of those over the cache)
                        *reinterpret_cast<uint32_t *>(sp + (s * kRows + t) * kRows + i * 8 + 2 * c4) = tc::pack_half2(p0, p1);
                    }
                    z += __shfl_xor_sync(0xffffffffu, z, 1);
                    z += __shfl_xor_sync(0xffffffffu, z, 2);
                    if (c4 == 0 && t < n) { own[s * T + t] = m; own[(4 + s) * T + t] = z; }
                }
            }
        }
    }
    __syncthreads();
    // up the tree node by node; a column's thread needs no other column
    if (tid < D) {
        const int col = tid, gc = col / ds;
        const __nv_bfloat16 *v = reinterpret_cast<const __nv_bfloat16 *>(sm + L::oV) + col;
        const unsigned long long fold = nd->fold, keep = nd->keep;
        constexpr int kAhead = 8;
        float next[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) next[i] = i < n ? base[(size_t)i * D + col] : 0.f;
        for (int t0 = 0; t0 < n; t0 += kAhead) {
            float o8[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                o8[i] = next[i];
                next[i] = t0 + kAhead + i < n ? base[(size_t)(t0 + kAhead + i) * D + col] : 0.f;
            }
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                const int t = t0 + i;
                if (t >= n) break;
                float u = su[t * D + col], o = o8[i], s = 0.f;
                for (unsigned long long w = nd->above[t]; w; w &= w - 1) {
                    const int j = __ffsll(w) - 1;
                    if (fold >> j & 1) {
                        const float x = su[j * D + col];
                        u = fmaf(-sa[t * kRows + j], x, u);
                        o = fmaf(sb[t * kRows + j], x, o);
                    }
                    if (keep >> j & 1) s = fmaf(__half2float(sp[(gc * kRows + t) * kRows + j]), to_f32(v[j * (L::kPitch / 2)]), s);
                }
                if (fold >> t & 1) o = fmaf(sb[t * kRows + t], u, o);
                else u = 0.f;
                if (keep >> t & 1) s = fmaf(__half2float(sp[(gc * kRows + t) * kRows + t]), to_f32(v[t * (L::kPitch / 2)]), s);
                su[t * D + col] = u;
                base[(size_t)t * D + col] = o;
                own[8 * T + (size_t)t * D + col] = s;
                if (a.u) a.u[(((size_t)b * T + t) * a.H + h) * D + col] = u;
            }
        }
    }
}

template <int D, int G, bool kNorm, int R>
__global__ void __launch_bounds__(kThreads, 2) tree_tc_kernel(Args a) {
    extern __shared__ __align__(128) uint8_t dyn_tc[];
    __shared__ Nodes nodes;
    const int per_pair = a.parts + 1, bh = blockIdx.x / per_pair, part = blockIdx.x - bh * per_pair - 1;   // part -1: the tree
    const int b = bh / a.H, h = bh - b * a.H, n = nodes_of(a, b);
    if (part < 0) {
        tree_item<D, G, kNorm, R>(a, dyn_tc, &nodes, b, h, n);
    } else {
        const Cut c = cut_of(a.cache_len[bh], a.cap, a.parts, a.least_tiles);
        if (part < c.np && n > 0) cache_item<D, G, kNorm, R>(a, dyn_tc, b, h, part, n, c);
    }
    if (last_of_pair(a, bh)) join_pair<__nv_bfloat16, D>(a, b, h, n);
}

template <int D, int G, bool kNorm, int R>
cudaError_t launch(const Args &a, int BH, cudaStream_t st) {
    auto kernel = tree_tc_kernel<D, G, kNorm, R>;
    cudaError_t e = allow_smem(kernel, Layout<D, R>::kTotal);
    if (e != cudaSuccess) return e;
    kernel<<<BH * (a.parts + 1), kThreads, Layout<D, R>::kTotal, st>>>(a);
    count_launch();
    return cudaGetLastError();
}
template <int D, int G, bool kNorm>
cudaError_t by_rows(const Args &a, int BH, cudaStream_t st) {
    if (a.T <= 16) return launch<D, G, kNorm, 1>(a, BH, st);
    if (a.T <= 32) return launch<D, G, kNorm, 2>(a, BH, st);
    return launch<D, G, kNorm, 4>(a, BH, st);
}

}  // namespace

cudaError_t launch_tree_tc(const tree::Args &a, int BH, int d, cudaStream_t st) {
    const bool norm = a.norm_eps >= 0.f;
    if (d == 128) {
        if (a.G == 1) return norm ? by_rows<128, 1, true>(a, BH, st) : by_rows<128, 1, false>(a, BH, st);
        return norm ? by_rows<128, 2, true>(a, BH, st) : by_rows<128, 2, false>(a, BH, st);
    }
    if (a.G == 1) return norm ? by_rows<64, 1, true>(a, BH, st) : by_rows<64, 1, false>(a, BH, st);
    return norm ? by_rows<64, 2, true>(a, BH, st) : by_rows<64, 2, false>(a, BH, st);
}

}  // namespace natsl
