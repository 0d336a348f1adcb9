// The accepted path p_1 .. p_m of a drafted tree goes into the two hidden states (Section 4.3's recurrence, unrolled):
//   S <- D S0 + sum_j D_j k_(p_j)^T u_(p_j)   over the folded tokens, D_j the decay behind token j, D the whole one;
// the tree step has left u, so the tokens do not depend on each other and no product with the state is needed.
// K/V rows of the retained tokens are appended to the cache.
//
// Bound by the state's round trip (8 d^2 bytes per pair).  One CTA per pair, four per multiprocessor: a thread has four columns
// and kRows neighbouring rows, read before the path is, four rows at a time afterwards.  B200: 64 x 16 pairs of 128 columns,
// paths of up to 32 nodes, 37 to 39 us (146 MB: 3.8 to 3.9 TB/s; a wave of CTAs is short, and each begins with the chain length of the
// path -> rows -> products); one CTA per multiprocessor with the state in registers took 64 us.  16 pairs take 5.4 us.
#include "tree_common.cuh"

namespace natsl {
namespace {

using namespace tree;

constexpr int kCommitThreads = 256;

// V neighbouring elements of a row.
template <typename ST, int V> struct RowPiece;
template <> struct RowPiece<float, 4> { using type = uint4; };
template <> struct RowPiece<float, 2> { using type = uint2; };
template <> struct RowPiece<__nv_bfloat16, 4> { using type = uint2; };
template <> struct RowPiece<__nv_bfloat16, 2> { using type = uint32_t; };
template <int V> __device__ __forceinline__ void unpack(uint4 y, float (&x)[V]) {
    x[0] = __uint_as_float(y.x); x[1] = __uint_as_float(y.y); x[2] = __uint_as_float(y.z); x[3] = __uint_as_float(y.w);
}
template <int V> __device__ __forceinline__ void unpack(uint32_t y, float (&x)[V]) {
    x[0] = __uint_as_float(y << 16);
    x[1] = __uint_as_float(y & 0xffff0000u);
}
template <int V> __device__ __forceinline__ void unpack(uint2 y, float (&x)[V]) {
    if constexpr (V == 2) {                       // two fp32
        x[0] = __uint_as_float(y.x);
        x[1] = __uint_as_float(y.y);
    } else {                                      // four bf16
        x[0] = __uint_as_float(y.x << 16); x[1] = __uint_as_float(y.x & 0xffff0000u);
        x[2] = __uint_as_float(y.y << 16); x[3] = __uint_as_float(y.y & 0xffff0000u);
    }
}

template <typename ST, int D>
__global__ void __launch_bounds__(kCommitThreads, 4)
tree_commit_kernel(const ST *__restrict__ k, const ST *__restrict__ v, const float *__restrict__ g,
                   const uint8_t *__restrict__ route, const float *__restrict__ u, const int32_t *__restrict__ path,
                   const int32_t *__restrict__ n_path, float *__restrict__ state, ST *__restrict__ k_cache,
                   ST *__restrict__ v_cache, int32_t *__restrict__ cache_len, int cap, int H, int T, float norm_eps,
                   int32_t *status) {
    constexpr int kVec = D / 4, kGroups = kCommitThreads / kVec, kRows = D / kGroups, V = D / 32;
    using Piece = typename RowPiece<ST, V>::type;
    extern __shared__ __align__(16) float dyn[];  // [T][D] keys, times what the token counts; [T][D] u
    __shared__ int s_node[kMaxNodes];
    __shared__ float s_alpha[kMaxNodes], s_after[kMaxNodes];
    __shared__ unsigned long long s_fold, s_keep;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bh = blockIdx.x, b = bh / H, h = bh - b * H;
    float *sk = dyn, *su = dyn + T * D;
    float4 *S = reinterpret_cast<float4 *>(state + (size_t)bh * D * D) + tid % kVec;
    const int row0 = tid / kVec * kRows;
    float4 s[4];
    auto load = [&](int q) {
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = S[(size_t)(row0 + 4 * q + r) * kVec];
    };
    tc::grid_dependency_wait();
    tc::launch_dependents();
    load(0);

    const int m_raw = n_path[b], m = min(max(m_raw, 0), T), n_raw = cache_len[bh], n_old = min(max(n_raw, 0), cap);
    bool bad = m_raw != m;
    if (tid < kMaxNodes) {
        int node = -1, rv = 1;
        if (tid < m) {
            node = path[(size_t)b * T + tid];
            const int before = tid ? path[(size_t)b * T + tid - 1] : -1;
            if (node <= before || node >= T || before < -1) {      // a path climbs: no node twice, none outside the tree
                bad = true;
            } else {
                const size_t at = ((size_t)b * T + node) * H + h;
                rv = route[at];
                s_alpha[tid] = expf(g[at]);
            }
        }
        s_node[tid] = node;
        const unsigned f = __ballot_sync(0xffffffffu, tid < m && rv != 1), kp = __ballot_sync(0xffffffffu, tid < m && rv != 0);
        if (lane == 0) {
            reinterpret_cast<unsigned *>(&s_fold)[warp] = f;
            reinterpret_cast<unsigned *>(&s_keep)[warp] = kp;
        }
    }
    bad = __syncthreads_or(bad);
    const int kept = __popcll(s_keep);
    if (tid == 0) {
        if (bad) atomicMin(status, (int)NATSL_ERR_TREE);
        if (n_raw != n_old || (!bad && kept > cap - n_old)) atomicMin(status, (int)NATSL_ERR_CACHE_FULL);
    }
    // (the same for the whole CTA) What is reported is left untouched, so that the caller can mend it and commit again.
    if (bad || n_raw != n_old || kept > cap - n_old) return;
    if (m == 0) return;
    if (tid < m) {
        float x = 1.f;
        for (int j = tid + 1; j < m; ++j) x *= s_alpha[j];
        s_after[tid] = x;
    }
    __syncthreads();
    const float whole = s_after[0] * s_alpha[0];
    for (int j = warp; j < m; j += kCommitThreads / 32) {
        const size_t row = (((size_t)b * T + s_node[j]) * H + h) * D + lane * V;
        const bool fold = s_fold >> j & 1, keep = s_keep >> j & 1;
        const Piece kp = *reinterpret_cast<const Piece *>(k + row), vp = *reinterpret_cast<const Piece *>(v + row);
        float x[V], y[V], ss = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) y[i] = fold ? u[row + i] : 0.f;
        unpack<V>(kp, x);
#pragma unroll
        for (int i = 0; i < V; ++i) ss = fmaf(x[i], x[i], ss);
        float f = s_after[j];
        if (norm_eps >= 0.f) f *= rsqrtf(warp_sum(ss) + norm_eps);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            sk[j * D + lane * V + i] = fold ? f * x[i] : 0.f;
            su[j * D + lane * V + i] = y[i];
        }
        if (keep) {
            const size_t at = ((size_t)bh * cap + n_old + __popcll(s_keep & ((1ull << j) - 1))) * D + lane * V;
            *reinterpret_cast<Piece *>(k_cache + at) = kp;
            *reinterpret_cast<Piece *>(v_cache + at) = vp;
        }
    }
    if (tid == 0 && kept) cache_len[bh] = n_old + kept;
    __syncthreads();
#pragma unroll
    for (int q = 0; q < kRows / 4; ++q) {
        float4 o[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) o[r] = make_float4(whole * s[r].x, whole * s[r].y, whole * s[r].z, whole * s[r].w);
        if (q + 1 < kRows / 4) load(q + 1);
        for (int j = 0; j < m; ++j) {
            const float4 uu = *reinterpret_cast<const float4 *>(su + j * D + tid % kVec * 4);
            const float4 k4 = *reinterpret_cast<const float4 *>(sk + j * D + row0 + 4 * q);
            const float kk[4] = {k4.x, k4.y, k4.z, k4.w};
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                o[r].x = fmaf(kk[r], uu.x, o[r].x); o[r].y = fmaf(kk[r], uu.y, o[r].y);
                o[r].z = fmaf(kk[r], uu.z, o[r].z); o[r].w = fmaf(kk[r], uu.w, o[r].w);
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) S[(size_t)(row0 + 4 * q + r) * kVec] = o[r];
    }
}

template <typename ST, int D>
cudaError_t launch(const void *k, const void *v, const float *g, const uint8_t *route, const float *u, const int32_t *path,
                   const int32_t *n_path, float *state, void *k_cache, void *v_cache, int32_t *cache_len, int cap, Shape s,
                   float norm_eps, void *ws, cudaStream_t st) {
    cudaError_t e = allow_smem(tree_commit_kernel<ST, D>, 2 * kMaxNodes * D * 4);
    if (e != cudaSuccess) return e;
    e = launch_kernel(tree_commit_kernel<ST, D>, dim3(s.B * s.H), dim3(kCommitThreads), 2 * s.L * D * 4, st, true, (const ST *)k,
                      (const ST *)v, g, route, u, path, n_path, state, (ST *)k_cache, (ST *)v_cache, cache_len, cap, s.H, s.L, norm_eps,
                      reinterpret_cast<int32_t *>(ws));
    count_launch();
    return e;
}

}  // namespace

cudaError_t launch_tree_commit(const void *k, const void *v, const float *g, const uint8_t *route, const float *u,
                               const int32_t *path, const int32_t *n_path, float *state, void *k_cache, void *v_cache,
                               int32_t *cache_len, int cap, Shape s, float norm_eps, void *ws, cudaStream_t st) {
#define ARGS k, v, g, route, u, path, n_path, state, k_cache, v_cache, cache_len, cap, s, norm_eps, ws, st
    if (s.bf16) return s.d == 128 ? launch<__nv_bfloat16, 128>(ARGS) : launch<__nv_bfloat16, 64>(ARGS);
    return s.d == 128 ? launch<float, 128>(ARGS) : launch<float, 64>(ARGS);
#undef ARGS
}

}  // namespace natsl
