// The accepted path p_1 .. p_m of a drafted tree goes into the two hidden states (Section 4.3's recurrence, unrolled):
//   S <- D S0 + sum_j D_j k_(p_j)^T u_(p_j)   over the folded tokens, D_j the decay behind token j, D the whole one;
// the tree step has left u, so the tokens do not depend on each other and no product with the state is needed.
// K/V rows of the retained tokens are appended to the cache.
//
// Bound by the state's round trip (8 d^2 bytes per pair): one CTA per pair, every thread's share of the state in flight
// before the path is read.
#include "tree_common.cuh"

namespace natsl {
namespace {

using namespace tree;

constexpr int kCommitThreads = 512;

template <typename ST, int D>
__global__ void __launch_bounds__(kCommitThreads)
tree_commit_kernel(const ST *__restrict__ k, const ST *__restrict__ v, const float *__restrict__ g,
                   const uint8_t *__restrict__ route, const float *__restrict__ u, const int32_t *__restrict__ path,
                   const int32_t *__restrict__ n_path, float *__restrict__ state, ST *__restrict__ k_cache,
                   ST *__restrict__ v_cache, int32_t *__restrict__ cache_len, int cap, int H, int T, float norm_eps,
                   int32_t *status) {
    constexpr int kVec = D / 4, kGroups = kCommitThreads / kVec, kRows = D / kGroups;
    extern __shared__ __align__(16) float dyn[];  // [T][D] keys, times what the token counts; [T][D] u
    __shared__ int s_node[kMaxNodes];
    __shared__ float s_alpha[kMaxNodes], s_after[kMaxNodes];
    __shared__ unsigned long long s_fold, s_keep;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bh = blockIdx.x, b = bh / H, h = bh - b * H;
    float *sk = dyn, *su = dyn + T * D;
    float4 *S = reinterpret_cast<float4 *>(state + (size_t)bh * D * D) + tid % kVec;
    const int row0 = tid / kVec;
    float4 s[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) s[r] = S[(size_t)(row0 + r * kGroups) * kVec];

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
        if (n_raw != n_old || (!bad && n_old + kept > cap)) atomicMin(status, (int)NATSL_ERR_CACHE_FULL);
    }
    if (bad || kept > cap - n_old) return;        // (the same for the whole CTA) the pair is left untouched
    float whole = 1.f;
    for (int j = 0; j < m; ++j) whole *= s_alpha[j];
    if (tid < m) {
        float x = 1.f;
        for (int j = tid + 1; j < m; ++j) x *= s_alpha[j];
        s_after[tid] = x;
    }
    __syncthreads();
    for (int j = warp; j < m; j += kCommitThreads / 32) {
        const size_t row = (((size_t)b * T + s_node[j]) * H + h) * D + lane * (D / 32);
        const bool fold = s_fold >> j & 1, keep = s_keep >> j & 1;
        float x[D / 32], ss = 0.f;
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            x[i] = to_f32(k[row + i]);
            ss = fmaf(x[i], x[i], ss);
        }
        float f = s_after[j];
        if (norm_eps >= 0.f) f *= rsqrtf(warp_sum(ss) + norm_eps);
#pragma unroll
        for (int i = 0; i < D / 32; ++i) {
            sk[j * D + lane * (D / 32) + i] = fold ? f * x[i] : 0.f;
            su[j * D + lane * (D / 32) + i] = fold ? u[row + i] : 0.f;
        }
        if (keep) {
            const int at = n_old + __popcll(s_keep & ((1ull << j) - 1));
            ST *kc = k_cache + ((size_t)bh * cap + at) * D + lane * (D / 32), *vc = v_cache + ((size_t)bh * cap + at) * D + lane * (D / 32);
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                kc[i] = k[row + i];
                vc[i] = v[row + i];
            }
        }
    }
    if (tid == 0 && kept) cache_len[bh] = n_old + kept;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kRows; ++r) { s[r].x *= whole; s[r].y *= whole; s[r].z *= whole; s[r].w *= whole; }
    for (int j = 0; j < m; ++j) {
        const float4 uu = *reinterpret_cast<const float4 *>(su + j * D + tid % kVec * 4);
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const float kk = sk[j * D + row0 + r * kGroups];
            s[r].x = fmaf(kk, uu.x, s[r].x); s[r].y = fmaf(kk, uu.y, s[r].y);
            s[r].z = fmaf(kk, uu.z, s[r].z); s[r].w = fmaf(kk, uu.w, s[r].w);
        }
    }
    if (m == 0) return;
#pragma unroll
    for (int r = 0; r < kRows; ++r) S[(size_t)(row0 + r * kGroups) * kVec] = s[r];
}

template <typename ST, int D>
cudaError_t launch(const void *k, const void *v, const float *g, const uint8_t *route, const float *u, const int32_t *path,
                   const int32_t *n_path, float *state, void *k_cache, void *v_cache, int32_t *cache_len, int cap, Shape s,
                   float norm_eps, void *ws, cudaStream_t st) {
    cudaError_t e = allow_smem(tree_commit_kernel<ST, D>, 2 * kMaxNodes * D * 4);
    if (e != cudaSuccess) return e;
    tree_commit_kernel<ST, D><<<s.B * s.H, kCommitThreads, 2 * s.L * D * 4, st>>>(
        (const ST *)k, (const ST *)v, g, route, u, path, n_path, state, (ST *)k_cache, (ST *)v_cache, cache_len, cap, s.H, s.L,
        norm_eps, reinterpret_cast<int32_t *>(ws));
    count_launch();
    return cudaGetLastError();
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
