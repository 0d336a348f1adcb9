// A bounded retained cache: attention weights added up per entry, and eviction by them.
//
// natsl_cache_weights adds to an entry's weight what the given query rows' softmax gives it,
//   weight_j += sum_t sum_s exp(scale q_ts.k_js - lse_ts)   over the rows that see it,
// from the log-sum-exps that the attention itself has left, so K is read once and V not at all.
//
// natsl_cache_evict keeps the first entries, the latest ones and the heaviest of the rest.  Two kernels: one selects (a
// radix select of the threshold on the weights' bits, ties to the lowest index) and lists the entries that stay; one
// moves them to the front, in order and in place.
#include "common.cuh"
#include "natsl_internal.h"
#include "tc_common.cuh"

namespace natsl {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ------------------------------------------------------------------------------------------
// Weights, fp32 CUDA cores: eight lanes share a key, each with D / 8 neighbouring columns; the query rows pass through
// shared memory in blocks.
// ------------------------------------------------------------------------------------------
constexpr int kWThreads = 128, kWKeys = kWThreads / 8, kWRows = 16;

template <typename ST, int D>
__global__ void __launch_bounds__(kWThreads)
cache_weights_simt_kernel(const ST *__restrict__ q, const float *__restrict__ lse, const int32_t *__restrict__ visible,
                          const ST *__restrict__ k_cache, const int32_t *__restrict__ cache_len, int cap,
                          float *__restrict__ weight, int H, int T, int G, float scale, float norm_eps, int blocks) {
    constexpr int kE = D / 8;
    __shared__ __align__(16) float sq[kWRows][D];
    __shared__ float s_lse[4][kWRows];
    __shared__ int s_vis[kWRows];
    const int tid = threadIdx.x, l8 = tid & 7, bh = blockIdx.x / blocks, b = bh / H, h = bh - b * H, ds = D / G, lanes = 8 / G;
    const int n = min(max(cache_len[bh], 0), cap), j0 = (blockIdx.x - bh * blocks) * kWKeys, j = j0 + tid / 8;
    if (j0 >= n) return;
    float kx[kE], sum = 0.f;
    {
        const ST *row = k_cache + ((size_t)bh * cap + min(j, n - 1)) * D + l8 * kE;
        float ss = 0.f;
#pragma unroll
        for (int x = 0; x < kE; x += 4) {
            const float4 y = load4(row + x);
            kx[x] = y.x; kx[x + 1] = y.y; kx[x + 2] = y.z; kx[x + 3] = y.w;
            ss += y.x * y.x + y.y * y.y + y.z * y.z + y.w * y.w;
        }
        if (norm_eps >= 0.f) {
            for (int o = lanes / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
            const float f = rsqrtf(ss / ds + norm_eps);
#pragma unroll
            for (int x = 0; x < kE; ++x) kx[x] *= f;
        }
    }
    for (int t0 = 0; t0 < T; t0 += kWRows) {
        const int rows = min(kWRows, T - t0);
        __syncthreads();
        for (int i = tid; i < rows * D; i += kWThreads) {
            const int t = i / D, x = i - t * D;
            sq[t][x] = to_f32(q[(((size_t)b * T + t0 + t) * H + h) * D + x]);
        }
        for (int i = tid; i < rows; i += kWThreads) s_vis[i] = visible ? min(visible[((size_t)b * T + t0 + i) * H + h], n) : n;
        for (int i = tid; i < rows * G; i += kWThreads)
            s_lse[i / rows][i % rows] = lse[((size_t)bh * G + i / rows) * T + t0 + i % rows];
        __syncthreads();
        if (norm_eps >= 0.f) {
            for (int i = tid; i < rows * G; i += kWThreads) {
                float *row = &sq[i % rows][i / rows * ds], ss = 0.f;
                for (int x = 0; x < ds; ++x) ss = fmaf(row[x], row[x], ss);
                const float f = rsqrtf(ss / ds + norm_eps);
                for (int x = 0; x < ds; ++x) row[x] *= f;
            }
            __syncthreads();
        }
        for (int t = 0; t < rows; ++t) {
            float s = 0.f;
#pragma unroll
            for (int x = 0; x < kE; x += 4) {
                const float4 y = *reinterpret_cast<const float4 *>(&sq[t][l8 * kE + x]);
                s = fmaf(y.x, kx[x], fmaf(y.y, kx[x + 1], fmaf(y.z, kx[x + 2], fmaf(y.w, kx[x + 3], s))));
            }
            for (int o = lanes / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            const float l = s_lse[l8 / lanes][t];
            // (a row without a finite log-sum-exp sees nothing; every lane of a head has the head's logit, one counts)
            if (l8 % lanes == 0 && j < s_vis[t] && isfinite(l)) sum += tc::ex2_ftz((s * scale - l) * kLog2e);
        }
    }
    for (int o = 4; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (l8 == 0 && j < n) weight[(size_t)bh * cap + j] += sum;
}

// ------------------------------------------------------------------------------------------
// Eviction: selection
// ------------------------------------------------------------------------------------------
constexpr int kSThreads = 1024, kBins = 2048;

// Weights in the order of unsigned words: a NaN below everything, both zeros equal.
__device__ __forceinline__ uint32_t order_key(float w) {
    if (isnan(w)) return 0u;
    const uint32_t x = __float_as_uint(w + 0.f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

__global__ void __launch_bounds__(kSThreads)
evict_select_kernel(const float *__restrict__ weight, int32_t *__restrict__ cache_len, int cap, int keep, int first, int recent,
                    int32_t *__restrict__ kept) {
    __shared__ int hist[kBins], s_warp[2][32], s_pick[2];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bh = blockIdx.x;
    const float *w = weight + (size_t)bh * cap;
    int32_t *list = kept + (size_t)bh * keep;
    const int n = min(max(cache_len[bh], 0), cap);
    if (n <= keep) {
        for (int i = tid; i < n; i += kSThreads) list[i] = i;
        return;
    }
    // the threshold: the weight of rank `need` among the entries that are not safe anyway, from its high bits down
    const int lo = first, hi = n - recent;
    int need = keep - first - recent;             // (entries still to be taken with the bits found so far)
    uint32_t prefix = 0;
    for (int pass = 0; pass < 3 && need > 0; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11, above = shift + bits;
        for (int i = tid; i < kBins; i += kSThreads) hist[i] = 0;
        __syncthreads();
        for (int j = lo + tid; j < hi; j += kSThreads) {
            const uint32_t x = order_key(w[j]);
            if (pass == 0 || x >> above == prefix) atomicAdd(&hist[x >> shift & ((1u << bits) - 1u)], 1);
        }
        __syncthreads();
        // thread i holds bins 2 i, 2 i + 1, counted from the top
        const int c0 = hist[kBins - 1 - 2 * tid], c1 = hist[kBins - 2 - 2 * tid];
        int sum = c0 + c1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, sum, o);
            if (lane >= o) sum += y;
        }
        if (lane == 31) s_warp[0][warp] = sum;
        __syncthreads();
        if (warp == 0) {
            int x = s_warp[0][lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int y = __shfl_up_sync(0xffffffffu, x, o);
                if (lane >= o) x += y;
            }
            s_warp[0][lane] = x;
        }
        __syncthreads();
        const int upto = sum + (warp ? s_warp[0][warp - 1] : 0), before = upto - c0 - c1;
        if (before < need && need <= upto) {
            const bool second = need > before + c0;
            s_pick[0] = kBins - 1 - 2 * tid - second;
            s_pick[1] = need - before - (second ? c0 : 0);
        }
        __syncthreads();
        prefix = prefix << bits | (uint32_t)s_pick[0];
        need = s_pick[1];
        __syncthreads();
    }
    // prefix: the threshold; need: how many of its equals stay.  Warps own runs of entries: count, scan, list.
    const bool none = keep - first - recent <= 0;
    const int run = ((n + 31) / 32 + 31) / 32 * 32, j0 = min(n, warp * run), j1 = min(n, j0 + run);
    auto look = [&](int j, bool &over, bool &equal) {
        over = j < n && (j < lo || j >= hi);
        equal = false;
        if (!over && j < n && !none) {
            const uint32_t x = order_key(w[j]);
            over = x > prefix;
            equal = x == prefix;
        }
    };
    int overs = 0, equals = 0;
    for (int j = j0; j < j1; j += 32) {
        bool o, e;
        look(j + lane, o, e);
        overs += __popc(__ballot_sync(0xffffffffu, o));
        equals += __popc(__ballot_sync(0xffffffffu, e));
    }
    if (lane == 0) { s_warp[0][warp] = overs; s_warp[1][warp] = equals; }
    __syncthreads();
    int at_over = 0, at_equal = 0;
    for (int i = 0; i < warp; ++i) { at_over += s_warp[0][i]; at_equal += s_warp[1][i]; }
    for (int j = j0; j < j1; j += 32) {
        bool o, e;
        look(j + lane, o, e);
        const unsigned mo = __ballot_sync(0xffffffffu, o), me = __ballot_sync(0xffffffffu, e), below = (1u << lane) - 1u;
        const int eq = at_equal + __popc(me & below), ov = at_over + __popc(mo & below);
        if (o || (e && eq < need)) list[ov + min(eq, need)] = j + lane;
        at_over += __popc(mo);
        at_equal += __popc(me);
    }
    if (tid == 0) cache_len[bh] = keep;           // (every thread has read the old length: barriers above)
}

// ------------------------------------------------------------------------------------------
// Eviction: the move.  Entry r comes from kept[r] >= r.  A wave of rows is read into shared memory by the CTAs of a pair
// (a cluster), and written after the cluster's barrier.  What a wave writes lies below everything that later waves read:
// their sources are no lower than their own places.
// ------------------------------------------------------------------------------------------
constexpr int kMThreads = 256;

__device__ __forceinline__ void cp_async16(void *dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::smem_u32(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }

template <int kRowBytes, int kRows>
__global__ void __launch_bounds__(kMThreads)
evict_move_kernel(uint8_t *k_cache, uint8_t *v_cache, float *weight, const int32_t *__restrict__ cache_len,
                  const int32_t *__restrict__ kept, int cap, int keep, int cluster) {
    extern __shared__ __align__(16) uint8_t rows[];   // [2][kRows][kRowBytes]
    constexpr int kPieces = kRowBytes / 16;
    const int tid = threadIdx.x, bh = blockIdx.x / cluster, rank = blockIdx.x - bh * cluster;
    const int n = min(max(cache_len[bh], 0), keep);
    const int32_t *list = kept + (size_t)bh * keep;
    uint8_t *kc = k_cache + (size_t)bh * cap * kRowBytes, *vc = v_cache + (size_t)bh * cap * kRowBytes;
    float *w = weight + (size_t)bh * cap;
    const int wave = cluster * kRows;
    for (int r0 = 0; r0 < n; r0 += wave) {        // (every CTA of the cluster: the same number of barriers)
        const int mine = r0 + rank * kRows;
        float x = 0.f;
        bool move = false;
        if (tid < kRows && mine + tid < n) {
            const int src = list[mine + tid];
            move = src != mine + tid;
            if (move) x = w[src];
        }
        for (int i = tid; i < kRows * kPieces; i += kMThreads) {
            const int r = i / kPieces, c = i - r * kPieces;
            if (mine + r >= n) break;
            const int src = list[mine + r];
            if (src == mine + r) continue;
            cp_async16(rows + i * 16, kc + (size_t)src * kRowBytes + c * 16);
            cp_async16(rows + (kRows * kPieces + i) * 16, vc + (size_t)src * kRowBytes + c * 16);
        }
        cp_async_wait_all();
        if (cluster > 1) {
            asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
        } else {
            __syncthreads();
        }
        if (move) w[mine + tid] = x;
        for (int i = tid; i < kRows * kPieces; i += kMThreads) {
            const int r = i / kPieces, c = i - r * kPieces;
            if (mine + r >= n) break;
            if (list[mine + r] == mine + r) continue;
            *reinterpret_cast<uint4 *>(kc + (size_t)(mine + r) * kRowBytes + c * 16) = *reinterpret_cast<const uint4 *>(rows + i * 16);
            *reinterpret_cast<uint4 *>(vc + (size_t)(mine + r) * kRowBytes + c * 16) =
                *reinterpret_cast<const uint4 *>(rows + (kRows * kPieces + i) * 16);
        }
        __syncthreads();                          // (the next wave fills the same rows)
    }
}

template <int kRowBytes>
cudaError_t launch_move(void *k_cache, void *v_cache, float *weight, const int32_t *cache_len, const int32_t *kept, int cap,
                        int keep, int BH, cudaStream_t st) {
    constexpr int kRows = 32 * 1024 / kRowBytes;  // 64 KB of rows per CTA and wave
    auto kernel = evict_move_kernel<kRowBytes, kRows>;
    cudaError_t e = allow_smem(kernel, 2 * kRows * kRowBytes);
    if (e != cudaSuccess) return e;
    int cluster = 1;                              // few pairs: as many CTAs for each as the machine has room for
    while (cluster < 8 && BH * cluster * 2 <= 2 * sm_count() && cluster * kRows < keep) cluster *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(BH * cluster);
    cfg.blockDim = dim3(kMThreads);
    cfg.dynamicSmemBytes = 2 * kRows * kRowBytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, kernel, (uint8_t *)k_cache, (uint8_t *)v_cache, weight, cache_len, kept, cap, keep, cluster);
    count_launch();
    return e;
}

}  // namespace

cudaError_t launch_cache_weights(const void *q, const float *lse, const int32_t *visible, const void *k_cache,
                                 const int32_t *cache_len, int cap, float *weight, float scale, Shape s, HeadGroups hg,
                                 bool tensor_cores, cudaStream_t st) {
    const int blocks = (cap + kWKeys - 1) / kWKeys;
#define RUN(ST, D)                                                                                                   \
    cache_weights_simt_kernel<ST, D><<<s.B * s.H * blocks, kWThreads, 0, st>>>((const ST *)q, lse, visible, (const ST *)k_cache, \
                                                                               cache_len, cap, weight, s.H, s.L, hg.G, scale, \
                                                                               hg.norm_eps, blocks)
    if (s.bf16) {
        if (s.d == 128) RUN(__nv_bfloat16, 128);
        else RUN(__nv_bfloat16, 64);
    } else {
        if (s.d == 128) RUN(float, 128);
        else RUN(float, 64);
    }
#undef RUN
    count_launch();
    return cudaGetLastError();
}

cudaError_t launch_cache_evict(void *k_cache, void *v_cache, float *weight, int32_t *cache_len, int cap, int keep, int first,
                               int recent, int32_t *kept, Shape s, cudaStream_t st) {
    const int BH = s.B * s.H, row = s.d * (s.bf16 ? 2 : 4);
    evict_select_kernel<<<BH, kSThreads, 0, st>>>(weight, cache_len, cap, keep, first, recent, kept);
    count_launch();
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    if (row == 512) return launch_move<512>(k_cache, v_cache, weight, cache_len, kept, cap, keep, BH, st);
    if (row == 256) return launch_move<256>(k_cache, v_cache, weight, cache_len, kept, cap, keep, BH, st);
    return launch_move<128>(k_cache, v_cache, weight, cache_len, kept, cap, keep, BH, st);
}

}  // namespace natsl
