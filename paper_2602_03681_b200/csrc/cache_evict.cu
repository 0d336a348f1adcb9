// A bounded retained cache: attention weights added up per entry, and eviction by them.
//
// natsl_cache_weights adds to an entry's weight what the given query rows' softmax gives it,
//   weight_j += sum_t sum_s exp(scale q_ts.k_js - lse_ts)   over the rows that see it,
// from the log-sum-exps that the attention itself has left, so K is read once and V not at all.
//
// natsl_cache_evict keeps the first entries, the latest ones and the heaviest of the rest (a radix select on the
// weights' bits finds the threshold; ties to the lowest index) and moves them to the front, in order and in place.
//
// B200 (a range is what several of them gave): the weights of 64 x 16 caches of 1638 entries of 128 columns for up to 16 rows 72 to
// 75 us (444 MB: 5.9 to 6.2 TB/s, 91 to 94 % of a copy's rate); an eviction over 64 x 16 caches of up to 1638 150 to 184 us (up to
// 1.09 GB, entries before the first gap stay), and 39 to 44 us where it has been cut already and only the latest entries move; of 16
// caches of 8192 entries 34 to 35 us, and 20 to 23.
#include <algorithm>
#include "common.cuh"
#include "natsl_internal.h"
#include "tc_common.cuh"
#include "tree_common.cuh"

namespace natsl {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// 16 bytes global -> shared past the registers
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float square_sum(uint32_t bf16x2, float s) {
    const float lo = __uint_as_float(bf16x2 << 16), hi = __uint_as_float(bf16x2 & 0xffff0000u);
    return fmaf(lo, lo, fmaf(hi, hi, s));
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

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
// Weights of up to 16 rows, tensor cores (bf16 storage, one or two softmax heads per linear head).  Bound by reading K once.  A CTA
// takes a run of a pair's keys through a ring of asynchronous copies, tiles of 64, the rows of q as fragments in registers; its
// warps share the tile by keys.  (More rows: cache_weights_umma.cu, which has both sides' times.)
// ------------------------------------------------------------------------------------------
constexpr int kTTile = 64, kTStages = 3, kMaxRun = 1024;

template <int D, int G, bool kNorm>
__global__ void __launch_bounds__(kWThreads, 4)
cache_weights_tc_kernel(const uint8_t *__restrict__ q, const float *__restrict__ lse, const int32_t *__restrict__ visible,
                        const uint8_t *__restrict__ k_cache, const int32_t *__restrict__ cache_len, int cap,
                        float *__restrict__ weight, int H, int T, float scale, float norm_eps, int runs, int run) {
    constexpr int ds = D / G, kKs = ds / 16, kRows = 16, kKeys = kTTile / 4, kNt = kKeys / 8;
    constexpr int kRowBytes = D * 2, kPieces = kRowBytes / 16, kStep = kWThreads / kPieces, kTileBytes = kTTile * kRowBytes;
    extern __shared__ __align__(128) uint8_t dyn_w[];      // the ring; then the sums [run]
    __shared__ float2 s_row[G][kRows];            // factor to base-2 logits, log-sum-exp in base 2
    __shared__ int s_vis[G][kRows];
    __shared__ __align__(8) float s_key[kNorm ? G : 1][kTTile];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, c4 = lane & 3;
    tc::grid_dependency_wait();
    tc::launch_dependents();
    const int bh = blockIdx.x / runs, b = bh / H, h = bh - b * H, n = min(max(cache_len[bh], 0), cap);
    const int from = (blockIdx.x - bh * runs) * run, to = min(n, from + run), tiles = (to - from + kTTile - 1) / kTTile;
    if (from >= n) return;
    float *s_sum = reinterpret_cast<float *>(dyn_w + kTStages * kTileBytes);
    const uint32_t ring = tc::smem_u32(dyn_w);
    const int piece = tid % kPieces, row0 = tid / kPieces;
    const uint8_t *kc = k_cache + ((size_t)bh * cap + from) * kRowBytes + piece * 16;
    const uint32_t dst0 = row0 * kRowBytes + ((piece ^ (row0 & 7)) << 4);
    auto fetch = [&](int t) {
        if (t < tiles) {
#pragma unroll
            for (int i = 0; i < kTTile / kStep; ++i) {
                const int j = t * kTTile + row0 + i * kStep;
                cp_async16(ring + t % kTStages * kTileBytes + dst0 + i * kStep * kRowBytes,
                           kc + (size_t)min(j, to - from - 1) * kRowBytes);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kTStages - 1; ++i) fetch(i);
    for (int e = tid; e < kRows * G; e += kWThreads) {
        const int g = e / kRows, t = e - g * kRows;
        int vis = 0;
        float l = 0.f;
        if (t < T) {
            l = lse[((size_t)bh * G + g) * T + t];
            vis = visible ? max(min(visible[((size_t)b * T + t) * H + h], n), 0) : n;
            if (!isfinite(l)) vis = 0;            // (a row that sees nothing)
        }
        s_vis[g][t] = vis - from;
        s_row[g][t] = make_float2(scale * kLog2e, l * kLog2e);
    }
    // (q passes through the ring's last place, which the first tile's turn fills)
    constexpr int kQ = (kTStages - 1) * kTileBytes;
    for (int e = tid; e < kRows * kPieces; e += kWThreads) {
        const int t = e / kPieces, c = e - t * kPieces;
        *reinterpret_cast<uint4 *>(dyn_w + kQ + t * kRowBytes + ((c ^ (t & 7)) << 4)) =
            t < T ? *reinterpret_cast<const uint4 *>(q + (((size_t)b * T + t) * H + h) * kRowBytes + c * 16) : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    uint32_t qf[D / 16][4];
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        const int t = lane & 15;
        tc::ldmatrix_x4(ring + kQ + t * kRowBytes + (((2 * k + (lane >> 4)) ^ (t & 7)) << 4), qf[k]);
    }
    float2 f[G][2];
    int vis[G][2];
    int least = 0x7fffffff;                       // keys that all rows see
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            f[g][r] = s_row[g][r * 8 + g4];
            vis[g][r] = s_vis[g][r * 8 + g4] - warp * kKeys - 2 * c4;
            least = min(least, vis[g][r]);
            if (kNorm) {
                float ss = 0.f;
#pragma unroll
                for (int k = g * kKs; k < (g + 1) * kKs; ++k)
#pragma unroll
                    for (int x = 0; x < 2; ++x) ss = square_sum(qf[k][r + 2 * x], ss);
                ss += __shfl_xor_sync(0xffffffffu, ss, 1);
                ss += __shfl_xor_sync(0xffffffffu, ss, 2);
                f[g][r].x *= rsqrtf(ss / ds + norm_eps);
            }
        }
    least = __reduce_min_sync(0xffffffffu, least + 2 * c4);
    for (int t = 0; t < tiles; ++t) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kTStages - 2) : "memory");
        __syncthreads();                          // tile t is there, and every warp is done with tile t - 1 ...
        fetch(t + kTStages - 1);                  // ... whose place this one takes
        const uint32_t kt = ring + t % kTStages * kTileBytes;
        if (kNorm) {                              // a key's RMS factors: two threads each, half a row
            const int key = tid >> 1, half = tid & 1;
            const uint8_t *row = dyn_w + (kt - ring) + key * kRowBytes;
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < kPieces / 2; ++i) {
                const int p = half * (kPieces / 2) + ((i + 4 * half) & (kPieces / 2 - 1));
                const uint4 y = *reinterpret_cast<const uint4 *>(row + ((p ^ (key & 7)) << 4));
                ss = square_sum(y.x, square_sum(y.y, square_sum(y.z, square_sum(y.w, ss))));
            }
            if (G == 1) ss += __shfl_xor_sync(0xffffffffu, ss, 1);
            s_key[G == 2 ? half : 0][key] = rsqrtf(ss / ds + norm_eps);
            __syncthreads();
        }
        float sum[kNt][2];
#pragma unroll
        for (int i = 0; i < kNt; ++i) sum[i][0] = sum[i][1] = 0.f;
        const bool all = (t + 1) * kTTile <= least;              // (uniform)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float x[kNt][4];
#pragma unroll
            for (int i = 0; i < kNt; ++i)
#pragma unroll
                for (int y = 0; y < 4; ++y) x[i][y] = 0.f;
#pragma unroll
            for (int k = g * kKs; k < (g + 1) * kKs; ++k)
#pragma unroll
                for (int i = 0; i < kNt; i += 2) {
                    const int row = warp * kKeys + i * 8 + (lane & 7) + (lane >> 4) * 8;
                    uint32_t bf[4];
                    tc::ldmatrix_x4(kt + row * kRowBytes + (((2 * k + ((lane >> 3) & 1)) ^ (row & 7)) << 4), bf);
                    mma_bf16(x[i], qf[k], bf[0], bf[1]);
                    mma_bf16(x[i + 1], qf[k], bf[2], bf[3]);
                }
#pragma unroll
            for (int i = 0; i < kNt; ++i) {
                float2 w = make_float2(1.f, 1.f);
                if (kNorm) w = *reinterpret_cast<const float2 *>(&s_key[g][warp * kKeys + i * 8 + 2 * c4]);
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const float z = kNorm ? x[i][2 * r + y] * (y ? w.y : w.x) : x[i][2 * r + y];
                        const float e = tc::ex2_ftz(fmaf(z, f[g][r].x, -f[g][r].y));
                        sum[i][y] += all || t * kTTile + i * 8 + y < vis[g][r] ? e : 0.f;
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < kNt; ++i)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) sum[i][y] += __shfl_xor_sync(0xffffffffu, sum[i][y], o);
            }
        if (g4 == 0) {
#pragma unroll
            for (int i = 0; i < kNt; ++i)
                *reinterpret_cast<float2 *>(s_sum + t * kTTile + warp * kKeys + i * 8 + 2 * c4) = make_float2(sum[i][0], sum[i][1]);
        }
    }
    cp_async_wait_all();
    __syncthreads();
    for (int j = tid; j < to - from; j += kWThreads) weight[(size_t)bh * cap + from + j] += s_sum[j];
}

template <int D, int G, bool kNorm>
cudaError_t launch_weights_tc(const void *q, const float *lse, const int32_t *visible, const void *k_cache, const int32_t *cache_len,
                              int cap, float *weight, float scale, Shape s, float norm_eps, cudaStream_t st) {
    // Runs of 128 to 1024 keys: as short as one resident set of CTAs allows.
    const long long BH = (long long)s.B * s.H, resident = 148 * 4, per = (BH * cap + resident - 1) / resident;
    const int run = (int)std::min<long long>(kMaxRun, std::max<long long>(128, (per + kTTile - 1) / kTTile * kTTile));
    const int runs = (cap + run - 1) / run, ring = kTStages * kTTile * D * 2;
    auto kernel = cache_weights_tc_kernel<D, G, kNorm>;
    cudaError_t e = allow_smem(kernel, ring + kMaxRun * 4);
    if (e != cudaSuccess) return e;
    e = launch_kernel(kernel, dim3((unsigned)(BH * runs)), dim3(kWThreads), ring + run * 4, st, true, (const uint8_t *)q,
                      lse, visible, (const uint8_t *)k_cache, cache_len, cap, weight, s.H, s.L, scale, norm_eps, runs, run);
    count_launch();
    return e;
}

// ------------------------------------------------------------------------------------------
// Eviction.  A pair is the work of one CTA, or of a cluster where pairs are few: its CTAs share the entries to find what stays and
// list it, then they move the rows in waves: a wave of rows is read into shared memory by the CTAs, and written behind the
// cluster's barrier.  Entry r comes from kept[r] >= r, so what a wave writes lies below everything that later waves read.  And
// once one entry is gone all behind it move: what lies before the first gap is left in place.
// ------------------------------------------------------------------------------------------
constexpr int kEThreads = 512, kEWarps = kEThreads / 32, kBins = 256;

// Weights in the order of unsigned words: a NaN below everything (0), both zeros equal.
__device__ __forceinline__ uint32_t order_key(float w) {
    if (isnan(w)) return 0u;
    const uint32_t x = __float_as_uint(w + 0.f);
    return x & 0x80000000u ? ~x : x | 0x80000000u;
}

// kHeld: entries per lane whose keys stay in registers (512 kHeld per CTA); more lie in shared memory where the rows will be, and
// what does not fit there is read again.
template <int kRowBytes, int kHeld>
__global__ void __launch_bounds__(kEThreads)
evict_kernel(uint8_t *k_cache, uint8_t *v_cache, float *weight, int32_t *cache_len, int cap, int keep, int first, int recent,
             int32_t *kept, int cluster, int rows) {
    extern __shared__ __align__(16) uint8_t dyn_e[];       // [2][rows][kRowBytes], then the rows' weights and sources
    __shared__ int hist[2][kBins], s_warp[2][kEWarps], s_pick[2], s_total[2], s_gap;
    __shared__ uint32_t s_all, s_any;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, bh = blockIdx.x / cluster, rank = blockIdx.x - bh * cluster;
    tc::grid_dependency_wait();
    tc::launch_dependents();
    float *w = weight + (size_t)bh * cap;
    int32_t *list = kept + (size_t)bh * keep;
    const int n = min(max(cache_len[bh], 0), cap);
    if (n <= keep) {                              // (the same for the whole cluster)
        for (int i = rank * kEThreads + tid; i < n; i += cluster * kEThreads) list[i] = i;
        return;
    }
    auto meet = [&] {                             // the cluster's barrier
        if (cluster > 1) { tree::cluster_arrive(); tree::cluster_wait(); }
        else __syncthreads();
    };
    auto of_rank = [&](const void *p, int r) { return __float_as_int(tree::ld_remote(tree::remote(p, r))); };
    if (tid == 0) { s_all = 0xffffffffu; s_any = 0u; s_gap = keep; }
    // ---- a warp owns a run of entries, a lane every 32nd of them ----
    const int lo = first, hi = n - recent, want = keep - first - recent;      // candidates; how many of them stay
    const int warps = cluster * kEWarps, run = ((n + warps - 1) / warps + 31) / 32 * 32;
    const int j0 = (int)min((long long)n, (long long)(rank * kEWarps + warp) * run), j1 = min(n, j0 + run), steps = (j1 - j0 + 31) / 32;
    auto is_candidate = [&](int j) { return (j < j1) & (j >= lo) & (j < hi); };
    auto key_of = [&](int j) { return is_candidate(j) ? order_key(w[j]) : 0u; };
    uint32_t held[kHeld];
#pragma unroll
    for (int i = 0; i < kHeld; ++i) held[i] = key_of(j0 + i * 32 + lane);
    const int room = rows * (2 * kRowBytes + 8) / (kEWarps * 128), spare = max(0, min(steps - kHeld, room));
    uint32_t *more = reinterpret_cast<uint32_t *>(dyn_e) + warp * room * 32 + lane;
    for (int i = 0; i < spare; ++i) more[i * 32] = key_of(j0 + (kHeld + i) * 32 + lane);
    auto each = [&](auto &&f) {                   // f(entry, its key), the warp together
#pragma unroll
        for (int i = 0; i < kHeld; ++i) f(j0 + i * 32 + lane, held[i]);
        for (int i = kHeld; i < steps; ++i) {
            const int j = j0 + i * 32 + lane;
            f(j, i < kHeld + spare ? more[(i - kHeld) * 32] : key_of(j));
        }
    };
    // ---- the threshold, eight bits at a time from the highest in which two candidates differ: a histogram in each CTA, summed by
    // all of them over distributed shared memory.  (From the first bit on, weights meet in a few bins and their counters queue;
    // a bit at a time, over all of a pair's entries in each CTA, took 23 of a call's 34 us at 16 pairs of 8192.) ----
    int need = want;
    uint32_t prefix = 0xffffffffu;                // (nothing is over it or equal to it where nothing more is wanted)
    __syncthreads();
    if (want > 0) {
        uint32_t all = 0xffffffffu, any = 0u;
        each([&](int j, uint32_t x) {
            all &= is_candidate(j) ? x : 0xffffffffu;
            any |= x;
        });
        all = __reduce_and_sync(0xffffffffu, all);
        any = __reduce_or_sync(0xffffffffu, any);
        if (lane == 0) { atomicAnd(&s_all, all); atomicOr(&s_any, any); }
        meet();
        all = __reduce_and_sync(0xffffffffu, lane < cluster ? (uint32_t)of_rank(&s_all, lane) : 0xffffffffu);
        any = __reduce_or_sync(0xffffffffu, lane < cluster ? (uint32_t)of_rank(&s_any, lane) : 0u);
        const int top = 31 - __clz((int)(all ^ any));                          // (-1: all alike)
        prefix = top < 0 ? all : top == 31 ? 0u : all & ~((2u << top) - 1u);
        for (int above = top + 1, set = 0; above > 0; set ^= 1) {              // bits from `above` on are found
            const int shift = max(0, above - 8);
            if (tid < kBins) hist[set][tid] = 0;
            __syncthreads();
            each([&](int j, uint32_t x) {
                const bool in = is_candidate(j) & ((above < 32 ? (x ^ prefix) >> above : 0u) == 0u);
                if (in) atomicAdd(&hist[set][x >> shift & (above - shift < 8 ? (1u << (above - shift)) - 1u : 255u)], 1);
            });
            meet();                               // (a set is filled again two passes on: whoever does has seen everyone read it)
            int c = 0, sum = 0;
            if (tid < kBins) {                    // thread i: bin 255 - i
                for (int r = 0; r < cluster; ++r) c += of_rank(&hist[set][kBins - 1 - tid], r);
                sum = c;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int y = __shfl_up_sync(0xffffffffu, sum, o);
                    if (lane >= o) sum += y;
                }
                if (lane == 31) s_warp[0][warp] = sum;
            }
            __syncthreads();
            if (tid < kBins) {
                const int before = sum - c + __reduce_add_sync(0xffffffffu, lane < warp ? s_warp[0][lane] : 0);
                if (before < need && need <= before + c) { s_pick[0] = kBins - 1 - tid; s_pick[1] = need - before; }
            }
            __syncthreads();
            prefix |= (uint32_t)s_pick[0] << shift;
            need = s_pick[1];
            above = shift;
        }
    }
    // prefix: the threshold; need: how many of its equals stay, the lowest
    auto over = [&](int j, uint32_t x) { return (j < j1) & ((j < lo) | (j >= hi) | (x > prefix)); };
    auto equal = [&](int j, uint32_t x) { return is_candidate(j) & (x == prefix) & (want > 0); };
    int overs = 0, equals = 0;
    each([&](int j, uint32_t x) {
        overs += over(j, x);
        equals += equal(j, x);
    });
    overs = __reduce_add_sync(0xffffffffu, overs);
    equals = __reduce_add_sync(0xffffffffu, equals);
    __syncthreads();
    if (lane == 0) { s_warp[0][warp] = overs; s_warp[1][warp] = equals; }
    __syncthreads();
    if (warp == 0) {
        overs = __reduce_add_sync(0xffffffffu, lane < kEWarps ? s_warp[0][lane] : 0);
        equals = __reduce_add_sync(0xffffffffu, lane < kEWarps ? s_warp[1][lane] : 0);
        if (lane == 0) { s_total[0] = overs; s_total[1] = equals; }
    }
    meet();
    // ---- the list: entry j goes to the number of overs below it and of the equals that stay.  The first gap is the first place
    // whose entry comes from behind it. ----
    int at_over = __reduce_add_sync(0xffffffffu, (lane < warp ? s_warp[0][lane] : 0) + (lane < rank ? of_rank(&s_total[0], lane) : 0));
    int at_equal = __reduce_add_sync(0xffffffffu, (lane < warp ? s_warp[1][lane] : 0) + (lane < rank ? of_rank(&s_total[1], lane) : 0));
    int gap = keep;
    each([&](int j, uint32_t x) {
        const bool o = over(j, x), e = equal(j, x);
        const unsigned mo = __ballot_sync(0xffffffffu, o), me = __ballot_sync(0xffffffffu, e), below = (1u << lane) - 1u;
        const int eq = at_equal + __popc(me & below), to = at_over + __popc(mo & below) + min(eq, need);
        at_over += __popc(mo);
        at_equal += __popc(me);
        if (o | (e & (eq < need))) {
            list[to] = j;
            gap = to < j ? min(gap, to) : gap;
        }
    });
    gap = __reduce_min_sync(0xffffffffu, gap);
    if (lane == 0 && gap < keep) atomicMin(&s_gap, gap);
    meet();                                       // (the list is there, too)
    gap = __reduce_min_sync(0xffffffffu, lane < cluster ? of_rank(&s_gap, lane) : keep);
    const int wave = cluster * rows;
    // ---- the move ----
    constexpr int kPieces = kRowBytes / 16;
    float *s_w = reinterpret_cast<float *>(dyn_e + 2 * rows * kRowBytes);
    int *s_from = reinterpret_cast<int *>(s_w + rows);
    const uint32_t buffer = tc::smem_u32(dyn_e);
    uint8_t *kc = k_cache + (size_t)bh * cap * kRowBytes, *vc = v_cache + (size_t)bh * cap * kRowBytes;
    for (int r0 = gap; r0 < keep || r0 == gap; r0 += wave) {   // (once at least; every CTA of the cluster as often)
        const int to = r0 + rank * rows, count = max(0, min(rows, keep - to));
        for (int r = tid; r < count; r += kEThreads) {
            const int src = __ldcg(list + to + r);
            s_from[r] = src;
            s_w[r] = w[src];
        }
        __syncthreads();
        for (int i = tid; i < count * kPieces; i += kEThreads) {
            const int r = i / kPieces, c = i - r * kPieces;
            const size_t at = (size_t)s_from[r] * kRowBytes + c * 16;
            cp_async16(buffer + i * 16, kc + at);
            cp_async16(buffer + (rows * kPieces + i) * 16, vc + at);
        }
        cp_async_wait_all();
        meet();
        for (int r = tid; r < count; r += kEThreads) w[to + r] = s_w[r];
        for (int i = tid; i < count * kPieces; i += kEThreads) {
            const size_t at = (size_t)to * kRowBytes + i * 16;
            *reinterpret_cast<uint4 *>(kc + at) = *reinterpret_cast<const uint4 *>(dyn_e + i * 16);
            *reinterpret_cast<uint4 *>(vc + at) = *reinterpret_cast<const uint4 *>(dyn_e + (rows * kPieces + i) * 16);
        }
        if (r0 == gap && rank == 0 && tid == 0) cache_len[bh] = keep;     // (behind the barrier: everyone has read the old one)
        __syncthreads();                          // (the next wave fills the same places)
    }
}

template <int kRowBytes>
cudaError_t launch_evict(void *k_cache, void *v_cache, float *weight, int32_t *cache_len, int cap, int keep, int first, int recent,
                         int32_t *kept, int BH, cudaStream_t st) {
    // Few pairs: a cluster for each, as large as can be resident for all of them with two CTAs per multiprocessor (with 192 KB of
    // rows, one, the sixteenth cluster of eight waits for another's end) and as leaves a CTA some 400 entries; many: four CTAs
    // per multiprocessor.  Half of 8192 entries dropped, cluster / half as many: 48 pairs 55 / 73 us, 100 pairs 104 / 167; of
    // 1638 entries 20 pairs (eight / four) 22 / 16, 48 (four / two) 20 / 20, 100 (two / one) 27 / 31.
    int cluster = BH <= 28 ? 8 : BH <= 66 ? 4 : BH <= 148 ? 2 : 1;
    while (cluster > 1 && cap < 400 * cluster) cluster /= 2;
    const int rows = (cluster > 1 ? 104 : 48) * 1024 / (2 * kRowBytes + 8), bytes = rows * (2 * kRowBytes + 8);
    auto kernel = cap <= 2048 * cluster ? evict_kernel<kRowBytes, 4> : evict_kernel<kRowBytes, 16>;
    cudaError_t e = allow_smem(kernel, 104 * 1024);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(BH * cluster);
    cfg.blockDim = dim3(kEThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, kernel, (uint8_t *)k_cache, (uint8_t *)v_cache, weight, cache_len, cap, keep, first,
                           recent, kept, cluster, rows);
    count_launch();
    return e;
}

}  // namespace

cudaError_t launch_cache_weights(const void *q, const float *lse, const int32_t *visible, const void *k_cache,
                                 const int32_t *cache_len, int cap, float *weight, float scale, Shape s, HeadGroups hg,
                                 bool tensor_cores, cudaStream_t st) {
    if (tensor_cores && hg.G <= 2) {
        if (s.L > 16) return launch_weights_umma(q, lse, visible, k_cache, cache_len, cap, weight, scale, s, hg, st);
#define ARGS q, lse, visible, k_cache, cache_len, cap, weight, scale, s, hg.norm_eps, st
#define BY_NORM(D, G) return hg.norm_eps >= 0.f ? launch_weights_tc<D, G, true>(ARGS) : launch_weights_tc<D, G, false>(ARGS)
        if (s.d == 128) {
            if (hg.G == 2) BY_NORM(128, 2);
            BY_NORM(128, 1);
        }
        if (hg.G == 2) BY_NORM(64, 2);
        BY_NORM(64, 1);
#undef BY_NORM
#undef ARGS
    }
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
#define ARGS k_cache, v_cache, weight, cache_len, cap, keep, first, recent, kept, BH, st
    return row == 512 ? launch_evict<512>(ARGS) : row == 256 ? launch_evict<256>(ARGS) : launch_evict<128>(ARGS);
#undef ARGS
}

}  // namespace natsl
