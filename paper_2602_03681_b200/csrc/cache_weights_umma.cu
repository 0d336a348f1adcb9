// Attention weight of the retained entries for more than 16 query rows (bf16 storage, one or two softmax heads): the transposed
// logits K q^T as tcgen05 MMAs, so that a thread has a key, its sum over the rows needs no neighbour and the key's RMS factor is
// a register.
//
//   weight_j += sum_t sum_s exp2(f_ts k_js.q_ts - l_ts),   f = scale log2(e) (/ RMS(q)), l = lse log2(e)
//
// Bound by memory up to some 64 exponentials a key, then by those: a multiprocessor takes 11 cycles to get a key's 256 bytes and
// one for 16 exponentials.  Two CTAs per multiprocessor, each with 64 rows of q at a time as the B operand and a ring of five
// slices of K (128 keys, 64 columns).  Two groups of four warps take tiles in turns; one warp issues copies, one MMAs.
//
// B200: 64 rows, two heads, 4 x 16 caches of up to 3277 keys 20 to 21 us: of a CTA's 24000 cycles 12300 are the exponentials of its
// multiprocessor, 4000 the start up to the rows' factors.  Against warp-level MMAs with the rows in registers, 64 x 16 caches of
// up to 1638 keys of 128 columns, one head / two normalised: 16 rows 62 / 80 us where those take 59 / 70; 17 rows 62 / 80 and
// 70 / 99, 64 rows 65 / 106 and 92 / 135, 128 rows 107 / 201 and 171 / 258.
#include <algorithm>
#include "common.cuh"
#include "natsl_internal.h"
#include "tc_common.cuh"

namespace natsl {
namespace {

using namespace tc;

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kRows = 64, kKeys = 128, kStages = 5, kSlice = kKeys * 128, kQSlice = kRows * 128;      // (slices: 64 columns)
constexpr int kWorkers = 256, kThreads = kWorkers + 64;

struct Bars {
    uint64_t full[kStages], empty[kStages], q_full, q_empty, s[4], free[4], drain;
    uint32_t tmem;
    int abort[2];
};

__device__ __forceinline__ float square_sum(uint32_t bf16x2, float s) {
    const float lo = __uint_as_float(bf16x2 << 16), hi = __uint_as_float(bf16x2 & 0xffff0000u);
    return fmaf(lo, lo, fmaf(hi, hi, s));
}
// ss[head] += the squares of row r of slice c (rows of 128 bytes, 16-byte pieces swizzled by row).
template <int D, int G> __device__ __forceinline__ void row_squares(const uint8_t *slice, int c, int r, float (&ss)[G]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint4 y = *reinterpret_cast<const uint4 *>(slice + r * 128 + ((i ^ (r & 7)) << 4));
        float &s = ss[(c * 64 + i * 8) / (D / G)];
        s = square_sum(y.x, square_sum(y.y, square_sum(y.z, square_sum(y.w, s))));
    }
}

// withhold (a test's): neither logits nor free places are announced, so that what waits for them gives up.
template <int D, int G, bool kNorm>
__global__ void __launch_bounds__(kThreads, 2)
cache_weights_umma_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                          const float *__restrict__ lse, const int32_t *__restrict__ visible, const int32_t *__restrict__ cache_len,
                          int cap, float *__restrict__ weight, int H, int T, float scale, float norm_eps, int runs, int run,
                          int wait_kcycles, int withhold) {
    constexpr int ds = D / G, kSlices = D / 64, kCols = kRows * G;       // kCols: columns of a tile's logits
    extern __shared__ __align__(1024) uint8_t dyn_u[];    // q, slice by slice; then the ring
    __shared__ Bars bar;
    __shared__ __align__(16) float2 s_row[kCols];         // factor to base-2 logits, log-sum-exp in base 2
    __shared__ __align__(8) int s_vis[kCols];             // keys of the run that the row sees
    __shared__ int s_least[kCols / 32], s_most[kCols / 32];
    const int tid = threadIdx.x, warp = tid >> 5;
    grid_dependency_wait();
    const int bh = blockIdx.x / runs, b = bh / H, h = bh - b * H, n = min(max(cache_len[bh], 0), cap);
    const int from = (blockIdx.x - bh * runs) * run, to = min(n, from + run);
    if (from >= n) return;
    if (warp == kWorkers / 32) {
        if (elect_one()) {
            for (int i = 0; i < kStages; ++i) { mbar_init(&bar.full[i], 1); mbar_init(&bar.empty[i], kNorm ? 129 : 1); }
            for (int i = 0; i < 4; ++i) { mbar_init(&bar.s[i], 1); mbar_init(&bar.free[i], 128); }
            mbar_init(&bar.q_full, 1);
            mbar_init(&bar.q_empty, kNorm ? 1 + kCols : 1);
            mbar_init(&bar.drain, 1);
            bar.abort[0] = 0;
            bar.abort[1] = wait_kcycles;
            fence_mbar_init();
            prefetch_tmap(&map_q);
            prefetch_tmap(&map_k);
        }
        __syncwarp();
        tmem_alloc(&bar.tmem, 256);
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    launch_dependents();
    const uint32_t tmem = bar.tmem;
    volatile int *abort_flag = bar.abort;
    uint8_t *ring = dyn_u + kSlices * kQSlice;
    const int tiles = (to - from + kKeys - 1) / kKeys, chunks = (T + kRows - 1) / kRows;
    // Tiles are counted through the chunks of rows: u = chunk tiles + tile; slice kSlices u + c.
    auto place_of = [](int u) { return (u & 1) * 2 + (G == 1 ? (u >> 1) & 1 : 0); };         // of the logits, 64 columns each
    auto place_phase = [](int u) { return (uint32_t)(G == 1 ? u >> 2 : u >> 1) & 1; };

    if (tid >= kWorkers + 32) {                   // ---- copies ----
        const int nt = (int)uniform((uint32_t)tiles), all = nt * (int)uniform((uint32_t)chunks);
        int i = 0, q = 0;                         // slices and chunks of q asked for
        bool ok = true;
        for (; i < kSlices * all; ++i) {
            const int u = i / kSlices, t = u % nt, s = i % kStages;
            if (t == 0 && i % kSlices == 0) {
                ok = q == 0 || wait_all(&bar.q_empty, (q - 1) & 1, abort_flag);
                if (!ok) break;
                if (elect_one()) {
                    mbar_arrive_expect_tx(&bar.q_full, kSlices * kQSlice);
                    for (int c = 0; c < kSlices; ++c) tma_load_4d(dyn_u + c * kQSlice, &map_q, &bar.q_full, c * 64, h, q * kRows, b);
                }
                ++q;
                __syncwarp();
            }
            ok = i < kStages || wait_all(&bar.empty[s], (i / kStages - 1) & 1, abort_flag);
            if (!ok) break;
            if (elect_one()) {
                mbar_arrive_expect_tx(&bar.full[s], kSlice);
                tma_load_2d(ring + s * kSlice, &map_k, &bar.full[s], i % kSlices * 64, bh * cap + from + t * kKeys);
            }
            __syncwarp();
        }
        // no copy in flight when the CTA retires, whoever has given up
        if (q > 0) mbar_wait_drain(&bar.q_full, (q - 1) & 1);
        for (int e = max(0, i - kStages); e < i; ++e) mbar_wait_drain(&bar.full[e % kStages], (e / kStages) & 1);
    } else if (tid >= kWorkers) {                 // ---- products ----
        constexpr uint32_t idesc = make_idesc(kFmtBF16, kKeys, kRows, false, false);
        const int nt = (int)uniform((uint32_t)tiles), all = nt * (int)uniform((uint32_t)chunks);
        const uint32_t tm = uniform(tmem), aq = uniform(smem_u32(dyn_u));
        bool ok = true;
        for (int u = 0, t = 0, q = 0; ok && u < all; ++u) {
            const int place = place_of(u);
            if (t == 0) ok = wait_all(&bar.q_full, q & 1, abort_flag);
            if (u >= (G == 1 ? 4 : 2)) ok = ok && wait_all(&bar.free[place], place_phase(u) ^ 1, abort_flag);
            tc_fence_after_sync();
#pragma unroll
            for (int c = 0; c < kSlices; ++c) {
                const int i = kSlices * u + c, s = i % kStages;
                ok = ok && wait_all(&bar.full[s], (i / kStages) & 1, abort_flag);
                if (!ok) break;
                const uint32_t ak = uniform(smem_u32(ring + s * kSlice)), ts = tm + 64 * place;
                if (elect_one()) {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        mma_ss(ts + (c * 64 + k * 16) / ds * 64, desc_kmajor(ak + k * 32), desc_kmajor(aq + c * kQSlice + k * 32), idesc,
                               (c * 64 + k * 16) % ds != 0);
                    mma_commit(&bar.empty[s]);
                    if (c == kSlices - 1 && !withhold) mma_commit(&bar.s[place]);
                    if (c == kSlices - 1 && t == nt - 1) mma_commit(&bar.q_empty);
                }
                __syncwarp();
            }
            if (++t == nt) { t = 0; ++q; }
        }
        if (elect_one()) {                        // no MMA in flight when tensor memory goes
            mma_commit(&bar.drain);
            mbar_wait_drain(&bar.drain, 0);
        }
        __syncwarp();
    } else {                                      // ---- the sums ----
        // (Who has given up announces nothing any more: arrivals without the waits between them would let the copies' warp take
        // places for free whose copies are in flight, and arm their barriers a second time.)
        const int g = warp >> 2, r = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        bool ok = true;
        for (int chunk = 0, u0 = 0; chunk < chunks; ++chunk, u0 += tiles) {
            const int t0 = chunk * kRows;
            if (chunk) named_barrier_sync(1, kWorkers);          // (the last rows' factors have been read, their sums written)
            if (tid < kCols) {
                const int s = tid / kRows, t = tid % kRows;
                int vis = 0;
                float l = 0.f, f = scale * kLog2e;
                if (t0 + t < T) {
                    l = lse[((size_t)bh * G + s) * T + t0 + t];
                    vis = visible ? max(min(visible[((size_t)b * T + t0 + t) * H + h], n) - from, 0) : n - from;
                    if (!isfinite(l)) vis = 0;    // (a row that sees nothing)
                }
                if (kNorm) {
                    ok = wait_all(&bar.q_full, chunk & 1, abort_flag) && ok;
                    float ss[G] = {};
#pragma unroll
                    for (int c = 0; c < kSlices; ++c) row_squares<D, G>(dyn_u + c * kQSlice, c, t, ss);
                    f *= rsqrtf(ss[G == 2 ? s : 0] / ds + norm_eps);
                    if (ok) mbar_arrive(&bar.q_empty);
                }
                s_row[tid] = make_float2(f, l * kLog2e);
                s_vis[tid] = vis;
                const int least = __reduce_min_sync(0xffffffffu, vis), most = __reduce_max_sync(0xffffffffu, vis);
                if (tid % 32 == 0) { s_least[tid / 32] = least; s_most[tid / 32] = most; }
            }
            named_barrier_sync(1, kWorkers);
            for (int u = u0; u < u0 + tiles; ++u) {
                if ((u & 1) != g) continue;
                const int first = (u - u0) * kKeys, j = first + r;       // from the run's start
                float *at = weight + (size_t)bh * cap + from + j;
                const bool mine = from + j < to;
                const float was = mine ? *at : 0.f;
                float fk[G];
                if (kNorm) {
                    float ss[G] = {};
#pragma unroll
                    for (int c = 0; c < kSlices; ++c) {
                        const int i = kSlices * u + c;
                        ok = ok && wait_all(&bar.full[i % kStages], (i / kStages) & 1, abort_flag);
                        row_squares<D, G>(ring + i % kStages * kSlice, c, r, ss);
                        if (ok) mbar_arrive(&bar.empty[i % kStages]);
                    }
#pragma unroll
                    for (int s = 0; s < G; ++s) fk[s] = rsqrtf(ss[s] / ds + norm_eps);
                }
                ok = ok && wait_all(&bar.s[place_of(u)], place_phase(u), abort_flag);
                tc_fence_after_sync();
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < G; ++s)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int part = 2 * s + hf;
                        if (s_most[part] <= first) continue;             // (nobody sees them)
                        uint32_t x[32];
                        tmem_ld32(tmem + 64 * (place_of(u) + s) + 32 * hf + lanes, x);
                        tmem_wait_ld();
                        const bool whole = s_least[part] >= first + kKeys;
#pragma unroll
                        for (int c = 0; c < 32; c += 2) {
                            const float4 w = *reinterpret_cast<const float4 *>(&s_row[part * 32 + c]);
                            float z0 = __uint_as_float(x[c]), z1 = __uint_as_float(x[c + 1]);
                            if (kNorm) { z0 *= fk[s]; z1 *= fk[s]; }
                            z0 = fmaf(z0, w.x, -w.y);
                            z1 = fmaf(z1, w.z, -w.w);
                            if (!whole) {
                                const int2 v = *reinterpret_cast<const int2 *>(&s_vis[part * 32 + c]);
                                if (j >= v.x) z0 = -INFINITY;
                                if (j >= v.y) z1 = -INFINITY;
                            }
                            sum[c & 2] += ex2_ftz(z0);
                            sum[(c & 2) + 1] += ex2_ftz(z1);
                        }
                    }
                tc_fence_before_sync();
                if (ok && !withhold) mbar_arrive(&bar.free[place_of(u)]);
                // (no status word: a wait that has run out shows as a NaN)
                if (mine) *at = ok && !abort_flag[0] ? was + ((sum[0] + sum[1]) + (sum[2] + sum[3])) : NAN;
            }
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kWorkers / 32) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, 256);
    }
}

template <int D, int G, bool kNorm>
cudaError_t launch(const CUtensorMap &map_q, const CUtensorMap &map_k, const float *lse, const int32_t *visible,
                   const int32_t *cache_len, int cap, float *weight, float scale, Shape s, float norm_eps, cudaStream_t st) {
    // Runs of 256 to 2048 keys: as short as one resident set of CTAs allows.
    const long long BH = (long long)s.B * s.H, resident = 148 * 2, per = (BH * cap + resident - 1) / resident;
    const int run = (int)std::min<long long>(2048, std::max<long long>(256, (per + kKeys - 1) / kKeys * kKeys));
    const int runs = (cap + run - 1) / run;
    constexpr int kSmem = D / 64 * kQSlice + kStages * kSlice;
    auto kernel = cache_weights_umma_kernel<D, G, kNorm>;
    cudaError_t e = allow_smem(kernel, kSmem);
    if (e != cudaSuccess) return e;
    e = launch_kernel(kernel, dim3((unsigned)(BH * runs)), dim3(kThreads), kSmem, st, true, map_q, map_k, lse, visible, cache_len, cap,
                      weight, s.H, s.L, scale, norm_eps, runs, run, debug_wait_kcycles(),
                      debug_withhold());
    count_launch();
    return e;
}

}  // namespace

cudaError_t launch_weights_umma(const void *q, const float *lse, const int32_t *visible, const void *k_cache,
                                const int32_t *cache_len, int cap, float *weight, float scale, Shape s, HeadGroups hg, cudaStream_t st) {
    CUtensorMap map_q, map_k;
    if (!tch::make_map_blhd(&map_q, q, s.B, s.L, s.H, s.d, kRows) ||
        !tch::make_map_2d(&map_k, k_cache, (uint64_t)s.B * s.H * cap, s.d, kKeys))
        return cudaErrorInvalidValue;
    const bool norm = hg.norm_eps >= 0.f;
    auto run = s.d == 128 ? hg.G == 2 ? norm ? launch<128, 2, true> : launch<128, 2, false> : norm ? launch<128, 1, true> : launch<128, 1, false>
                          : hg.G == 2 ? norm ? launch<64, 2, true> : launch<64, 2, false> : norm ? launch<64, 1, true> : launch<64, 1, false>;
    return run(map_q, map_k, lse, visible, cache_len, cap, weight, scale, s, hg.norm_eps, st);
}

}  // namespace natsl
