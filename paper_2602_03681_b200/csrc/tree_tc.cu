// Tree step on the tensor cores (bf16 storage): the hybrid layer over a tree of up to 64 drafted tokens.  The mathematics is
// tree_simt.cu's.
//
// A CTA has two parts that work side by side and meet at the end.  Some warps read the CTA's share of the cache, in tiles of 64
// keys.  Up to 32 nodes they are half of the warps and use warp-level MMAs: a tree has few query rows
// for a tcgen05 tile of 128, and the call is bound by reading K/V once.  K and V pass in turns through a ring of asynchronous
// copies; the warps share the tile by keys (and, beyond 16 nodes, by two groups of 16), each with its own running maximum and
// sum, so that a key's row leaves shared memory once (twice) whatever the number of nodes, and their results meet at the
// end.  Beyond 32 nodes that arithmetic takes twice the time of the bytes, and tcgen05 takes it over (below).
// A running maximum moves only when a logit exceeds it by 2^8.  Probabilities meet V rounded to bf16 (2^-8 of themselves, V's
// own precision); their sum is taken before the rounding.
//
// The other warps compute the tree's own part, for the CTA's columns: the T x T tables as MMAs; k S0 and q S0 with the fp32
// state as three bf16 terms that together hold all of its 24 bits, so that u, which goes into the state at the commit, is as
// exact as on CUDA cores; the substitution for u in fp32, a thread per column, by blocks of 16 nodes without a look at the
// tree's shape (the table is zero off the path); the read-outs as MMAs again, u and the table as two bf16 terms each (2^-16).
// Zeros in the place of what a node does not see would let an infinity or a NaN through, so values that are not finite take
// a slower way that looks at the paths.
//
// B200 (a range is what several of them gave): one token of 64 x 16 heads over 1638 keys 155 to 166 us (930 MB: 5.6 to 6.0 TB/s,
// 86 to 92 % of a copy's rate); 32 nodes 216 to 236 us (4.1 to 4.5 TB/s: of a CTA's 53000 cycles the last 10000 are the join, which
// no load overlaps but the neighbour CTA's); 64 nodes of 8 x 16 heads over up to 6554 keys 91 to 95 us (161 us with warp-level MMAs;
// with 64 columns 63 to 67, and 100 to 106); 16 nodes of 16 heads 11 us.
#include <algorithm>
#include "tree_common.cuh"

namespace natsl {
namespace {

using namespace tree;

constexpr int kTileKeys = 64;
using tc::ldmatrix_x4;
using tc::ldmatrix_x4_trans;

__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The first sixteen lanes give the rows: two 8x8 matrices, transposed.
__device__ __forceinline__ void ldmatrix_x2_trans(uint32_t saddr, uint32_t (&r)[2]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(saddr) : "memory");
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
    using S = Sums<2, kRows>;
    using N = Nodes<2, kRows>;
    // Two CTAs of 8 warps per multiprocessor, or one of 16: half of a CTA's warps read the cache, each 16 rows and a share of the
    // tile's keys.  Beyond 32 nodes the cache's products are tcgen05 MMAs: four warps of softmax and four that issue
    // the copies of K and V and the two products, beside eight for the tree's own part.  (The same for 17 to 32 nodes, with one
    // softmax warp a CTA: 224 us for 64 x 16 heads over 1638 keys, where warp-level MMAs take 216.)
    static constexpr bool kUmma = R == 4;
    static constexpr int kCtas = R == 4 ? 1 : 2, kWarps = R == 4 ? 8 : 4;      // kWarps: of the tree's part
    static constexpr int kHalf = 32 * kWarps, kReaders = kUmma ? 256 : kHalf, kThreads = kReaders + kHalf;
    static constexpr int kKeyGroups = kUmma ? 2 : kWarps / R, kWarpKeys = kTileKeys / kKeyGroups;
    static constexpr int kRowBytes = D * 2, kTileBytes = kTileKeys * kRowBytes;
    static constexpr int kSlots = kUmma ? D == 128 ? 7 : 12 : D == 128 ? 4 : 6;
    static constexpr int kAccPitch = D + 4;
    static constexpr int kCols = D / 2;                      // columns of a CTA, at most
    static constexpr int kPitch = kRowBytes + 16;            // (an odd number of 16-byte pieces: eight rows, eight banks)
    static constexpr int kPitchV = kCols * 2 + 16;
    static constexpr int oK = sizeof(S), oV = oK + kRows * kPitch;
    // q: padded rows, or an MMA operand: 64 columns after another, rows of 128 bytes, 16-byte pieces swizzled by row
    static constexpr int oQ = (oV + kRows * kPitchV + (kUmma ? 1023 : 15)) / (kUmma ? 1024 : 16) * (kUmma ? 1024 : 16);
    static constexpr int oTab = oQ + kRows * (kUmma ? kRowBytes : kPitch);
    __host__ __device__ static constexpr int q_piece(int t, int c) {         // of piece c of row t, from oQ
        return kUmma ? (c >> 3) * (kRows * 128) + t * 128 + (((c & 7) ^ (t & 7)) << 4) : t * kPitch + c * 16;
    }
    // u and the linear read-out of the CTA's columns (the sums over the tree's V: over k); the probabilities over the tree, bf16
    static constexpr int oU = oTab + kRows * kRows * 4, oO = oU + kRows * kCols * 4, oP = oO + kRows * kCols * 4;
    static constexpr int kPitchP = kRows * 2 + 16;
    // the ring (16-byte pieces swizzled by row); at the end the key groups' results, the first one's place the CTA's
    static constexpr int oRing = (oP + kRows * kPitchP + 1023) / 1024 * 1024, kRing = kSlots * kTileBytes;
    static constexpr int kMerge = kKeyGroups * kRows * kAccPitch * 4;
    static_assert(kMerge <= kRing, "the key groups' results lie in the ring");
    static constexpr int kTotal = oRing + kRing;
    static_assert(!kUmma || kTotal + 9216 <= 232448, "a multiprocessor's shared memory, with the static part");
};

// The CTA's share of the cache: units 0, 1, 2, ... are K of tile 0, V of tile 0, K of tile 1, ...
template <int D, int R> struct Stream {
    using L = Layout<D, R>;
    static constexpr int kPieces = L::kRowBytes / 16, kStep = L::kHalf / kPieces;
    const uint8_t *kc, *vc;
    uint32_t ring, dst0;
    int row0, from, to, units;
    __device__ Stream(const Args &a, uint8_t *sm, int bh, int tid, const Share &c) {
        const int piece = tid % kPieces;          // thread = 16-byte piece of every kStep-th row of a tile
        row0 = tid / kPieces;
        kc = reinterpret_cast<const uint8_t *>(a.k_cache) + (size_t)bh * a.cap * L::kRowBytes + piece * 16;
        vc = reinterpret_cast<const uint8_t *>(a.v_cache) + (size_t)bh * a.cap * L::kRowBytes + piece * 16;
        ring = tc::smem_u32(sm + L::oRing);
        dst0 = row0 * L::kRowBytes + ((piece ^ (row0 & 7)) << 4);
        from = c.from;
        to = c.to;
        units = (c.to - c.from + kTileKeys - 1) / kTileKeys * 2;
    }
    __device__ uint32_t slot(int u) const { return ring + u % L::kSlots * L::kTileBytes; }
    __device__ void fetch(int u) const {
        if (u < units) {
            const uint32_t at = slot(u) + dst0;
            const uint8_t *src = u & 1 ? vc : kc;
#pragma unroll
            for (int i = 0; i < kTileKeys / kStep; ++i) {
                const int j = from + (u >> 1) * kTileKeys + row0 + i * kStep;
                const bool in = j < to;           // rows past the end count as zeros: what lies there may be anything
                cp_async16(at + i * kStep * L::kRowBytes, src + (size_t)(in ? j : from) * L::kRowBytes, in);
            }
        }
        cp_async_commit();
    }
};

// The key groups' results -> the CTA's.  group_m, group_z [G][key groups][rows]; acc [key groups][rows][pitch], the result in the
// first one's place.
template <int D, int G, int R>
__device__ __forceinline__ void merge_groups(typename Layout<D, R>::S *sums, float *acc, const float *group_m, const float *group_z,
                                             int n_nodes, int tid, int threads) {
    using L = Layout<D, R>;
    for (int i = tid; i < n_nodes * (D / 4); i += threads) {
        const int t = i / (D / 4), x = (i - t * (D / 4)) * 4, s = x / (D / G);
        float M = -INFINITY;
#pragma unroll
        for (int k = 0; k < L::kKeyGroups; ++k) M = fmaxf(M, group_m[(s * L::kKeyGroups + k) * L::kRows + t]);
        const float mu = M == -INFINITY ? 0.f : M;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        float Z = 0.f;
#pragma unroll
        for (int k = 0; k < L::kKeyGroups; ++k) {
            const int at = (s * L::kKeyGroups + k) * L::kRows + t;
            const float e = tc::ex2_ftz(group_m[at] - mu);
            const float4 w = *reinterpret_cast<const float4 *>(acc + (k * L::kRows + t) * L::kAccPitch + x);
            Z = fmaf(group_z[at], e, Z);
            y.x = fmaf(w.x, e, y.x); y.y = fmaf(w.y, e, y.y);
            y.z = fmaf(w.z, e, y.z); y.w = fmaf(w.w, e, y.w);
        }
        *reinterpret_cast<float4 *>(acc + t * L::kAccPitch + x) = y;
        if (x % (D / G) == 0) { sums->cache_m[s][t] = M; sums->cache_z[s][t] = Z; }
    }
}

template <int D, int G, bool kNorm, int R>
__device__ void cache_part(const Args &a, typename Layout<D, R>::S *sums, uint8_t *sm, const Stream<D, R> &in, int n_nodes) {
    using L = Layout<D, R>;
    constexpr int ds = D / G, kNt = L::kWarpKeys / 8, kKs = ds / 16, kHalf = L::kHalf;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, c4 = lane & 3;
    const int rg = warp / L::kKeyGroups, kg = warp - rg * L::kKeyGroups, r0 = rg * 16;
    const uint32_t q_at = tc::smem_u32(sm + L::oQ) ;
    auto load_q = [&](int k, uint32_t (&x)[4]) { ldmatrix_x4(q_at + L::q_piece(r0 + (lane & 15), 2 * k + (lane >> 4)), x); };

    // each row's factor to base-2 logits
    float f[2][kNorm ? G : 1];
    f[0][0] = f[1][0] = a.scale_sm * kLog2e;
    if (kNorm) {
#pragma unroll
        for (int s = 0; s < G; ++s) {
            float ss[2] = {0.f, 0.f};
#pragma unroll
            for (int k = s * kKs; k < (s + 1) * kKs; ++k) {
                uint32_t x[4];
                load_q(k, x);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 y = bf2(x[i]);
                    ss[i & 1] = fmaf(y.x, y.x, fmaf(y.y, y.y, ss[i & 1]));
                }
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                ss[r] += __shfl_xor_sync(0xffffffffu, ss[r], 1);
                ss[r] += __shfl_xor_sync(0xffffffffu, ss[r], 2);
                f[r][s] = a.scale_sm * kLog2e * rsqrtf(ss[r] / ds + a.norm_eps);
            }
        }
    }
    float o[D / 8][4], mx[G][2], z[G][2];
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
        for (int x = 0; x < 4; ++x) o[i][x] = 0.f;
#pragma unroll
    for (int s = 0; s < G; ++s)
#pragma unroll
        for (int r = 0; r < 2; ++r) { mx[s][r] = -INFINITY; z[s][r] = 0.f; }
    const int key0 = kg * L::kWarpKeys;
    uint32_t pf[G][kNt / 2][4];
    auto turn = [&](int u) {                      // unit u is there, and every warp is done with unit u - 1 ...
        cp_async_wait<L::kSlots - 2>();
        tc::named_barrier_sync(1, kHalf);
        in.fetch(u + L::kSlots - 1);              // ... whose place this one takes
    };
    for (int u = 0; u < in.units; u += 2) {
        const int left = in.to - in.from - (u >> 1) * kTileKeys - key0;      // of the warp's keys
        turn(u);
        if (left > 0) {
            const uint32_t kt = in.slot(u);
#pragma unroll
            for (int s = 0; s < G; ++s) {
                float x[kNt][4], kk[kNt];
#pragma unroll
                for (int i = 0; i < kNt; ++i) {
                    kk[i] = 0.f;
#pragma unroll
                    for (int y = 0; y < 4; ++y) x[i][y] = 0.f;
                }
#pragma unroll
                for (int k = s * kKs; k < (s + 1) * kKs; ++k) {
                    uint32_t qf[4];
                    load_q(k, qf);
#pragma unroll
                    for (int i = 0; i < kNt; i += 2) {
                        const int row = key0 + i * 8 + (lane & 7) + (lane >> 4) * 8;
                        uint32_t bf[4];
                        ldmatrix_x4(kt + row * L::kRowBytes + (((2 * k + ((lane >> 3) & 1)) ^ (row & 7)) << 4), bf);
                        mma_bf16(x[i], qf, bf[0], bf[1]);
                        mma_bf16(x[i + 1], qf, bf[2], bf[3]);
                        if (kNorm) {              // the key's sum of squares rides along
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
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float fr = f[r][kNorm ? s : 0];
                        x[i][2 * r] *= fr * w0;
                        x[i][2 * r + 1] *= fr * w1;
                    }
                }
                if (left < L::kWarpKeys) {
#pragma unroll
                    for (int i = 0; i < kNt; ++i)
#pragma unroll
                        for (int y = 0; y < 4; ++y)
                            if (i * 8 + 2 * c4 + (y & 1) >= left) x[i][y] = -INFINITY;
                }
                bool raise = false;
                float top[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float y = x[0][2 * r];
#pragma unroll
                    for (int i = 0; i < kNt; ++i) y = tc::max3(y, x[i][2 * r], x[i][2 * r + 1]);
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 1));
                    top[r] = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 2));
                    raise |= top[r] > mx[s][r] + 8.f;
                }
                if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float m1 = fmaxf(mx[s][r], top[r]);
                        const float e = mx[s][r] == m1 ? 1.f : tc::ex2_ftz(mx[s][r] - m1);
                        mx[s][r] = m1;
                        z[s][r] *= e;
#pragma unroll
                        for (int i = s * ds / 8; i < (s + 1) * ds / 8; ++i) {
                            o[i][2 * r] *= e;
                            o[i][2 * r + 1] *= e;
                        }
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float mu = mx[s][r] == -INFINITY ? 0.f : mx[s][r];
#pragma unroll
                    for (int i = 0; i < kNt; ++i) {
                        const float p0 = tc::ex2_ftz(x[i][2 * r] - mu), p1 = tc::ex2_ftz(x[i][2 * r + 1] - mu);
                        z[s][r] += p0 + p1;
                        pf[s][i / 2][(i & 1) * 2 + r] = tc::pack_bf162(p0, p1);
                    }
                }
            }
        }
        turn(u + 1);
        if (left > 0) {
            const uint32_t vt = in.slot(u + 1);
#pragma unroll
            for (int i = 0; i < kNt / 2; ++i) {
                const int row = key0 + i * 16 + (lane & 15);
#pragma unroll
                for (int n = 0; n < D / 16; ++n) {
                    uint32_t bf[4];
                    ldmatrix_x4_trans(vt + row * L::kRowBytes + (((2 * n + (lane >> 4)) ^ (row & 7)) << 4), bf);
                    mma_bf16(o[2 * n], pf[n * 16 / ds][i], bf[0], bf[1]);
                    mma_bf16(o[2 * n + 1], pf[n * 16 / ds][i], bf[2], bf[3]);
                }
            }
        }
    }
    // the key groups' results -> the CTA's
    __shared__ float s_m[G][L::kKeyGroups][L::kRows], s_z[G][L::kKeyGroups][L::kRows];
    cp_async_wait<0>();
    tc::named_barrier_sync(1, kHalf);
    float *acc = reinterpret_cast<float *>(sm + L::oRing);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int t = r0 + r * 8 + g4;
        float *to = acc + (kg * L::kRows + t) * L::kAccPitch + 2 * c4;
#pragma unroll
        for (int i = 0; i < D / 8; ++i) *reinterpret_cast<float2 *>(to + 8 * i) = make_float2(o[i][2 * r], o[i][2 * r + 1]);
#pragma unroll
        for (int s = 0; s < G; ++s) {
            float y = z[s][r];
            y += __shfl_xor_sync(0xffffffffu, y, 1);
            y += __shfl_xor_sync(0xffffffffu, y, 2);
            if (c4 == 0) { s_m[s][kg][t] = mx[s][r]; s_z[s][kg][t] = y; }
        }
    }
    tc::named_barrier_sync(1, kHalf);
    merge_groups<D, G, R>(sums, acc, &s_m[0][0][0], &s_z[0][0][0], n_nodes, tid, kHalf);
}

// ------------------------------------------------------------------------------------------
// The CTA's share of the cache with tcgen05 (33 to 64 nodes).  An MMA has 128 rows: the even tiles' logits use rows
// 0 .. 63 of it, the odd ones' 64 .. 127 -- the operand is q behind, or ahead of, whatever shared memory holds there, and what the
// other rows get is never looked at -- so that all four warps have a row per thread and tiles of their own, two key groups with a
// running maximum each.  Probabilities take the logits' place in tensor memory as the second product's operand.  Per tile the
// MMAs take 256 cycles; with warp-level MMAs a tile of 64 rows took 2900, twice the time that its bytes need.
// ------------------------------------------------------------------------------------------
struct UmmaBars {
    uint64_t full[2][6], empty[2][6];             // [K, V][stage]
    uint64_t s[4], p[4], o[4], drain[2];          // per place of logits: logits there, probabilities there, product done
    uint32_t tmem;
    int abort[2];
};
constexpr int kTmemCols = 512, kTmemO = 256;      // logits: four places of 64 columns; then the two groups' sums

template <int D> struct UmmaShare {
    using L = Layout<D, 4>;
    static constexpr int kStagesV = L::kSlots / 2, kStagesK = L::kSlots - kStagesV;      // (K is read twice if normalised)
    static constexpr int kSlices = D / 64, kSlice = kTileKeys * 128;                     // of 64 columns
    static_assert(kStagesK <= 6, "");
    const CUtensorMap *map[2];
    UmmaBars *bar;
    uint8_t *sm, *ring;
    int row, keys, tiles;                         // first row, keys, tiles of the share
    static __device__ constexpr int stages(int kv) { return kv ? kStagesV : kStagesK; }
    __device__ int stage(int kv, int t) const { return kv ? t % kStagesV : t % kStagesK; }
    __device__ uint32_t phase(int kv, int t) const { return (kv ? t / kStagesV : t / kStagesK) & 1; }
    __device__ uint8_t *at(int kv, int t) const { return ring + (kv * kStagesK + stage(kv, t)) * L::kTileBytes; }
};
// A head's sums: with 64 columns and two heads both get all columns (an operand of 32 would start inside the swizzle).
template <int D, int G> struct UmmaSums {
    static constexpr int kCols = D == 128 ? 128 / G : 64;
    static __device__ constexpr int at(int s) { return kCols * s + (D == 128 ? 0 : s * (D / G)); }       // of its own columns
};

__device__ __forceinline__ void umma_init(UmmaBars *bar, bool norm, int wait_kcycles) {      // (one thread)
    for (int s = 0; s < 6; ++s)
        for (int kv = 0; kv < 2; ++kv) { tc::mbar_init(&bar->full[kv][s], 1); tc::mbar_init(&bar->empty[kv][s], kv == 0 && norm ? 65 : 1); }
    for (int s = 0; s < 4; ++s) {
        tc::mbar_init(&bar->s[s], 1);
        tc::mbar_init(&bar->p[s], 64);
        tc::mbar_init(&bar->o[s], 1);
    }
    for (int i = 0; i < 2; ++i) tc::mbar_init(&bar->drain[i], 1);
    bar->abort[0] = 0;
    bar->abort[1] = wait_kcycles;
    tc::fence_mbar_init();
}
// Places of a tile's logits: with one softmax head two per group, in turns; with two, one for each.
template <int G> __device__ __forceinline__ int place_of(int t) { return (t & 1) * 2 + (G == 1 ? (t >> 1) & 1 : 0); }
template <int G> __device__ __forceinline__ uint32_t place_phase(int t) { return (G == 1 ? t >> 2 : t >> 1) & 1; }

// The issuing warps.  One that did all four took 2600 cycles a tile, half of them for issuing itself: 145 us where four take 92.
// Copies of K (0) or V (1).
template <int D> __device__ void umma_load(const UmmaShare<D> &in, int kv) {
    using namespace tc;
    UmmaBars *bar = in.bar;
    const int tiles = (int)uniform((uint32_t)in.tiles), stages = in.stages(kv);
    int t = 0;
    for (; t < tiles; ++t) {
        const int s = in.stage(kv, t);
        if (t >= stages && !wait_all(&bar->empty[kv][s], in.phase(kv, t) ^ 1, bar->abort)) break;
        if (elect_one()) {
            mbar_arrive_expect_tx(&bar->full[kv][s], UmmaShare<D>::L::kTileBytes);
            for (int c = 0; c < in.kSlices; ++c) tma_load_2d(in.at(kv, t) + c * in.kSlice, in.map[kv], &bar->full[kv][s], c * 64, in.row + t * kTileKeys);
        }
        __syncwarp();
    }
    // no copy in flight when the CTA retires, whoever has given up
    for (int i = max(0, t - stages); i < t; ++i) mbar_wait_drain(&bar->full[kv][in.stage(kv, i)], in.phase(kv, i));
}

__device__ __forceinline__ void umma_drain(uint64_t *bar) {              // nor an MMA
    if (tc::elect_one()) {
        tc::mma_commit(bar);
        tc::mbar_wait_drain(bar, 0);
    }
    __syncwarp();
}

// Logits = q K^T into a tile's place, once the product that read the probabilities of the place's last tile is done.
template <int D, int G>
__device__ void umma_logits(const UmmaShare<D> &in, uint32_t tmem, uint32_t q_at) {
    using namespace tc;
    UmmaBars *bar = in.bar;
    constexpr uint32_t idesc = make_idesc(kFmtBF16, 128, kTileKeys, false, false);
    const int tiles = (int)uniform((uint32_t)in.tiles);
    const uint32_t tm = uniform(tmem), aq = uniform(q_at);
    bool ok = true;
    for (int t = 0; ok && t < tiles; ++t) {
        const int place = place_of<G>(t);
        if (t >= (G == 1 ? 4 : 2)) ok = wait_all(&bar->o[place], place_phase<G>(t) ^ 1, bar->abort);
        ok = ok && wait_all(&bar->full[0][in.stage(0, t)], in.phase(0, t), bar->abort);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t ak = uniform(smem_u32(in.at(0, t))), a0 = aq - (t & 1) * (64 * 128), ts = tm + 64 * place;
        if (elect_one()) {
#pragma unroll
            for (int c = 0; c < in.kSlices; ++c)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_ss(ts + (c * 64 + k * 16) / (D / G) * 64, desc_kmajor(a0 + c * (64 * 128) + k * 32), desc_kmajor(ak + c * in.kSlice + k * 32),
                           idesc, (c * 64 + k * 16) % (D / G) != 0);
            mma_commit(&bar->s[place]);
            mma_commit(&bar->empty[0][in.stage(0, t)]);
        }
        __syncwarp();
    }
    umma_drain(&bar->drain[0]);
}

// The group's sums += probabilities V.
template <int D, int G>
__device__ void umma_sums(const UmmaShare<D> &in, uint32_t tmem) {
    using namespace tc;
    UmmaBars *bar = in.bar;
    constexpr int kCols = UmmaSums<D, G>::kCols;
    constexpr uint32_t idesc = make_idesc(kFmtBF16, 128, kCols, false, true);
    const int tiles = (int)uniform((uint32_t)in.tiles);
    const uint32_t tm = uniform(tmem);
    bool ok = true;
    for (int t = 0; ok && t < tiles; ++t) {
        const int place = place_of<G>(t);
        ok = wait_all(&bar->full[1][in.stage(1, t)], in.phase(1, t), bar->abort) && wait_all(&bar->p[place], place_phase<G>(t), bar->abort);
        if (!ok) break;
        // Rows past the end count as zeros: what lies there may be anything.  (This warp follows every phase of V's barriers.  The
        // softmax warps, which do not, are up to four tiles ahead with one softmax head, V has three places at 128 columns: to
        // them the barrier's last phase but one looks like the one to come, and they cleared rows of a tile on its way.)
        const int left = in.keys - t * kTileKeys;
        if (left < kTileKeys) {
            uint8_t *tile = in.at(1, t);
            for (int e = threadIdx.x & 31; e < (kTileKeys - left) * (D / 8); e += 32) {
                const int c = e % (D / 8), j = left + e / (D / 8);
                *reinterpret_cast<uint4 *>(tile + c / 8 * in.kSlice + j * 128 + c % 8 * 16) = make_uint4(0, 0, 0, 0);
            }
            fence_proxy_async_smem();
            __syncwarp();
        }
        tc_fence_after_sync();
        const uint32_t av = uniform(smem_u32(in.at(1, t))), ts = tm + 64 * place, to = tm + kTmemO + 128 * (t & 1);
        if (elect_one()) {
#pragma unroll
            for (int s = 0; s < G; ++s)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    mma_ts(to + kCols * s, ts + 64 * s + k * 8, desc_mnmajor(av + (D == 128 ? s * in.kSlice : 0) + k * 2048, in.kSlice), idesc,
                           t > 1 || k != 0);
            mma_commit(&bar->o[place]);
            mma_commit(&bar->empty[1][in.stage(1, t)]);
        }
        __syncwarp();
    }
    umma_drain(&bar->drain[1]);
}

// The four softmax warps: thread = row of a key group.  withhold (a test's): no tile's probabilities are announced, so that
// what waits for them gives up.
template <int D, int G, bool kNorm>
__device__ void umma_softmax(const Args &a, typename Layout<D, 4>::S *sums, const UmmaShare<D> &in, uint32_t tmem, int n_nodes, bool withhold) {
    using namespace tc;
    using L = Layout<D, 4>;
    constexpr int ds = D / G, kSlices = D / 64;
    __shared__ float s_m[G][2][64], s_z[G][2][64];
    __shared__ __align__(16) float s_rk[kNorm ? 2 : 1][2][G][64];      // [group][in turns]: the keys' RMS factors
    UmmaBars *bar = in.bar;
    volatile int *abort_flag = bar->abort;
    const int tid = threadIdx.x, warp = tid >> 5, g = warp >> 1, r = tid & 63;
    const uint32_t lanes = (uint32_t)(warp * 32) << 16, to = tmem + kTmemO + 128 * g + lanes;
    auto row_squares = [&](const uint8_t *slice, int x, int row, float (&ss)[G]) {       // += those of slice x
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            const uint4 y = *reinterpret_cast<const uint4 *>(slice + row * 128 + ((c ^ (row & 7)) << 4));
            const float2 y0 = bf2(y.x), y1 = bf2(y.y), y2 = bf2(y.z), y3 = bf2(y.w);
            ss[(x * 64 + c * 8) / ds] += y0.x * y0.x + y0.y * y0.y + y1.x * y1.x + y1.y * y1.y + y2.x * y2.x + y2.y * y2.y + y3.x * y3.x + y3.y * y3.y;
        }
    };
    float f[G], m[G], z[G];
    {
        float ss[G] = {};
        if (kNorm)
#pragma unroll
            for (int c = 0; c < kSlices; ++c) row_squares(in.sm + L::oQ + c * (64 * 128), c, r, ss);
#pragma unroll
        for (int s = 0; s < G; ++s) {
            f[s] = a.scale_sm * kLog2e;
            if (kNorm) f[s] *= rsqrtf(ss[s] / ds + a.norm_eps);
            m[s] = -INFINITY;
            z[s] = 0.f;
        }
    }
    bool ok = true;
    int i = 0;                                    // the group's tiles so far
    for (int t = g; t < in.tiles; t += 2, ++i) {
        const int left = in.keys - t * kTileKeys;
        ok = ok && wait_all(&bar->s[place_of<G>(t)], place_phase<G>(t), abort_flag);
        if (kNorm) {                              // (the barrier below is everyone's, however the waits end)
            ok = ok && wait_all(&bar->full[0][in.stage(0, t)], in.phase(0, t), abort_flag);
            if (ok) {
                float ss[G] = {};
#pragma unroll
                for (int c = 0; c < kSlices; ++c) row_squares(in.at(0, t) + c * in.kSlice, c, r, ss);
#pragma unroll
                for (int s = 0; s < G; ++s) s_rk[g][i & 1][s][r] = rsqrtf(ss[s] / ds + a.norm_eps);
                mbar_arrive(&bar->empty[0][in.stage(0, t)]);
            }
            named_barrier_sync(3 + g, 64);
        }
        if (!ok) continue;
        tc_fence_after_sync();
#pragma unroll
        for (int s = 0; s < G; ++s) {
            const uint32_t ts = tmem + 64 * (place_of<G>(t) + s) + lanes;
            float x[2][32];
            float top = -INFINITY;
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                tmem_ld32(ts + 32 * hf, reinterpret_cast<uint32_t(&)[32]>(x[hf]));
                tmem_wait_ld();
#pragma unroll
                for (int c = 0; c < 32; c += 4) {
                    float4 w = make_float4(1.f, 1.f, 1.f, 1.f);
                    if (kNorm) w = *reinterpret_cast<const float4 *>(&s_rk[g][i & 1][s][32 * hf + c]);
                    x[hf][c] *= f[s] * w.x; x[hf][c + 1] *= f[s] * w.y;
                    x[hf][c + 2] *= f[s] * w.z; x[hf][c + 3] *= f[s] * w.w;
                }
                if (left < kTileKeys) {
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (32 * hf + c >= left) x[hf][c] = -INFINITY;
                }
                float m4[4] = {x[hf][0], x[hf][1], x[hf][2], x[hf][3]};
#pragma unroll
                for (int c = 4; c < 28; c += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) m4[e] = max3(m4[e], x[hf][c + e], x[hf][c + 4 + e]);
#pragma unroll
                for (int e = 0; e < 4; ++e) top = max3(top, m4[e], x[hf][28 + e]);
            }
            const float m_old = m[s];
            if (top > m_old + 8.f) m[s] = fmaxf(m_old, top);
            const float mu = m[s] == -INFINITY ? 0.f : m[s], e = m[s] == m_old ? 1.f : ex2_ftz(m_old - mu);
            uint32_t p[32];
            float z2[2] = {0.f, 0.f};
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
#pragma unroll
                for (int c = 0; c < 32; c += 2) {
                    const float p0 = ex2_ftz(x[hf][c] - mu), p1 = ex2_ftz(x[hf][c + 1] - mu);
                    z2[hf] += p0 + p1;
                    p[16 * hf + c / 2] = pack_bf162(p0, p1);
                }
            z[s] = fmaf(z[s], e, z2[0] + z2[1]);
            tmem_st32(ts, p);
            if (i > 0 && __any_sync(0xffffffffu, e != 1.f)) {
                ok = wait_all(&bar->o[place_of<G>(t - 2)], place_phase<G>(t - 2), abort_flag);
                if (ok) {
                    tc_fence_after_sync();
#pragma unroll 1
                    for (int c = 0; c < ds; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(to + UmmaSums<D, G>::at(s) + c, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int y = 0; y < 32; ++y) o[y] = __float_as_uint(__uint_as_float(o[y]) * e);
                        tmem_st32(to + UmmaSums<D, G>::at(s) + c, o);
                    }
                }
            }
        }
        tmem_wait_st();
        tc_fence_before_sync();
        if (ok && !withhold) mbar_arrive(&bar->p[place_of<G>(t)]);
    }
    const int t_last = g + 2 * (i - 1);           // (products are done in their order)
    if (ok && i > 0) ok = wait_all(&bar->o[place_of<G>(t_last)], place_phase<G>(t_last), abort_flag);
    tc_fence_after_sync();
    named_barrier_sync(1, 128);                   // (both groups' tiles have been read: the ring is free)
    float *acc = reinterpret_cast<float *>(in.ring), *mine = acc + (g * 64 + r) * L::kAccPitch;
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        if (i > 0) {                              // (uniform)
            tmem_ld32(to + UmmaSums<D, G>::at(c / ds) + c % ds, o);
            tmem_wait_ld();
        } else {
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = 0u;
        }
#pragma unroll
        for (int y = 0; y < 32; y += 4) *reinterpret_cast<uint4 *>(mine + c + y) = make_uint4(o[y], o[y + 1], o[y + 2], o[y + 3]);
    }
    tc_fence_before_sync();
    named_barrier_arrive(5, 192);                 // (an issuing warp gives tensor memory back)
#pragma unroll
    for (int s = 0; s < G; ++s) { s_m[s][g][r] = m[s]; s_z[s][g][r] = z[s]; }
    named_barrier_sync(1, 128);
    merge_groups<D, G, 4>(sums, acc, &s_m[0][0][0], &s_z[0][0][0], n_nodes, tid, 128);
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

// ... and as two (2^-16 of x is left over).
__device__ __forceinline__ void split2(float x0, float x1, uint32_t (&t)[2]) {
    t[0] = tc::pack_bf162(x0, x1);
    const float2 y = bf2(t[0]);
    t[1] = tc::pack_bf162(x0 - y.x, x1 - y.y);
}
__device__ __forceinline__ bool finite(float x) { return fabsf(x) <= 3.402823466e38f; }
__device__ __forceinline__ bool finite_bf16x2(uint32_t x) { return (x & 0x7f80u) != 0x7f80u && (x & 0x7f800000u) != 0x7f800000u; }

// The tree's own part, for columns c0 .. c0 + cols - 1 (cols = D / cluster).  q, k and the columns of v are in shared memory;
// odd: a value of those is not finite.
template <int D, int G, bool kNorm, int R>
__device__ void tree_part(const Args &a, typename Layout<D, R>::S *sums, uint8_t *sm, typename Layout<D, R>::N *nd, int b, int h, int n,
                          int rank, bool odd, const NodeRow &node) {
    using L = Layout<D, R>;
    constexpr int ds = D / G, kRows = L::kRows, kNt = 2 * R, kKs = D / 16, kPieces = L::kRowBytes / 16, kHalf = L::kHalf, kWarps = L::kWarps;
    const int tid = threadIdx.x - L::kReaders, warp = tid >> 5, lane = tid & 31, g4 = lane >> 2, c4 = lane & 3, T = a.T;
    const int bh = b * a.H + h, cols = D / a.cluster, c0 = rank * cols, sc = c0 / ds;   // sc: the columns' softmax head
    auto sync = [] { tc::named_barrier_sync(2, kHalf); };
    float *tab = reinterpret_cast<float *>(sm + L::oTab);    // [j][i], i > j: what u_i takes from u_j
    float *su = reinterpret_cast<float *>(sm + L::oU), *so = reinterpret_cast<float *>(sm + L::oO);
    float *st = reinterpret_cast<float *>(sm + L::oK);       // (over k)

    // A tile of eight state columns as the B fragments of all products with it: rows 2 c4, + 1, + 8, + 9 of a step of 16.
    __shared__ int s_odd;
    if (tid == 0) s_odd = 0;
    const float *S = a.state + (size_t)bh * D * D + c0 + g4;
    auto load = [&](int tile, int k, float (&y)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __ldg(S + (size_t)(16 * k + 2 * c4 + (i & 1) + (i >> 1) * 8) * D + tile * 8);
    };
    const int tiles = cols / 8, tile0 = warp < R ? tiles : kWarps - 1 - warp;       // (the first R warps have the tables)
    constexpr int kStride = kWarps - R;
    float s[kKs][4];
    if (tile0 < tiles)
#pragma unroll
        for (int k = 0; k < kKs; ++k) load(tile0, k, s[k]);
    if (kNorm && tid < 2 * kRows) {               // a row's norms, thread = row of q or k
        const int t = tid % kRows;
        const bool is_k = tid >= kRows;
        float all = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float ss = 0.f;
#pragma unroll
            for (int c = g * kPieces / G; c < (g + 1) * kPieces / G; ++c) {
                const uint4 y = *reinterpret_cast<const uint4 *>(is_k ? sm + L::oK + t * L::kPitch + c * 16 : sm + L::oQ + L::q_piece(t, c));
                const float2 y0 = bf2(y.x), y1 = bf2(y.y), y2 = bf2(y.z), y3 = bf2(y.w);
                ss += y0.x * y0.x + y0.y * y0.y + y1.x * y1.x + y1.y * y1.y + y2.x * y2.x + y2.y * y2.y + y3.x * y3.x + y3.y * y3.y;
            }
            (is_k ? nd->rk_sm : nd->rq_sm)[g][t] = rsqrtf(ss / ds + a.norm_eps);
            all += ss;
        }
        (is_k ? nd->rk_la : nd->rq_la)[t] = rsqrtf(all + a.norm_eps);
    }
    walk_nodes(a, b, h, n, tid, node, nd, sync);
    sync();
    auto rq_la = [&](int t) { return kNorm ? nd->rq_la[t] : 1.f; };
    auto rk_la = [&](int t) { return kNorm ? nd->rk_la[t] : 1.f; };
    const uint32_t q_at = tc::smem_u32(sm + L::oQ), k_at = tc::smem_u32(sm + L::oK), v_at = tc::smem_u32(sm + L::oV);

    // ---- the tables: the first R warps have 16 rows each, all columns.  What u takes from u and the probabilities go to shared
    // memory; what the read-out takes from u (two terms) stays in registers, as the A fragments of the read-out. ----
    uint32_t bh_f[kNt / 2][4], bl_f[kNt / 2][4];
    auto tables = [&] {
        // bit 8 i + x of a row's words: column 8 i + 2 c4 + x
        const int t0 = warp * 16 + g4, sh = G > 1 ? sc : 0;
        unsigned fold[2][2], seen[2][2];
        float bt[2], fq[2], f[2], m[2] = {-INFINITY, -INFINITY}, z[2] = {0.f, 0.f};
        float2 total[2];
        int wipes[2];
        float y[kNt][4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int t = t0 + 8 * r;
            const unsigned long long path = t < n ? nd->above[t] | 1ull << t : 0ull;
            const unsigned long long pf = (path & nd->fold) >> (2 * c4), ps = (path & nd->keep) >> (2 * c4);
            fold[r][0] = (unsigned)pf; fold[r][1] = (unsigned)(pf >> 32);
            seen[r][0] = (unsigned)ps; seen[r][1] = (unsigned)(ps >> 32);
            bt[r] = nd->beta[t] * rk_la(t);
            fq[r] = a.scale_la * rq_la(t);
            f[r] = a.scale_sm * kLog2e * (kNorm ? nd->rq_sm[sh][t] : 1.f);
            total[r] = nd->total[t];
            wipes[r] = nd->wipes[t];
        }
        constexpr int kPart = 2;                  // (16 columns at a time: registers)
#pragma unroll
        for (int i0 = 0; i0 < kNt; i0 += kPart) {
            float kk[kPart][4], qk[G][kPart][4];
#pragma unroll
            for (int i = 0; i < kPart; ++i)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    kk[i][x] = 0.f;
#pragma unroll
                    for (int g = 0; g < G; ++g) qk[g][i][x] = 0.f;
                }
#pragma unroll
            for (int k = 0; k < kKs; k += 2) {
                uint32_t ak[2][4], aq[2][4], bf[kPart][4];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int t = warp * 16 + (lane & 15), c = 2 * (k + x) + (lane >> 4);
                    ldmatrix_x4(k_at + t * L::kPitch + c * 16, ak[x]);
                    ldmatrix_x4(q_at + L::q_piece(t, c), aq[x]);
                }
#pragma unroll
                for (int i = 0; i < kPart; ++i) ldmatrix_x4(k_at + ((i0 + i) * 8 + (lane & 7)) * L::kPitch + (2 * k + (lane >> 3)) * 16, bf[i]);
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int i = 0; i < kPart; ++i) {
                        mma_bf16(kk[i], ak[x], bf[i][2 * x], bf[i][2 * x + 1]);
                        mma_bf16(qk[k * 16 / ds][i], aq[x], bf[i][2 * x], bf[i][2 * x + 1]);
                    }
            }
#pragma unroll
            for (int i = 0; i < kPart; ++i) {
                float w[2][2];
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int j = (i0 + i) * 8 + 2 * c4 + x, bit = 8 * ((i0 + i) & 3) + x;
                    const float2 total_j = nd->total[j];
                    const int wipes_j = nd->wipes[j];
                    const float rk = rk_la(j), rs = kNorm ? nd->rk_sm[sh][j] : 1.f;
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const bool folds = fold[r][i0 / 4] >> bit & 1u, sees = seen[r][i0 / 4] >> bit & 1u;
                        float q = qk[0][i][2 * r + x], own = q;
                        if (G > 1) {
                            own = sc ? qk[G - 1][i][2 * r + x] : q;
                            q += qk[G - 1][i][2 * r + x];
                        }
                        const float decay = decay_between(total[r], wipes[r], total_j, wipes_j) * rk;
                        w[r][x] = folds ? fq[r] * decay * q : 0.f;
                        if (j < t0 + 8 * r) tab[j * kRows + t0 + 8 * r] = folds ? bt[r] * decay * kk[i][2 * r + x] : 0.f;
                        y[i0 + i][2 * r + x] = sees ? own * f[r] * rs : -INFINITY;
                        m[r] = fmaxf(m[r], y[i0 + i][2 * r + x]);
                    }
                }
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    uint32_t w2[2];
                    split2(w[r][0], w[r][1], w2);
                    bh_f[(i0 + i) / 2][(i & 1) * 2 + r] = w2[0];
                    bl_f[(i0 + i) / 2][(i & 1) * 2 + r] = w2[1];
                }
            }
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            m[r] = fmaxf(m[r], __shfl_xor_sync(0xffffffffu, m[r], 1));
            m[r] = fmaxf(m[r], __shfl_xor_sync(0xffffffffu, m[r], 2));
            const float mu = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
            for (int i = 0; i < kNt; ++i) {
                const float p0 = tc::ex2_ftz(y[i][2 * r] - mu), p1 = tc::ex2_ftz(y[i][2 * r + 1] - mu);
                z[r] += p0 + p1;
                *reinterpret_cast<uint32_t *>(sm + L::oP + (t0 + 8 * r) * L::kPitchP + (i * 8 + 2 * c4) * 2) = tc::pack_bf162(p0, p1);
            }
            z[r] += __shfl_xor_sync(0xffffffffu, z[r], 1);
            z[r] += __shfl_xor_sync(0xffffffffu, z[r], 2);
            if (c4 == 0) { sums->tree_m[sc][t0 + 8 * r] = m[r]; sums->tree_z[sc][t0 + 8 * r] = z[r]; }
        }
    };
    // ---- k S0 and q S0, a warp's tiles of eight columns for all rows: the right-hand sides and the start of the read-out ----
    auto state_products = [&] {
        for (int tile = tile0; tile < tiles; tile += kStride) {
            float acc[2 * R][4];
#pragma unroll
            for (int m = 0; m < 2 * R; ++m)
#pragma unroll
                for (int x = 0; x < 4; ++x) acc[m][x] = 0.f;
#pragma unroll
            for (int k = 0; k < kKs; ++k) {
                uint32_t b0[3], b1[3];
                split3(s[k][0], s[k][1], b0);
                split3(s[k][2], s[k][3], b1);
                if (tile + kStride < tiles) load(tile + kStride, k, s[k]);
                constexpr int kM = R == 4 ? 4 : 2 * R;       // (row tiles at a time: registers)
#pragma unroll
                for (int m0 = 0; m0 < 2 * R; m0 += kM) {
                    uint32_t af[kM][4];
#pragma unroll
                    for (int m = 0; m < kM; ++m) {
                            const int t = (m0 + m) % R * 16 + (lane & 15), c = 2 * k + (lane >> 4);
                            ldmatrix_x4(m0 + m < R ? k_at + t * L::kPitch + c * 16 : q_at + L::q_piece(t, c), af[m]);
                        }
#pragma unroll
                    for (int x = 2; x >= 0; --x)
#pragma unroll
                        for (int m = 0; m < kM; ++m) mma_bf16(acc[m0 + m], af[m], b0[x], b1[x]);
                }
            }
            const int at = tile * 8 + 2 * c4;
#pragma unroll
            for (int m = 0; m < 2 * R; ++m)
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int t = (m % R) * 16 + r * 8 + g4;
                    const float x0 = acc[m][2 * r], x1 = acc[m][2 * r + 1];
                    if (m < R) {
                        const float fk = nd->whole[t] * rk_la(t), bt = nd->beta[t];
                        const float2 v = bf2(*reinterpret_cast<const uint32_t *>(sm + L::oV + t * L::kPitchV + at * 2));
                        *reinterpret_cast<float2 *>(su + t * cols + at) =
                            t < n ? make_float2(bt * (v.x - fk * x0), bt * (v.y - fk * x1)) : make_float2(0.f, 0.f);
                    } else {
                        const float fq = a.scale_la * nd->whole[t] * rq_la(t);
                        *reinterpret_cast<float2 *>(so + t * cols + at) = make_float2(fq * x0, fq * x1);
                    }
                }
        }
    };
    if (warp < R) tables();
    else state_products();
    sync();                                       // (k has been read: the sums over the tree's V take its place)
    // ---- the substitution: a thread's column, by blocks of 16 nodes.  A node that u_j does not reach has a zero in the table; a
    // block in which something is not finite is done again, along the paths. ----
    if (tid < cols) {
        const unsigned long long fold = nd->fold;
        float *col = su + tid;
        for (int t0 = 0; t0 < n; t0 += 16) {
            const unsigned folds = (unsigned)(fold >> t0);
            float r[16], sum = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = col[(t0 + i) * cols];
#pragma unroll 4
            for (int j = 0; j < t0; ++j) {
                const float u = col[j * cols], *row = tab + j * kRows + t0;
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const float4 w = *reinterpret_cast<const float4 *>(row + i);
                    r[i] = fmaf(-w.x, u, r[i]); r[i + 1] = fmaf(-w.y, u, r[i + 1]);
                    r[i + 2] = fmaf(-w.z, u, r[i + 2]); r[i + 3] = fmaf(-w.w, u, r[i + 3]);
                }
            }
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float *row = tab + (t0 + j) * kRows + t0;
                r[j] = folds >> j & 1u ? r[j] : 0.f;
                sum = fmaf(r[j], 0.f, sum);       // (NaN from what is not finite)
#pragma unroll
                for (int i = (j + 1) / 4 * 4; i < 16; i += 4) {
                    const float4 w = *reinterpret_cast<const float4 *>(row + i);
                    if (i > j) r[i] = fmaf(-w.x, r[j], r[i]);
                    if (i + 1 > j) r[i + 1] = fmaf(-w.y, r[j], r[i + 1]);
                    if (i + 2 > j) r[i + 2] = fmaf(-w.z, r[j], r[i + 2]);
                    if (i + 3 > j) r[i + 3] = fmaf(-w.w, r[j], r[i + 3]);
                }
            }
            if (sum == 0.f) {
#pragma unroll
                for (int i = 0; i < 16; ++i) col[(t0 + i) * cols] = r[i];
            } else {
                odd = true;
                for (int t = t0; t < min(n, t0 + 16); ++t) {
                    float x = col[t * cols];
                    for (unsigned long long w = nd->above[t] & fold; w; w &= w - 1) {
                        const int j = __ffsll(w) - 1;
                        x = fmaf(-tab[j * kRows + t], col[j * cols], x);
                    }
                    col[t * cols] = fold >> t & 1 ? x : 0.f;
                }
            }
        }
    }
    // ---- the sums over the tree's V, by the warps that the substitution leaves.  (Here and below a row's own non-finite entries
    // spoil that row alone; those of V and u are taken as zeros and added afterwards to the rows that see them.) ----
    constexpr int kSums = kWarps == 4 ? 2 : 4;    // these warps (64 columns keep two busy with the substitution)
    if (warp >= kWarps - kSums)
        for (int item = warp - (kWarps - kSums); item < R * tiles; item += kSums) {
            const int m = item % R, tile = item / R;
            float o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k > m) break;                 // (parents come first)
                uint32_t af[4], bf[2];
                ldmatrix_x4(tc::smem_u32(sm + L::oP) + (m * 16 + (lane & 15)) * L::kPitchP + (2 * k + (lane >> 4)) * 16, af);
                ldmatrix_x2_trans(v_at + (k * 16 + (lane & 15)) * L::kPitchV + tile * 16, bf);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if ((bf[x] & 0x7f80u) == 0x7f80u) bf[x] &= 0xffff0000u;
                    if ((bf[x] & 0x7f800000u) == 0x7f800000u) bf[x] &= 0xffffu;
                }
                mma_bf16(o, af, bf[0], bf[1]);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r)
                *reinterpret_cast<float2 *>(st + (m * 16 + r * 8 + g4) * cols + tile * 8 + 2 * c4) = make_float2(o[2 * r], o[2 * r + 1]);
        }
    if (odd) s_odd = 1;
    sync();
    odd = s_odd != 0;
    // ---- the linear read-out ----
    if (warp < R) {
        auto clean = [&](float x) { return odd && !finite(x) ? 0.f : x; };
        for (int tile = 0; tile < tiles; ++tile) {
            const int at = tile * 8 + 2 * c4;
            float o[4], lo[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float2 y = *reinterpret_cast<const float2 *>(so + (warp * 16 + r * 8 + g4) * cols + at);
                o[2 * r] = y.x;
                o[2 * r + 1] = y.y;
            }
#pragma unroll
            for (int k = 0; k < R; ++k) {
                if (k > warp) break;
                const float *y = su + (k * 16 + 2 * c4) * cols + tile * 8 + g4;
                uint32_t b0[2], b1[2];
                split2(clean(y[0]), clean(y[cols]), b0);
                split2(clean(y[8 * cols]), clean(y[9 * cols]), b1);
                mma_bf16(lo, bl_f[k], b0[0], b1[0]);
                mma_bf16(o, bh_f[k], b0[0], b1[0]);
                mma_bf16(lo, bh_f[k], b0[1], b1[1]);
            }
#pragma unroll
            for (int r = 0; r < 2; ++r)
                *reinterpret_cast<float2 *>(so + (warp * 16 + r * 8 + g4) * cols + at) = make_float2(o[2 * r] + lo[2 * r], o[2 * r + 1] + lo[2 * r + 1]);
        }
    }
    if (a.u)
        for (int i = kHalf - 1 - tid; i < n * (cols / 4); i += kHalf) {      // (the last warps first)
            const int t = i / (cols / 4), c = (i - t * (cols / 4)) * 4;
            *reinterpret_cast<float4 *>(a.u + (((size_t)b * T + t) * a.H + h) * D + c0 + c) =
                *reinterpret_cast<const float4 *>(su + t * cols + c);
        }
    if (odd) {
        sync();
        if (warp < R)                             // what the read-out takes from u, in the table's place, [t][j]
#pragma unroll
            for (int k = 0; k < kNt / 2; ++k)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float2 y = bf2(bh_f[k][x]), w = bf2(bl_f[k][x]);
                    float *to = tab + (warp * 16 + (x & 1) * 8 + g4) * kRows + k * 16 + (x >> 1) * 8 + 2 * c4;
                    to[0] = y.x + w.x;
                    to[1] = y.y + w.y;
                }
        sync();
        for (int i = tid; i < n * cols; i += kHalf) {
            const int t = i / cols, c = i - t * cols;
            const unsigned long long path = nd->above[t] | 1ull << t;
            for (unsigned long long w = path & nd->fold; w; w &= w - 1) {
                const int j = __ffsll(w) - 1;
                if (!finite(su[j * cols + c])) so[i] += tab[t * kRows + j] * su[j * cols + c];
            }
            for (unsigned long long w = path & nd->keep; w; w &= w - 1) {
                const int j = __ffsll(w) - 1;
                const float v = to_f32(*reinterpret_cast<const __nv_bfloat16 *>(sm + L::oV + j * L::kPitchV + c * 2));
                if (!finite(v)) st[i] += to_f32(*reinterpret_cast<const __nv_bfloat16 *>(sm + L::oP + t * L::kPitchP + j * 2)) * v;
            }
        }
    }
}

template <int D, int G, bool kNorm, int R>
__global__ void __launch_bounds__(Layout<D, R>::kThreads, Layout<D, R>::kCtas)
tree_tc_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, Args a, int wait_kcycles,
               int withhold) {
    using L = Layout<D, R>;
    constexpr int kReaders = L::kReaders, kThreads = L::kThreads;
    extern __shared__ __align__(1024) uint8_t dyn_tc[];
    __shared__ typename L::N nodes;
    __shared__ UmmaBars bars;
    const int bh = blockIdx.x / a.cluster, rank = blockIdx.x - bh * a.cluster, b = bh / a.H, h = bh - b * a.H, tid = threadIdx.x;
    if (L::kUmma && tid == 128) {
        umma_init(&bars, kNorm, wait_kcycles);
        tc::prefetch_tmap(&map_k);
        tc::prefetch_tmap(&map_v);
    }
    tc::grid_dependency_wait();
    if (L::kUmma && tid / 32 == 4) {
        __syncwarp();                             // (one lane comes from the branch above; an allocation is the whole warp's)
        tc::tmem_alloc(&bars.tmem, kTmemCols);
    }
    const NodeRow node = load_node(a, b, h, tid >= kReaders ? tid - kReaders : a.T);
    const int n = nodes_of(a, b), cols = D / a.cluster;
    const Share share = share_of(a.cache_len[bh], a.cap, a.cluster, rank);
    const Stream<D, R> in(a, dyn_tc, bh, tid, share);
    typename L::S *sums = reinterpret_cast<typename L::S *>(dyn_tc);
    if (!L::kUmma && tid < kReaders)
#pragma unroll
        for (int u = 0; u < L::kSlots - 1; ++u) in.fetch(u);
    // q, k and the columns of v
    constexpr int kPieces = L::kRowBytes / 16, kLoads = (L::kRows * kPieces + kThreads - 1) / kThreads;
    const uint4 zero = make_uint4(0, 0, 0, 0);
    uint4 x[2][kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int e = tid + i * kThreads, t = e / kPieces;
        const size_t at = (((size_t)b * a.T + t) * a.H + h) * kPieces + e - t * kPieces;
        x[0][i] = t < n ? reinterpret_cast<const uint4 *>(a.q)[at] : zero;
        x[1][i] = t < n ? reinterpret_cast<const uint4 *>(a.k)[at] : zero;
    }
    bool odd = false;                             // something that is not finite may meet a zero
    for (int e = tid; e < L::kRows * (cols / 8); e += kThreads) {
        const int t = e / (cols / 8), c = e - t * (cols / 8);
        const uint4 y = t < n ? reinterpret_cast<const uint4 *>(a.v)[(((size_t)b * a.T + t) * a.H + h) * kPieces + rank * cols / 8 + c] : zero;
        odd |= !(finite_bf16x2(y.x) && finite_bf16x2(y.y) && finite_bf16x2(y.z) && finite_bf16x2(y.w));
        *reinterpret_cast<uint4 *>(dyn_tc + L::oV + t * L::kPitchV + c * 16) = y;
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int e = tid + i * kThreads, t = e / kPieces, c = e - t * kPieces;
        if (t < L::kRows) {
            *reinterpret_cast<uint4 *>(dyn_tc + L::oQ + L::q_piece(t, c)) = x[0][i];
            *reinterpret_cast<uint4 *>(dyn_tc + L::oK + t * L::kPitch + c * 16) = x[1][i];
        }
    }
    if (L::kUmma) {
        tc::fence_proxy_async_smem();             // (q is an operand of the MMAs)
        tc::tc_fence_before_sync();
    }
    odd = __syncthreads_or(odd);
    tc::launch_dependents();
    if (tid >= kReaders) {
        tree_part<D, G, kNorm, R>(a, sums, dyn_tc, &nodes, b, h, n, rank, odd, node);
    } else if constexpr (L::kUmma) {
        tc::tc_fence_after_sync();
        const uint32_t tmem = bars.tmem;
        const int keys = share.to - share.from;
        const UmmaShare<D> u{{&map_k, &map_v}, &bars, dyn_tc, dyn_tc + L::oRing, bh * a.cap + share.from, keys, (keys + kTileKeys - 1) / kTileKeys};
        if (tid < 128) {
            umma_softmax<D, G, kNorm>(a, sums, u, tmem, n, withhold != 0);
        } else if (tid < 160) {
            umma_sums<D, G>(u, tmem);
            tc::named_barrier_sync(5, 192);
            tc::tc_fence_after_sync();
            tc::tmem_dealloc(tmem, kTmemCols);
        } else if (tid < 192) {
            umma_logits<D, G>(u, tmem, tc::smem_u32(dyn_tc + L::oQ));
            tc::named_barrier_arrive(5, 192);
        } else {
            umma_load<D>(u, (tid >> 5) & 1);
        }
    } else {
        cache_part<D, G, kNorm, R>(a, sums, dyn_tc, in, n);
    }
    join_rows<__nv_bfloat16, D>(a, b, h, n, rank, sums, reinterpret_cast<const float *>(dyn_tc + L::oRing), L::kAccPitch,
                                reinterpret_cast<const float *>(dyn_tc + L::oO), reinterpret_cast<const float *>(dyn_tc + L::oK));
    if (L::kUmma && tid == 0 && bars.abort[0]) atomicMin(a.status, (int)NATSL_ERR_TIMEOUT);
}

template <int D, int G, bool kNorm, int R>
cudaError_t launch(const Args &a, int BH, cudaStream_t st) {
    auto kernel = tree_tc_kernel<D, G, kNorm, R>;
    cudaError_t e = allow_smem(kernel, Layout<D, R>::kTotal);
    if (e != cudaSuccess) return e;
    CUtensorMap map_k = {}, map_v = {};
    if (Layout<D, R>::kUmma && (!tch::make_map_2d(&map_k, a.k_cache, (uint64_t)BH * a.cap, D, kTileKeys) ||
                                !tch::make_map_2d(&map_v, a.v_cache, (uint64_t)BH * a.cap, D, kTileKeys)))
        return cudaErrorInvalidValue;
    return launch_clusters(kernel, BH * a.cluster, a.cluster, Layout<D, R>::kThreads, Layout<D, R>::kTotal, st, map_k, map_v, a,
                           debug_wait_kcycles(), debug_withhold());
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
