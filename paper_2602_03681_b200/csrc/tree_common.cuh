// What the two tree-step kernels (tensor cores, fp32 CUDA cores) share: how a pair's work is cut, the walk up the drafted
// tree, and the join of the partial results.
#pragma once
#include "common.cuh"
#include "natsl_internal.h"
#include "tc_common.cuh"

namespace natsl {
namespace tree {

constexpr int kMaxNodes = 64;        // one machine word of ancestors per node
constexpr int kThreads = 128;
constexpr int kTileKeys = 64;        // keys the cut of a cache is counted in
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Cache items per (sequence, head) that the workspace has room for, by the number of pairs alone.
__host__ __device__ inline int max_parts(int BH) {
    const int p = 592 / BH;
    return p < 4 ? 4 : (p > 64 ? 64 : p);
}
// Workspace: [0,256) status word; tickets [BH] i32; per pair the linear read-outs [T][D], then parts + 1 partial results
// (the last one is the tree's own): m [4][T] in base-2 units, z [4][T], acc [T][D].
__host__ __device__ inline size_t off_pairs(size_t BH) { return (256 + BH * 4 + 255) / 256 * 256; }
__host__ __device__ inline size_t part_floats(int T, int D) { return (size_t)T * (8 + D); }
__host__ __device__ inline size_t pair_floats(int T, int D, int parts) { return (size_t)T * D + (parts + 1) * part_floats(T, D); }

// A stored length outside [0, cap] counts as the nearer of both.  Of `parts` items the first np take tpp tiles each.
struct Cut { int n, tpp, np; };
__device__ __forceinline__ Cut cut_of(int n_raw, int cap, int parts, int least_tiles) {
    Cut c;
    c.n = min(max(n_raw, 0), cap);
    const int tiles = (c.n + kTileKeys - 1) / kTileKeys;
    c.tpp = max(least_tiles, (tiles + parts - 1) / parts);
    c.np = (tiles + c.tpp - 1) / c.tpp;
    return c;
}

struct Args {
    const void *q, *k, *v;
    const float *g, *beta;
    const uint8_t *route;
    const int32_t *parent, *n_nodes;
    const float *w, *state;
    const void *k_cache, *v_cache;
    const int32_t *cache_len;
    void *out;
    float *u, *lse;
    uint8_t *ws;
    int H, T, cap, G, parts, least_tiles;
    float scale_la, scale_sm, eps, norm_eps;      // norm_eps < 0: q, k as given
};

// Shared-memory head of a CTA: the tree.
struct Nodes {
    unsigned long long above[kMaxNodes];          // strict ancestors
    unsigned long long fold, keep;                // nodes that update the state; nodes whose K/V count as retained
    float beta[kMaxNodes], alpha[kMaxNodes], whole[kMaxNodes];   // whole: decay from the context up to and with the node
    float rq_la[kMaxNodes], rk_la[kMaxNodes];     // L2 factors; RMS factors per softmax head
    float rq_sm[4][kMaxNodes], rk_sm[4][kMaxNodes];
    int parent[kMaxNodes];
};

// Nodes of a sequence's tree; a count outside [0, T] counts as the nearer of both and is reported.
__device__ __forceinline__ int nodes_of(const Args &a, int b) {
    const int n = a.n_nodes ? a.n_nodes[b] : a.T;
    return min(max(n, 0), a.T);
}

// Reads the tree of (b, h) into `nd`, walks every node's path (a parent is always a lower index, so a walk ends) and puts
// the decay D_ij = exp(sum of g on the path from j, exclusive, to i) of every ancestor j of i at decay[i * pitch + j]:
// products along the path, so that a decay of zero (g = -inf) stays zero and long paths lose nothing by cancellation.
__device__ __forceinline__ void read_nodes(const Args &a, int b, int h, int n, Nodes *nd, float *decay, int pitch) {
    const int tid = threadIdx.x;
    int32_t *status = reinterpret_cast<int32_t *>(a.ws);
    if (tid < kMaxNodes) {
        int par = -1, rv = 0;
        if (tid < n) {
            const size_t at = ((size_t)b * a.T + tid) * a.H + h;
            par = a.parent[(size_t)b * a.T + tid];
            if (par < -1 || par >= tid) {         // not a tree: reported, and taken as a child of the context
                par = -1;
                atomicMin(status, (int)NATSL_ERR_TREE);
            }
            rv = a.route[at];
            nd->beta[tid] = a.beta[at];
            nd->alpha[tid] = expf(a.g[at]);
        }
        nd->parent[tid] = par;
        const unsigned f = __ballot_sync(0xffffffffu, tid < n && rv != 1), k = __ballot_sync(0xffffffffu, tid < n && rv != 0);
        if ((tid & 31) == 0) {
            reinterpret_cast<unsigned *>(&nd->fold)[tid >> 5] = f;
            reinterpret_cast<unsigned *>(&nd->keep)[tid >> 5] = k;
        }
    }
    if (tid == 0) {
        if (a.n_nodes && a.n_nodes[b] != n) atomicMin(status, (int)NATSL_ERR_TREE);
        const int len = a.cache_len[(size_t)b * a.H + h];
        if (len < 0 || len > a.cap) atomicMin(status, (int)NATSL_ERR_CACHE_FULL);
    }
    __syncthreads();
    if (tid < n) {
        unsigned long long up = 0;
        float prod = nd->alpha[tid];
        for (int x = nd->parent[tid]; x >= 0; x = nd->parent[x]) {
            up |= 1ull << x;
            decay[tid * pitch + x] = prod;
            prod *= nd->alpha[x];
        }
        decay[tid * pitch + tid] = 1.f;
        nd->above[tid] = up;
        nd->whole[tid] = prod;
    } else if (tid < kMaxNodes) {
        nd->above[tid] = 0;
        nd->whole[tid] = 0.f;
    }
}

// Pair bh is finished by whichever of its parts + 1 items comes last (an atomic ticket, nobody waits); true in that CTA.
__device__ __forceinline__ bool last_of_pair(const Args &a, int bh) {
    __shared__ int s_last;
    __syncthreads();                              // every thread's partial results are written
    if (threadIdx.x == 0) {
        int32_t *ticket = reinterpret_cast<int32_t *>(a.ws + 256) + bh;
        __threadfence();
        const int last = tc::atom_add_acq_rel(ticket, 1) == a.parts;
        if (last) *ticket = 0;                    // ready for the next call
        __threadfence();
        s_last = last;
    }
    __syncthreads();
    return s_last != 0;
}

// Joins the partial results of pair (b, h): softmax over cache items and the tree, both branches normalised and combined.
// A warp takes a row; lane l owns columns V l .. V l + V - 1.
template <typename ST, int D>
__device__ __forceinline__ void join_pair(const Args &a, int b, int h, int n) {
    constexpr int V = D / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int bh = b * a.H + h, G = a.G, ls = 32 / G, sg = lane / ls;
    const Cut c = cut_of(a.cache_len[bh], a.cap, a.parts, a.least_tiles);
    const float *base = reinterpret_cast<const float *>(a.ws + off_pairs((size_t)gridDim.x / (a.parts + 1))) +
                        (size_t)bh * pair_floats(a.T, D, a.parts);
    const size_t pf = part_floats(a.T, D);
    const float *first = base + (size_t)a.T * D, *own = first + a.parts * pf;
    for (int t = warp; t < n; t += kThreads / 32) {
        float M = __ldcg(own + sg * a.T + t), Z = 0.f, o[V], ol[V];
        for (int p = 0; p < c.np; ++p) M = fmaxf(M, __ldcg(first + p * pf + sg * a.T + t));
        const float Mu = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int x = 0; x < V; ++x) {
            o[x] = 0.f;
            ol[x] = __ldcg(base + (size_t)t * D + lane * V + x);
        }
        for (int p = 0; p <= c.np; ++p) {         // (in this order whoever joins: the same sums on every call)
            const float *pp = p < c.np ? first + p * pf : own;
            const float f = tc::ex2_ftz(__ldcg(pp + sg * a.T + t) - Mu);
            Z = fmaf(__ldcg(pp + (4 + sg) * a.T + t), f, Z);
            const float *acc = pp + 8 * a.T + (size_t)t * D + lane * V;
#pragma unroll
            for (int x = 0; x < V; ++x) o[x] = fmaf(__ldcg(acc + x), f, o[x]);
        }
        const float iz = Z == 0.f ? 0.f : 1.f / Z;     // (no visible key: o_nla = 0)
        float sn = 0.f, sl = 0.f;
#pragma unroll
        for (int x = 0; x < V; ++x) {
            o[x] *= iz;
            sn = fmaf(o[x], o[x], sn);
            sl = fmaf(ol[x], ol[x], sl);
        }
        for (int s = ls / 2; s > 0; s >>= 1) sn += __shfl_xor_sync(0xffffffffu, sn, s);
        sl = warp_sum(sl);
        const size_t row = ((size_t)b * a.T + t) * a.H + h;
        const float wn = a.w ? a.w[row * 2] : 0.5f, wl = a.w ? a.w[row * 2 + 1] : 0.5f;
        const float fn = wn * rsqrtf(sn / (D / G) + a.eps), fl = wl * rsqrtf(sl / D + a.eps);
        ST *out = reinterpret_cast<ST *>(a.out) + row * D + lane * V;
#pragma unroll
        for (int x = 0; x < V; ++x) out[x] = from_f32<ST>(fn * o[x] + fl * ol[x]);
        if (a.lse && lane % ls == 0)
            a.lse[((size_t)bh * G + sg) * a.T + t] = Z == 0.f ? -INFINITY : (M + log2f(Z)) * kLn2;
    }
}

}  // namespace tree

// tree_tc.cu: bf16 storage, one or two softmax heads per linear head
cudaError_t launch_tree_tc(const tree::Args &a, int BH, int d, cudaStream_t st);

}  // namespace natsl
