// What the two tree-step kernels (tensor cores, fp32 CUDA cores) share: how a pair's work is cut, the walk up the drafted
// tree, and the join of the partial results.
//
// A (sequence, head) pair is the work of one cluster of 2, 4 or 8 CTAs.  Each takes a slice of the retained K/V for all nodes,
// and d / cluster columns of the tree's own part (linear branch, and the softmax over the tree's own tokens).  The partial
// results stay in shared memory; behind the cluster's barrier each CTA joins every cluster-th row of the tree, reading its
// neighbours' shares over distributed shared memory.  So a call is one launch, needs no scratch and no atomics, and the sums
// have the same order on every call.  (With partial results in global memory and the last of a pair's CTAs, by a ticket,
// joining them alone, 16 nodes of 16 pairs took 44 us, 25 of them in that join; now 11 us, 3000 cycles a row of the join, most
// of it the neighbours' shared memory, which gives some 14 bytes a cycle.)
#pragma once
#include "common.cuh"
#include "natsl_internal.h"
#include "tc_common.cuh"

namespace natsl {
namespace tree {

constexpr int kMaxNodes = 64;        // one machine word of ancestors per node
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

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
    int32_t *status;
    int H, T, cap, G, cluster;
    float scale_la, scale_sm, eps, norm_eps;      // norm_eps < 0: q, k as given
};

// A cache's share of CTA `rank`: keys [from, to).  A stored length outside [0, cap] counts as the nearer of both.
struct Share { int from, to; };
__device__ __forceinline__ Share share_of(int n_raw, int cap, int cluster, int rank) {
    const int n = min(max(n_raw, 0), cap), blocks = n / 16 + (n % 16 != 0), per = (blocks + cluster - 1) / cluster;
    const int from = (int)min((long long)rank * per * 16, (long long)n);
    return Share{from, (int)min((long long)from + (long long)per * 16, (long long)n)};
}

// Read by the whole cluster: running maxima (base 2) and sums of the CTA's cache share, and those of the softmax over the tree's
// own tokens for the softmax heads of the CTA's columns.
template <int kHeads, int kRows> struct Sums {
    float cache_m[kHeads][kRows], cache_z[kHeads][kRows], tree_m[kHeads][kRows], tree_z[kHeads][kRows];
};

template <int kHeads, int kRows> struct Nodes {
    unsigned long long above[kRows];              // strict ancestors
    unsigned long long fold, keep;                // nodes that update the state; nodes whose K/V count as retained
    float2 total[kRows];                          // sum of g from the context up to and with the node, as two fp32 terms; a g whose
    int wipes[kRows];                             // exp is zero is left out and counted here
    float whole[kRows], beta[kRows], g[kRows];    // whole: exp of that sum; g: -inf where its exp is zero
    float rq_la[kRows], rk_la[kRows];             // L2 factors; RMS factors per softmax head
    float rq_sm[kHeads][kRows], rk_sm[kHeads][kRows];
    int parent[kRows];
};

// What is read of a node (lane-wise, ahead of the number of nodes: rows behind the last node exist, and are not looked at).
struct NodeRow { int parent, route; float beta, g; };
__device__ __forceinline__ NodeRow load_node(const Args &a, int b, int h, int t) {
    NodeRow x{-1, 0, 0.f, 0.f};
    if (t < a.T) {
        const size_t at = ((size_t)b * a.T + t) * a.H + h;
        x = NodeRow{a.parent[(size_t)b * a.T + t], a.route[at], a.beta[at], a.g[at]};
    }
    return x;
}
// Walks every node's path (a parent is always a lower index, so a walk ends).  tid: of 64 threads or more, whose barrier `sync`
// is; row: load_node's of node tid.  Another barrier is due before the result is read.
template <int kHeads, int kRows, typename Sync>
__device__ __forceinline__ void walk_nodes(const Args &a, int b, int h, int n, int tid, const NodeRow &row, Nodes<kHeads, kRows> *nd, Sync sync) {
    if (tid < 64) {                               // (two whole warps, for the ballots)
        int par = tid < n ? row.parent : -1;
        if (par < -1 || par >= tid) {             // not a tree: reported, and taken as a child of the context
            if (tid < n) atomicMin(a.status, (int)NATSL_ERR_TREE);
            par = -1;
        }
        if (tid < kRows) {
            nd->parent[tid] = par;
            nd->beta[tid] = tid < n ? row.beta : 0.f;
            // A decay that is zero in fp32 (g below -104) ends what comes from above, as one of -inf does: left in the sums, a large
            // enough g would take the others' bits with it.  So they are sums of at most 64 values above -104.
            nd->g[tid] = expf(row.g) == 0.f ? -INFINITY : row.g;
        }
        const unsigned f = __ballot_sync(0xffffffffu, tid < n && row.route != 1), k = __ballot_sync(0xffffffffu, tid < n && row.route != 0);
        if ((tid & 31) == 0) {
            reinterpret_cast<unsigned *>(&nd->fold)[tid >> 5] = f;
            reinterpret_cast<unsigned *>(&nd->keep)[tid >> 5] = k;
        }
    }
    if (tid == 0) {
        if (a.n_nodes && a.n_nodes[b] != n) atomicMin(a.status, (int)NATSL_ERR_TREE);
        const int len = a.cache_len[(size_t)b * a.H + h];
        if (len < 0 || len > a.cap) atomicMin(a.status, (int)NATSL_ERR_CACHE_FULL);
    }
    sync();
    if (tid < kRows) {
        unsigned long long up = 0;
        double sum = 0.0;                         // (in 64 bits: nothing of a short stretch far from the context is lost)
        int wipes = 0;
        for (int x = tid < n ? tid : -1; x >= 0;) {
            const float g = nd->g[x];
            wipes += g == -INFINITY;
            sum += g == -INFINITY ? 0.f : g;
            x = nd->parent[x];
            up |= x >= 0 ? 1ull << x : 0ull;
        }
        const float hi = (float)sum;
        nd->above[tid] = up;
        nd->total[tid] = make_float2(hi, (float)(sum - (double)hi));
        nd->wipes[tid] = wipes;
        nd->whole[tid] = wipes || tid >= n ? 0.f : expf(hi);
    }
}
// Decay on the path from its node j (exclusive) to i, and zero as soon as a zero one lies on it.
__device__ __forceinline__ float decay_between(float2 total_i, int wipes_i, float2 total_j, int wipes_j) {
    const float x = expf((total_i.x - total_j.x) + (total_i.y - total_j.y));
    return wipes_i != wipes_j ? 0.f : x;
}

// Nodes of a sequence's tree; a count outside [0, T] counts as the nearer of both and is reported.
__device__ __forceinline__ int nodes_of(const Args &a, int b) {
    const int n = a.n_nodes ? a.n_nodes[b] : a.T;
    return min(max(n, 0), a.T);
}

// The cluster's barrier: what its threads have written to shared memory is there for all of them.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire;" ::: "memory"); }
// `p`'s counterpart in CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t remote(const void *p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(tc::smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float ld_remote(uint32_t p) {
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(p) : "memory");
    return x;
}
template <int V> __device__ __forceinline__ void ld_remote(uint32_t p, float (&x)[V]) {
    if constexpr (V == 4)
        asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x[0]), "=f"(x[1]), "=f"(x[2]), "=f"(x[3]) : "r"(p) : "memory");
    else
        asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x[0]), "=f"(x[1]) : "r"(p) : "memory");
}

// Joins the rows rank, rank + cluster, ... of pair (b, h): softmax over the cache shares and the tree, both branches normalised
// and combined.  A warp takes a row; lane l owns columns V l .. V l + V - 1.  acc [rows][acc_pitch]: the CTA's sums over its
// cache share, all columns; o_la, o_tree [rows][D / cluster]: the linear read-out and the sums over the tree, its own columns.
template <typename ST, int D, int kCluster, typename S>
__device__ __forceinline__ void join_rows_of(const Args &a, int b, int h, int n, int rank, const S *sums, const float *acc,
                                             int acc_pitch, const float *o_la, const float *o_tree) {
    constexpr int V = D / 32, cols = D / kCluster;
    const int lane = threadIdx.x & 31, G = a.G, ls = 32 / G, sg = lane / ls, step = kCluster * (blockDim.x >> 5);
    const int owner = lane * V / cols, at = lane * V - owner * cols;
    struct Row {
        float m[kCluster], z[kCluster], x[kCluster][V], mt, zt, o[V], la[V];
    };
    auto load = [&](int t, Row &y) {
#pragma unroll
        for (int r = 0; r < kCluster; ++r) {
            y.m[r] = ld_remote(remote(&sums->cache_m[sg][t], r));
            y.z[r] = ld_remote(remote(&sums->cache_z[sg][t], r));
            ld_remote<V>(remote(acc + t * acc_pitch + lane * V, r), y.x[r]);
        }
        y.mt = ld_remote(remote(&sums->tree_m[sg][t], owner));
        y.zt = ld_remote(remote(&sums->tree_z[sg][t], owner));
        ld_remote<V>(remote(o_tree + t * cols + at, owner), y.o);
        ld_remote<V>(remote(o_la + t * cols + at, owner), y.la);
    };
    auto finish = [&](int t, Row &y, bool last) {
        float M = y.mt;
#pragma unroll
        for (int r = 0; r < kCluster; ++r) M = fmaxf(M, y.m[r]);
        const float Mu = M == -INFINITY ? 0.f : M, ft = tc::ex2_ftz(y.mt - Mu);
        float Z = y.zt * ft;
#pragma unroll
        for (int i = 0; i < V; ++i) y.o[i] *= ft;
#pragma unroll
        for (int r = 0; r < kCluster; ++r) {
            const float f = tc::ex2_ftz(y.m[r] - Mu);
            Z = fmaf(y.z[r], f, Z);
#pragma unroll
            for (int i = 0; i < V; ++i) y.o[i] = fmaf(y.x[r][i], f, y.o[i]);
        }
        const float iz = Z == 0.f ? 0.f : 1.f / Z;     // (no visible key: o_nla = 0)
        float sn = 0.f, sl = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            y.o[i] *= iz;
            sn = fmaf(y.o[i], y.o[i], sn);
            sl = fmaf(y.la[i], y.la[i], sl);
        }
        if (last) cluster_arrive();               // (the warp has read its last row)
        for (int s = ls / 2; s > 0; s >>= 1) sn += __shfl_xor_sync(0xffffffffu, sn, s);
        sl = warp_sum(sl);
        const float *w = a.w + (((size_t)b * a.T + t) * a.H + h) * 2;
        const float fn = (a.w ? w[0] : 0.5f) * rsqrtf(sn / (D / G) + a.eps), fl = (a.w ? w[1] : 0.5f) * rsqrtf(sl / D + a.eps);
        ST *out = reinterpret_cast<ST *>(a.out) + (((size_t)b * a.T + t) * a.H + h) * D + lane * V;
#pragma unroll
        for (int i = 0; i < V; ++i) y.o[i] = fmaf(fn, y.o[i], fl * y.la[i]);
        if constexpr (V == 4) {
            store4(out, make_float4(y.o[0], y.o[1], y.o[2], y.o[3]));
        } else {
            out[0] = from_f32<ST>(y.o[0]);
            out[1] = from_f32<ST>(y.o[1]);
        }
        if (a.lse && lane % ls == 0)
            a.lse[(((size_t)b * a.H + h) * G + sg) * a.T + t] = Z == 0.f ? -INFINITY : (M + log2f(Z)) * kLn2;
    };
    int t = rank + kCluster * (threadIdx.x >> 5);
    Row y;
    cluster_arrive();
    cluster_wait();
    if (t >= n) cluster_arrive();                 // (no row for this warp)
    else load(t, y);
    for (; t < n; t += step) {                    // (with two CTAs, where rows are many, a row is on its way while one is finished)
        if constexpr (kCluster == 2) {
            Row next;
            if (t + step < n) load(t + step, next);
            finish(t, y, t + step >= n);
            y = next;
        } else {
            finish(t, y, t + step >= n);
            if (t + step < n) load(t + step, y);
        }
    }
    cluster_wait();                               // nobody's shared memory goes while a neighbour still reads it
}
template <typename ST, int D, typename S>
__device__ __forceinline__ void join_rows(const Args &a, int b, int h, int n, int rank, const S *sums, const float *acc, int acc_pitch,
                                          const float *o_la, const float *o_tree) {
    if (a.cluster == 2) join_rows_of<ST, D, 2>(a, b, h, n, rank, sums, acc, acc_pitch, o_la, o_tree);
    else if (a.cluster == 4) join_rows_of<ST, D, 4>(a, b, h, n, rank, sums, acc, acc_pitch, o_la, o_tree);
    else join_rows_of<ST, D, 8>(a, b, h, n, rank, sums, acc, acc_pitch, o_la, o_tree);
}

// One cluster per pair, placed while the work before it in the stream finishes.
template <typename K, typename... A>
cudaError_t launch_clusters(K kernel, int grid, int cluster, int threads, size_t smem, cudaStream_t st, const A &...args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
    count_launch();
    return e;
}

}  // namespace tree

// tree_tc.cu: bf16 storage, one or two softmax heads per linear head
cudaError_t launch_tree_tc(const tree::Args &a, int BH, int d, cudaStream_t st);

}  // namespace natsl
