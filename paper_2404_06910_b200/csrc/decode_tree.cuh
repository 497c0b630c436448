// What the kernels of sp_pruned_decode_tree share: arguments, the check of a prompt's tree, the table of its key segments, the sets of
// ancestors and the merge of partial results over a cluster.
#pragma once

#include <cooperative_groups.h>

#include "common.cuh"
#include "tc_ptx.cuh"

namespace sp {

constexpr int kTreeMaxNodes = 64;                // a node's ancestors are the bits of one 64-bit word
constexpr int kTtPad = 8;                        // the bf16 kernel's segments start at multiples of this: the smallest TMA box's rows
constexpr float kLog2eT = 1.4426950408889634f;
constexpr float kLn2T = 0.6931471805599453f;

struct TreeArgs {
    const void *q, *k_cache, *v_cache, *tail_k, *tail_v;
    const int32_t *ppo, *pre_start, *pre_len, *path_start, *doc_len, *qry_len;
    const int32_t *kept_idx, *tail_len, *parent, *n_nodes;
    void *out;
    float *lse;
    uint32_t *status;
    int k, tail_cap, max_nodes, n_heads, n_kv_heads, n_prompts, n_paths, max_pre_len, max_path_len;
    int64_t total_tokens;
    float scale_log2e;
};

// Number of nodes of prompt b, committed rows of its tail; false where the tree or the tail is impossible (the prompt is then skipped and
// reported).  All 32 lanes of a warp; parents of node lane and lane + 32 in par.
__device__ __forceinline__ bool tree_of_prompt(const TreeArgs &a, int b, int &n, int &committed, int (&par)[2])
{
    const int lane = threadIdx.x & 31;
    // all places' parents, before it is known how many nodes there are: one round trip to memory instead of two
#pragma unroll
    for (int i = 0; i < 2; ++i) par[i] = lane + 32 * i < a.max_nodes ? a.parent[(int64_t)b * a.max_nodes + lane + 32 * i] : -1;
    n = a.n_nodes ? a.n_nodes[b] : a.max_nodes;
    committed = a.tail_len[b];
    bool good = n >= 0 && n <= a.max_nodes && committed >= 0 && (int64_t)committed + n <= a.tail_cap;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int node = lane + 32 * i;
        if (node >= n) par[i] = -1;
        good = good && par[i] >= -1 && (par[i] < node || node >= n);
    }
    return __all_sync(0xffffffffu, good);
}

// Segment s of prompt b (0: the preamble, then the kept paths): its first row in the cache and its length.  False where the layout's arrays put it outside
// the cache or make it longer than the host was told: the segment is then empty and reported.  A kept index that is none of the prompt's paths is an
// empty segment too, and fine, as in sp_pruned_decode.
__device__ __forceinline__ bool tree_segment(const TreeArgs &a, int b, int s, int64_t &row, int64_t &len)
{
    int most = a.max_path_len;
    bool good = true;
    row = len = 0;
    if (s == 0) {
        row = a.pre_start[b]; len = a.pre_len[b]; most = a.max_pre_len;
    } else {
        const int i = a.kept_idx[(int64_t)b * a.k + s - 1], p0 = a.ppo[b], p1 = a.ppo[b + 1];
        if (i >= max(p0, 0) && i < min(p1, a.n_paths)) {
            const int doc = a.doc_len[i], qry = a.qry_len[i];
            good = doc >= 0 && qry >= 0;
            row = a.path_start[i]; len = (int64_t)doc + qry;
        }
    }
    good = good && row >= 0 && len >= 0 && len <= most && row + len <= a.total_tokens;
    if (!good) len = 0;
    return good;
}

// The grid's first layer (z = 0; prompts follow) reports: it is scheduled before every other block, so that its plain store comes before any
// other block could have something to add.
__device__ __forceinline__ void tree_report(const TreeArgs &a)
{
    if (blockIdx.x || blockIdx.y) return;
    // A thread takes segments and places of nodes one by one, whatever prompt they are of, several loads under way at a time: with thousands of prompts of few
    // keys this block would otherwise be the last to end.
    bool good = true;
    const uint32_t per = a.k + 1, segments = (uint32_t)a.n_prompts * per, nodes = (uint32_t)a.n_prompts * a.max_nodes;
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < segments; i += blockDim.x) {
        int64_t row, len;
        good &= tree_segment(a, i / per, i % per, row, len);
    }
#pragma unroll 4
    for (uint32_t i = threadIdx.x; i < nodes; i += blockDim.x) {
        const int b = i / a.max_nodes, node = i % a.max_nodes, n = a.n_nodes ? a.n_nodes[b] : a.max_nodes, committed = a.tail_len[b], parent = a.parent[i];
        good &= n >= 0 && n <= a.max_nodes && committed >= 0 && (int64_t)committed + n <= a.tail_cap && (node >= n || (parent >= -1 && parent < node));
    }
    good = __syncthreads_and(good);
    if (threadIdx.x == 0) *a.status = good ? STATUS_OK : STATUS_BAD_LAYOUT;
}

// Shared memory of a block's prompt: the sets of ancestors, then the key segments [preamble | kept paths | tail and nodes].  Keys are numbered so
// that every segment starts at a multiple of `pad`; numbers between a segment's end and the next one's start stand for no key.
struct TreeTable {
    struct Head { unsigned long long anc[kTreeMaxNodes]; signed char ptr[kTreeMaxNodes]; int n, committed, good, ctx; } *head;      // ctx: number of node 0
    int *lo;                                     // [k + 3]: first number of every segment, and the end
    int *end;                                    // [k + 2]: behind its last key
    int *row;                                    // [k + 2]: its first row in the cache or in the prompt's tail
    __host__ __device__ static size_t bytes(int k) { return round_up(sizeof(Head) + (3 * (size_t)k + 7) * 4, 16); }
    __device__ TreeTable(unsigned char *p, int k) : head(reinterpret_cast<Head *>(p)), lo(reinterpret_cast<int *>(p + sizeof(Head))), end(lo + k + 3), row(end + k + 2) {}

    // All threads of the block, 64 at least.  False: nothing to do for this prompt.
    __device__ bool fill(const TreeArgs &a, int b, int pad)
    {
        const int n_seg = a.k + 2, lane = threadIdx.x & 31;
        if (threadIdx.x < 32) {
            int par[2], n, committed;
            const bool good = tree_of_prompt(a, b, n, committed, par);
            unsigned long long anc[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                anc[i] = 1ull << (lane + 32 * i);
                head->anc[lane + 32 * i] = anc[i];
                head->ptr[lane + 32 * i] = (signed char)par[i];
            }
            // ancestors by doubling: after round r a set holds 2^(r+1) of them and the pointer leads to the next
            for (int span = 1; good && span < n; span *= 2) {
                __syncwarp();
                unsigned long long up[2] = {0, 0};
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (par[i] >= 0) { up[i] = head->anc[par[i]]; par[i] = head->ptr[par[i]]; }
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    anc[i] |= up[i];
                    head->anc[lane + 32 * i] = anc[i];
                    head->ptr[lane + 32 * i] = (signed char)par[i];
                }
            }
            if (lane == 0) { head->n = n; head->committed = committed; head->good = good; }
        }
        // lengths first, in end[]; the first warp is busy with the tree
        for (int s = (int)threadIdx.x - 32; threadIdx.x >= 32 && s < n_seg - 1; s += blockDim.x - 32) {
            int64_t r, len;
            tree_segment(a, b, s, r, len);
            row[s] = (int)r;
            end[s] = (int)len;
        }
        __syncthreads();
        if (!head->good || head->n == 0) return false;
        if (threadIdx.x < 32) {
            int sum = 0;
            for (int s = 0; s < n_seg - 1; s += 32) {
                const int len = s + lane < n_seg - 1 ? end[s + lane] : 0, room = (len + pad - 1) / pad * pad;
                int v = room;
#pragma unroll
                for (int o = 1; o < 32; o *= 2) { const int w = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += w; }
                if (s + lane < n_seg - 1) { lo[s + lane] = sum + v - room; end[s + lane] = sum + v - room + len; }
                sum += __shfl_sync(0xffffffffu, v, 31);
            }
            if (lane == 0) {
                row[n_seg - 1] = 0;
                lo[n_seg - 1] = sum;
                head->ctx = sum + head->committed;
                end[n_seg - 1] = lo[n_seg] = head->ctx + head->n;
            }
        }
        __syncthreads();
        return true;
    }
    // Segment of number u < lo[last]: from a segment at or before it; from nowhere.
    __device__ __forceinline__ int find(int seg, int u) const { while (u >= lo[seg + 1]) ++seg; return seg; }
    __device__ __forceinline__ int search(int u, int n_seg) const
    {
        int a = 0, b = n_seg;                    // lo[a] <= u < lo[b]
        while (b - a > 1) { const int m = (a + b) / 2; if (lo[m] <= u) a = m; else b = m; }
        return a;
    }
    // Which of the numbers u0 .. u0 + 63 stand for keys; seg: a segment at or before u0's, moved on to it.  All lanes of a warp.
    __device__ __forceinline__ unsigned long long exists(int &seg, int u0, int total) const
    {
        seg = find(seg, u0);
        if (u0 + 64 <= end[seg]) return ~0ull;
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int u = u0 + 32 * i + (threadIdx.x & 31);
            w[i] = __ballot_sync(0xffffffffu, u < total && u < end[find(seg, min(u, total - 1))]);
        }
        return w[0] | (unsigned long long)w[1] << 32;
    }
};

// Which of the keys u0 .. u0 + 63 a node sees: all of the context, its ancestors and itself, nothing behind the nodes.
__device__ __forceinline__ unsigned long long tree_sees(unsigned long long anc, int ctx, int u0)
{
    const int d = ctx - u0;                      // keys of the context from u0 on
    if (d >= 64) return ~0ull;
    if (d >= 0) return ((1ull << d) - 1) | anc << d;
    return d > -64 ? anc >> -d : 0ull;
}

__device__ __forceinline__ float ex2t(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// 16 bytes into shared memory, zeros where there is nothing.
__device__ __forceinline__ void cp_async16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Four elements as floats.
__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(__nv_bfloat16 *p, const float (&v)[4]) { *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])); }

template <int N> struct TreeConst { static constexpr int value = N; };
// Partial results of a piece of a row: outputs that are not normalised, their reference (log2 units) and sum.
struct TreePartial {
    float m, l, o[4];
    float2 ml[8];
    float4 v[8];
    template <int N, typename F> __device__ __forceinline__ void load(F at, int c, int d)           // at(i): the i-th of N to join
    {
#pragma unroll
        for (int i = 0; i < N; ++i) { const float *p = at(i); ml[i] = *reinterpret_cast<const float2 *>(p + d); v[i] = *reinterpret_cast<const float4 *>(p + c); }
    }
    template <int N> __device__ __forceinline__ void join()
    {
        m = -INFINITY;
        l = o[0] = o[1] = o[2] = o[3] = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) m = fmaxf(m, ml[i].x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (ml[i].x == -INFINITY && ml[i].y == 0.f) continue;     // keys that this row sees nothing of
            const float w = ex2t(ml[i].x - m);
            l += ml[i].y * w;
            o[0] += v[i].x * w; o[1] += v[i].y * w; o[2] += v[i].z * w; o[3] += v[i].w * w;
        }
    }
};

// Partial results of a block: [rows][D + 4] floats (outputs, reference, sum), COPIES of them, 128 / COPIES rows apart.  They are joined in the
// block, then over the cluster, whose blocks share the rows out among themselves: always in the same order, so that results do not depend on
// scheduling.  Called by all threads of all blocks; first_row: row of the prompt's (node, head of the group) sequence that row 0 stands for.
template <typename T, int D, int COPIES>
__device__ __forceinline__ void tree_merge(const TreeArgs &a, float *part, int rows, int first_row, int b, int hk)
{
    namespace cg = cooperative_groups;
    constexpr int PS = D + 4, PIECES = D / 4;
    cg::cluster_group cluster = cg::this_cluster();
    const int n = gridDim.x, me = blockIdx.x, group = a.n_heads / a.n_kv_heads;
    const auto write = [&](const TreePartial &x, int r, int c) {
        const float inv = x.l == 0.f ? 0.f : 1.f / x.l;
        const float o[4] = {x.o[0] * inv, x.o[1] * inv, x.o[2] * inv, x.o[3] * inv};
        const int g = (first_row + r) / group, h = hk * group + (first_row + r) % group;
        const int64_t at = ((int64_t)b * a.max_nodes + g) * a.n_heads + h;
        store4(static_cast<T *>(a.out) + at * D + c, o);
        if (c == 0 && a.lse) a.lse[at] = x.l == 0.f ? -INFINITY : (x.m + log2f(x.l)) * kLn2T;
    };
    __syncthreads();
    if (COPIES > 1 || n == 1) {
        for (int i = threadIdx.x; i < rows * PIECES; i += blockDim.x) {           // a row's pieces are neighbours in a warp
            const int r = i / PIECES, c = i % PIECES * 4;
            TreePartial x;
            x.load<COPIES>([&](int j) { return part + (r + j * (128 / COPIES)) * PS; }, c, D);
            x.join<COPIES>();
            if (n == 1) { write(x, r, c); continue; }
            // all pieces' threads have read reference and sum: a row's are 16 or 32 neighbouring lanes, all of which are here
            __syncwarp(PIECES == 32 ? 0xffffffffu : 0xffffu << (threadIdx.x & 16));
            float *p = part + r * PS;
            *reinterpret_cast<float4 *>(p + c) = make_float4(x.o[0], x.o[1], x.o[2], x.o[3]);
            if (c == 0) { p[D] = x.m; p[D + 1] = x.l; }
        }
    }
    if (n == 1) return;
    cluster.sync();
    // my rows: pieces of several at once, since reads from another block's shared memory take long
    const int items = (rows - me + n - 1) / n * PIECES;
    const auto mine = [&](auto shares, auto at_once) {
        constexpr int N = decltype(shares)::value, U = decltype(at_once)::value;
        for (int i0 = threadIdx.x; i0 < items; i0 += U * blockDim.x) {
            TreePartial x[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = min(i0 + k * (int)blockDim.x, items - 1), r = me + i / PIECES * N, c = i % PIECES * 4;
                x[k].template load<N>([&](int s) { return cluster.map_shared_rank(part, s) + r * PS; }, c, D);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int i = i0 + k * (int)blockDim.x;
                if (i < items) { x[k].template join<N>(); write(x[k], me + i / PIECES * N, i % PIECES * 4); }
            }
        }
    };
    if (n == 2) mine(TreeConst<2>{}, TreeConst<4>{}); else if (n == 4) mine(TreeConst<4>{}, TreeConst<2>{}); else mine(TreeConst<8>{}, TreeConst<1>{});
    cluster.sync();                              // nobody leaves while its shared memory is read
}

int launch_tree_tc(const TreeArgs &a, int head_dim, int64_t max_keys, cudaStream_t st);       // decode_tree_tc.cu

}  // namespace sp
