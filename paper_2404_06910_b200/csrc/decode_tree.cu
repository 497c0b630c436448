// sp_pruned_decode_tree: attention of a tree of drafted tokens over the pruned cache (Section 3.2.3, Algorithm 3: the response attends to
// the preamble, the kept paths and the response so far; here several candidates for its next tokens do so at once).
//
// Every node sees the same context and, of the nodes, its ancestors and itself.  The context's K and V are read once for all nodes and all
// query heads of a KV head: with N nodes and G heads per KV head a step has N G flop per byte where a single token has G.
//
// bf16 runs in decode_tree_tc.cu.  The kernel here serves fp32 (the reference type, small problems): a block takes 16 rows of (node, head of the
// group) and a share of the keys, 32 keys at a time through a double buffer in shared memory; half a warp owns a row: each lane has two keys' scores
// and D / 16 columns of the output.  Products run in fp32 FMA from shared memory, two 16-byte reads for eight of them, which bounds it where there
// are many keys; key shares of a row tile are the blocks of a cluster.  One prompt of 70 keys, 6 nodes, 4 heads of 64: 8.5 us, of which launch and
// dependent index loads are some 6.
#include "decode_tree.cuh"

namespace sp {

constexpr int kTsRows = 16, kTsKeys = 32, kTsThreads = 256;
constexpr int kTsMaxSmem = 200 * 1024;          // allowed to the kernel once and for all: see kDecMaxSmem in decode.cu

template <int D> struct TsConfig {
    static constexpr int KS = D + 4, TILE = kTsKeys * KS;      // elements of a row in shared memory: 16 bytes off, so that eight lanes' pieces meet no bank twice
    static constexpr size_t KV_OFF = kTsRows * KS * 4, P_OFF = KV_OFF + 4 * TILE * 4, TABLE_OFF = P_OFF + kTsRows * kTsKeys * 4;
    static_assert(4 * TILE >= kTsRows * KS, "the partial result takes the place of the tiles");
};

template <int D>
__global__ void __launch_bounds__(kTsThreads) tree_simt_kernel(const __grid_constant__ TreeArgs a)
{
    using C = TsConfig<D>;
    constexpr int NC = D / 64;                   // pieces of 4 columns per lane
    extern __shared__ __align__(16) unsigned char smem_raw[];
    float *sq = reinterpret_cast<float *>(smem_raw), *s_p = reinterpret_cast<float *>(smem_raw + C::P_OFF);
    float *skv = reinterpret_cast<float *>(smem_raw + C::KV_OFF);
    pdl_wait();
    if (blockIdx.z == 0) { tree_report(a); return; }
    TreeTable table(smem_raw + C::TABLE_OFF, a.k);
    const int b = blockIdx.z - 1, hk = blockIdx.y % a.n_kv_heads, first_row = blockIdx.y / a.n_kv_heads * kTsRows;
    if (!table.fill(a, b, 1)) return;               // the same for all blocks of the cluster
    const int group = a.n_heads / a.n_kv_heads, rows = min(table.head->n * group - first_row, kTsRows);
    if (rows <= 0) return;
    const int n_seg = a.k + 2, ctx = table.head->ctx, total = table.lo[n_seg];
    const int tiles = (total + kTsKeys - 1) / kTsKeys, t0 = (int)((int64_t)tiles * blockIdx.x / gridDim.x), t1 = (int)((int64_t)tiles * (blockIdx.x + 1) / gridDim.x);

    // a thread copies one 16-byte piece of every RPT-th key row
    constexpr int N = 4, PIECES = D / N, RPT = kTsThreads / PIECES, PASSES = kTsKeys / RPT;
    const int piece = threadIdx.x % PIECES, row0 = threadIdx.x / PIECES;
    const int64_t kv_row = (int64_t)a.n_kv_heads * D;
    const float *kc = static_cast<const float *>(a.k_cache) + hk * D, *vc = static_cast<const float *>(a.v_cache) + hk * D;
    const float *tk = static_cast<const float *>(a.tail_k) + (int64_t)b * a.tail_cap * kv_row + hk * D;
    const float *tv = static_cast<const float *>(a.tail_v) + (int64_t)b * a.tail_cap * kv_row + hk * D;
    auto load = [&](int t) {
        float *dst = skv + (t & 1) * 2 * C::TILE;
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
            const int r = row0 + i * RPT, u = t * kTsKeys + r;
            const float *ks = kc, *vs = vc;
            if (u < total) {
                const int s = table.search(u, n_seg);
                const int64_t off = ((int64_t)table.row[s] + (u - table.lo[s])) * kv_row;
                ks = (s == n_seg - 1 ? tk : kc) + off;
                vs = (s == n_seg - 1 ? tv : vc) + off;
            }
            cp_async16(ptx::smem_u32(dst + r * C::KS + piece * N), ks + piece * N, u < total);
            cp_async16(ptx::smem_u32(dst + C::TILE + r * C::KS + piece * N), vs + piece * N, u < total);
        }
        cp_async_commit();
    };
    if (t0 < t1) load(t0);
    for (int i = threadIdx.x; i < kTsRows * (D / 4); i += kTsThreads) {           // queries; rows that do not exist: zeros
        const int r = i / (D / 4), c = i % (D / 4) * 4, gr = first_row + r;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows) v = load4(static_cast<const float *>(a.q) + (((int64_t)b * a.max_nodes + gr / group) * a.n_heads + hk * group + gr % group) * D + c);
        *reinterpret_cast<float4 *>(sq + r * C::KS + c) = v;
    }
    const int r = threadIdx.x / 16, sub = threadIdx.x % 16;
    const unsigned long long anc = r < rows ? table.head->anc[(first_row + r) / group] : 0ull;
    const float *qr = sq + r * C::KS;
    float *pr = s_p + r * kTsKeys;
    float m = -INFINITY, l = 0.f, acc[NC][4] = {};
    for (int t = t0; t < t1; ++t) {
        if (t + 1 < t1) { load(t + 1); cp_async_wait<1>(); } else cp_async_wait<0>();
        __syncthreads();
        const float *kt = skv + (t & 1) * 2 * C::TILE, *vt = kt + C::TILE;
        float s[2] = {0.f, 0.f};
#pragma unroll 8
        for (int c = 0; c < D; c += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(qr + c);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float4 k = load4(kt + (sub + 16 * i) * C::KS + c);
                s[i] = fmaf(q.x, k.x, s[i]); s[i] = fmaf(q.y, k.y, s[i]); s[i] = fmaf(q.z, k.z, s[i]); s[i] = fmaf(q.w, k.w, s[i]);
            }
        }
        const unsigned long long sees = tree_sees(anc, ctx, t * kTsKeys);
        bool seen[2];
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            seen[i] = sees >> (sub + 16 * i) & 1 && t * kTsKeys + sub + 16 * i < total;
            s[i] = seen[i] ? s[i] * a.scale_log2e : -INFINITY;
            top = fmaxf(top, s[i]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (top > m) {
            const float f = ex2t(m - top);
            l *= f;
#pragma unroll
            for (int i = 0; i < NC; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][e] *= f;
            m = top;
        }
        const float minus = m == -INFINITY ? 0.f : -m;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float p = ex2t(s[i] + minus);
            if (seen[i]) l += p;
            pr[sub + 16 * i] = seen[i] ? p : -1.f;                    // a key that is not seen is left out: its V may hold anything
        }
        __syncwarp();
#pragma unroll 4
        for (int j = 0; j < kTsKeys; ++j) {
            const float p = pr[j];
            if (p < 0.f) continue;
#pragma unroll
            for (int i = 0; i < NC; ++i) {
                const float4 v = load4(vt + j * C::KS + sub * 4 + 64 * i);
                acc[i][0] = fmaf(p, v.x, acc[i][0]); acc[i][1] = fmaf(p, v.y, acc[i][1]);
                acc[i][2] = fmaf(p, v.z, acc[i][2]); acc[i][3] = fmaf(p, v.w, acc[i][3]);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    float *part = reinterpret_cast<float *>(smem_raw + C::KV_OFF);
#pragma unroll
    for (int i = 0; i < NC; ++i) *reinterpret_cast<float4 *>(part + r * (D + 4) + sub * 4 + 64 * i) = make_float4(acc[i][0], acc[i][1], acc[i][2], acc[i][3]);
    if (sub == 0) { part[r * (D + 4) + D] = m; part[r * (D + 4) + D + 1] = l; }
    tree_merge<float, D, 1>(a, part, rows, first_row, b, hk);
}

template <int D> static int launch_tree_simt(const TreeArgs &a, int64_t max_keys, cudaStream_t st)
{
    const int group = a.n_heads / a.n_kv_heads, row_tiles = (a.max_nodes * group + kTsRows - 1) / kTsRows;
    const size_t smem = TsConfig<D>::TABLE_OFF + TreeTable::bytes(a.k);
    SP_REQUIRE(smem <= kTsMaxSmem, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: k = %d needs too much shared memory", a.k);
    // Shares of the keys: as many as two blocks per SM allow, eight at most, two tiles at least.
    const int64_t units = (int64_t)row_tiles * a.n_kv_heads * a.n_prompts;
    int n = 1;
    while (n < 8 && 2 * n * units <= 2 * num_sms() && 2 * n * 2 * kTsKeys <= max_keys) n *= 2;
    SP_CUDA(cudaFuncSetAttribute(tree_simt_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTsMaxSmem));
    return launch(tree_simt_kernel<D>, dim3(n, row_tiles * a.n_kv_heads, a.n_prompts + 1), kTsThreads, smem, st, n, a);
}

}  // namespace sp

extern "C" size_t sp_decode_tree_workspace_bytes(int n_prompts, int max_nodes, int n_heads, int head_dim)
{
    (void)n_prompts; (void)max_nodes; (void)n_heads; (void)head_dim;
    return 256;                                  // the status word: partial results are merged in shared memory
}

extern "C" int sp_pruned_decode_tree(const void *q, const void *k_cache, const void *v_cache, const sp_layout *lay,
                                     const int32_t *kept_idx, int k, const void *tail_k, const void *tail_v,
                                     const int32_t *tail_len, int tail_cap, const int32_t *parent, const int32_t *n_nodes,
                                     int max_nodes, int64_t max_keys, int n_heads, int n_kv_heads, int head_dim, float scale,
                                     void *out, float *lse, void *ws, size_t ws_bytes, int dtype, void *stream)
{
    using namespace sp;
    SP_REQUIRE(dtype == SP_F32 || dtype == SP_BF16, SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: unknown dtype %d", dtype);
    if (int rc = check_layout(lay)) return rc;
    SP_REQUIRE(head_dim == 64 || head_dim == 128, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: head_dim %d (64 or 128 supported)", head_dim);
    SP_REQUIRE(n_heads > 0 && n_kv_heads > 0 && n_heads % n_kv_heads == 0, SP_ERR_INVALID_ARG,
               "sp_pruned_decode_tree: n_heads %d must be a positive multiple of n_kv_heads %d", n_heads, n_kv_heads);
    SP_REQUIRE(k >= 0 && k <= 4096, SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: k %d out of range [0, 4096]", k);
    SP_REQUIRE(max_nodes >= 0 && tail_cap >= 0 && max_keys >= 0, SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: negative max_nodes / tail_cap / max_keys");
    SP_REQUIRE(max_nodes <= kTreeMaxNodes, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: %d nodes (at most %d supported)", max_nodes, kTreeMaxNodes);
    SP_REQUIRE(lay->n_prompts <= 65534, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: more than 65534 prompts");
    SP_REQUIRE((int64_t)max_nodes * n_heads <= 65535, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: more than 65535 rows of nodes and heads");
    if (lay->n_prompts == 0 || max_nodes == 0) return SP_OK;
    SP_REQUIRE(q && out, SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: q / out is NULL");
    SP_REQUIRE(k_cache && v_cache, SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: cache pointer is NULL");
    SP_REQUIRE(k == 0 || kept_idx, SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: kept_idx is NULL with k > 0");
    SP_REQUIRE(tail_k && tail_v && tail_len && parent, SP_ERR_INVALID_ARG,
               "sp_pruned_decode_tree: the nodes' keys lie in the tail: tail_k, tail_v, tail_len and parent are required");
    SP_REQUIRE(aligned16(q) && aligned16(out) && aligned16(k_cache) && aligned16(v_cache) && aligned16(tail_k) && aligned16(tail_v),
               SP_ERR_INVALID_ARG, "sp_pruned_decode_tree: data pointers must be 16-byte aligned");
    const int64_t bound = (int64_t)lay->max_pre_len + (int64_t)k * lay->max_path_len + tail_cap;
    // Numbers of keys are 32 bits: with the gaps that TreeTable leaves in front of multiples of kTtPad, and what a tile reaches behind the last one.
    const int64_t numbers = bound + (dtype == SP_BF16 ? (int64_t)(kTtPad - 1) * (k + 1) : 0);
    SP_REQUIRE(numbers < (int64_t)INT32_MAX - 256, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: up to %lld keys per prompt", (long long)bound);
    SP_REQUIRE(ws && aligned256(ws) && ws_bytes >= sp_decode_tree_workspace_bytes(lay->n_prompts, max_nodes, n_heads, head_dim), SP_ERR_WORKSPACE,
               "sp_pruned_decode_tree: workspace of %zu bytes (256-byte aligned) required", sp_decode_tree_workspace_bytes(lay->n_prompts, max_nodes, n_heads, head_dim));

    TreeArgs a;
    a.q = q; a.k_cache = k_cache; a.v_cache = v_cache; a.tail_k = tail_k; a.tail_v = tail_v;
    a.ppo = lay->prompt_path_off; a.pre_start = lay->pre_start; a.pre_len = lay->pre_len;
    a.path_start = lay->path_start; a.doc_len = lay->doc_len; a.qry_len = lay->qry_len;
    a.kept_idx = kept_idx; a.tail_len = tail_len; a.parent = parent; a.n_nodes = n_nodes;
    a.out = out; a.lse = lse; a.status = static_cast<uint32_t *>(ws);
    a.k = k; a.tail_cap = tail_cap; a.max_nodes = max_nodes; a.n_heads = n_heads; a.n_kv_heads = n_kv_heads;
    a.n_prompts = lay->n_prompts; a.n_paths = lay->n_paths; a.max_pre_len = lay->max_pre_len; a.max_path_len = lay->max_path_len;
    a.total_tokens = lay->total_tokens; a.scale_log2e = scale * kLog2eT;
    if (max_keys == 0 || max_keys > bound) max_keys = bound;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == SP_BF16) return launch_tree_tc(a, head_dim, max_keys, st);
    return head_dim == 128 ? launch_tree_simt<128>(a, max_keys, st) : launch_tree_simt<64>(a, max_keys, st);
}
