// sp_tree_accept: the walk down a tree of drafted tokens as far as drafts and samples agree, and the K / V rows of the nodes on it moved
// together in the tails of all layers, in place.
//
// Latency-sized: a few rows of every layer.  One launch does both: every block walks its prompt's tree itself (a warp, two nodes per lane, a
// ballot per step) and then moves its share of the columns.  A thread owns 16 bytes of a row and takes the moves in ascending order, four loads
// before four stores: node j of the path goes to row j <= its own, so what a store overwrites has been read, by the same thread.
// 64 prompts x 32 nodes, 16 layers of 8 x 128: 5.3 us, of which launch and the walk's dependent loads are all but 1.6 (the moved rows' bytes).
#include <cstdlib>

#include "common.cuh"

namespace sp {

constexpr int kAccThreads = 256, kAccMaxNodes = 64;

struct AcceptArgs {
    const int32_t *draft, *sampled, *parent, *n_nodes, *tail_len;
    int32_t *path, *n_accepted, *next_token, *new_tail_len;
    unsigned char *tail_k, *tail_v;
    int64_t layer_bytes;
    int max_nodes, tail_cap, n_layers, row_vecs;             // row_vecs: 16-byte pieces of a row
};

__global__ void __launch_bounds__(kAccThreads) tree_accept_kernel(const __grid_constant__ AcceptArgs a)
{
    __shared__ int moves[kAccMaxNodes], n_moves, first_move, base;            // from moves[i] to first_move + i
    pdl_wait();
    const int b = blockIdx.y;
    if (threadIdx.x < 32) {
        const int lane = threadIdx.x;
        int n = a.n_nodes ? a.n_nodes[b] : a.max_nodes;
        const int len = a.tail_len ? a.tail_len[b] : 0;
        if (n < 0 || n > a.max_nodes || (a.tail_len && (len < 0 || (int64_t)len + n > a.tail_cap))) n = 0;
        const int64_t at0 = (int64_t)b * a.max_nodes;
        int par[2] = {-2, -2}, draft[2] = {0, 0}, got[2] = {0, 0}, line[2] = {-1, -1};
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (lane + 32 * i < n) { par[i] = a.parent[at0 + lane + 32 * i]; draft[i] = a.draft[at0 + lane + 32 * i]; got[i] = a.sampled[at0 + lane + 32 * i]; }
        int at = 0, count = 0, token = -1, first = kAccMaxNodes;
        while (count < n) {
            if (lane == (count & 31)) line[count >> 5] = at;
            if (first == kAccMaxNodes && at != count) first = count;
            ++count;
            token = at < 32 ? __shfl_sync(0xffffffffu, got[0], at) : __shfl_sync(0xffffffffu, got[1], at - 32);
            const uint32_t lo = __ballot_sync(0xffffffffu, lane > at && par[0] == at && draft[0] == token);
            const uint32_t hi = __ballot_sync(0xffffffffu, lane + 32 > at && par[1] == at && draft[1] == token);
            if (!(lo | hi)) break;
            at = lo ? __ffs(lo) - 1 : 31 + __ffs(hi);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int j = lane + 32 * i;
            if (j >= first && j < count) moves[j - first] = line[i];
            if (blockIdx.x == 0 && j < a.max_nodes) a.path[at0 + j] = line[i];
        }
        if (lane == 0) {
            n_moves = first < count ? count - first : 0;
            first_move = first;
            base = len;
            if (blockIdx.x == 0) {
                a.n_accepted[b] = count;
                a.next_token[b] = token;
                if (a.new_tail_len) a.new_tail_len[b] = len + count;
            }
        }
    }
    __syncthreads();
    const int n = n_moves;
    if (n == 0) return;
    const int64_t row_bytes = (int64_t)a.row_vecs * 16, from = ((int64_t)b * a.tail_cap + base) * row_bytes;
    const int64_t columns = 2LL * a.n_layers * a.row_vecs;
    for (int64_t c = (int64_t)blockIdx.x * kAccThreads + threadIdx.x; c < columns; c += (int64_t)gridDim.x * kAccThreads) {
        const int64_t tensor = c / a.row_vecs;
        unsigned char *p = (tensor & 1 ? a.tail_v : a.tail_k) + (tensor >> 1) * a.layer_bytes + from + (c - tensor * a.row_vecs) * 16;
        for (int i = 0; i < n; i += 4) {
            uint4 w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) if (i + e < n) w[e] = *reinterpret_cast<const uint4 *>(p + moves[i + e] * row_bytes);
#pragma unroll
            for (int e = 0; e < 4; ++e) if (i + e < n) *reinterpret_cast<uint4 *>(p + (first_move + i + e) * row_bytes) = w[e];
        }
    }
}

}  // namespace sp

extern "C" int sp_tree_accept(const int32_t *draft, const int32_t *sampled, const int32_t *parent, const int32_t *n_nodes,
                              int n_prompts, int max_nodes, int32_t *path, int32_t *n_accepted, int32_t *next_token,
                              void *tail_k, void *tail_v, const int32_t *tail_len, int32_t *new_tail_len, int tail_cap,
                              int n_layers, int64_t ld_layer, int n_kv_heads, int head_dim, int dtype, void *stream)
{
    using namespace sp;
    SP_REQUIRE(dtype == SP_F32 || dtype == SP_BF16, SP_ERR_INVALID_ARG, "sp_tree_accept: unknown dtype %d", dtype);
    SP_REQUIRE(n_prompts >= 0 && max_nodes >= 0 && n_layers >= 0 && tail_cap >= 0, SP_ERR_INVALID_ARG, "sp_tree_accept: negative size");
    SP_REQUIRE(max_nodes <= kAccMaxNodes, SP_ERR_UNSUPPORTED, "sp_tree_accept: %d nodes (at most %d supported)", max_nodes, kAccMaxNodes);
    SP_REQUIRE(n_prompts <= 65535, SP_ERR_UNSUPPORTED, "sp_tree_accept: more than 65535 prompts");
    if (n_prompts == 0) return SP_OK;
    SP_REQUIRE(n_accepted && next_token, SP_ERR_INVALID_ARG, "sp_tree_accept: NULL pointer");
    SP_REQUIRE(max_nodes == 0 || (draft && sampled && parent && path), SP_ERR_INVALID_ARG, "sp_tree_accept: NULL pointer");
    SP_REQUIRE((tail_len == nullptr) == (new_tail_len == nullptr), SP_ERR_INVALID_ARG, "sp_tree_accept: tail_len and new_tail_len come together");
    int64_t row_bytes = 0;
    if (n_layers > 0) {
        SP_REQUIRE(tail_k && tail_v && tail_len, SP_ERR_INVALID_ARG, "sp_tree_accept: tail pointers are NULL with n_layers > 0");
        SP_REQUIRE(n_kv_heads > 0 && head_dim > 0, SP_ERR_INVALID_ARG, "sp_tree_accept: bad n_kv_heads / head_dim");
        row_bytes = (int64_t)n_kv_heads * head_dim * elt_bytes(dtype);
        SP_REQUIRE(row_bytes % 16 == 0 && row_bytes < (1 << 24), SP_ERR_UNSUPPORTED, "sp_tree_accept: rows of %lld bytes", (long long)row_bytes);
        SP_REQUIRE(aligned16(tail_k) && aligned16(tail_v), SP_ERR_INVALID_ARG, "sp_tree_accept: tails must be 16-byte aligned");
        SP_REQUIRE(n_layers == 1 || (ld_layer >= (int64_t)n_prompts * tail_cap * n_kv_heads * head_dim && ld_layer * elt_bytes(dtype) % 16 == 0),
                   SP_ERR_INVALID_ARG, "sp_tree_accept: ld_layer %lld is too small or not a multiple of 16 bytes", (long long)ld_layer);
        // K and V of two layers l and m lie |d + (m - l) stride| apart: of the differences m - l the two nearest to -d / stride
        const int64_t size = (int64_t)n_prompts * tail_cap * row_bytes, stride = n_layers > 1 ? ld_layer * elt_bytes(dtype) : 0;
        const int64_t d = static_cast<char *>(tail_v) - static_cast<char *>(tail_k);
        bool apart = stride || std::abs(d) >= size;
        for (int64_t j = stride ? d / stride - 1 : 0; stride && j <= d / stride + 1; ++j)
            apart &= std::abs(j) >= n_layers || std::abs(d - j * stride) >= size;
        SP_REQUIRE(apart, SP_ERR_INVALID_ARG, "sp_tree_accept: the K and V tails overlap");
    }
    // every block reads the inputs and one writes the outputs
    const struct { const void *p; int64_t n; } in[] = {{draft, max_nodes}, {sampled, max_nodes}, {parent, max_nodes}, {n_nodes, 1}, {tail_len, 1}},
                                               to[] = {{path, max_nodes}, {n_accepted, 1}, {next_token, 1}, {new_tail_len, 1}};
    for (const auto &o : to)
        for (const auto &i : in) {
            const char *x = static_cast<const char *>(o.p), *y = static_cast<const char *>(i.p);
            SP_REQUIRE(!x || !y || x + 4 * o.n * n_prompts <= y || y + 4 * i.n * n_prompts <= x, SP_ERR_INVALID_ARG,
                       "sp_tree_accept: outputs must not overlap the inputs");
        }
    AcceptArgs a = {};
    a.draft = draft; a.sampled = sampled; a.parent = parent; a.n_nodes = n_nodes; a.tail_len = tail_len;
    a.path = path; a.n_accepted = n_accepted; a.next_token = next_token; a.new_tail_len = new_tail_len;
    a.tail_k = static_cast<unsigned char *>(tail_k); a.tail_v = static_cast<unsigned char *>(tail_v);
    a.layer_bytes = ld_layer * elt_bytes(dtype);
    a.max_nodes = max_nodes; a.n_layers = n_layers; a.row_vecs = (int)(row_bytes / 16);
    a.tail_cap = n_layers > 0 ? tail_cap : INT32_MAX;       // lengths alone need no room, but have to stay numbers
    // a column per thread, as far as eight blocks per SM go
    const int64_t columns = 2LL * n_layers * a.row_vecs, want = (columns + kAccThreads - 1) / kAccThreads;
    const int64_t most = std::max<int64_t>(1, 8LL * num_sms() / n_prompts);
    return launch(tree_accept_kernel, dim3((unsigned)std::max<int64_t>(1, std::min(want, most)), n_prompts), kAccThreads, 0,
                  static_cast<cudaStream_t>(stream), 1, a);
}
