// sp_pruned_decode_tree in bf16: both products on tcgen05.
//
// A block takes up to 128 rows of (node, query head of the group), all of which read the same keys, and a share of those:
//   S [rows x 64 keys] = Q K^T     tcgen05.mma, Q and K from shared memory
//   P                              a thread per row: the row's 64 scores in registers, no exchange; P as the sum of two bf16 numbers over S
//   O [rows x D] += P V            tcgen05.mma, P from tensor memory, V as it lies (MN-major)
// Two bf16 numbers hold 16 bits of P.  Over 760 random keys that is 4.5e-6 of the output's norm, where fp32 weights are 4e-7 and the rounding of the
// output to bf16 1.65e-3, of which it changes nothing: one element in 240 goes to its other neighbour.  A third number would make the second product
// half as long again, and has no room: scores, P and O of two blocks are all of the tensor memory's 512 columns.
// With few rows most of the 128 are empty, which costs nothing that shows: per 64 keys the products take some 400 clk and a row's softmax about
// 1 000, where the keys' 32 KB take 1 350 clk of half an SM's share of HBM.  Two blocks share an SM, so that one's start, chain and end lie under
// the other's loads.
// Keys are numbered so that every segment starts at a multiple of eight (TreeTable), and arrive by TMA in slots K0 V0 K1 V1 ... of a ring: a tile
// inside one segment as one box, other tiles as boxes of 32, 16 and 8 rows, which may bring up to seven rows along that nobody needs.
// (Gathered by cp.async the rows kept the loading warps busy, 107 clk per instruction and warp, and as TMA gathers of four rows too, 74 clk
// each: 64 prompts x 16 nodes 285 and 271 us.)
// 64 prompts x 16 nodes, 32 heads of 128, eight tiles a unit: 141 us, 3.7 TB/s, bound by the units' starts and ends; contexts of 7 900 keys stream at
// 0.9 of the copy bandwidth.  Heads of 64 have half the bytes and the same softmax, starts and ends: 0.77 of the time (cold L2: 115 us against 150).
// Key shares of a row tile are the blocks of a cluster, merged as in decode_tree.cuh.
// What a row does not see has P = 0, and 0 x Inf would reach O all the same.  So tiles of V with the end of a segment or nodes are cleaned first:
// rows that stand for no key become zeros; values of nodes that are not finite are taken out, and added at the end by the
// rows that see them.
// Roles: warps 0-3 queries, softmax and output, 4 loads, 5 cleaning, 6 products.  Every mbarrier wait is bounded: on expiry the block records a
// timeout in the workspace status word and unwinds.
#include "decode_tree.cuh"
#include "tensor_map.cuh"

namespace sp {

using namespace ptx;

extern bool g_stall_producer;                 // test hook, see prefill_tc.cu

constexpr int kTtLoadWarp = 4, kTtCleanWarp = 5, kTtMmaWarp = 6, kTtThreads = 224;
constexpr int kTtKeys = 64, kTtMaxSlots = 12;
constexpr int kTtTmem = 256;                  // columns: two S / P buffers of 64, O
constexpr int kTtHalfSm = 228 * 1024 / 2 - 1024, kTtMaxSmem = 227 * 1024;

struct TreeTcArgs {
    CUtensorMap cache[2][4], tail[2][4];      // [K, V][box: a whole tile, 32, 16, 8 rows x 64 columns]
    TreeArgs t;
    int tile_rows, n_slots, stall;            // rows of a tile, slots of the ring
    uint32_t q_and, q_xor;                    // two queries' bits: a negative scale is positive with negated queries, a scale of zero any with zeros
};
struct TreeTcShared {
    uint64_t full[kTtMaxSlots], empty[kTtMaxSlots], clean[kTtMaxSlots], s_full[2], p_ready[2], o_done[2], q_full, drain;
    unsigned long long not_finite;            // nodes with values that are not finite, of this block's keys
    uint32_t tmem;
};

// D[tmem] (+)= A[tmem] * B[smem] where the lanes whose bit in `off` (a word per lane quarter) is set keep what they hold.
__device__ __forceinline__ void umma_ts_lanes(uint32_t lead, uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate, const uint32_t (&off)[4])
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %5, 0;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%6, %7, %8, %9}, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead), "r"(off[0]), "r"(off[1]), "r"(off[2]), "r"(off[3]) : "memory");
}
// Largest of three, NaN left out.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Two bf16 numbers: a mask over those that are not finite.
__device__ __forceinline__ uint32_t bf16_not_finite(uint32_t w)
{
    return ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u) | ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u);
}

// Softmax of a warp: `copies` warps share the 64 keys of a tile for the same rows (each lane quarter of the tile then holds the same queries), so
// that few rows still keep four warps busy.  A copy has its own reference, sum and output, whose lanes only the products over its keys update; copies
// are merged like key shares.
template <int D, int COPIES> struct TreeSoftmax {
    static constexpr int W = kTtKeys / COPIES;               // keys of this warp
    // P of the slice's keys over their scores: per 16 keys 8 columns of high numbers, then 8 of low ones
    __device__ __forceinline__ static void weigh(uint32_t buf, const uint32_t (&s)[W], uint64_t scale2, float minus, uint64_t (&l2)[2])
    {
        const uint64_t minus2 = pack_f32x2(minus, minus);
#pragma unroll
        for (int h = 0; h < W; h += 16) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                float x, y;
                unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[h + i]), __uint_as_float(s[h + i + 1])), scale2, minus2), x, y);
                x = ex2t(x);
                y = ex2t(y);
                l2[i / 2 & 1] = add_f32x2(l2[i / 2 & 1], pack_f32x2(x, y));
                split_bf16(x, y, w[i / 2], w[8 + i / 2]);
            }
            tmem_st16(buf + h, w);
        }
    }
    // false: a wait ran out
    __device__ __forceinline__ static bool run(TreeTcShared &sh, uint32_t t_lane, int slice, int steps, int t0, const TreeTable &table, int n_seg, unsigned long long anc, float scale, float &m, float &l)
    {
        bool ok = true;
        uint64_t l2[2] = {0ull, 0ull};           // the sum in four parts
        const uint64_t scale2 = pack_f32x2(scale, scale);
        const int lane = threadIdx.x & 31, ctx = table.head->ctx, total = table.lo[n_seg];
        int seg = steps > 0 ? table.search(t0 * kTtKeys, n_seg) : 0;
#pragma unroll 1
        for (int g = 0; g < steps; ++g) {
            const uint32_t buf = t_lane + (g & 1) * kTtKeys;
            const unsigned long long sees = (tree_sees(anc, ctx, (t0 + g) * kTtKeys) & table.exists(seg, (t0 + g) * kTtKeys, total)) >> (slice * W);
            if (!(ok = mbar_wait_warp(&sh.s_full[g & 1], g >> 1 & 1))) break;
            tc_fence_after();
            uint32_t s[W];
            if constexpr (W == 16) tmem_ld16(buf + slice * W, s);
            else
#pragma unroll
                for (int i = 0; i < W; i += 32) tmem_ld32(buf + slice * W + i, reinterpret_cast<uint32_t (&)[32]>(s[i]));
            tmem_ld_wait();
            const bool whole = W == 64 ? sees == ~0ull : (sees & ((1ull << (W & 63)) - 1)) == (1ull << (W & 63)) - 1;
            if (!__all_sync(0xffffffffu, whole)) {
#pragma unroll
                for (int i = 0; i < W; ++i) s[i] = (uint32_t)(sees >> (i & 32)) >> (i & 31) & 1 ? s[i] : 0xff800000u;
            }
            // (the scale is not negative: see the queries)
            float tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < W; i += 8)
#pragma unroll
                for (int j = 0; j < 4; ++j) tops[j] = max3(tops[j], __uint_as_float(s[i + 2 * j]), __uint_as_float(s[i + 2 * j + 1]));
            const float top = max3(fmaxf(tops[0], tops[1]), tops[2], tops[3]) * scale;
            // the reference moves only when it has to: a weight may be up to 2^8
            const bool grown = top > m + 8.f || (m == -INFINITY && top > m);
            if (__any_sync(0xffffffffu, grown)) {
                const float now = grown ? top : m, f = grown ? ex2t(m - now) : 1.f;
                m = now;
                l2[0] = mul_f32x2(l2[0], pack_f32x2(f, f));
                l2[1] = mul_f32x2(l2[1], pack_f32x2(f, f));
                if (g > 0) {
                    if (!(ok = mbar_wait_warp(&sh.o_done[(g - 1) & 1], (g - 1) >> 1 & 1))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c = 0; c < D; c += 16) {
                        uint32_t o[16];
                        tmem_ld16(t_lane + 2 * kTtKeys + c, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        tmem_st16(t_lane + 2 * kTtKeys + c, o);
                    }
                }
            }
            const float minus = m == -INFINITY ? 0.f : -m;
            weigh(buf + slice * W, s, scale2, minus, l2);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.p_ready[g & 1]);
        }
        float x, y;
        unpack_f32x2(add_f32x2(l2[0], l2[1]), x, y);
        l = x + y;
        if (steps > 0) ok = ok && mbar_wait_warp(&sh.o_done[(steps - 1) & 1], (steps - 1) >> 1 & 1);
        tc_fence_after();
        return ok;
    }
};

template <int D>
__global__ void __launch_bounds__(kTtThreads, 2) tree_tc_kernel(const __grid_constant__ TreeTcArgs p)
{
    constexpr int SLOT = kTtKeys * D * 2, PIECES = D / 8;         // bytes of a tile of K or V; 16-byte pieces of a row
    extern __shared__ __align__(1024) unsigned char smem[];
    const TreeArgs &a = p.t;
    unsigned char *ring = smem + 128 * D * 2;    // behind the queries
    TreeTcShared &sh = *reinterpret_cast<TreeTcShared *>(ring + p.n_slots * SLOT);
    TreeTable table(reinterpret_cast<unsigned char *>(&sh) + round_up(sizeof(TreeTcShared), 16), a.k);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x < kTtMaxSlots) {
        mbar_init(&sh.full[threadIdx.x], 1); mbar_init(&sh.empty[threadIdx.x], 2); mbar_init(&sh.clean[threadIdx.x], 1);
        if (threadIdx.x < 2) { mbar_init(&sh.s_full[threadIdx.x], 1); mbar_init(&sh.p_ready[threadIdx.x], 4); mbar_init(&sh.o_done[threadIdx.x], 1); }
        if (threadIdx.x == 0) { mbar_init(&sh.q_full, 4); mbar_init(&sh.drain, 1); sh.not_finite = 0ull; }
        fence_mbar_init();
    } else if (threadIdx.x >= 32 && threadIdx.x < 48) {
        prefetch_tmap(&p.cache[0][0] + (threadIdx.x - 32));
    }
    pdl_wait();
    if (blockIdx.z == 0) { tree_report(a); return; }
    const int b = blockIdx.z - 1, hk = blockIdx.y % a.n_kv_heads, first_row = blockIdx.y / a.n_kv_heads * p.tile_rows;
    // Tensor memory is taken behind pdl_wait() and given back before the cluster's barrier: no block holds it while it waits for another.  Two
    // blocks of this kernel fit on an SM, whose 512 columns are enough for both.
    if (warp == kTtMmaWarp) { tmem_alloc(&sh.tmem, kTtTmem); tmem_relinquish(); }
    tc_fence_before();
    const bool some = table.fill(a, b, kTtPad);       // the same for all blocks of the cluster, as is rows; two barriers, behind which barriers and tensor memory are everybody's
    const int group = a.n_heads / a.n_kv_heads, rows = some ? min(table.head->n * group - first_row, p.tile_rows) : 0;
    if (rows <= 0) {
        if (warp == kTtMmaWarp) tmem_dealloc(sh.tmem, kTtTmem);
        return;
    }
    const int copies = rows <= 32 ? 4 : (rows <= 64 ? 2 : 1), stride = 128 / copies;
    const int n_seg = a.k + 2, ctx = table.head->ctx, total = table.lo[n_seg], committed = table.head->committed;
    const int tiles = (total + kTtKeys - 1) / kTtKeys;
    const int t0 = (int)((uint32_t)tiles * blockIdx.x / gridDim.x), t1 = (int)((uint32_t)tiles * (blockIdx.x + 1) / gridDim.x);       // at most 2^25 tiles, 8 shares
    const int steps = t1 - t0;
    // V rows of a tile that do not all stand for keys which every row sees; seg: as for exists()
    const auto needs_cleaning = [&](int &seg, int u0) { seg = table.find(seg, u0); return u0 + kTtKeys > min(ctx, table.end[seg]); };
    const auto key_steps = [&](int u0) { return (min(total - u0, kTtKeys) + 15) >> 4; };        // of 16 keys that the tile's products take
    const int seg0 = steps > 0 ? table.search(t0 * kTtKeys, n_seg) : 0;

    // softmax warps: their rows, and which of the keys of a tile
    const int row = threadIdx.x & (stride - 1), slice = warp * 32 / stride;
    const bool live = warp < 4 && row < rows, live_w = warp < 4 && (warp * 32 & (stride - 1)) < rows;
    tc_fence_after();
    const uint32_t tb = sh.tmem;
    bool ok = (smem_u32(smem) & 1023u) == 0;     // the swizzle atoms need it; reported like an expired wait

    float m = -INFINITY, l = 0.f;
    const unsigned long long anc = live ? table.head->anc[(first_row + row) / group] : 0ull;
    const uint32_t t_lane = tb + ((uint32_t)(warp & 3) * 32 << 16);
    if (warp < 4) {
        // ------------------------------------------------------------------------ queries, a row of the tile for each of its copies; softmax
        // (rows that do not exist: zeros, whose scores do not move a reference)
        // eight pieces a thread are under way together, so that 128 rows come at two latencies instead of sixteen
        const int pieces = steps > 0 ? (copies > 1 ? stride : (rows + 31) & ~31) * PIECES : 0;
#pragma unroll 1
        for (int i0 = threadIdx.x; i0 < pieces; i0 += 1024) {
            uint4 w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + j * 128, r = i / PIECES, c = i % PIECES, gr = first_row + r, node = gr / group;
                w[j] = make_uint4(0u, 0u, 0u, 0u);
                if (r < rows) w[j] = *reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(a.q) + (((int64_t)b * a.max_nodes + node) * a.n_heads + hk * group + (gr - node * group)) * D + c * 8);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = i0 + j * 128, r = i / PIECES, c = i % PIECES;
                if (i >= pieces) break;
                const uint4 x = make_uint4((w[j].x & p.q_and) ^ p.q_xor, (w[j].y & p.q_and) ^ p.q_xor, (w[j].z & p.q_and) ^ p.q_xor, (w[j].w & p.q_and) ^ p.q_xor);
                unsigned char *dst = smem + (c >> 3) * (128 * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4);
                for (int k = 0; k < copies; ++k) *reinterpret_cast<uint4 *>(dst + k * stride * 128) = x;
            }
        }
        fence_proxy_async();                     // ordinary stores -> visible to the products' reads
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full);
        if (!live_w) {                           // no rows: keeps step
            for (int g = 0; g < steps && (ok = mbar_wait_warp(&sh.s_full[g & 1], g >> 1 & 1)); ++g)
                if (lane == 0) mbar_arrive(&sh.p_ready[g & 1]);
        } else if (ok) {
            if (copies == 4) ok = TreeSoftmax<D, 4>::run(sh, t_lane, slice, steps, t0, table, n_seg, anc, a.scale_log2e, m, l);
            else if (copies == 2) ok = TreeSoftmax<D, 2>::run(sh, t_lane, slice, steps, t0, table, n_seg, anc, a.scale_log2e, m, l);
            else ok = TreeSoftmax<D, 1>::run(sh, t_lane, 0, steps, t0, table, n_seg, anc, a.scale_log2e, m, l);
        }
    } else if (warp == kTtLoadWarp) {
        // ------------------------------------------------------------------------ loads
        // Tiles of several segments: lane j looks after rows 8 (j % 8) to 8 (j % 8) + 7 and half j / 8, and loads the box that starts there, if one
        // does: a segment's L groups of eight rows are boxes of 4, 2 and 1 groups in this order.
        if (!p.stall) {
            const uint32_t lead = elect_one();
            const uint64_t keep = l2_policy_evict_normal();
            const int half = lane >> 3, first = (lane & 7) * 8;
            int seg = seg0, slot = 0;
            uint32_t ph = 1, fills = 0;
#pragma unroll 1
            for (int g = 0; g < steps && ok; ++g) {
                const int u0 = (t0 + g) * kTtKeys, have = min(kTtKeys, (total - u0 + 7) & ~7);
                seg = table.find(seg, u0);
                int s = seg, u = u0, box = 0, at_row = 0, z = 0;
                uint32_t mine = lead;
                if (u0 + kTtKeys > ((table.end[seg] + 7) & ~7)) {
                    z = half;
                    at_row = first;
                    mine = half < D / 64 && first < have;
                    if (mine) {
                        u = u0 + first;
                        s = table.find(seg, u);
                        const int from = max(table.lo[s], u0), groups = (min((table.end[s] + 7) & ~7, u0 + kTtKeys) - from) >> 3, left = groups - ((u - from) >> 3);
                        const int bit = 31 - __clz(left);
                        mine = (groups & ((2 << bit) - 1)) == left;
                        box = 3 - bit;
                    }
                }
                const bool in_tail = s == n_seg - 1;
                const int at = table.row[s] + u - table.lo[s] + (in_tail ? b * a.tail_cap : 0);
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    if (!(ok = mbar_wait_warp(&sh.empty[slot], ph))) break;
                    if (lead) mbar_expect_tx(&sh.full[slot], have * D * 2);
                    __syncwarp();
                    tma_load_3d_hint(mine, ring + slot * SLOT + z * (kTtKeys * 128) + at_row * 128, (in_tail ? p.tail[kv] : p.cache[kv]) + box, 0, at,
                                     hk * (D / 64) + z, &sh.full[slot], keep);
                    ++fills;
                    if (++slot == p.n_slots) { slot = 0; ph ^= 1; }
                }
            }
            // a wait ran out: the copies in flight must land before the block may exit (bounded)
            if (!ok)
                for (uint32_t f = fills - min(fills, (uint32_t)p.n_slots); f < fills; ++f) mbar_wait_warp(&sh.full[f % p.n_slots], f / p.n_slots & 1);
        }
    } else if (warp == kTtCleanWarp) {
        // ------------------------------------------------------------------------ cleaning of V: lane j piece j % PIECES of every 32 / PIECES-th row
        // Every fill of the ring is waited for in order, and its slot released too: a waiter that left out fills of a two-phase barrier could
        // mistake an older one.
        constexpr int RPW = 32 / PIECES;         // rows at a time
        const int c = lane % PIECES;
        int slot = 0, seg = seg0;
        uint32_t ph = 0;
#pragma unroll 1
        for (int item = 0; item < 2 * steps && ok; ++item) {
            if (!(ok = mbar_wait_warp(&sh.full[slot], ph))) break;
            const int u0 = (t0 + item / 2) * kTtKeys;
            if ((item & 1) && needs_cleaning(seg, u0)) {
                const auto piece = [&](int r) { return reinterpret_cast<uint4 *>(ring + slot * SLOT + (c >> 3) * (kTtKeys * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); };
                // rows that stand for no key, as far as the products read
                unsigned long long none = ~table.exists(seg, u0, total);
                const int used = key_steps(u0) * 16;
                if (used < kTtKeys) none &= (1ull << used) - 1;
                while (none) {
                    int r = 0;
#pragma unroll
                    for (int i = 0; i < RPW; ++i)
                        if (none) { if (lane / PIECES >= i) r = __ffsll(none) - 1; none &= none - 1; }
                    *piece(r) = make_uint4(0u, 0u, 0u, 0u);
                }
                // nodes
                const int r1 = min(total - u0, kTtKeys);
#pragma unroll 1
                for (int r = max(ctx - u0, 0) + lane / PIECES; r < r1; r += 4 * RPW) {
                    uint4 w[4];
                    uint32_t odd = 0u;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        w[i] = *piece(min(r + i * RPW, r1 - 1));
                        odd |= bf16_not_finite(w[i].x) | bf16_not_finite(w[i].y) | bf16_not_finite(w[i].z) | bf16_not_finite(w[i].w);
                    }
                    if (odd)
                        for (int i = 0; i < 4 && r + i * RPW < r1; ++i) {
                            const uint4 v = *piece(r + i * RPW);
                            const uint32_t x = bf16_not_finite(v.x), y = bf16_not_finite(v.y), z = bf16_not_finite(v.z), q = bf16_not_finite(v.w);
                            if (!(x | y | z | q)) continue;
                            *piece(r + i * RPW) = make_uint4(v.x & ~x, v.y & ~y, v.z & ~z, v.w & ~q);
                            atomicOr(&sh.not_finite, 1ull << (u0 + r + i * RPW - ctx));
                        }
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sh.clean[slot]);
            }
            if (lane == 0) mbar_arrive(&sh.empty[slot]);
            __syncwarp();
            if (++slot == p.n_slots) { slot = 0; ph ^= 1; }
        }
    } else {
        // ------------------------------------------------------------------------ products
        const uint32_t lead = elect_one();
        // High word: stride-dimension offset 1024 B (8-row groups), descriptor version 1, 128-byte swizzle.  V: leading dimension, the next half.
        const uint64_t d_hi = (uint64_t)((1024u >> 4) | (1u << 14) | (2u << 29)) << 32;
        const uint64_t qd = d_hi | uniform(((smem_u32(smem) & 0x3ffffu) >> 4) | (1u << 16));
        const uint32_t k_lo = ((smem_u32(ring) & 0x3ffffu) >> 4) | (1u << 16), v_lo = ((smem_u32(ring) & 0x3ffffu) >> 4) | ((uint32_t)(kTtKeys * 128) >> 4 << 16);
        const uint32_t id_s = idesc_bf16(128, kTtKeys, 0, 0), id_o = idesc_bf16(128, D, 0, 1);
        int slot = 0, seg = seg0;                // of the next K tile; its V tile is in the one behind it
        uint32_t ph = 0;
        auto scores = [&](int g) {
            if (!(ok = mbar_wait_warp(&sh.full[slot], ph))) return;
            tc_fence_after();
            const uint64_t kd = d_hi | uniform(k_lo + slot * (SLOT >> 4));
            const uint32_t d = uniform(tb + (g & 1) * kTtKeys);
#pragma unroll
            for (int kk = 0; kk < D / 16; ++kk)                 // contraction over head_dim
                umma_ss(lead, d, qd + (kk >> 2) * ((128 * 128) >> 4) + (kk & 3) * 2, kd + (kk >> 2) * ((kTtKeys * 128) >> 4) + (kk & 3) * 2, id_s, kk > 0 ? 1u : 0u);
            if (lead) { umma_commit(&sh.s_full[g & 1]); umma_commit(&sh.empty[slot]); }
            __syncwarp();
        };
        uint32_t cleaned = 0;                    // parity of the slots' cleanings
        ok = ok && (steps == 0 || mbar_wait_warp(&sh.q_full, 0));
        if (steps > 0 && ok) scores(0);
#pragma unroll 1
        for (int g = 0; g < steps && ok; ++g) {
            int vs = slot + 1;
            uint32_t v_ph = ph;
            if (vs == p.n_slots) { vs = 0; v_ph ^= 1; }
            slot = vs + 1; ph = v_ph;
            if (slot == p.n_slots) { slot = 0; ph ^= 1; }
            // the next scores are under way while this tile's softmax runs; they go where P of the tile before was read by products issued earlier
            if (g + 1 < steps) { scores(g + 1); if (!ok) break; }
            if (!(ok = mbar_wait_warp(&sh.full[vs], v_ph))) break;
            if (needs_cleaning(seg, (t0 + g) * kTtKeys)) {
                if (!(ok = mbar_wait_warp(&sh.clean[vs], cleaned >> vs & 1))) break;
                cleaned ^= 1u << vs;
            }
            if (!(ok = mbar_wait_warp(&sh.p_ready[g & 1], g >> 1 & 1))) break;
            tc_fence_after();
            const uint64_t vd = d_hi | uniform(v_lo + vs * (SLOT >> 4));
            const uint32_t at = uniform(tb + (g & 1) * kTtKeys), d = uniform(tb + 2 * kTtKeys), fresh = uniform((uint32_t)(g == 0)), n = uniform(key_steps((t0 + g) * kTtKeys));
            // contraction over keys, with the high and the low numbers
            if (copies == 1) {
#pragma unroll
                for (int kk = 0; kk < kTtKeys / 16; ++kk) {
                    if (kk >= n) break;
                    umma_ts(lead, d, at + kk * 16, vd + kk * (2048 >> 4), id_o, kk > 0 || !fresh ? 1u : 0u);
                    umma_ts(lead, d, at + kk * 16 + 8, vd + kk * (2048 >> 4), id_o, 1u);
                }
            } else {
#pragma unroll
                for (int kk = 0; kk < kTtKeys / 16; ++kk) {
                    if (kk >= n) break;
                    uint32_t off[4];             // all lanes but the copy's whose keys these are
#pragma unroll
                    for (int i = 0; i < 4; ++i) off[i] = uniform((copies == 4 ? i == kk : i >> 1 == kk >> 1) ? 0u : ~0u);
                    umma_ts_lanes(lead, d, at + kk * 16, vd + kk * (2048 >> 4), id_o, fresh && (copies == 4 || !(kk & 1)) ? 0u : 1u, off);
                    umma_ts_lanes(lead, d, at + kk * 16 + 8, vd + kk * (2048 >> 4), id_o, 1u, off);
                }
            }
            if (lead) { umma_commit(&sh.o_done[g & 1]); umma_commit(&sh.empty[vs]); }
            __syncwarp();
        }
        if (!ok) {
            // a wait ran out: every product must finish (bounded) before the tensor memory is freed
            if (lead) umma_commit(&sh.drain);
            __syncwarp();
            mbar_wait_warp(&sh.drain, 0);
        }
    }
    __syncwarp();
    if (!ok && lane == 0) atomicExch(a.status, (uint32_t)STATUS_TIMEOUT);
    __syncthreads();

    // ---------------------------------------------------------------------------- output
    const bool merge = gridDim.x > 1 || copies > 1;
    constexpr int PS = D + 4;
    float *part = reinterpret_cast<float *>(smem);
    if (live_w) {
        unsigned long long odd = sh.not_finite & anc;             // nodes that the row sees whose values were taken out ...
        if (odd && copies > 1) {                                  // ... in this warp's share of their tile
            unsigned long long mine = 0ull;
            for (unsigned long long left = odd; left; left &= left - 1) {
                const int node = __ffsll(left) - 1;
                if (((ctx + node) & (kTtKeys - 1)) / (kTtKeys / copies) == slice) mine |= 1ull << node;
            }
            odd = mine;
        }
        const int gr = first_row + min(row, rows - 1), h = hk * group + gr % group;
        const int64_t at = ((int64_t)b * a.max_nodes + gr / group) * a.n_heads + h;
        const float inv = merge ? 1.f : (l == 0.f ? 0.f : 1.f / l);
        unsigned char *dst = static_cast<unsigned char *>(a.out) + at * D * 2;
        float *mine = part + (row + slice * stride) * PS;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
            uint32_t o[32];
            if (steps > 0) {
                tmem_ld32(t_lane + 2 * kTtKeys + c, o);
                tmem_ld_wait();
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0u;
            }
            if (live) {
                for (unsigned long long left = odd; left; left &= left - 1) {
                    const int64_t r = (int64_t)b * a.tail_cap + committed + __ffsll(left) - 1;
                    const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.tail_v) + (r * a.n_kv_heads + hk) * D + c;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const float x = __bfloat162float(v[i]);
                        if (!(fabsf(x) < INFINITY)) o[i] = __float_as_uint(__uint_as_float(o[i]) + x);
                    }
                }
                if (merge) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) *reinterpret_cast<uint4 *>(mine + c + i) = make_uint4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = pack_bf16x2(__uint_as_float(o[i + 2 * j]) * inv, __uint_as_float(o[i + 2 * j + 1]) * inv);
                        *reinterpret_cast<uint4 *>(dst + (c + i) * 2) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
        }
        if (live && merge) { mine[D] = m; mine[D + 1] = l; }
        if (live && !merge && a.lse) a.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2T;
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kTtMmaWarp) { tc_fence_after(); tmem_dealloc(tb, kTtTmem); }
    if (copies == 4) tree_merge<__nv_bfloat16, D, 4>(a, part, rows, first_row, b, hk);
    else if (copies == 2) tree_merge<__nv_bfloat16, D, 2>(a, part, rows, first_row, b, hk);
    else if (merge) tree_merge<__nv_bfloat16, D, 1>(a, part, rows, first_row, b, hk);
}

template <int D> static int launch_tc(const TreeArgs &a, int64_t max_keys, cudaStream_t st)
{
    constexpr int SLOT = kTtKeys * D * 2, Q_BYTES = 128 * D * 2;
    const int all_rows = a.max_nodes * (a.n_heads / a.n_kv_heads), row_tiles = (all_rows + 127) / 128;
    TreeTcArgs p;
    p.t = a;
    p.tile_rows = (all_rows + row_tiles - 1) / row_tiles;
    p.stall = g_stall_producer ? 1 : 0;
    p.q_and = a.scale_log2e == 0.f ? 0u : ~0u;
    p.q_xor = a.scale_log2e < 0.f ? 0x80008000u : 0u;
    p.t.scale_log2e = a.scale_log2e == 0.f ? 1.f : std::fabs(a.scale_log2e);
    const size_t extra = round_up(sizeof(TreeTcShared), 16) + TreeTable::bytes(a.k);
    // Ring: what half an SM's shared memory has room for; a table of thousands of kept paths takes a whole one.
    const auto slots = [&](size_t room) { return room < Q_BYTES + extra ? 0 : (int)std::min<size_t>(kTtMaxSlots, (room - Q_BYTES - extra) / SLOT); };
    p.n_slots = slots(kTtHalfSm);
    if (p.n_slots < 4) p.n_slots = slots(kTtMaxSmem);
    SP_REQUIRE(p.n_slots >= 4, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: k = %d needs too much shared memory", a.k);
    static_assert(Q_BYTES + 4 * SLOT >= 128 * (D + 4) * 4, "the partial result takes the place of queries and ring");
    // not so little that a third block fits, whose tensor memory would not
    const size_t smem = std::max<size_t>(Q_BYTES + p.n_slots * SLOT + extra, 80 * 1024);
    const int64_t units = (int64_t)row_tiles * a.n_kv_heads * a.n_prompts;
    int n = 1;
    while (n < 8 && 2 * n * units <= 2 * num_sms() && 2 * n * kTtKeys <= max_keys) n *= 2;
    const int64_t columns = (int64_t)a.n_kv_heads * D, tail_rows = std::max<int64_t>((int64_t)a.n_prompts * a.tail_cap, 1);       // (a tail without rows is not read)
    SP_REQUIRE(tail_rows < (int64_t)INT32_MAX, SP_ERR_UNSUPPORTED, "sp_pruned_decode_tree: %lld tail rows (fewer than 2^31 supported)", (long long)tail_rows);
    for (int i = 0; i < 2; ++i) {
        const void *tail = i ? a.tail_v : a.tail_k, *cache = i ? a.v_cache : a.k_cache;
        for (int box = 0; box < 4; ++box) {
            if (int rc = encode_rows_map(&p.tail[i][box], tail, tail_rows, columns, kTtKeys >> box, box ? 1 : D / 64)) return rc;
            // a cache without rows is not read
            if (int rc = encode_rows_map(&p.cache[i][box], a.total_tokens ? cache : tail, a.total_tokens ? a.total_tokens : tail_rows, columns, kTtKeys >> box, box ? 1 : D / 64)) return rc;
        }
    }
    SP_CUDA(cudaFuncSetAttribute(tree_tc_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, kTtMaxSmem));
    return launch(tree_tc_kernel<D>, dim3(n, row_tiles * a.n_kv_heads, a.n_prompts + 1), kTtThreads, smem, st, n, p);
}

int launch_tree_tc(const TreeArgs &a, int head_dim, int64_t max_keys, cudaStream_t st)
{
    return head_dim == 128 ? launch_tc<128>(a, max_keys, st) : launch_tc<64>(a, max_keys, st);
}

}  // namespace sp
