// sp_sample_tokens: one token per row of logits, with temperature, top-k, top-p and min-p, from one given uniform number per row.
//
// A block (a cluster of two to eight where a row does not fit: see launch_sample) holds its row in shared memory, so that the logits leave HBM once however many
// passes the filters take.
// All three filters keep a prefix of one order (value descending, index ascending), so the kept set is a threshold value and the last index
// among its ties; and the token is the first one in index order whose running sum of kept weights w = exp((x - max) / T) passes u W.
//   top-k   While a row is loaded every thread notes the maxima of four quarters of its elements; the k-th largest of all these bounds the k-th
//           largest element from below and leaves little more than k elements.  Up to 1 536 of them are listed and sorted, and everything
//           else happens on the list; more go through a radix select by counts.
//   top-p   Where the noted maxima alone reach p W, the elements above the bound of the 128-th are listed and sorted.  Else: elements with
//           w < (1 - p) W / V weigh less than (1 - p) W together, so none of them is needed to reach p W.  A histogram of the others over
//           1 024 ranges of values, with the elements' number and their mean place in each, says in which few p W is reached; what lies
//           above is summed and what lies in them listed and sorted.  Lists that come out too long (thousands of ties, a temperature that
//           makes all weights alike) go through a radix select by exact weights instead.
//   min-p   w >= min_p, looked at where the rest is known.
// Which token that is must not depend on rounding: next to u W there is a border between tokens every 1 / V, and with weights of fp32 accuracy
// (6e-8) one row in some hundred of 50 000 tokens came out one token off.  So what counts are weights in fp64 (2^(j/16) from a table times a
// polynomial of degree 6, 1e-15), rounded once to multiples of 2^-44, and sums of 64-bit integers: exact, in any order, atomics included.  fp64
// costs several times what fp32 does (a pass over 50432 elements by a block alone on its SM 3 and some 15 us), so rows are tried with fp32
// weights and a bound on what their sums are off by; only sums that leave a doubt (in 1 to 2 rows of a hundred) are taken again, exactly.
// Two rows share an SM where they fit (100 KB: 51 000 elements in bf16, 25 000 in fp32); a longer one has it to itself.  What bounds a row is its
// chain of passes over shared memory (each some 4 us for two rows, by the exponentials' 16 per clk) and of short steps of the whole block between
// barriers.  1024 bf16 rows of 50432, us with cold L2 (floor 16): greedy 33, nothing left out 76, k = 20 59, k = 1000 143, p = 0.9 199, settings as
// requests have them 122; those of 65000: 174, of 128000, a cluster of two a row: 460.  256 fp32 rows of 32000, top-p and min-p: 64 (two waves).
#include <cooperative_groups.h>

#include <cfloat>

#include "common.cuh"

namespace sp {

namespace cg = cooperative_groups;

constexpr int kSmpThreads = 512, kSmpWarps = kSmpThreads / 32;
constexpr int kSmpBits = 9, kSmpBins = 1 << kSmpBits;         // of a radix level
constexpr int kSmpFine = 2 * kSmpThreads;        // bins of the histogram over values: two a thread
constexpr int kSmpList = 3 * kSmpThreads;        // elements that can be listed
constexpr int kSmpSmall = 256;                   // kept elements that the list alone deals with to the end
constexpr int kSmpGroups = 4;                    // maxima that a thread notes
constexpr int kSmpMaxVocab = 1 << 18;            // sums of weights stay below 2^63, and eight blocks hold an fp32 row
constexpr int kSmpMaxSmem = 200 * 1024;          // allowed to the kernel once and for all: see kDecMaxSmem in decode.cu
constexpr uint32_t kSmpLeastCode = 0x00800000u;  // code of the lowest finite number
constexpr double kSmpUnit = 17592186044416.0;    // 2^44

struct SampleArgs {
    const void *logits;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t *top_k;
    int32_t *tokens;
    float *logp;
    int64_t ld;
    int vocab, vecs;                             // 16-byte pieces of a row that a block holds
};

// Larger number, larger code; -0 as +0; NaN and -inf below everything that may be kept.
__device__ __forceinline__ uint32_t sample_code(float x)
{
    if (!(x > -INFINITY)) return 0u;
    if (x == 0.f) x = 0.f;
    const uint32_t b = __float_as_uint(x);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float sample_value(uint32_t code) { return __uint_as_float(code & 0x80000000u ? code & 0x7fffffffu : ~code); }

typedef unsigned long long u64;

struct SampleShared {
    union {                                      // one after the other
        u64 hist[kSmpBins];
        uint32_t count[kSmpFine];
        u64 list[kSmpList];                      // code << 32 | ~index: descending order of these is the order of the filters
    };
    double exp2_table[16];                       // 2^(j / 16): a bank each, so that no two lanes' reads meet
    u64 warp_sum[kSmpWarps], warp_sum2[kSmpWarps], total2, total;              // total: this block's, for the other blocks of the cluster
    u64 above, left;                             // results of a select; what is left of a goal in front of the thread that reaches it
    uint32_t bin, bin_to;
    int winner;                                  // that thread
    int index, listed, found;
    float max;
};

// What every row needs several times is called, not inlined: a row runs through most of the code once, and what is not in the instruction cache costs
// as much as it does.  x: inclusive sum over the block's threads, in thread order; y: the block's total.
__device__ __noinline__ ulonglong2 sample_block_scan(SampleShared *sh, u64 v)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) { const u64 w = __shfl_up_sync(0xffffffffu, v, o); if (lane >= o) v += w; }
    __syncthreads();
    if (lane == 31) sh->warp_sum[warp] = v;
    __syncthreads();
    // every warp sums up the warps' sums: the last lane's for the lanes in front
    u64 s = lane < kSmpWarps ? sh->warp_sum[lane] : 0ull;
#pragma unroll
    for (int o = 1; o < kSmpWarps; o *= 2) { const u64 w = __shfl_up_sync(0xffffffffu, s, o); if (lane >= o) s += w; }
    const u64 all = __shfl_sync(0xffffffffu, s, kSmpWarps - 1), front = __shfl_sync(0xffffffffu, s, max(warp - 1, 0));
    return make_ulonglong2(warp ? v + front : v, all);
}
// Sum over a warp, in all lanes: three 32-bit additions of the hardware's (22, 22 and 20 bits of each number), which take a fifth of the time of
// five rounds of exchange.
__device__ __forceinline__ u64 sample_warp_sum(u64 v)
{
    const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)v & 0x3fffffu), b = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 22) & 0x3fffffu),
                   c = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 44));
    return (u64)a + ((u64)b << 22) + ((u64)c << 44);
}
// Sorts the list's n keys (all different), descending.
__device__ __noinline__ void sample_sort(SampleShared *sh, int n)
{
    u64 *list = sh->list;
    __syncthreads();
    if (n <= kSmpThreads / 2) {
        // an element's place is the number of larger ones; two or four threads an element
        const int log_t = n <= kSmpThreads / 4 ? 2 : 1, i = threadIdx.x >> log_t, t = threadIdx.x & ((1 << log_t) - 1);
        const u64 mine = i < n ? list[i] : 0ull;
        int place = 0;
        if (((threadIdx.x & ~31) >> log_t) < n)
#pragma unroll 4
            for (int j = t; j < n; j += 1 << log_t) place += list[j] > mine;
        place += __shfl_xor_sync(0xffffffffu, place, 1);
        if (log_t > 1) place += __shfl_xor_sync(0xffffffffu, place, 2);
        __syncthreads();
        if (i < n && t == 0) list[place] = mine;
        __syncthreads();
        return;
    }
    // By bins of codes, then every element among those of its bin.  The keys stay in registers while the bins are where the list was.  (1 300 keys: 4 us,
    // the exchanges below 17.)
    u64 key[3];
    uint32_t hi = 0u, lo = ~0u, slot[3], start[3], end[3];
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        const int i = threadIdx.x + j * kSmpThreads;
        key[j] = i < n ? list[i] : 0ull;
        if (i < n) { hi = max(hi, (uint32_t)(key[j] >> 32)); lo = min(lo, (uint32_t)(key[j] >> 32)); }
    }
    hi = __reduce_max_sync(0xffffffffu, hi);
    lo = __reduce_min_sync(0xffffffffu, lo);
    if ((threadIdx.x & 31) == 0) { sh->warp_sum[threadIdx.x >> 5] = hi; sh->warp_sum2[threadIdx.x >> 5] = lo; }
    __syncthreads();                             // the keys are read too
    sh->count[threadIdx.x] = sh->count[threadIdx.x + kSmpThreads] = 0u;
#pragma unroll
    for (int w = 0; w < kSmpWarps; ++w) { hi = max(hi, (uint32_t)sh->warp_sum[w]); lo = min(lo, (uint32_t)sh->warp_sum2[w]); }
    __syncthreads();
    const float per = (float)kSmpFine / ((float)(hi - lo) + 1.f);
    const auto bin_of = [&](u64 k) { return min((int)((float)(hi - (uint32_t)(k >> 32)) * per), kSmpFine - 1); };
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if ((int)threadIdx.x + j * kSmpThreads < n) slot[j] = atomicAdd(&sh->count[bin_of(key[j])], 1u);
    __syncthreads();
    const uint32_t c0 = sh->count[2 * threadIdx.x], c1 = sh->count[2 * threadIdx.x + 1];
    const bool crowded = __syncthreads_or(max(c0, c1) > 64u);
    if (!crowded) {
        const uint32_t upto = (uint32_t)sample_block_scan(sh, c0 + c1).x;
        sh->count[2 * threadIdx.x] = upto - c0 - c1;
        sh->count[2 * threadIdx.x + 1] = upto - c1;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if ((int)threadIdx.x + j * kSmpThreads < n) {
                const int bin = bin_of(key[j]);
                start[j] = sh->count[bin];
                end[j] = bin + 1 < kSmpFine ? sh->count[bin + 1] : (uint32_t)n;
            }
        __syncthreads();
    } else {
#pragma unroll
        for (int j = 0; j < 3; ++j) { start[j] = threadIdx.x + j * kSmpThreads; slot[j] = 0u; }
    }
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if ((int)threadIdx.x + j * kSmpThreads < n) list[start[j] + slot[j]] = key[j];
    __syncthreads();
    if (!crowded) {
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            if ((int)threadIdx.x + j * kSmpThreads >= n) break;
            slot[j] = 0u;
            for (uint32_t i = start[j]; i < end[j]; ++i) slot[j] += list[i] > key[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if ((int)threadIdx.x + j * kSmpThreads < n) list[start[j] + slot[j]] = key[j];
        __syncthreads();
        return;
    }
    // Many elements in one bin (ties, one value far from the others).
    // Bitonic, with every comparison putting the larger element first (the first step of a merge compares mirrored places), so that the places
    // up to the next power of two that hold nothing stay behind the others and need no look.
    // A warp's comparisons lie together, so that steps that stay within their elements need no barrier of the block.
    int size = 2 * kSmpThreads;
    while (size < n) size *= 2;
    const int of_warp = size / 2 / kSmpWarps, first = (threadIdx.x >> 5) * of_warp + (threadIdx.x & 31);
#pragma unroll 1
    for (int run = 2; run <= size; run *= 2)
#pragma unroll 1
        for (int step = run / 2; step > 0; step /= 2) {
            for (int i = first; i < first + of_warp; i += 32) {
                const int j = i & (step - 1), lo = 2 * i - j, hi = step == run / 2 ? (lo | (run - 1)) - j : lo + step;
                if (hi >= n) continue;
                const u64 x = list[lo], y = list[hi];
                if (x < y) { list[lo] = y; list[hi] = x; }
            }
            // (the next step, or the next run's first, reaches as far as this one's run at least)
            if (step > of_warp || (step == 1 && run > of_warp) || step / 2 > of_warp) __syncthreads(); else __syncwarp();
        }
}

template <typename T, bool CLUSTER> struct Sampler {
    static constexpr int N = Vec<T>::N;
    const SampleArgs &a;
    SampleShared &sh;
    const T *data;                               // [a.vecs * N]
    int n_vec, per_thread, first;                // pieces that this block holds, that a thread looks after; index in the row of the first element
    float top;                                   // the row's maximum
    double scale;                                // log2(e) / T
    float fast_scale, nothing, least_weighed;    // nothing: a number that weighs 0; least_weighed: one that weighs some 2^-60
    bool exact;                                  // weights in fp64 and sums exact; else in fp32, with a bound on what they are off by

    __device__ __forceinline__ void row_sync() const { if (CLUSTER) cg::this_cluster().sync(); else __syncthreads(); }
    __device__ __forceinline__ int blocks() const { return CLUSTER ? (int)cg::this_cluster().num_blocks() : 1; }
    __device__ __forceinline__ int rank() const { return CLUSTER ? (int)cg::this_cluster().block_rank() : 0; }
    template <typename V> __device__ __forceinline__ const V *at(const V *p, int r) const { return CLUSTER ? cg::this_cluster().map_shared_rank(const_cast<V *>(p), r) : p; }

    // exp((x - max) / T) in fp64 as a product, of an x that is not below least_weighed.  Without branches: many are under way at once.
    __device__ __forceinline__ double weight_parts(float x, double &power) const
    {
        const double d = (double)x - (double)top, t = fma(d, scale, 0x1.8p48);       // the exponent in multiples of 1/16 in the low bits
        const int k = __double2loint(t);
        const double r = fma(d, scale, 0x1.8p48 - t);            // |r| <= 1/32
        double p = 1.5403530393381608e-4;        // ln2^6 / 720, ln2^5 / 120, ln2^4 / 24, ln2^3 / 6, ln2^2 / 2, ln2
        p = fma(p, r, 1.3333558146428443e-3);
        p = fma(p, r, 9.618129107628477e-3);
        p = fma(p, r, 5.550410866482158e-2);
        p = fma(p, r, 2.402265069591007e-1);
        p = fma(p, r, 6.931471805599453e-1);
        p = fma(p, r, 1.0);
        power = sh.exp2_table[k & 15];
        power = __hiloint2double(__double2hiint(power) + (k >> 4) * (1 << 20), __double2loint(power));
        return p;
    }
    __device__ __forceinline__ double weight(float x) const
    {
        if (top == INFINITY) return x == INFINITY ? 1.0 : 0.0;
        double power;
        const double p = weight_parts(fmaxf(x, least_weighed), power);
        return x >= least_weighed ? p * power : 0.0;
    }
    // In multiples of 2^-44, to the nearest.
    __device__ __forceinline__ u64 weigh(float x) const
    {
        if (top == INFINITY) return x == INFINITY ? 1ull << 44 : 0ull;
        double power;
        const double p = weight_parts(fmaxf(x, least_weighed), power);
        return x >= least_weighed ? (u64)(__double_as_longlong(fma(p, power, 0x1.8p8)) - __double_as_longlong(0x1.8p8)) : 0ull;
    }
    // The same in fp32 and what it may be off by, relative: three roundings of the exponent (of the difference, the factor and the product), 2^-22
    // of the exponential, three additions one after another in a piece's sum; a tenth more of each.  Exponents end at -150, where weights are 0.
    __device__ __forceinline__ float fast_weight(float x, float &exponent) const
    {
        exponent = (x - top) * fast_scale;
        float w;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(exponent));
        return w;
    }
    static constexpr double kOffPerExponent = 3 * 0x1p-24 * 0.6931471805599453 * 1.1, kOffAdded = 3 * 0x1p-24 * 1.1, kOff = 0x1p-22 * 1.1 + kOffAdded;

    // f(piece's four words, index of its first element) for this thread's pieces, which lie together, so that threads are in index order; an odd
    // number of them each, so that eight neighbours' pieces meet no bank twice.
    template <typename F> __device__ __forceinline__ void pieces(F f) const
    {
        const int v0 = threadIdx.x * per_thread, v1 = min(v0 + per_thread, n_vec);
#pragma unroll 2
        for (int v = v0; v < v1; ++v) f(*reinterpret_cast<const uint4 *>(data + v * N), first + v * N);
    }
    __device__ __forceinline__ static void unpack(const uint4 &w, float (&x)[N]) { Vec<T>::load(reinterpret_cast<const T *>(&w), x); }
    // f(x, index) for this thread's elements from `least` to `most`, where most are not: a bit per element of some pieces first, then the elements whose bits are
    // set, each lane its own, so that a warp's hits are dealt with side by side.
    template <typename F> __device__ __forceinline__ void each(float least, float most, F f) const
    {
        constexpr int CHUNK = 32 / N;            // pieces that 32 bits stand for
        // bf16: against thresholds cut to bf16, which leaves no number out; f sees to the rest
        const uint32_t cut = __float_as_uint(least) >> 16, both = cut | cut << 16, cut_most = __float_as_uint(most) >> 16, both_most = cut_most | cut_most << 16;
        const auto two = [](const uint32_t &x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
        const int v0 = threadIdx.x * per_thread, v1 = min(v0 + per_thread, n_vec);
#pragma unroll 1
        for (int v = v0; v < v1; v += CHUNK) {
            uint32_t hits = 0;
#pragma unroll
            for (int j = 0; j < CHUNK; ++j) {
                if (v + j >= v1) break;
                const uint4 w = *reinterpret_cast<const uint4 *>(data + (v + j) * N);
                const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (N == 8) {
                        const uint32_t h = __hge2_mask(two(ws[e]), two(both)) & __hle2_mask(two(ws[e]), two(both_most));
                        hits |= ((h & 1u) | (h >> 30 & 2u)) << (8 * j + 2 * e);
                    } else {
                        hits |= __uint_as_float(ws[e]) >= least && __uint_as_float(ws[e]) <= most ? 1u << (4 * j + e) : 0u;
                    }
                }
            }
            for (; hits; hits &= hits - 1) {
                const int bit = __ffs(hits) - 1;
                f(to_float(data[v * N + bit]), first + v * N + bit);
            }
        }
    }
    // A sum of weights in units, and what it may be off by.
    struct Sum { u64 units, off; };
    // Elements that are kept: x >= at up to index `last`, x >= above behind it.  -150 as above.
    struct Cut { float at, above; int last; };
    __device__ __forceinline__ Cut cut_of(float least, int tie_last, float floor_x) const
    {
        const float base = fmaxf(floor_x, exact ? -FLT_MAX : nothing);
        if (base > least) return Cut{base, base, INT32_MAX};
        return Cut{least, sample_value(sample_code(least) + 1), tie_last};
    }
    __device__ __forceinline__ static bool kept(const Cut &c, float x, int i) { return x >= (i <= c.last ? c.at : c.above); }
    // f(piece's elements, -inf those behind the last of the ties, threshold)
    template <typename F> __device__ __forceinline__ void pieces_of(const Cut &cut, F f) const
    {
        pieces([&](const uint4 &w, int i) {
            float x[N];
            unpack(w, x);
            if (i <= cut.last && i + N - 1 > cut.last)       // the piece with the last of the ties
#pragma unroll
                for (int e = 0; e < N; ++e) if (i + e > cut.last && !(x[e] >= cut.above)) x[e] = -INFINITY;
            f(x, i <= cut.last ? cut.at : cut.above);
        });
    }
    // Sum of this thread's elements that are kept.
    __device__ __forceinline__ Sum weigh_all(const Cut &cut) const
    {
        double all = 0.0;
        float weighted[2] = {0.f, 0.f};          // by the size of the exponent
        pieces_of(cut, [&](const float (&x)[N], float t) {
            float g[N];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float y;
                g[e] = fast_weight(x[e] >= t ? x[e] : nothing, y);
                weighted[e & 1] = fmaf(-y, g[e], weighted[e & 1]);
            }
            float s = (g[0] + g[1]) + (g[2] + g[3]);
            if constexpr (N == 8) s += (g[4] + g[5]) + (g[6] + g[7]);
            all += (double)s;
        });
        return Sum{(u64)(all * kSmpUnit), (u64)((all * kOff + (double)(weighted[0] + weighted[1]) * kOffPerExponent) * kSmpUnit) + 1};
    }
    // The same exactly, and of those above `high`.  Not inlined: seldom needed, see select().
    __device__ __forceinline__ ulonglong2 weigh_exactly(const Cut &cut, float high) const { return weigh_exactly_of(*this, cut, high); }
    __device__ __noinline__ static ulonglong2 weigh_exactly_of(Sampler s, Cut cut, float high)
    {
        u64 sum = 0, above = 0;
        s.pieces_of(cut, [&](const float (&x)[N], float t) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const u64 g = s.weigh(x[e] >= t ? x[e] : -INFINITY);
                sum += g;
                above += x[e] > high ? g : 0ull;
            }
        });
        return make_ulonglong2(sum, above);
    }
    // Inclusive sum over the block's threads, in thread order; all: the block's total.
    __device__ __forceinline__ u64 block_scan(u64 v, u64 &all) const
    {
        const ulonglong2 r = sample_block_scan(&sh, v);
        all = r.y;
        return r.x;
    }
    // Inclusive sum over the row's threads, in index order; all: the row's total.
    __device__ __forceinline__ u64 row_scan(u64 v, u64 &all)
    {
        v = block_scan(v, all);
        if (!CLUSTER) return v;
        if (threadIdx.x == 0) sh.total = all;
        row_sync();
        all = 0;
        for (int r = 0; r < blocks(); ++r) {
            const u64 t = *at(&sh.total, r);
            if (r < rank()) v += t;
            all += t;
        }
        row_sync();
        return v;
    }
    // Sums over the row, two at a time.
    __device__ __forceinline__ void row_sums(u64 &v, u64 &w)
    {
        v = sample_warp_sum(v);
        w = sample_warp_sum(w);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) { sh.warp_sum[threadIdx.x >> 5] = v; sh.warp_sum2[threadIdx.x >> 5] = w; }
        __syncthreads();
        const int lane = threadIdx.x & 31;
        v = sample_warp_sum(lane < kSmpWarps ? sh.warp_sum[lane] : 0ull);
        w = sample_warp_sum(lane < kSmpWarps ? sh.warp_sum2[lane] : 0ull);
        if (!CLUSTER) return;
        if (threadIdx.x == 0) { sh.total = v; sh.total2 = w; }
        row_sync();
        v = w = 0;
        for (int r = 0; r < blocks(); ++r) { v += *at(&sh.total, r); w += *at(&sh.total2, r); }
        row_sync();
    }
    __device__ __forceinline__ Sum row_sum(Sum s) { row_sums(s.units, s.off); return s; }
    // A bound from below on the k-th largest element: the k-th largest of the noted maxima, to the upper 20 bits of its code; -inf where there are fewer.
    // Over several warps (few) or blocks every one takes its share of k, and the least of their bounds holds.
    __device__ __forceinline__ float bound_of_kth(int k, uint4 top4) const
    {
        const uint32_t tops[kSmpGroups] = {top4.x, top4.y, top4.z, top4.w};
        const int share = (k + blocks() - 1) / blocks();
        uint32_t t = 0;
        if (share <= kSmpGroups * kSmpThreads / 8) {
            // by warps: no barriers, and some three times as many elements at or above the bound as needed
            // (up to a quarter of the lanes: their largest alone say nearly as much)
            const uint32_t n = (share + kSmpWarps - 1) / kSmpWarps, largest = max(max(tops[0], tops[1]), max(tops[2], tops[3]));
#pragma unroll 1
            for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 12); --bit) {
                const uint32_t c = t | 1u << bit;
                uint32_t m = 0;
                if (n <= 8) {
                    m = __popc(__ballot_sync(0xffffffffu, largest >= c));
                } else {
#pragma unroll
                    for (int i = 0; i < kSmpGroups; ++i) m += __popc(__ballot_sync(0xffffffffu, tops[i] >= c));
                }
                if (m >= n) t = c;
            }
            __syncthreads();
            if ((threadIdx.x & 31) == 0) sh.warp_sum[threadIdx.x >> 5] = t;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < kSmpWarps; ++w) t = min(t, (uint32_t)sh.warp_sum[w]);
        } else if (share <= kSmpGroups * kSmpThreads) {
            uint32_t *part = reinterpret_cast<uint32_t *>(sh.hist);
#pragma unroll 1
            for (int bit = 31; bit >= (sizeof(T) == 2 ? 16 : 12); --bit) {
                const uint32_t c = t | 1u << bit;
                uint32_t n = 0;
#pragma unroll
                for (int i = 0; i < kSmpGroups; ++i) n += tops[i] >= c;
                n = __reduce_add_sync(0xffffffffu, n);
                uint32_t *p = part + (bit & 1) * kSmpWarps;
                if ((threadIdx.x & 31) == 0) p[threadIdx.x >> 5] = n;
                __syncthreads();
                n = 0;
#pragma unroll
                for (int w = 0; w < kSmpWarps; ++w) n += p[w];
                if (n >= (uint32_t)share) t = c;
            }
        }
        if (CLUSTER) {
            __syncthreads();
            if (threadIdx.x == 0) sh.bin = t;
            row_sync();
            for (int r = 0; r < blocks(); ++r) t = min(t, *at(&sh.bin, r));
            row_sync();
        }
        return t < kSmpLeastCode ? -INFINITY : sample_value(t);
    }
    __device__ __forceinline__ void append(float x, int i)
    {
        const int n = atomicAdd(&sh.listed, 1);
        if (n < kSmpList) sh.list[n] = (u64)sample_code(x) << 32 | (uint32_t)~i;
    }
    // Before and behind a pass that appends: empties the list; makes it the row's in every block.  Returns the number of elements, and no list where
    // it is above kSmpList.  The list's order is any.
    __device__ __forceinline__ void clear_list()
    {
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
    }
    __device__ __forceinline__ int join_list()
    {
        row_sync();
        if (!CLUSTER) return sh.listed;
        int n = sh.listed, all = 0;
        for (int r = 0; r < blocks(); ++r) all += *at(&sh.listed, r);
        if (all <= kSmpList)                     // behind its own elements, the others'
            for (int r = 0; r < blocks(); ++r) {
                if (r == rank()) continue;
                const int m = *at(&sh.listed, r);
                for (int i = threadIdx.x; i < m; i += kSmpThreads) sh.list[n + i] = at(sh.list, r)[i];
                n += m;
            }
        row_sync();
        return all;
    }
    __device__ __forceinline__ void sort(int n) const { sample_sort(&sh, n); }
    __device__ __forceinline__ float listed_value(int i) const { return sample_value((uint32_t)(sh.list[i] >> 32)); }
    __device__ __forceinline__ int listed_index(int i) const { return (int)~(uint32_t)sh.list[i]; }
    // The sorted list's first n elements: exact weights of those of this thread (three neighbours), and their sum over the threads in front.
    __device__ __forceinline__ u64 weigh_listed(int n, u64 (&w)[3], u64 &all) const
    {
        u64 sum = 0;
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            const int j = 3 * threadIdx.x + i;
            w[i] = 0;
            if (j < n) w[i] = weigh(listed_value(j));
            sum += w[i];
        }
        return block_scan(sum, all) - sum;
    }
    // How many of the sorted list's first n elements have a sum of weights below goal in front of them (one at least); -1: that, or that all of them
    // reach it, is not certain where sums and goal may be off by `off`, or is not so.
    __device__ __forceinline__ int reach(int n, u64 goal, u64 off) const
    {
        u64 w[3], all, front = weigh_listed(n, w, all);
        u64 c = 0;                               // 32 bits: certainly below, 32 bits: doubtful
#pragma unroll
        for (int i = 0; i < 3; ++i) {
            if (3 * (int)threadIdx.x + i < n) c += front + off < goal ? 1ull : (front < goal + off && off ? 1ull << 32 : 0ull);
            front += w[i];
        }
        u64 total;
        block_scan(c, total);
        return total >> 32 || all < goal + off ? -1 : max((int)(uint32_t)total, 1);
    }
    // Threshold and last index where the sorted list's first n elements, behind others whose weight is `above`, reach goal.  0: found, 1: not there, 2: not
    // certain.
    __device__ __forceinline__ int settle(int n, u64 above, u64 goal, u64 off, float &least, int &tie_last) const
    {
        const int needed = above + off < goal ? reach(n, goal - above, off) : -1;
        if (needed < 0) return off ? 2 : 1;
        const int last = min(needed, n) - 1;
        least = listed_value(last);
        tie_last = listed_index(last);
        __syncthreads();
        return 0;
    }
    // One level of a select: from the top the bin of the histogram that add() makes in which the running sum reaches goal.  Leaves sh.bin and
    // sh.above (the sum in front of that bin).
    template <bool COUNTS, typename F> __device__ __forceinline__ void select_level(u64 goal, F add)
    {
        static_assert(kSmpBins == kSmpThreads, "a bin per thread");
        __syncthreads();
        if (COUNTS) sh.count[threadIdx.x] = 0; else sh.hist[threadIdx.x] = 0;
        if (threadIdx.x == 0) { sh.bin = 0; sh.above = 0; }
        __syncthreads();
        add();
        row_sync();
        const int bin = kSmpBins - 1 - threadIdx.x;
        u64 h = 0, all;
        for (int r = 0; r < blocks(); ++r) h += COUNTS ? at(sh.count, r)[bin] : at(sh.hist, r)[bin];
        row_sync();                              // nobody's histogram is read behind this
        const u64 upto = block_scan(h, all);
        if (upto - h < goal && upto >= goal) { sh.bin = bin; sh.above = upto - h; }
        __syncthreads();
    }
    // The largest number t such that the amounts of elements x >= t (COUNTS: one each; else their exact weights) reach goal, -inf where there are not as
    // many; above: the sum of elements x > t.  Not inlined, as nth(): seldom needed.  They get the sampler by value, since one whose address is
    // known somewhere lives in memory everywhere.  (64-bit additions in shared memory take turns, 32-bit ones are the hardware's.)
    struct Selected { float value; u64 above; };
    template <bool COUNTS> __device__ __forceinline__ Selected select(float least, u64 goal) const { return select_of<COUNTS>(*this, least, goal); }
    template <bool COUNTS> __device__ __noinline__ static Selected select_of(Sampler s, float least, u64 goal) { return s.template do_select<COUNTS>(least, goal); }
    template <bool COUNTS> __device__ __forceinline__ Selected do_select(float least, u64 goal)
    {
        u64 above;
        uint32_t prefix = 0;
        above = 0;
        int shift = 32, left = sizeof(T) == 2 ? 16 : 32;              // bf16: the low half of a code says nothing
#pragma unroll 1
        while (left > 0) {
            const int bits = min(left, kSmpBits), down = shift - bits;
            select_level<COUNTS>(goal - above, [&]() {
                each(least, INFINITY, [&](float x, int) {
                    const uint32_t c = sample_code(x);
                    if (!c || (shift < 32 && c >> shift != prefix >> shift)) return;
                    const uint32_t bin = c >> down & ((1u << bits) - 1);
                    if (COUNTS) atomicAdd(&sh.count[bin], 1u); else atomicAdd(&sh.hist[bin], weigh(x));
                });
            });
            above += sh.above;
            prefix |= sh.bin << down;
            shift = down;
            left -= bits;
        }
        // bf16: codes of negative numbers have ones in the low half
        if (sizeof(T) == 2 && !(prefix & 0x80000000u)) prefix |= 0xffffu;
        return Selected{prefix < kSmpLeastCode ? -INFINITY : sample_value(prefix), above};
    }
    // Where a running sum over the row's threads passes goal: sh.winner in the block that has the place (else none), and what is left of goal there.
    __device__ __forceinline__ void find_thread(u64 mine, u64 upto, u64 goal)
    {
        __syncthreads();
        if (threadIdx.x == 0) sh.winner = -1;
        __syncthreads();
        if (goal < upto && goal >= upto - mine) { sh.winner = threadIdx.x; sh.left = goal - (upto - mine); }
        __syncthreads();
    }
    // Index of the n-th (from 1) element in index order that equals t; there are that many in the row.
    __device__ __forceinline__ int nth(int n, float t) const { return nth_of(*this, n, t); }
    __device__ __noinline__ static int nth_of(Sampler s, int n, float t) { return s.do_nth(n, t); }
    __device__ __forceinline__ int do_nth(int n, float t)
    {
        u64 mine = 0, all;
        each(t, t, [&](float x, int) { mine += x == t; });
        const u64 upto = row_scan(mine, all);
        find_thread(mine, upto, (u64)(n - 1));
        if (threadIdx.x == 0) sh.index = INT32_MAX;
        __syncthreads();
        if (sh.winner >= 0 && threadIdx.x < 32) {
            // the thread's elements, a piece per lane
            const int lane = threadIdx.x, v = sh.winner * per_thread + lane;
            const bool there = lane < per_thread && v < n_vec;
            float x[N];
            unpack(there ? *reinterpret_cast<const uint4 *>(data + v * N) : make_uint4(0u, 0u, 0u, 0u), x);
            int c = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) c += there && x[e] == t;
            int run = c;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) { const int w = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += w; }
            int left = (int)sh.left - (run - c);
            if (left >= 0 && left < c)
#pragma unroll
                for (int e = 0; e < N; ++e) if (x[e] == t && left-- == 0) sh.index = first + v * N + e;
        }
        row_sync();
        int found = INT32_MAX;
        for (int r = 0; r < blocks(); ++r) found = min(found, *at(&sh.index, r));
        row_sync();
        return found;
    }
    // What the difference of a partial sum and `share` of the total may be off by, if the partial sum is off by `part` and the total by `all`: (1 -
    // share) of the first error and share of the rest's, as the total's terms are the partial sum's too; a unit for each element, for the exact
    // sums' own roundings.
    __device__ __forceinline__ u64 doubt(double share, u64 part, u64 all) const
    {
        const double p = (double)part, rest = fmax((double)all - p, 0.0);
        return (u64)(((1.0 - share) * p + share * rest) * 1.001) + a.vocab;
    }
    // The same where the two sums are of two passes: the elements' weights are alike in both, but not the additions in pieces of which only one
    // pass takes all elements, nor the units that the threads' sums are cut to.
    __device__ __forceinline__ u64 doubt_apart(double share, const Sum &part, const Sum &all) const
    {
        return doubt(share, part.off, all.off) + (u64)(((double)part.units + share * (double)all.units) * kOffAdded) + 2 * kSmpThreads * blocks();
    }
    // Where the elements' weights, in the order of the filters, reach goal, which is `share` of `all`, found among those down to `low`.  Threshold and last
    // index.  0: found, 1: not there, or too many elements lie there for the list, 2: not certain where in the list, which is sorted: n elements, the largest
    // that are not above x_from.
    __device__ __forceinline__ int fine_select(float low, u64 goal, double share, Sum all, float &x_from, int &n, float &least, int &tie_last)
    {
        // A bin's word: its elements' number in the upper half, the sum of their places in the bin, in 32nds, in the lower half.  One that runs over
        // (65 536 elements, 2 048 at the end of a bin) makes this look in the wrong place, which shows in the exact sums at the end.
        const float high = top, per = kSmpFine / (high - low), per32 = 32.f * per;
        const Cut inside = cut_of(least, tie_last, -INFINITY);
        __syncthreads();
        sh.count[threadIdx.x] = sh.count[threadIdx.x + kSmpThreads] = 0;
        __syncthreads();
        pieces([&](const uint4 &w, int i) {
            float x[N];
            unpack(w, x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float pos = (high - x[e]) * per32;
                if (!(pos < 32.f * kSmpFine - 1.f) || !kept(inside, x[e], i + e)) continue;
                const uint32_t at = __float_as_uint(pos + 0x1p23f) & 0x7fffffu;           // to the nearest
                atomicAdd(&sh.count[at >> 5], 0x10000u | (at & 31u));
            }
        });
        row_sync();
        // Two bins' weights in fp64 per thread.  d: what a bin is long, in powers of e.  An element is off its place by up to half a 32nd and the
        // roundings of the place, and a bin's weights are taken as linear in it.
        const double d = scale / per * 0.6931471805599453, off_place = d * (0.53 / 32.0) + d * d * 0.5;
        u64 mass[2], slack[2], total;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            u64 c = 0, q = 0;
            for (int r = 0; r < blocks(); ++r) { const uint32_t h = at(sh.count, r)[2 * threadIdx.x + j]; c += h >> 16; q += h & 0xffffu; }
            const double w0 = exp2((-(double)(2 * threadIdx.x + j) / per) * scale) * kSmpUnit;
            mass[j] = (u64)(w0 * fmax((double)c - (double)q * d * 0x1p-5, 0.0));
            slack[j] = (u64)(w0 * (double)c * off_place) + 2;
        }
        row_sync();
        const u64 upto = block_scan(mass[0] + mass[1], total);
        const u64 s_upto = block_scan(slack[0] + slack[1], total) + all.off;
        if (threadIdx.x == 0) { sh.bin = kSmpFine; sh.bin_to = kSmpFine - 1; }
        __syncthreads();
        // the first in which the sum may, and the first in which it must have reached goal
        if (upto + s_upto >= goal) atomicMin(&sh.bin, 2 * threadIdx.x + (upto - mass[1] + s_upto < goal));
        if (upto >= goal + s_upto) atomicMin(&sh.bin_to, 2 * threadIdx.x + (upto - mass[1] < goal + s_upto));
        clear_list();
        if (sh.bin == kSmpFine) return 1;
        const float around = 0.6f / per32 + (high - low) * 1e-6f, x_to = fmaxf(high - ((float)sh.bin_to + 1.f) / per - around, low);
        x_from = high - (float)sh.bin / per + around;
        // What lies above them is summed, what lies in them listed.  (The list takes elements behind tie_last at the threshold of top-k too: goal
        // is reached in front of them.)
        const Sum part = row_sum(weigh_all(Cut{sample_value(sample_code(x_from) + 1), 0.f, INT32_MAX}));
        each(x_to, x_from, [&](float x, int i) { if (x >= x_to && x <= x_from) append(x, i); });
        n = join_list();
        if (n == 0 || n > kSmpList) return 1;
        sort(n);
        return settle(n, part.units, goal, doubt_apart(share, part, all), least, tie_last);
    }
    // The token, by one thread of the row.
    __device__ __forceinline__ void write(int64_t r, float x, int index, float temperature, u64 total) const
    {
        a.tokens[r] = index;
        if (!a.logp) return;
        const double y = top == INFINITY ? 0.0 : ((double)x - (double)top) / (double)temperature;
        a.logp[r] = (float)(y - log((double)total / kSmpUnit));
    }
};

template <typename T, bool CLUSTER>
__global__ void __launch_bounds__(kSmpThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a)
{
    constexpr int N = Vec<T>::N;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    SampleShared &sh = *reinterpret_cast<SampleShared *>(smem_raw);
    T *data = reinterpret_cast<T *>(smem_raw + round_up(sizeof(SampleShared), 16));
    pdl_wait();
    Sampler<T, CLUSTER> s{a, sh, data};
    const int blocks = s.blocks(), rank = s.rank();
    const int64_t r = blockIdx.x / blocks;

    // The row in pieces of 16 bytes from the boundary in front of it; what the first and the last piece hold of other rows counts as -inf.
    const T *row = static_cast<const T *>(a.logits) + r * a.ld;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    const int all_vecs = (a.vocab + skew + N - 1) / N, v0 = min(rank * a.vecs, all_vecs);
    s.n_vec = min(a.vecs, all_vecs - v0);
    s.per_thread = (s.n_vec + kSmpThreads - 1) / kSmpThreads | 1;
    s.first = v0 * N - skew;
    for (int v = threadIdx.x; v < s.n_vec; v += kSmpThreads) {
        const int at = s.first + v * N;
        if (at >= 0 && at + N <= a.vocab) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(data + v * N)), "l"(row + at) : "memory");
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) { store_val(data + v * N + e, -INFINITY); if (at + e >= 0 && at + e < a.vocab) data[v * N + e] = row[at + e]; }
        }
    }
    if (threadIdx.x < 16) sh.exp2_table[threadIdx.x] = exp2(threadIdx.x / 16.0);
    const float temperature = a.temperature ? a.temperature[r] : 1.f;
    const int k = a.top_k ? a.top_k[r] : 0;
    const float p = a.top_p ? a.top_p[r] : 1.f, min_p = a.min_p ? a.min_p[r] : 0.f;
    const float u = fmaxf(a.u[r], 0.f);
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float top[kSmpGroups];                       // maxima of four groups of pieces, as evenly as they come
#pragma unroll
    for (int i = 0; i < kSmpGroups; ++i) top[i] = -INFINITY;
    {
        for (int v = threadIdx.x; v < s.n_vec; v += kSmpGroups * kSmpThreads)
#pragma unroll
            for (int i = 0; i < kSmpGroups; ++i) {
                if (v + i * kSmpThreads >= s.n_vec) break;
                const uint4 w = *reinterpret_cast<const uint4 *>(data + (v + i * kSmpThreads) * N);
                if constexpr (N == 8) {
                    const auto two = [](const uint32_t &x) { return *reinterpret_cast<const __nv_bfloat162 *>(&x); };
                    const __nv_bfloat162 m2 = __hmax2(__hmax2(two(w.x), two(w.y)), __hmax2(two(w.z), two(w.w)));
                    top[i] = fmaxf(top[i], fmaxf(__low2float(m2), __high2float(m2)));
                } else {
                    top[i] = fmaxf(top[i], fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w))));
                }
            }
        const float m = warp_max(fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])));
        if ((threadIdx.x & 31) == 0) sh.warp_sum[threadIdx.x >> 5] = __float_as_uint(m);
        __syncthreads();
        float all_max = -INFINITY;
#pragma unroll
        for (int w = 0; w < kSmpWarps; ++w) all_max = fmaxf(all_max, __uint_as_float((uint32_t)sh.warp_sum[w]));
        if (CLUSTER) {
            if (threadIdx.x == 0) sh.max = all_max;
            s.row_sync();
            for (int i = 0; i < blocks; ++i) all_max = fmaxf(all_max, *s.at(&sh.max, i));
        }
        s.top = all_max;
    }
    const bool writer = rank == 0 && threadIdx.x == 0;
    if (!(s.top > -INFINITY) || !(temperature > 0.f)) {
        // the maximum's first index, by the threads that have noted it
        if (threadIdx.x == 0) sh.index = INT32_MAX;
        __syncthreads();
        if (s.top > -INFINITY)
#pragma unroll
            for (int i = 0; i < kSmpGroups; ++i) {
                if (top[i] != s.top) continue;
                for (int v = threadIdx.x + i * kSmpThreads; v < s.n_vec; v += kSmpGroups * kSmpThreads) {
                    float x[N];
                    s.unpack(*reinterpret_cast<const uint4 *>(data + v * N), x);
                    int e = N;
#pragma unroll
                    for (int j = N - 1; j >= 0; --j) if (x[j] == s.top) e = j;
                    if (e < N) { atomicMin(&sh.index, s.first + v * N + e); break; }
                }
            }
        s.row_sync();
        int token = sh.index;
        for (int i = 0; i < blocks; ++i) token = min(token, *s.at(&sh.index, i));
        if (token == INT32_MAX) token = -1;
        if (writer) {
            a.tokens[r] = token;
            if (a.logp) a.logp[r] = token < 0 ? -INFINITY : 0.f;
        }
        if (CLUSTER) s.row_sync();               // nobody leaves while its shared memory is read
        return;
    }
    s.scale = 1.4426950408889634 / (double)temperature;
    s.fast_scale = (float)s.scale;
    s.least_weighed = fmaxf((float)((double)s.top - 60.0 / s.scale), -FLT_MAX);       // what lies below weighs less than 2^-46 for certain, however this is rounded
    // Kept: elements above `least`, and of those that equal it the ones up to index tie_last.
    float least = -INFINITY;
    int tie_last = -1;
    // w >= min_p is x >= floor_x, the smallest number that weighs as much: between two numbers a millionth apart around its logarithm
    float floor_x = -INFINITY;
    if (min_p > 0.f && s.top < INFINITY) {
        const double low = fmin((double)min_p, 1.0);
        const float guess = (float)((double)s.top + log2(low) / s.scale);
        if (guess > -INFINITY) {
            uint32_t lo = sample_code(guess - fabsf(guess) * 1e-6f - 1e-37f), hi = sample_code(s.top);              // the maximum weighs 1
            const uint32_t near = sample_code(guess + fabsf(guess) * 1e-6f + 1e-37f);
            if (near < hi && s.weight(sample_value(near)) >= low) hi = near;
            if (s.weight(sample_value(lo)) >= low) lo = kSmpLeastCode;
#pragma unroll 1
            while (hi - lo > 1) {                // w(lo) < low <= w(hi)
                const uint32_t mid = lo + (hi - lo) / 2;
                if (s.weight(sample_value(mid)) >= low) hi = mid; else lo = mid;
            }
            floor_x = sample_value(hi);
        }
    } else if (min_p > 0.f) {
        floor_x = INFINITY;
    }
    bool cut = p < 1.f;                          // top-p is still to be done
    const uint4 tops = make_uint4(sample_code(top[0]), sample_code(top[1]), sample_code(top[2]), sample_code(top[3]));
    if (k > 0 && k < a.vocab) {
        const float bound = s.bound_of_kth(k, tops);
        int n = kSmpList + 1;
        if (bound > -INFINITY || a.vocab <= kSmpList) {
            s.clear_list();
            s.each(bound, INFINITY, [&](float x, int i) { if (x > -INFINITY) s.append(x, i); });
            n = s.join_list();
        }
        if (n <= kSmpList) {
            s.sort(n);
            n = min(n, k);
            if (cut) {
                u64 w[3], total;
                s.weigh_listed(n, w, total);
                n = min(n, s.reach(n, max((u64)ceil(fmax((double)p, 0.0) * (double)total), 1ull), 0));
                cut = false;
            }
            least = s.listed_value(n - 1);
            tie_last = s.listed_index(n - 1);
            if (n <= kSmpSmall) {
                // the few that are kept, in index order
                u64 c = 0, w[3], total;
                if ((int)threadIdx.x < n) c = s.listed_value(threadIdx.x) >= floor_x;
                s.block_scan(c, total);
                n = (int)total;
                __syncthreads();
                if ((int)threadIdx.x < n) sh.list[threadIdx.x] = sh.list[threadIdx.x] << 32 | sh.list[threadIdx.x] >> 32;           // ~index first
                s.sort(n);
                u64 sum = 0;
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const int j = 3 * threadIdx.x + i;
                    w[i] = j < n ? s.weigh(sample_value((uint32_t)sh.list[j])) : 0ull;
                    sum += w[i];
                }
                u64 front = s.block_scan(sum, total) - sum;
                const u64 goal = min((u64)((double)u * (double)total), total - 1);
#pragma unroll
                for (int i = 0; i < 3; ++i) {
                    const int j = 3 * threadIdx.x + i;
                    if (rank == 0 && goal >= front && goal < front + w[i]) s.write(r, sample_value((uint32_t)sh.list[j]), (int)~(uint32_t)(sh.list[j] >> 32), temperature, total);
                    front += w[i];
                }
                if (CLUSTER) s.row_sync();
                return;
            }
        } else {
            const auto found = s.template select<true>(bound, k);
            least = found.value;
            if (least > -INFINITY) tie_last = s.nth((int)(k - (int64_t)found.above), least);
        }
    }
    // With fp32 weights first.  What comes of them is what comes of exact ones unless a sum ends as near to its goal as both may be off
    // together (doubt()).  Then those sums are taken again, exactly.  A maximum of +inf and temperatures beyond fp32's reach go there at once.
    s.nothing = s.top - 150.f / s.fast_scale;
    s.exact = !(s.top < INFINITY && s.fast_scale < 1e30f && s.fast_scale > 1e-30f && (s.top - s.nothing) * s.fast_scale > 140.f);
    if (cut) {
        const double share = fmax((double)p, 0.0);
        const auto goal_of = [&](u64 all) { return min(max((u64)ceil(share * (double)all), 1ull), all); };
        int outcome = 1, n = 0;
        float x_from = INFINITY;
        if (!s.exact) {
            // Some hundred of the largest elements may be enough: those above the bound of the 128-th.  The noted maxima among them are most of their weight.
            const float bound = fmaxf(s.bound_of_kth(128, tops), least);
            float noted_w = 0.f, no_matter;
            const auto note = [&](uint32_t code) { const float x = sample_value(code); if (x > bound) noted_w += s.fast_weight(x, no_matter); };
            note(tops.x); note(tops.y); note(tops.z); note(tops.w);
            const auto all = s.row_sum(s.weigh_all(s.cut_of(least, tie_last, -INFINITY)));
            u64 noted = (u64)((double)noted_w * kSmpUnit), none = 0;
            s.row_sums(noted, none);
            const u64 goal = goal_of(all.units);
            if (noted >= goal + all.off) {
                s.clear_list();
                s.each(bound, INFINITY, [&](float x, int i) { if (x > bound) s.append(x, i); });
                n = s.join_list();
                if (n > 0 && n <= kSmpList) {
                    s.sort(n);
                    outcome = s.settle(n, 0, goal, s.doubt(share, 0, all.off), least, tie_last);
                }
            }
            // What weighs less than (1 - p) W / V is not needed; 0.1 % below, for the roundings on the way: half a unit for each of V
            // elements is no more than that as long as this weight is 500 units or more.
            const double floor_w = (1.0 - share) * ((double)all.units / kSmpUnit) / a.vocab * 0.999;
            if (outcome == 1 && floor_w >= 0x1p-34) {
                const float lowest = s.top - fmaxf((float)(-log2(floor_w) / s.scale) * 1.00001f, 1e-30f);
                if (lowest < s.top) outcome = s.fine_select(lowest, goal, share, all, x_from, n, least, tie_last);
            }
        }
        if (outcome) {
            const bool exact = s.exact;
            s.exact = true;
            const auto mine = s.weigh_exactly(s.cut_of(least, tie_last, -INFINITY), x_from);
            u64 all = mine.x, above = mine.y;
            s.row_sums(all, above);
            const u64 goal = goal_of(all);
            if (outcome == 2) outcome = s.settle(n, above, goal, 0, least, tie_last);
            if (outcome) {
                const auto found = s.template select<false>(least, goal);
                const float t = found.value;
                const u64 one = max(s.weigh(t), 1ull);
                const int last = s.nth((int)min((goal - found.above + one - 1) / one, (u64)a.vocab), t);
                tie_last = t == least ? min(tie_last, last) : last;
                least = t;
            }
            s.exact = exact;
        }
    }
#pragma unroll 1
    while (true) {
        // the kept weights' sums, in index order
        const auto kept = s.cut_of(least, tie_last, floor_x);
        const auto mine = s.exact ? typename Sampler<T, CLUSTER>::Sum{s.weigh_exactly(kept, INFINITY).x, 0} : s.weigh_all(kept);
        u64 total, all_off = 0, part_off = 0;
        const u64 upto = s.row_scan(mine.units, total);
        // the token's running sum is the first above goal
        const u64 goal = min((u64)((double)u * (double)total), total - 1);
        if (!s.exact) part_off = s.row_scan(mine.off, all_off);
        s.find_thread(mine.units, upto, goal);
        if ((int)threadIdx.x == sh.winner) sh.above = part_off - mine.off;         // of the sums in front: the winner's own elements are weighed exactly below
        if (threadIdx.x == 0) sh.found = 0;
        __syncthreads();
        if (sh.winner >= 0 && threadIdx.x < 32) {
            // the winner's elements, a piece per lane; their weights exact
            const u64 doubt = s.exact ? 0 : s.doubt(fmin((double)u, 1.0), sh.above, all_off);
            const int lane = threadIdx.x, v = sh.winner * s.per_thread + lane;
            const bool there = lane < s.per_thread && v < s.n_vec;
            u64 left = sh.left;
            float x[N];
            u64 c[N], sum = 0;
            s.unpack(there ? *reinterpret_cast<const uint4 *>(data + v * N) : make_uint4(0u, 0u, 0u, 0u), x);
#pragma unroll
            for (int e = 0; e < N; ++e) { c[e] = there && s.kept(kept, x[e], s.first + v * N + e) ? s.weigh(x[e]) : 0ull; sum += c[e]; }
            u64 run = sum;
#pragma unroll
            for (int o = 1; o < 32; o *= 2) { const u64 t = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += t; }
            if (left >= run - sum && left < run) {
                left -= run - sum;
                bool open = true;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (open && left < c[e]) {
                        open = false;
                        if (s.exact || (left >= doubt && left + doubt < c[e])) {
                            sh.found = 1;
                            s.write(r, x[e], s.first + v * N + e, temperature, total);
                        }
                    }
                    left -= c[e];
                }
            }
        }
        s.row_sync();
        int found = s.exact;
        if (!s.exact)
            for (int i = 0; i < blocks; ++i) found += *s.at(&sh.found, i);
        s.row_sync();                            // nobody leaves, or goes on, while its shared memory is read
        if (found) return;
        s.exact = true;
    }
}

template <typename T> static int launch_sample(SampleArgs &a, int64_t rows, cudaStream_t st)
{
    constexpr int N = Vec<T>::N;
    const size_t head = round_up(sizeof(SampleShared), 16);
    // Blocks per row: one as long as the row fits into its shared memory, whether or not that leaves room for a second block on the SM; else as many as it
    // takes, eight at most.  (A cluster of two, so that two blocks share an SM again, costs the barriers of a cluster in every short step: 256 fp32 rows of
    // 32000, top-p and min-p, 72 us with one block and 102 with two; 64 of them 47 and 61; without filters 37 and 43; 1024 bf16 rows of 65000, mixed, 174 and
    // 225, of 80000 217 and 260; 64 bf16 rows of 65000, temperature only, 41 and 41.)
    int n = 1;
    const auto vecs = [&](int n) { return (a.vocab + N - 1 + N - 1 + n * N - 1) / (n * N); };          // a row may start anywhere in a piece
    while (n < 8 && head + (size_t)vecs(n) * 16 > kSmpMaxSmem) n *= 2;
    a.vecs = vecs(n);
    const size_t smem = head + (size_t)a.vecs * 16;
    SP_REQUIRE(smem <= kSmpMaxSmem, SP_ERR_UNSUPPORTED, "sp_sample_tokens: a row of %d logits does not fit", a.vocab);
    const auto kern = n > 1 ? sample_kernel<T, true> : sample_kernel<T, false>;
    SP_CUDA(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmpMaxSmem));
    return launch(kern, dim3((unsigned)(rows * n)), kSmpThreads, smem, st, n, a);
}

}  // namespace sp

extern "C" int sp_sample_tokens(const void *logits, int64_t ld_logits, int64_t n_rows, int vocab, const float *u,
                                const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p,
                                int32_t *tokens, float *logp, int dtype, void *stream)
{
    using namespace sp;
    SP_REQUIRE(dtype == SP_F32 || dtype == SP_BF16, SP_ERR_INVALID_ARG, "sp_sample_tokens: unknown dtype %d", dtype);
    SP_REQUIRE(n_rows >= 0 && vocab >= 1, SP_ERR_INVALID_ARG, "sp_sample_tokens: bad n_rows / vocab");
    SP_REQUIRE(ld_logits >= vocab, SP_ERR_INVALID_ARG, "sp_sample_tokens: ld_logits %lld < vocab %d", (long long)ld_logits, vocab);
    SP_REQUIRE(vocab <= kSmpMaxVocab, SP_ERR_UNSUPPORTED, "sp_sample_tokens: vocab %d (at most %d supported)", vocab, kSmpMaxVocab);
    SP_REQUIRE(n_rows < (1 << 28), SP_ERR_UNSUPPORTED, "sp_sample_tokens: too many rows");
    if (n_rows == 0) return SP_OK;
    SP_REQUIRE(logits && u && tokens, SP_ERR_INVALID_ARG, "sp_sample_tokens: NULL pointer");
    SP_REQUIRE(((uintptr_t)logits & (elt_bytes(dtype) - 1)) == 0, SP_ERR_INVALID_ARG, "sp_sample_tokens: logits are not aligned to their type");
    SampleArgs a = {};
    a.logits = logits; a.u = u; a.temperature = temperature; a.top_p = top_p; a.min_p = min_p; a.top_k = top_k;
    a.tokens = tokens; a.logp = logp; a.ld = ld_logits; a.vocab = vocab;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == SP_BF16 ? launch_sample<__nv_bfloat16>(a, n_rows, st) : launch_sample<float>(a, n_rows, st);
}
