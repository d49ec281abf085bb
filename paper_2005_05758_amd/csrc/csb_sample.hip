// Sampling from logits with temperature, top-k, top-p and min-p (csb_sample).
//
// A token's weight is a whole number of units, floor(2^38 e^((logit - max) / T)), so sums of units are the same in any order, and what is kept and
// drawn depends on nothing but the row and its numbers.  Top-k and top-p keep a beginning of the order by (logit, number); where it ends
// is searched for without sorting the row.  Buckets of (max - logit) / T, 1023 of them as far as weights have units, order tokens coarsely:
//   few:    for k of at most kFewest tokens the k-th largest of the maxima of groups of tokens bounds the k-th token from below; the tokens of the buckets up
//           to that one's, a few more than k, are ranked against each other, and all else happens among them;
//   many:   a histogram holds how many tokens and units each bucket has, sums over it find the bucket in which what is kept ends, and the
//           tokens of that one bucket are split again by their place in the order, 1024 parts at a time, until the part has one token.
// (A place is the logit's bits and the token's number in 64 bits, so places differ and ties need no care.)  Tokens of the last bucket have no whole unit:
// they are counted nowhere, and cannot be drawn.  Exponentials are binary64, which this card does as fast as binary32.
//
// Rows of up to kRowMost bytes: one launch, a workgroup a row, which it holds in LDS; what is kept goes into a list there if it fits, else its units stay in registers, so
// that the row is passed over twice or three times and no more (165 rows of 32003 bfloat16 tokens, top-p and their distributions, 38 us; by the kernels for larger rows
// 56).  Others, in chunks of 4096 tokens: maxima of groups; few, and beside them the histogram of the other rows (where nothing is cut: units of the chunks); the
// bucket's tokens and the units before it by chunk; the end of what is kept and the draw; the distribution, if it is asked for.  (64 rows of 131071 binary32
// tokens, four rows in five few: 43 us; all few, k of 40, 23; by histograms, k of 1000, 45, top-p of 0.9 61; alone, both of these, 126; nothing cut 31.)
// Bound by the issue of vector instructions where all of a row counts (36 a token and pass, 22 of them for the exponential), else by latencies: each launch is a chain of
// trips to memory and of barriers.
#include <algorithm>
#include <new>
#include <type_traits>

#include "csb_layer.hpp"

namespace csb {

constexpr int kRowMost = 98304, kRowSmall = kRowMost / 3;      // bytes of a row that a workgroup holds; of one that leaves room for another workgroup
constexpr int kBuckets = 1024, kChunk = 4096, kMaxChunks = 4096, kListMost = 4096, kFewMost = 1024, kFewest = 256, kRankMost = 320;
constexpr double kUnit = 274877906944.0;       // 2^38

enum RowState : uint32_t { ROW_WHOLE, ROW_CUT, ROW_ALONE };    // nothing is cut; by the histogram; by one workgroup

struct SampleDev {
    const void *logits;
    const float *temperature, *top_p, *min_p, *r;
    const int32_t *top_k;
    int32_t *tokens;
    void *probs;
    int64_t ld, ldp;
    int32_t rows, vocab, chunks;
    // workspace: [rows][chunks], [rows][chunks][256], [rows][kBuckets] (units, or tokens where k cuts), [rows], [rows][kListMost], [rows] (NULL: no row is few)
    float *maxes, *groups;
    unsigned long long *histogram, *sums;
    uint32_t *listed, *done;
    uint64_t *ends, *totals, *list;
};

// a b + c, the constant in scalar registers (the compiler copies it to vector registers each time, to add to it there: three instructions instead of one).
__device__ __forceinline__ double fma_of_constant(double a, double b, double c) {
    double d;
    asm("v_fma_f64 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "s"(c));
    return d;
}

// What a row's numbers ask for.
struct SampleRow {
    float m, per_bucket, part, part_of_m;      // (part: of logits, so that no difference of two overflows where the temperature makes numbers of such)
    double per_bit;                            // log2 e / T
    int32_t k;                                 // 0: all
    uint32_t p;                                // floor(top_p 2^24); 2^24: all
    double least;                              // units that min-p asks for
    __device__ __forceinline__ SampleRow(const SampleDev &a, int row, float max) : SampleRow(a, row) { largest(max); }
    // what does not need the largest logit
    __device__ __forceinline__ SampleRow(const SampleDev &a, int row) {
        const float T = a.temperature ? a.temperature[row] : 1.0f;
        k = a.top_k ? a.top_k[row] : 0;
        if (k < 1 || k >= a.vocab) k = 0;
        const float tp = a.top_p ? a.top_p[row] : 1.0f;
        p = tp < 1.0f ? (uint32_t)(fmaxf(tp, 0.0f) * 16777216.0f) : 1u << 24;
        const float mp = a.min_p ? a.min_p[row] : 0.0f;
        least = mp > 0.0f ? __builtin_floor((double)fminf(mp, 1.0f) * kUnit) : 0.0;
        if (T > 0.0f) {
            per_bit = 1.4426950408889634 / (double)T;
            part = T > 0x1p60f ? 0.5f : 1.0f;
            per_bucket = (float)((kBuckets - 1) / 26.5 / part / (double)T);    // e^-26.5 2^38 < 1
        } else {
            per_bit = per_bucket = __builtin_inff();           // the largest alone,
            k = 1;                                             // and the first of them
            part = 1.0f;
        }
    }
    __device__ __forceinline__ void largest(float max) {
        m = max;
        part_of_m = m * part;
    }
    __device__ __forceinline__ bool cut() const { return k || p < 1u << 24; }
    // units of a token; whole, below 2^39
    __device__ __forceinline__ double weight(float s) const {
        double y;
        const double w = weight_within(s, &y);
        return s == m ? kUnit : y > -40.0 ? w : 0.0;           // (infinite logits, and NaN of infinite temperatures)
    }
    // the same for finite ones; y: the weight's binary logarithm, 38 taken off
    __device__ __forceinline__ double weight_within(float s, double *log) const {
        const double y = ((double)s - (double)m) * per_bit, t = y + (0x1.8p52 + 38.0), f = y - (t - (0x1.8p52 + 38.0));  // (t: the nearest whole number, and its 32 bits)
        *log = y;
        double e = 1.0205905413765595e-07;                   // 2^f for |f| <= 1/2 to 2^-45, through ten of Chebyshev's points
        e = fma_of_constant(e, f, 1.325964524488711e-06);
        e = fma_of_constant(e, f, 1.5252672924850737e-05);
        e = fma_of_constant(e, f, 0.0001540343375125101);
        e = fma_of_constant(e, f, 0.0013333558200794592);
        e = fma_of_constant(e, f, 0.009618129193934313);
        e = fma_of_constant(e, f, 0.05550410866465167);
        e = fma_of_constant(e, f, 0.2402265069564034);
        e = fma_of_constant(e, f, 0.6931471805599462);
        e = fma_of_constant(e, f, 1.0000000000000135);
        return __builtin_floor(__builtin_amdgcn_ldexp(e, (int)(uint32_t)__builtin_bit_cast(uint64_t, t)));
    }
    // four at a time, side by side and for all lanes, whatever they are used for: one by one each instruction waits for the one before
    __device__ __forceinline__ void weights_within(const float *s, double *w, double *log) const {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = weight_within(s[j], log + j);
        asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = s[j] == m ? kUnit : w[j];
    }
    // a logit that no token up to bucket b is below (others may be above it, none of them infinite): the rounding of bucket() is 2^-22 of it, of the difference 2^-22 of m
    __device__ __forceinline__ float least_of(int b) const {
        const float t = m - (float)(b + 1) * 1.0001f / (per_bucket * part) - fabsf(m) * 0x1p-22f;
        return t > -0x1.fffffep127f ? t : -0x1.fffffep127f;
    }
    __device__ __forceinline__ int bucket(float s) const {
        float b = fminf(fmaf(s, -part, part_of_m) * per_bucket, (float)(kBuckets - 1));
        asm("" : "+v"(b));                                     // (a choice of two numbers, no branch around one)
        return (int)(s == m ? 0.0f : b);
    }
};

__device__ __forceinline__ uint64_t whole(double w) { return __builtin_bit_cast(uint64_t, w + 0x1p52) & 0xfffffffffffffull; }
// A logit as it counts: NaN as -infinity, -0 as 0.
__device__ __forceinline__ float logit(float s) { return s == s ? s + 0.0f : -__builtin_inff(); }
// A token's place in the order: larger ones come first.
__device__ __forceinline__ uint64_t place(float s, uint32_t v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, s);
    return (uint64_t)(b ^ (b >> 31 ? 0xffffffffu : 0x80000000u)) << 32 | (0xffffffffu - v);
}
__device__ __forceinline__ float logit_at(uint64_t place) {
    const uint32_t b = (uint32_t)(place >> 32);
    return __builtin_bit_cast(float, b ^ (b >> 31 ? 0x80000000u : 0xffffffffu));
}
// floor(all * m / 2^24), m <= 2^24
__device__ __forceinline__ uint64_t part_of(uint64_t all, uint32_t m) { return (all >> 24) * m + (((all & 0xffffff) * m) >> 24); }
__device__ __forceinline__ uint32_t draw_number(float r) { return r > 0.0f ? min((uint32_t)(fminf(r, 1.0f) * 16777216.0f), 16777215u) : 0u; }

// Four logits from v on; -infinity past `end`.
template <int VF> __device__ __forceinline__ void logits4(const void *row, int32_t v, int32_t end, float *s) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    const T *p = (const T *)row + v;
    if (v + 4 <= end) {
        const T4 x = load_any<T4>(p);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = logit((float)x[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = v + j < end ? logit((float)p[j]) : -__builtin_inff();
    }
}
template <int VF> __device__ __forceinline__ void probs4(void *row, int32_t v, int32_t end, const float *x) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    T *p = (T *)row + v;
    if (v + 4 <= end) {
        T4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (T)x[j];
        store_any(p, y);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) if (v + j < end) p[j] = (T)x[j];
    }
}

// v moved to other lanes: by CTRL, in the rows of 16 lanes of ROWS; zero where no lane's comes.
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, true); }
template <int CTRL, int ROWS> __device__ __forceinline__ uint64_t moved(uint64_t v) {
    return (uint64_t)moved<CTRL, ROWS>((uint32_t)(v >> 32)) << 32 | moved<CTRL, ROWS>((uint32_t)v);
}
// Sum over the lanes up to this one: within rows of 16, then over the rows.
template <typename N> __device__ __forceinline__ N upto_in_wave(N v) {
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v);
    v += moved<0x143, 0xc>(v);
    return v;
}
template <typename N> __device__ __forceinline__ N before_in_wave(N v) { return upto_in_wave(v) - v; }
template <typename N> __device__ __forceinline__ N of_lane(N v, int lane) {
    if constexpr (sizeof(N) == 8) return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
    else return (N)__builtin_amdgcn_readlane((int)v, lane);
}
template <typename N> __device__ __forceinline__ N sum_of_wave(N v) { return of_lane(upto_in_wave(v), 63); }
__device__ __forceinline__ uint64_t max_of_wave(uint64_t v) {  // (0: none)
    const auto larger = [](uint64_t x, uint64_t y) { return x > y ? x : y; };
    v = larger(v, moved<0x111, 0xf>(v));
    v = larger(v, moved<0x112, 0xf>(v));
    v = larger(v, moved<0x114, 0xf>(v));
    v = larger(v, moved<0x118, 0xf>(v));
    v = larger(v, moved<0x142, 0xa>(v));
    v = larger(v, moved<0x143, 0xc>(v));
    return of_lane(v, 63);
}

// A workgroup's memory for the searches of a row.
struct SampleShared {
    unsigned long long units[kBuckets], low, high, found, found_units, base_units;
    uint64_t part_units[16];
    uint32_t counts[kBuckets], part_counts[16];
    uint64_t few_units[64];
    uint32_t bin, bin_count, base_count, listed, few_tokens[64];
    int32_t token;
    float part_max[16];
};

// Of sixteen numbers, one for each wavefront: the sum of those before the caller's; *all: of all.
template <typename N> __device__ __forceinline__ N before_of_waves(const N *parts, N *all) {
    N v = parts[threadIdx.x & 15];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    v += moved<0x111, 0xf>(v);
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    *all = of_lane(v, 15);
    return wave ? of_lane(v, wave - 1) : 0;
}
// Sum over the threads below this one; *total: of all.
__device__ __forceinline__ uint64_t block_before(SampleShared &sh, uint64_t v, uint64_t *total) {
    const uint64_t before = before_in_wave(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.part_units[threadIdx.x >> 6] = before + v;
    __syncthreads();
    return before + before_of_waves(sh.part_units, total);
}

// The bin, of counts and units in LDS by thread, in which what is kept ends: of `target` tokens (BY_COUNT), or of those with fewer
// than `target` units before them; counted from what sh.base_* hold, which is moved up to the bin (UNITS: units too).  1024 threads, all of them.
template <bool BY_COUNT, bool UNITS = true> __device__ __forceinline__ void find_bin(SampleShared &sh, uint64_t target) {
    const int tid = threadIdx.x, wave = tid >> 6;
    const uint32_t c = sh.counts[tid];
    const uint64_t u = UNITS ? sh.units[tid] : 0;
    uint32_t cb = BY_COUNT ? before_in_wave(c) : 0;
    uint64_t ub = UNITS ? before_in_wave(u) : 0;
    if ((tid & 63) == 63) {
        if (BY_COUNT) sh.part_counts[wave] = cb + c;
        if (UNITS) sh.part_units[wave] = ub + u;
    }
    __syncthreads();
    uint32_t all_counts;
    uint64_t all_units;
    cb += sh.base_count;
    ub += sh.base_units;
    if (BY_COUNT) cb += before_of_waves(sh.part_counts, &all_counts);
    if (UNITS) ub += before_of_waves(sh.part_units, &all_units);
    __syncthreads();                                           // (base_* are read)
    if (BY_COUNT ? cb < target && cb + c >= target : ub < target && ub + u >= target) {   // one thread, or none
        sh.bin = tid;
        sh.bin_count = c;
        sh.base_count = cb;
        sh.base_units = ub;
    }
    __syncthreads();
}

// The same for a share of all units: returns the target.  sh.base_count: about how many tokens the buckets up to the bin have, by the units that a token has in the
// middle of a bucket (1.4 % off where a bucket's tokens lie at one of its ends).
__device__ __forceinline__ uint64_t find_share(SampleShared &sh, uint32_t p, uint64_t *all) {
    const int tid = threadIdx.x;
    const uint64_t u = sh.units[tid];
    const uint32_t about = (uint32_t)((float)u * __builtin_amdgcn_exp2f((float)tid * (float)(26.5 / (kBuckets - 1) * 1.4426950408889634) + (float)(0.5 * 26.5 / (kBuckets - 1) * 1.4426950408889634 - 38.0)) + 0.9f);
    const uint32_t count = before_in_wave(about) + about;
    if ((tid & 63) == 63) sh.part_counts[tid >> 6] = count;
    const uint64_t before = block_before(sh, u, all), share = part_of(*all, p), target = share ? share : 1;
    if (before < target && before + u >= target) {
        sh.bin = tid;
        sh.bin_count = count;
        sh.base_units = before;
    }
    __syncthreads();
    uint32_t total;
    if (tid >> 6 == (int)(sh.bin >> 6)) {
        const uint32_t below = before_of_waves(sh.part_counts, &total);
        if ((tid & 63) == 0) sh.base_count = below + sh.bin_count;
    }
    __syncthreads();
    return target;
}

// The last token kept, among those that tokens.each names (calls its argument with places and units): sh.found, and the units up to and
// with it: sh.found_units.  sh.base_* hold what comes before all of them.
template <bool BY_COUNT, typename Tokens> __device__ __forceinline__ void find_token(SampleShared &sh, uint64_t target, const Tokens &tokens) {
    const int tid = threadIdx.x;
    if (tid == 0) { sh.low = ~0ull; sh.high = 0; sh.found = 0; sh.found_units = 0; }
    __syncthreads();
    uint64_t low = ~0ull, high = 0;
    tokens.each([&](uint64_t at, double) { low = at < low ? at : low; high = at > high ? at : high; });
    low = ~max_of_wave(~low);
    high = max_of_wave(high);
    if ((tid & 63) == 0 && low <= high) { atomicMin(&sh.low, (unsigned long long)low); atomicMax(&sh.high, (unsigned long long)high); }
    __syncthreads();
    low = sh.low;
    high = sh.high;
    for (;;) {                                                 // (uniform; places differ, so a part of 2^shift places ends at one token)
        const uint64_t range = high - low;
        const int bits = range ? 64 - __builtin_clzll(range) : 0, shift = bits > 10 ? bits - 10 : 0;
        sh.counts[tid] = 0;
        sh.units[tid] = 0;
        __syncthreads();
        if (tid == 0) sh.bin = kBuckets;
        tokens.each([&](uint64_t at, double w) {
            if (at >= low && at <= high) {
                const uint32_t b = (uint32_t)((high - at) >> shift);
                atomicAdd(&sh.counts[b], 1u);
                atomicAdd(&sh.units[b], (unsigned long long)whole(w));
            }
        });
        __syncthreads();
        find_bin<BY_COUNT>(sh, target);
        if (sh.bin >= (uint32_t)kBuckets) break;               // (cannot be, unless the logits change meanwhile)
        high -= (uint64_t)sh.bin << shift;
        const uint64_t width = ((uint64_t)1 << shift) - 1;
        low = high - low > width ? high - width : low;
        if (sh.bin_count <= 1 || shift == 0) break;
    }
    tokens.each([&](uint64_t at, double w) {
        if (at >= low && at <= high) { sh.found = at; sh.found_units = sh.base_units + whole(w); }
    });
    __syncthreads();
}

// The same among the `n` tokens of a list in LDS, at most kRankMost: ranked against each other, then one sum (n^2 / 16 clocks: a search by parts
// takes as long from 400 tokens on).
template <bool BY_COUNT> __device__ __forceinline__ void find_ranked(SampleShared &sh, const SampleRow &row, uint64_t target, const uint64_t *list, uint32_t n) {
    const uint32_t tid = threadIdx.x;
    const uint64_t at = tid < n ? list[tid] : 0;
    uint32_t rank = 0;
    if (tid < n)
#pragma unroll 8
        for (uint32_t i = 0; i < n; ++i) rank += list[i] > at;
    if (tid < n) sh.units[rank] = whole(row.weight(logit_at(at)));
    const uint32_t base_count = sh.base_count;
    const uint64_t base_units = sh.base_units;
    __syncthreads();
    if (tid == 0) { sh.found = 0; sh.found_units = 0; sh.bin = kBuckets; }
    const uint64_t u = tid < n ? sh.units[tid] : 0;
    uint64_t all, before = block_before(sh, u, &all) + base_units;
    if (tid < n && (BY_COUNT ? base_count + tid + 1 == target : before < target && before + u >= target)) {     // one thread
        sh.bin = tid;
        sh.found_units = before + u;
    }
    __syncthreads();
    if (tid < n && rank == sh.bin) sh.found = at;
    __syncthreads();
}

// Where what is kept of a row ends: the last token's place (0: nothing is cut).  sh.units and sh.counts hold the row's histogram.
template <typename Tokens>
__device__ __forceinline__ uint64_t end_of_kept(SampleShared &sh, const SampleRow &row, Tokens &tokens) {
    const int tid = threadIdx.x;
    const uint32_t c = sh.counts[tid];
    const uint64_t u = sh.units[tid];
    uint64_t units = 0, target = (uint64_t)row.k, end = 0;
    if (tid == 0) { sh.base_count = 0; sh.base_units = 0; sh.bin = kBuckets; }
    __syncthreads();
    if (row.k) find_bin<true>(sh, target);
    else target = find_share(sh, row.p, &units);
#pragma unroll 1
    for (bool by_count = row.k != 0;; by_count = false) {      // (uniform) by count, then by share of what that leaves
        if (sh.bin < (uint32_t)kBuckets) {                     // (uniform; else fewer tokens than k have units)
            tokens.gather((int)sh.bin, by_count ? sh.base_count + sh.bin_count : row.k ? 0 : sh.base_count);
            const bool few = sh.listed <= (uint32_t)kRankMost;
            if (by_count) few ? find_ranked<true>(sh, row, target, tokens.near(), sh.listed) : find_token<true>(sh, target, tokens);
            else few ? find_ranked<false>(sh, row, target, tokens.near(), sh.listed) : find_token<false>(sh, target, tokens);
            end = sh.found;
            units = sh.found_units;
        } else if (by_count) block_before(sh, u, &units);
        if (!by_count || row.p == 1u << 24) return end;
        const uint64_t share = part_of(units, row.p);
        target = share ? share : 1;
        __syncthreads();
        sh.counts[tid] = c;                                    // (a search uses their place)
        sh.units[tid] = u;
        if (tid == 0) { sh.base_count = 0; sh.base_units = 0; sh.bin = kBuckets; }
        __syncthreads();
        find_bin<false>(sh, target);
    }
}

// ---- reading a row, four tokens at a time: -infinity behind its end ------------------------------------------------------------------------
template <int VF> struct RowInMemory {
    const void *p;
    int32_t vocab;
    __device__ __forceinline__ void operator()(int32_t v, float *s) const { logits4<VF>(p, v, vocab, s); }
    __device__ __forceinline__ void raw(int32_t v, float *s) const { logits4<VF>(p, v, vocab, s); }
};
template <int VF> struct RowInLds {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    const T *p;
    int32_t vocab;                             // (rounded up to four: the rest holds -infinity)
    __device__ __forceinline__ void operator()(int32_t v, float *s) const {
        raw(v, s);
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = logit(s[j]);
    }
    // as they are: NaN may be among them, and -0
    __device__ __forceinline__ void raw(int32_t v, float *s) const {
        if (v < vocab) {
            const T4 x = *(const T4 *)(p + v);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = (float)x[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = -__builtin_inff();
        }
    }
};

// Largest of the workgroup's (1024 threads).
__device__ __forceinline__ float block_max(SampleShared &sh, float m) {
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((threadIdx.x & 63) == 0) sh.part_max[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) m = fmaxf(m, sh.part_max[w]);
    return m;
}
// The tokens of a row that take() wants, in a list in LDS in any order; sh.listed: how many there are, which may be more than the list holds.
template <typename Read, typename Take>
__device__ __forceinline__ void list_tokens(SampleShared &sh, const Read &read, int32_t vocab, uint64_t *list, Take take) {
    __syncthreads();
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
#pragma unroll 1
    for (int32_t v0 = 0; v0 < vocab; v0 += 16384) {
        float s[4][4];
        uint32_t mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) read.raw(v0 + 4096 * i + 4 * (int)threadIdx.x, s[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) mine += take(s[i / 4][i % 4]);
        const uint32_t upto = upto_in_wave(mine);
        uint32_t at = 0;
        if ((threadIdx.x & 63) == 63 && upto) at = atomicAdd(&sh.listed, upto);
        at = of_lane(at, 63) + upto - mine;
        if (mine)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (take(s[i / 4][i % 4])) {
                    if (at < (uint32_t)kListMost) list[at] = place(s[i / 4][i % 4] + 0.0f, v0 + 4096 * (i / 4) + 4 * threadIdx.x + i % 4);
                    ++at;
                }
    }
    __syncthreads();
}

// The tokens of one bucket: from a list of all tokens up to it, from a list of its own, or from the row each time where neither holds them.
template <typename Read> struct BucketTokens {
    SampleShared &sh;
    const SampleRow &row;
    const Read &read;
    int32_t vocab;
    uint64_t *list, *own;                      // of kListMost, of kRankMost
    uint32_t upto = ~0u;                       // tokens in the first; more than it holds: it has the bucket's
    int bucket = 0;
    __device__ __forceinline__ bool whole() const { return upto <= (uint32_t)kListMost; }
    // `about`: how many tokens there are up to bucket b, more or less
    __device__ __forceinline__ void gather(int b, uint32_t about) {
        bucket = b;
        if (upto == ~0u && about <= (uint32_t)kListMost) {
            const float least = row.least_of(b);
            list_tokens(sh, read, vocab, list, [&](float s) { return s >= least; });
            upto = sh.listed;
        }
        if (!whole()) {
            list_tokens(sh, read, vocab, list, [&](float s) { return row.bucket(s) == bucket; });
            return;
        }
        __syncthreads();
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < upto; i += 1024) {
            const uint64_t at = list[i];
            if (row.bucket(logit_at(at)) == bucket) {
                const uint32_t n = atomicAdd(&sh.listed, 1u);
                if (n < (uint32_t)kRankMost) own[n] = at;
            }
        }
        __syncthreads();
    }
    __device__ __forceinline__ const uint64_t *near() const { return whole() ? own : list; }      // at most kRankMost of them
    template <typename Take> __device__ __forceinline__ void each(Take take) const {
        if (whole()) {                                         // (uniform)
            for (uint32_t i = threadIdx.x; i < upto; i += 1024) {
                const float s = logit_at(list[i]);
                if (row.bucket(s) == bucket) take(list[i], row.weight(s));
            }
            return;
        }
        if (sh.listed <= (uint32_t)kListMost) {
            for (uint32_t i = threadIdx.x; i < sh.listed; i += 1024) take(list[i], row.weight(logit_at(list[i])));
            return;
        }
#pragma unroll 1
        for (int32_t v = 4 * (int)threadIdx.x; v < vocab; v += 4096) {
            float s[4];
            read(v, s);
#pragma unroll
            for (int j = 0; j < 4; ++j) if (row.bucket(s[j]) == bucket) take(place(s[j], v + j), row.weight(s[j]));
        }
    }
};

// The last token that is kept (its place 0: nothing is cut).
struct SampleEnd {
    float s;
    uint32_t v;
    __device__ __forceinline__ explicit SampleEnd(uint64_t end) : s(end ? logit_at(end) : -__builtin_inff()), v(end ? 0xffffffffu - (uint32_t)end : 0xffffffffu) {}
    __device__ __forceinline__ bool keeps(float x, int32_t number) const { return x > s || (x == s && (uint32_t)number <= v); }
};
// Units of a token of a row.
__device__ __forceinline__ double kept_units(const SampleRow &row, float s, int32_t v, const SampleEnd &end) {
    if (!end.keeps(s, v)) return 0.0;
    const double w = row.weight(s);
    return w < row.least ? 0.0 : w;
}

struct Kept { uint64_t end, total; int32_t token; uint32_t listed; };   // the last token's place, units of all, the token drawn; tokens in a list that has all kept (0: none has)

// The first k tokens, and all else, among the `n` of the list, which has them; k and n at most kFewMost.
__device__ __forceinline__ Kept draw_of_few(SampleShared &sh, const SampleRow &row, const uint64_t *list, uint32_t n, uint32_t number) {
    const uint32_t tid = threadIdx.x;
    const uint64_t at = tid < n ? list[tid] : 0;
    const double w = tid < n ? row.weight(logit_at(at)) : 0.0;
    uint32_t rank = 0, turn = 0;                               // by place, and by number: larger last words are lower numbers
    if (tid < n)
#pragma unroll 8
        for (uint32_t i = 0; i < n; ++i) {
            const uint64_t other = list[i];
            rank += other > at;
            turn += (uint32_t)other > (uint32_t)at;
        }
    if (tid == 0) { sh.found = ~0ull; sh.token = -1; }
    if (tid < n) sh.units[rank] = whole(w);
    __syncthreads();
    const uint64_t u = tid < n ? sh.units[tid] : 0;
    uint64_t all;
    const uint64_t before = block_before(sh, u, &all);
    const uint32_t most = min((uint32_t)row.k, n);
    if (tid == most - 1) sh.base_units = before + u;           // units of the first k
    sh.units[tid] = before;
    __syncthreads();
    const uint64_t part = part_of(sh.base_units, row.p);
    const bool kept = tid < n && rank < most && (row.p == 1u << 24 || sh.units[rank] < (part ? part : 1)) && w >= row.least;
    const uint64_t mine = kept ? whole(w) : 0, last = ~max_of_wave(kept ? ~at : 0);
    if ((tid & 63) == 0) atomicMin(&sh.found, (unsigned long long)last);
    __syncthreads();
    sh.units[tid] = 0;
    __syncthreads();
    if (tid < n) sh.units[turn] = mine;
    __syncthreads();
    const uint64_t own = sh.units[tid], below = block_before(sh, own, &all), limit = part_of(all, number);
    if (below <= limit && limit < below + own) sh.bin = tid;   // one thread: there is a token of some weight
    __syncthreads();
    if (tid < n && turn == sh.bin) sh.token = (int32_t)(0xffffffffu - (uint32_t)at);
    __syncthreads();
    return {sh.found, all, sh.token, n};
}

// The same where the last token is known, from a list of up to kListMost with all that are kept.
__device__ __forceinline__ Kept draw_of_list(SampleShared &sh, const SampleRow &row, int32_t vocab, const uint64_t *list, uint32_t n, uint64_t end, uint32_t number) {
    const uint32_t tid = threadIdx.x;
    const int bits = 32 - __builtin_clz((uint32_t)vocab), shift = bits > 10 ? bits - 10 : 0;      // 1024 parts of the numbers, of up to 2^shift
    __syncthreads();
    sh.units[tid] = 0;
    if (tid == 0) { sh.token = -1; sh.listed = 0; }
    __syncthreads();
    uint64_t u[kListMost / 1024];
    uint32_t v[kListMost / 1024];
#pragma unroll
    for (int i = 0; i < kListMost / 1024; ++i) {
        u[i] = 0;
        v[i] = 0;
        if (1024 * i + tid < n) {
            const uint64_t at = list[1024 * i + tid];
            const double w = row.weight(logit_at(at));
            if (at >= end && w >= row.least) u[i] = whole(w);
            v[i] = 0xffffffffu - (uint32_t)at;
            if (u[i]) atomicAdd(&sh.units[v[i] >> shift], (unsigned long long)u[i]);
        }
    }
    __syncthreads();
    const uint64_t part = sh.units[tid];
    uint64_t all;
    const uint64_t before = block_before(sh, part, &all), limit = part_of(all, number);
    if (before <= limit && limit < before + part) { sh.bin = tid; sh.base_units = before; }       // one thread: the first token has some weight
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kListMost / 1024; ++i)
        if (u[i] && v[i] >> shift == sh.bin) {
            const uint32_t to = atomicAdd(&sh.listed, 1u);
            sh.few_units[to] = u[i];
            sh.few_tokens[to] = v[i];
        }
    __syncthreads();
    if (tid < sh.listed) {
        const uint32_t own = sh.few_tokens[tid];
        uint64_t upto = sh.base_units;
        for (uint32_t i = 0; i < sh.listed; ++i) upto += sh.few_tokens[i] <= own ? sh.few_units[i] : 0;
        if (upto > limit && limit >= upto - sh.few_units[tid]) sh.token = (int32_t)own;
    }
    __syncthreads();
    return {end, all, sh.token, n};
}

// A bucket that the first k tokens do not reach past, by the maxima of disjoint groups of tokens that `each` names.
template <typename Each> __device__ __forceinline__ int bucket_of_first(SampleShared &sh, const SampleRow &row, Each each) {
    const int tid = threadIdx.x;
    sh.counts[tid] = 0;
    if (tid == 0) { sh.base_count = 0; sh.base_units = 0; sh.bin = kBuckets - 2; }
    __syncthreads();
    each([&](float m) {
        const int b = row.bucket(m);
        if (b < kBuckets - 1) atomicAdd(&sh.counts[b], 1u);
    });
    __syncthreads();
    find_bin<true, false>(sh, (uint64_t)row.k);
    return (int)sh.bin;
}

// Tokens of one wavefront that come one by one to some lanes, worked on 64 at a time: `buffer` holds 128 of them.
template <typename Item> struct WaveStream {
    Item *buffer;
    uint32_t held = 0;
    template <typename Work> __device__ __forceinline__ void add(bool mine, const Item &item, Work work) {
        const uint64_t who = __ballot(mine);
        if (mine) buffer[held + __builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0))] = item;
        held += (uint32_t)__builtin_popcountll(who);
        if (held >= 64) {                                      // (uniform in the wavefront, whose own LDS accesses stay in order)
            const uint32_t lane = threadIdx.x & 63;
            __builtin_amdgcn_wave_barrier();
            const Item first = buffer[lane], next = buffer[64 + lane];
            __builtin_amdgcn_wave_barrier();
            work(first, true);
            held -= 64;
            if (lane < held) buffer[lane] = next;
            __builtin_amdgcn_wave_barrier();
        }
    }
    template <typename Work> __device__ __forceinline__ void rest(Work work) {
        __builtin_amdgcn_wave_barrier();
        const bool there = (threadIdx.x & 63) < held;
        work(buffer[threadIdx.x & 63], there);
        held = 0;
    }
};

// Where what is kept of a row ends, by one workgroup of 1024 threads.
template <typename Read> __device__ __forceinline__ uint64_t cut_row(SampleShared &sh, const SampleRow &row, const Read &read, int32_t vocab, BucketTokens<Read> &tokens) {
    const int tid = threadIdx.x;
    __syncthreads();
    sh.counts[tid] = 0;
    sh.units[tid] = 0;
    __syncthreads();
#pragma unroll 1
    for (int32_t v = 4 * tid; v < vocab; v += 4096) {
        float s[4];
        double w[4], log[4];
        read.raw(v, s);
        row.weights_within(s, w, log);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int b = row.bucket(s[j]);                    // (the last one for NaN)
            if (b < kBuckets - 1) {
                if (row.k) atomicAdd(&sh.counts[b], 1u);
                atomicAdd(&sh.units[b], (unsigned long long)whole(w[j]));
            }
        }
    }
    __syncthreads();
    return end_of_kept(sh, row, tokens);
}

// A row in memory by one workgroup.  Wavefront w draws from the `per` tokens from w per on, 256 at a time.
template <typename Read>
__device__ __forceinline__ Kept draw_alone(SampleShared &sh, const SampleRow &row, const Read &read, int32_t vocab, uint64_t *list, uint64_t *own, uint32_t number) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t end = 0;
    if (row.cut()) {
        BucketTokens<Read> tokens{sh, row, read, vocab, list, own};
        end = cut_row(sh, row, read, vocab, tokens);
    }
    const SampleEnd last(end);
    const int32_t per = (vocab + 4095) / 4096 * 256, first = wave * per, stop = min(first + per, vocab);
    uint64_t mine = 0;
    __syncthreads();                                           // (the list's place is the streams' now)
    WaveStream<float> stream{(float *)list + 128 * wave};
    const auto add_up = [&](float x, bool there) {
        const double w = row.weight(x);
        if (there && w >= row.least) mine += whole(w);
    };
#pragma unroll 1
    for (int32_t v0 = first; v0 < stop; v0 += 256) {
        float s[4];
        read(v0 + 4 * lane, s);
#pragma unroll
        for (int j = 0; j < 4; ++j) stream.add(s[j] > -__builtin_inff() && last.keeps(s[j], v0 + 4 * lane + j), s[j], add_up);
    }
    stream.rest(add_up);
    mine = sum_of_wave(mine);
    __syncthreads();
    if (lane == 0) sh.part_units[wave] = mine;
    if (tid == 0) sh.token = -1;
    __syncthreads();
    uint64_t all = 0, before = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) before += sh.part_units[w];
        all += sh.part_units[w];
    }
    const uint64_t limit = part_of(all, number);
    if (before <= limit && limit < before + mine) {            // one wavefront, if there is any weight
#pragma unroll 1
        for (int32_t v0 = first; v0 < stop; v0 += 256) {
            float s[4];
            uint64_t u[4], sum = 0;
            read(v0 + 4 * lane, s);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u[j] = whole(kept_units(row, s[j], v0 + 4 * lane + j, last));
                sum += u[j];
            }
            uint64_t at = before + before_in_wave(sum);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (at <= limit && limit < at + u[j]) sh.token = v0 + 4 * lane + j;
                at += u[j];
            }
            before = __shfl(at, 63);
            if (limit < before) break;
        }
    }
    __syncthreads();
    return {end, all, sh.token, 0};
}

// A row in LDS of which any number of tokens is kept: their units once, in registers for the distribution.  Run i of the row is tokens 4096 i and on, four a thread.
template <int VF, int RUNS>
__device__ __forceinline__ Kept draw_of_many(SampleShared &sh, const SampleRow &row, const RowInLds<VF> &read, int32_t vocab, uint64_t end, uint32_t number, void *probs) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const SampleEnd last(end);
    using Units = typename std::conditional<VF == CSB_VAL_F32, double, float>::type;       // (to 2^-24 of themselves for results of 16 bits, whose rounding is 2^-12 at least)
    Units units[RUNS][4];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < RUNS; ++i)
        if (4096 * i < vocab) {                                // (uniform)
            const int32_t v = 4096 * i + 4 * tid;
            float s[4];
            double w[4], log[4], sum = 0.0;                    // (of 256 weights at most: exact)
            read.raw(v, s);
            row.weights_within(s, w, log);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool more = s[j] > last.s, same = s[j] == last.s, before = (uint32_t)(v + j) <= last.v;
                const bool kept = (more | (same & before)) & ((log[j] > -40.0) | (s[j] == row.m)) & (w[j] >= row.least);
                const double u = kept ? w[j] : 0.0;
                sum += u;
                units[i][j] = (Units)u;
            }
            const uint64_t all = sum_of_wave(whole(sum));
            if (lane == 0) sh.units[16 * i + wave] = all;
        }
    if (tid == 0) { sh.token = -1; sh.bin = kBuckets; }
    __syncthreads();
    const uint64_t part = tid < 16 * RUNS && 4096 * (tid / 16) < vocab ? sh.units[tid] : 0;
    uint64_t all;
    const uint64_t before = block_before(sh, part, &all), limit = part_of(all, number);
    if (before <= limit && limit < before + part) { sh.bin = tid; sh.base_units = before; }
    __syncthreads();
    if (wave == 0 && sh.bin < (uint32_t)kBuckets) {            // the run's 256 tokens, by one wavefront
        const int32_t v = 256 * (int)sh.bin + 4 * lane;
        float s[4];
        uint64_t u[4], sum = 0;
        read(v, s);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum += u[j] = whole(kept_units(row, s[j], v + j, last));
        uint64_t at = sh.base_units + before_in_wave(sum);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (at <= limit && limit < at + u[j]) sh.token = v + j;
            at += u[j];
        }
    }
    if (probs) {
        const double per = all ? 1.0 / (double)all : 0.0;
#pragma unroll
        for (int i = 0; i < RUNS; ++i) {
            const int32_t v = 4096 * i + 4 * tid;
            float x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = (float)((double)units[i][j] * per);
            if (v < vocab) probs4<VF>(probs, v, vocab, x);
        }
    }
    __syncthreads();
    return {end, all, sh.token, 0};
}

template <int VF, int BYTES>
__global__ __launch_bounds__(1024) void sample_small_kernel(const SampleDev a) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    constexpr int RUNS = BYTES / (int)sizeof(T4) / 1024;
    __shared__ SampleShared sh;
    __shared__ uint64_t list[kListMost], own[kRankMost];
    __shared__ T4 held[BYTES / sizeof(T4)];
    const int number = blockIdx.x, tid = threadIdx.x;
    const T *from = (const T *)a.logits + (int64_t)number * a.ld;
    T *to = a.probs ? (T *)a.probs + (int64_t)number * a.ldp : nullptr;
    T4 x[RUNS];
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        const int32_t v = 4 * tid + 4096 * i;
        if (v + 4 <= a.vocab) x[i] = load_any<T4>(from + v);
        else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i][j] = v + j < a.vocab ? from[v + j] : (T)-__builtin_inff();
        }
    }
    float largest = -__builtin_inff();                         // of the thread's tokens
#pragma unroll
    for (int i = 0; i < RUNS; ++i) {
        const int32_t v = 4 * tid + 4096 * i;
        if (v < a.vocab) held[v / 4] = x[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) largest = fmaxf(largest, logit((float)x[i][j]));
    }
    const float m = block_max(sh, largest);                    // (the barrier is for the row too)
    const SampleRow row(a, number, m);
    const RowInLds<VF> read{(const T *)held, a.vocab};
    const uint32_t r = a.tokens ? draw_number(a.r[number]) : 0;
    Kept kept{0, 0, -1, 0};
    bool zeros = true;                                         // (all of what follows is uniform)
    if (m > -__builtin_inff()) {
        bool few = false;
        if (row.k && row.k <= kFewest) {
            const int b = bucket_of_first(sh, row, [&](auto take) { take(largest); });
            const float least = row.least_of(b);
            list_tokens(sh, read, a.vocab, list, [&](float s) { return s >= least; });
            few = sh.listed <= (uint32_t)kFewMost;
            if (few) kept = draw_of_few(sh, row, list, sh.listed, r);
        }
        if (!few) {
            uint64_t end = 0;
            BucketTokens<RowInLds<VF>> tokens{sh, row, read, a.vocab, list, own};
            if (row.cut()) end = cut_row(sh, row, read, a.vocab, tokens);
            if (end && tokens.whole()) kept = draw_of_list(sh, row, a.vocab, list, tokens.upto, end, r);
            else {
                kept = draw_of_many<VF, RUNS>(sh, row, read, a.vocab, end, r, to);
                zeros = false;
            }
        }
    }
    if (a.tokens && tid == 0) a.tokens[number] = kept.token;
    if (to && zeros) {                                         // zeros in the row's place, the kept over them
        const double per = kept.total ? 1.0 / (double)kept.total : 0.0;
        __syncthreads();
#pragma unroll 1
        for (int32_t v = 4 * tid; v < a.vocab; v += 4096) held[v / 4] = T4{};
        __syncthreads();
        for (uint32_t i = tid; i < kept.listed; i += 1024) {
            const uint64_t at = list[i];
            const double w = row.weight(logit_at(at));
            if (at >= kept.end) ((T *)held)[0xffffffffu - (uint32_t)at] = (T)(float)(w < row.least ? 0.0 : w * per);
        }
        __syncthreads();
#pragma unroll 1
        for (int32_t v = 4 * tid; v < a.vocab; v += 4096) {
            const T4 x = held[v / 4];
            if (v + 4 <= a.vocab) store_any(to + v, x);
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j) if (v + j < a.vocab) to[v + j] = x[j];
            }
        }
    }
}

// ---- larger rows: a workgroup of 256 threads a chunk, sixteen tokens a thread -----------------------------------------------------------------
__device__ __forceinline__ float max_of_wave(float m) {
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    return m;
}
// The row's largest logit, by every wavefront for itself.
__device__ __forceinline__ float max_of_row(const SampleDev &a, int row) {
    float m = -__builtin_inff();
    for (int i = threadIdx.x & 63; i < a.chunks; i += 64) m = fmaxf(m, a.maxes[(int64_t)row * a.chunks + i]);
    return max_of_wave(m);
}
// Sixteen tokens of a chunk: numbers chunk_number(c, 0 .. 15).
__device__ __forceinline__ int32_t chunk_number(int c, int i) { return c * kChunk + 1024 * (i / 4) + 4 * (int)(threadIdx.x & 255) + i % 4; }
template <int VF> __device__ __forceinline__ void chunk_tokens(const SampleDev &a, int row, int c, float (*s)[4]) {
    const void *from = (const typename Elem<VF>::T *)a.logits + (int64_t)row * a.ld;
#pragma unroll
    for (int i = 0; i < 4; ++i) logits4<VF>(from, chunk_number(c, 4 * i), a.vocab, s[i]);
}
__device__ __forceinline__ RowState state_of(const SampleRow &row) {      // (few that were too many, and both ends: the second is known when the first is)
    return !row.cut() ? ROW_WHOLE : row.k && (row.k <= kFewest || row.p < 1u << 24) ? ROW_ALONE : ROW_CUT;
}

template <int VF>
__global__ __launch_bounds__(256) void sample_max_kernel(const SampleDev a) {
    __shared__ float part[4];
    const int row = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    float s[4][4], m = -__builtin_inff();
    chunk_tokens<VF>(a, row, c, s);
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, s[i / 4][i % 4]);
    a.groups[(int64_t)blockIdx.x * 256 + tid] = m;
    m = max_of_wave(m);
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) a.maxes[blockIdx.x] = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    if (c == 0) {                                              // the row's histogram starts empty
#pragma unroll
        for (int i = 0; i < kBuckets / 256; ++i) a.histogram[(int64_t)row * kBuckets + 256 * i + tid] = 0;
        if (tid == 0) a.listed[row] = 0;
    }
}

// Few tokens of a row.
struct FewShared { SampleShared sh; uint64_t list[kFewMost]; uint32_t hits[kFewMost]; };
template <int VF> __device__ __forceinline__ void draw_few_row(const SampleDev &a, FewShared &few_shared, int number) {
    SampleShared &sh = few_shared.sh;
    uint64_t *list = few_shared.list;
    uint32_t *hits = few_shared.hits;
    const int tid = threadIdx.x, n_groups = a.chunks * 256;
    const float *groups = a.groups + (int64_t)number * n_groups;
    float g[8];                                                // the first 8192 groups stay in registers
#pragma unroll
    for (int i = 0; i < 8; ++i) g[i] = 1024 * i + tid < n_groups ? groups[1024 * i + tid] : -__builtin_inff();
    const float m = max_of_row(a, number);
    const SampleRow row(a, number, m);
    bool few = m == -__builtin_inff();                         // (nothing to draw from)
    Kept kept{0, 0, -1, 0};
    if (!few && row.k && row.k <= kFewest) {                   // (uniform)
        const auto each = [&](auto take) {
#pragma unroll
            for (int i = 0; i < 8; ++i) take(g[i], 1024 * i + tid);
#pragma unroll 1
            for (int i = 8192 + tid; i < n_groups; i += 1024) take(groups[i], i);
        };
        const int b = bucket_of_first(sh, row, [&](auto take) { each([&](float m, int) { take(m); }); });
        // the groups that have tokens up to that bucket, then their tokens, four to a thread
        if (tid == 0) { sh.listed = 0; sh.bin_count = 0; }
        __syncthreads();
        each([&](float m, int i) {
            if (row.bucket(m) <= b) {
                const uint32_t n = atomicAdd(&sh.bin_count, 1u);
                if (n < (uint32_t)kFewMost) hits[n] = i;
            }
        });
        __syncthreads();
        const uint32_t n = sh.bin_count;
        if (n <= (uint32_t)kFewMost) {
            const void *from = (const typename Elem<VF>::T *)a.logits + (int64_t)number * a.ld;
            for (uint32_t i = tid; i < n * 4; i += 1024) {
                const uint32_t h = hits[i / 4];
                const int32_t v = (int32_t)(h >> 8) * kChunk + 1024 * (int32_t)(i & 3) + 4 * (int32_t)(h & 255);
                float s[4];
                logits4<VF>(from, v, a.vocab, s);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (row.bucket(s[j]) <= b) {
                        const uint32_t at = atomicAdd(&sh.listed, 1u);
                        if (at < (uint32_t)kFewMost) list[at] = place(s[j], v + j);
                    }
            }
        }
        __syncthreads();
        few = n <= (uint32_t)kFewMost && sh.listed <= (uint32_t)kFewMost;
        if (few) kept = draw_of_few(sh, row, list, sh.listed, a.tokens ? draw_number(a.r[number]) : 0);
    }
    if (tid) return;
    a.done[number] = few;
    if (few) {
        if (a.tokens) a.tokens[number] = kept.token;
        a.ends[number] = kept.end;
        a.totals[number] = kept.total;
    }
}

// The histogram of a row that is cut, the chunks' units of one that is not: four chunks by 1024 threads.
struct HistogramShared { unsigned long long bins[kBuckets]; uint64_t part[16]; };
template <int VF> __device__ __forceinline__ void count_chunks(const SampleDev &a, HistogramShared &sh, int number, int c) {
    const int tid = threadIdx.x;
    float s[4][4];
    SampleRow row(a, number);
    const RowState state = state_of(row);
    if (state == ROW_ALONE) return;                            // (uniform)
    chunk_tokens<VF>(a, number, c, s);                         // (past the row's last chunk: of no weight)
    const float m = max_of_row(a, number);
    row.largest(m);
    const bool any = m > -__builtin_inff();
    if (state == ROW_WHOLE || !any) {
        const SampleEnd all(0);
        double here = 0.0;                                     // (16 weights: exact)
#pragma unroll 4
        for (int i = 0; i < 16; ++i) here += any ? kept_units(row, s[i / 4][i % 4], 0, all) : 0.0;
        const uint64_t sum = sum_of_wave(whole(here));
        if ((tid & 63) == 0) sh.part[tid >> 6] = sum;
        __syncthreads();
        const uint64_t *of_chunk = sh.part + (tid >> 8) * 4;
        if ((tid & 255) == 0 && c < a.chunks) a.sums[(int64_t)number * a.chunks + c] = of_chunk[0] + of_chunk[1] + of_chunk[2] + of_chunk[3];
        return;
    }
    sh.bins[tid] = 0;
    __syncthreads();
    if (row.k) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int b = row.bucket(s[i / 4][i % 4]);
            if (b < kBuckets - 1) atomicAdd(&sh.bins[b], 1ull);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            double w[4], log[4];
            row.weights_within(s[i], w, log);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = row.bucket(s[i][j]);
                if (b < kBuckets - 1) atomicAdd(&sh.bins[b], (unsigned long long)whole(w[j]));
            }
        }
    }
    __syncthreads();
    const unsigned long long v = sh.bins[tid];
    if (v) atomicAdd(&a.histogram[(int64_t)number * kBuckets + tid], v);
}

// Workgroups of few rows, and beside them those of other rows' chunks.
template <int VF>
__global__ __launch_bounds__(1024) void sample_few_kernel(const SampleDev a) {
    __shared__ union { FewShared few; HistogramShared histogram; } shared;
    const uint32_t few_rows = a.done ? (uint32_t)a.rows : 0u, quarters = (uint32_t)(a.chunks + 3) / 4;
    if (blockIdx.x < few_rows) draw_few_row<VF>(a, shared.few, (int)blockIdx.x);
    else {
        const uint32_t i = blockIdx.x - few_rows;
        count_chunks<VF>(a, shared.histogram, (int)(i / quarters), (int)(i % quarters) * 4 + (int)(threadIdx.x >> 8));
    }
}

// The bucket in which what is kept of a row ends, by 256 threads, four buckets each (kBuckets: nothing is cut).
__device__ __forceinline__ int bucket_of_256(const SampleDev &a, int number, const SampleRow &row, uint64_t *part, int *found) {
    const int tid = threadIdx.x, wave = tid >> 6;
    uint64_t u[4], mine = 0, all = 0, before;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] = a.histogram[(int64_t)number * kBuckets + 4 * tid + i];
        mine += u[i];
    }
    before = before_in_wave(mine);
    if ((tid & 63) == 63) part[wave] = before + mine;
    if (tid == 0) *found = kBuckets;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += part[w];
        all += part[w];
    }
    const uint64_t share = part_of(all, row.p), target = row.k ? (uint64_t)row.k : share ? share : 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (before < target && before + u[i] >= target) *found = 4 * tid + i;    // one thread, or none
        before += u[i];
    }
    __syncthreads();
    return *found;
}

// Rows that are cut: the tokens of the bucket in which what is kept ends, in any order, and the units of the chunk before it.
template <int VF>
__global__ __launch_bounds__(256) void sample_bucket_kernel(const SampleDev a) {
    __shared__ float kept[kChunk];
    __shared__ uint64_t part[4];
    __shared__ int found;
    __shared__ uint32_t n_kept, at;
    const int tid = threadIdx.x, number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks;
    float s[4][4];
    SampleRow row(a, number);
    if (state_of(row) != ROW_CUT) return;                      // (uniform)
    chunk_tokens<VF>(a, number, c, s);
    const float m = max_of_row(a, number);
    if (!(m > -__builtin_inff())) return;
    row.largest(m);
    if (tid == 0) n_kept = 0;
    const int bucket = bucket_of_256(a, number, row, part, &found);
    uint32_t mine = 0;                                     // which of the sixteen are the bucket's
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float x = s[i / 4][i % 4];
        const int b = row.bucket(x);
        if (b == bucket) mine |= 1u << i;
        if (b < bucket && b < kBuckets - 1) kept[atomicAdd(&n_kept, 1u)] = x;
    }
    const uint32_t count = __builtin_popcount(mine), below = before_in_wave(count);
    __syncthreads();
    if ((tid & 63) == 63) part[tid >> 6] = below + count;
    __syncthreads();
    if (tid == 0) {
        const uint32_t total = (uint32_t)(part[0] + part[1] + part[2] + part[3]);
        at = total ? atomicAdd(&a.listed[number], total) : 0;               // a place for the workgroup's
    }
    __syncthreads();
    uint32_t to = at + below;
    for (int w = 0; w < (tid >> 6); ++w) to += (uint32_t)part[w];
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (mine >> i & 1) {
            if (to < (uint32_t)kListMost) a.list[(int64_t)number * kListMost + to] = place(s[i / 4][i % 4], chunk_number(c, i));
            ++to;
        }
    const SampleEnd none(0);
    uint64_t sum = 0;                                      // the weights of the kept alone, side by side
    const uint32_t n = n_kept;
    for (uint32_t i = tid; i < n; i += 256) sum += whole(kept_units(row, kept[i], 0, none));
    __syncthreads();                                       // (part is read)
    sum = sum_of_wave(sum);
    if ((tid & 63) == 0) part[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) a.sums[(int64_t)number * a.chunks + c] = part[0] + part[1] + part[2] + part[3];
}

// Tokens of a bucket, in a list alone.
struct ListedTokens {
    const SampleRow &row;
    const uint64_t *list;
    uint32_t n;
    template <typename Take> __device__ __forceinline__ void each(Take take) const {
        for (uint32_t i = threadIdx.x; i < n; i += 1024) take(list[i], row.weight(logit_at(list[i])));
    }
};

template <int VF>
__global__ __launch_bounds__(1024) void sample_draw_kernel(const SampleDev a) {
    __shared__ SampleShared sh;
    __shared__ uint64_t list[kListMost], own[kRankMost];
    __shared__ unsigned long long sums[kMaxChunks];
    const int tid = threadIdx.x;
    const int number = blockIdx.x;
    // (requested together: what a row does not have is not used)
    const uint32_t done = a.done ? a.done[number] : 0, r = a.tokens ? draw_number(a.r[number]) : 0;
    const uint64_t histogram = a.histogram[(int64_t)number * kBuckets + tid];
    uint32_t listed = a.listed[number];
    const float m = max_of_row(a, number);
    const SampleRow row(a, number, m);
    uint64_t of_chunks[kMaxChunks / 1024];
#pragma unroll
    for (int i = 0; i < kMaxChunks / 1024; ++i) of_chunks[i] = 1024 * i + tid < a.chunks ? a.sums[(int64_t)number * a.chunks + 1024 * i + tid] : 0;
    if (done) return;
    const bool any = m > -__builtin_inff();
    const RowState state = any ? state_of(row) : ROW_WHOLE;
    if (state != ROW_CUT) listed = 0;
    if (state == ROW_ALONE || listed > (uint32_t)kListMost) {
        const RowInMemory<VF> read{(const typename Elem<VF>::T *)a.logits + (int64_t)number * a.ld, a.vocab};
        const Kept kept = draw_alone(sh, row, read, a.vocab, list, own, r);
        if (tid == 0) {
            if (a.tokens) a.tokens[number] = kept.token;
            a.ends[number] = kept.end;
            a.totals[number] = kept.total;
        }
        return;
    }
    uint64_t end = 0;
#pragma unroll
    for (int i = 0; i < kMaxChunks / 1024; ++i) sums[1024 * i + tid] = any ? of_chunks[i] : 0;
    if (state == ROW_CUT) {
        for (uint32_t i = tid; i < listed; i += 1024) list[i] = a.list[(int64_t)number * kListMost + i];
        const uint64_t u = sh.units[tid] = row.k ? 0 : histogram;
        sh.counts[tid] = row.k ? (uint32_t)histogram : 0;
        if (tid == 0) { sh.base_count = 0; sh.base_units = 0; sh.bin = kBuckets; }
        uint64_t all, target = (uint64_t)row.k;
        block_before(sh, u, &all);
        if (row.k) find_bin<true>(sh, target);
        else {
            const uint64_t share = part_of(all, row.p);
            target = share ? share : 1;
            find_bin<false>(sh, target);
        }
        if (sh.bin < (uint32_t)kBuckets) {                     // (uniform)
            const ListedTokens tokens{row, list, listed};
            const bool few = listed <= (uint32_t)kRankMost;
            if (row.k) few ? find_ranked<true>(sh, row, target, list, listed) : find_token<true>(sh, target, tokens);
            else few ? find_ranked<false>(sh, row, target, list, listed) : find_token<false>(sh, target, tokens);
            end = sh.found;
            const SampleEnd last(end);
            for (uint32_t i = tid; i < listed; i += 1024) {
                const uint32_t v = 0xffffffffu - (uint32_t)list[i];
                const uint64_t w = whole(kept_units(row, logit_at(list[i]), v, last));
                if (w) atomicAdd(&sums[v / kChunk], (unsigned long long)w);
            }
        }
    }
    __syncthreads();
    uint64_t all, mine[kMaxChunks / 1024], sum = 0;            // four chunks a thread
#pragma unroll
    for (int i = 0; i < kMaxChunks / 1024; ++i) sum += mine[i] = sums[kMaxChunks / 1024 * tid + i];
    uint64_t before = block_before(sh, sum, &all);
    const uint64_t limit = part_of(all, r);
    if (tid == 0) {
        a.ends[number] = end;
        a.totals[number] = all;
        sh.bin = kMaxChunks;
        sh.token = -1;
    }
    if (!a.tokens) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kMaxChunks / 1024; ++i) {
        if (before <= limit && limit < before + mine[i]) { sh.bin = kMaxChunks / 1024 * tid + i; sh.base_units = before; }
        before += mine[i];
    }
    __syncthreads();
    if (sh.bin < (uint32_t)kMaxChunks) {                       // (uniform: any weight) the chunk's tokens, four a thread
        const int32_t v = (int32_t)sh.bin * kChunk + 4 * tid;
        const SampleEnd last(end);
        float s[4];
        uint64_t u[4], here = 0, total;
        logits4<VF>((const typename Elem<VF>::T *)a.logits + (int64_t)number * a.ld, v, a.vocab, s);
#pragma unroll 1
        for (int j = 0; j < 4; ++j) here += u[j] = whole(kept_units(row, s[j], v + j, last));
        uint64_t at = sh.base_units + block_before(sh, here, &total);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (at <= limit && limit < at + u[j]) sh.token = v + j;
            at += u[j];
        }
    }
    __syncthreads();
    if (tid == 0) a.tokens[number] = sh.token;
}

// The distribution: zeros, and in their places the kept, side by side.
template <int VF>
__global__ __launch_bounds__(256) void sample_probs_kernel(const SampleDev a) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    struct Item { float s; int32_t v; };
    __shared__ T4 out[kChunk / 4];
    __shared__ Item items[4 * 128];
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    float s[4][4];
    chunk_tokens<VF>(a, number, c, s);
    const float m = max_of_row(a, number);
    const SampleRow row(a, number, m);
    const SampleEnd last(a.ends[number]);
    const uint64_t all = a.totals[number];
    const double per = all ? 1.0 / (double)all : 0.0;
    WaveStream<Item> stream{items + 128 * (tid >> 6)};
    const auto set = [&](const Item &x, bool there) {          // (the wavefront's own tokens: behind its zeros)
        const double w = row.weight(x.s);
        if (there) ((T *)out)[x.v] = (T)(float)(w < row.least ? 0.0 : w * per);
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) out[256 * i + tid] = T4{};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float x = s[i / 4][i % 4];
        stream.add(all && x > -__builtin_inff() && last.keeps(x, chunk_number(c, i)), Item{x, 1024 * (i / 4) + 4 * tid + i % 4}, set);
    }
    stream.rest(set);
    __syncthreads();
    void *to = (T *)a.probs + (int64_t)number * a.ldp;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const T4 x = out[256 * i + tid];
        const float y[4] = {(float)x[0], (float)x[1], (float)x[2], (float)x[3]};
        probs4<VF>(to, chunk_number(c, 4 * i), a.vocab, y);
    }
}

struct SamplePlaces { size_t maxes, groups, histogram, sums, listed, done, ends, totals, list, bytes; };
static SamplePlaces sample_places(int64_t rows, int64_t chunks) {
    SamplePlaces p{};
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    p.histogram = take((size_t)rows * kBuckets * 8);
    p.list = take((size_t)rows * kListMost * 8);
    p.sums = take((size_t)rows * chunks * 8);
    p.ends = take((size_t)rows * 8);
    p.totals = take((size_t)rows * 8);
    p.groups = take((size_t)rows * chunks * 256 * 4);
    p.maxes = take((size_t)rows * chunks * 4);
    p.listed = take((size_t)rows * 4);
    p.done = take((size_t)rows * 4);
    p.bytes = at;
    return p;
}
static int32_t sample_chunks(int32_t vocab) { return (vocab + kChunk - 1) / kChunk; }       // (at most kMaxChunks)

static int64_t first_workgroups(int64_t rows, int32_t chunks, bool few) { return rows * ((chunks + 3) / 4) + (few ? rows : 0); }   // of sample_few_kernel

template <int VF>
static void launch_sample(const SampleDev &d, hipStream_t st) {
    const int64_t bytes = (int64_t)d.vocab * (VF == CSB_VAL_F32 ? 4 : 2);
    const dim3 block(1024), rows((uint32_t)d.rows);
    if (bytes <= kRowSmall) {
        hipLaunchKernelGGL((sample_small_kernel<VF, kRowSmall>), rows, block, 0, st, d);
        return;
    }
    if (bytes <= kRowMost) {
        hipLaunchKernelGGL((sample_small_kernel<VF, kRowMost>), rows, block, 0, st, d);
        return;
    }
    const int64_t chunks = (int64_t)d.rows * d.chunks;
    const int64_t first = first_workgroups(d.rows, d.chunks, d.done);
    const dim3 few(256), all((uint32_t)chunks);
    hipLaunchKernelGGL(sample_max_kernel<VF>, all, few, 0, st, d);
    hipLaunchKernelGGL(sample_few_kernel<VF>, dim3((uint32_t)first), block, 0, st, d);
    if (d.top_k || d.top_p || d.temperature) hipLaunchKernelGGL(sample_bucket_kernel<VF>, all, few, 0, st, d);
    hipLaunchKernelGGL(sample_draw_kernel<VF>, rows, block, 0, st, d);
    if (d.probs) hipLaunchKernelGGL(sample_probs_kernel<VF>, all, few, 0, st, d);
}

}  // namespace csb

extern "C" size_t csb_sample_workspace_bytes(int32_t n_rows, int32_t vocab) {
    if (n_rows <= 0 || vocab <= csb::kRowMost / 4) return 0;
    return csb::sample_places(n_rows, csb::sample_chunks(vocab)).bytes;
}

extern "C" int csb_sample(int32_t type, const void *d_logits, int64_t ld, const float *d_temperature, const int32_t *d_top_k,
                          const float *d_top_p, const float *d_min_p, const float *d_r, int32_t n_rows, int32_t vocab,
                          int32_t *d_tokens, void *d_probs, int64_t ldprobs, void *d_ws, void *stream) {
    using namespace csb;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_sample: ") + what); return code; };
    if (!known_type(type)) return fail(CSB_EINVAL, "unknown type");
    if (n_rows < 0 || vocab < 1) return fail(CSB_EINVAL, "bad size");
    if (vocab > 1 << 24) return fail(CSB_EUNSUPPORTED, "vocabulary above 2^24 (its units would pass 63 bits)");
    if (ld < vocab || (d_probs && ldprobs < vocab)) return fail(CSB_EINVAL, "a leading dimension below the vocabulary");
    if (n_rows == 0) return CSB_OK;
    if (!d_logits || (!d_tokens && !d_probs) || (d_tokens && !d_r)) return fail(CSB_EINVAL, "NULL pointer");
    if (d_probs == d_logits && ldprobs != ld) return fail(CSB_EINVAL, "the distribution in place of the logits at another leading dimension");
    if (((uintptr_t)d_logits | (uintptr_t)d_probs) % (uintptr_t)type_size(type) ||
        ((uintptr_t)d_temperature | (uintptr_t)d_top_k | (uintptr_t)d_top_p | (uintptr_t)d_min_p | (uintptr_t)d_r | (uintptr_t)d_tokens) % 4)
        return fail(CSB_EINVAL, "misaligned pointer");
    SampleDev d{};
    d.logits = d_logits; d.ld = ld; d.temperature = d_temperature; d.top_k = d_top_k; d.top_p = d_top_p; d.min_p = d_min_p; d.r = d_r;
    d.rows = n_rows; d.vocab = vocab; d.tokens = d_tokens; d.probs = d_probs; d.ldp = ldprobs;
    d.chunks = sample_chunks(vocab);
    if (n_rows > 1 << 21 || (int64_t)n_rows * d.chunks > kMaxWorkgroups) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    if ((int64_t)vocab * type_size(type) > kRowMost) {
        if (first_workgroups(n_rows, d.chunks, true) >= 1 << 22) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");     // (of 1024 threads)
        if (!d_ws) return fail(CSB_EINVAL, "NULL workspace");
        if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
        const SamplePlaces p = sample_places(n_rows, d.chunks);
        char *ws = (char *)d_ws;
        d.histogram = (unsigned long long *)(ws + p.histogram); d.sums = (unsigned long long *)(ws + p.sums); d.list = (uint64_t *)(ws + p.list);
        d.ends = (uint64_t *)(ws + p.ends); d.totals = (uint64_t *)(ws + p.totals);
        d.groups = (float *)(ws + p.groups); d.maxes = (float *)(ws + p.maxes); d.listed = (uint32_t *)(ws + p.listed);
        if (d_top_k || d_temperature) d.done = (uint32_t *)(ws + p.done);  // (a temperature of zero asks for one token)
        try {
            static const char sample_user = 0;                 // this entry point as a user of workspaces
            workspace_changed_hands(d_ws, &sample_user);
        } catch (const std::bad_alloc &) {
            return fail(CSB_ENOMEM, "out of host memory");
        }
    }
    hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case CSB_VAL_F32: launch_sample<CSB_VAL_F32>(d, st); break;
        case CSB_VAL_F16: launch_sample<CSB_VAL_F16>(d, st); break;
        default: launch_sample<CSB_VAL_BF16>(d, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(CSB_EDEVICE, hipGetErrorString(e));
    return CSB_OK;
}
