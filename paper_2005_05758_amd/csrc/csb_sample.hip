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
// Rows of up to kRowSmall bytes, and of kRowMost with top-k: one launch, a workgroup a row, which it holds in LDS.  Others, in chunks of 16384 tokens: maxima of groups; few, or the
// histogram (rows that nothing is cut of: units of the chunks); the bucket's tokens and the units before it by chunk; the end of what is kept and the draw; the
// distribution, if it is asked for.  Workgroups whose row is done, or is another's, leave at once.
#include <algorithm>
#include <new>

#include "csb_layer.hpp"

namespace csb {

constexpr int kRowMost = 98304, kRowSmall = kRowMost / 3;      // bytes of a row that a workgroup may hold, and of one that it always does
constexpr int kBuckets = 1024, kChunk = 16384, kMaxChunks = 1024, kListMost = 4096, kFewMost = 1024, kFewest = 256;
constexpr double kUnit = 274877906944.0;       // 2^38

enum RowState : uint32_t { ROW_DONE, ROW_WHOLE, ROW_CUT, ROW_ALONE };    // drawn; nothing is cut; by the histogram; by one workgroup

struct SampleDev {
    const void *logits;
    const float *temperature, *top_p, *min_p, *r;
    const int32_t *top_k;
    int32_t *tokens;
    void *probs;
    int64_t ld, ldp;
    int32_t rows, vocab, chunks;
    // workspace: [rows][chunks], [rows][chunks][1024], [rows][kBuckets], [rows], [rows][kListMost]
    float *maxes, *groups;
    unsigned long long *units, *sums;
    uint32_t *counts, *listed, *state;
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
    float m, per_bucket;
    double per_bit;                            // log2 e / T
    int32_t k;                                 // 0: all
    uint32_t p;                                // floor(top_p 2^24); 2^24: all
    double least;                              // units that min-p asks for
    __device__ __forceinline__ SampleRow(const SampleDev &a, int row, float max) : m(max) {
        const float T = a.temperature ? a.temperature[row] : 1.0f;
        k = a.top_k ? a.top_k[row] : 0;
        if (k < 1 || k >= a.vocab) k = 0;
        const float tp = a.top_p ? a.top_p[row] : 1.0f;
        p = tp < 1.0f ? (uint32_t)(fmaxf(tp, 0.0f) * 16777216.0f) : 1u << 24;
        const float mp = a.min_p ? a.min_p[row] : 0.0f;
        least = mp > 0.0f ? __builtin_floor((double)fminf(mp, 1.0f) * kUnit) : 0.0;
        if (T > 0.0f) {
            per_bit = 1.4426950408889634 / (double)T;
            per_bucket = (float)((kBuckets - 1) / 26.5 / (double)T);           // e^-26.5 2^38 < 1
        } else {
            per_bit = per_bucket = __builtin_inff();           // the largest alone,
            k = 1;                                             // and the first of them
        }
    }
    __device__ __forceinline__ bool cut() const { return k || p < 1u << 24; }
    // units of a token; whole, below 2^39
    __device__ __forceinline__ double weight(float s) const {
        const double y = ((double)s - (double)m) * per_bit, n = __builtin_rint(y), f = y - n;
        double e = 4.4455382718708110e-10;                     // (ln 2)^i / i!: e^(f ln 2), |f| <= 1/2, to 2^-42
        e = fma_of_constant(e, f, 7.0549116208011233e-09);
        e = fma_of_constant(e, f, 1.0178086009239699e-07);
        e = fma_of_constant(e, f, 1.3215486790144309e-06);
        e = fma_of_constant(e, f, 1.5252733804059840e-05);
        e = fma_of_constant(e, f, 1.5403530393381609e-04);
        e = fma_of_constant(e, f, 1.3333558146428443e-03);
        e = fma_of_constant(e, f, 9.6181291076284772e-03);
        e = fma_of_constant(e, f, 5.5504108664821580e-02);
        e = fma_of_constant(e, f, 2.4022650695910071e-01);
        e = fma_of_constant(e, f, 6.9314718055994531e-01);
        e = fma_of_constant(e, f, 1.0);
        const double w = __builtin_floor(__builtin_amdgcn_ldexp(e, (int)n + 38));
        return s == m ? kUnit : y > -40.0 ? w : 0.0;           // (infinite logits, and NaN of infinite temperatures)
    }
    __device__ __forceinline__ int bucket(float s) const { return s == m ? 0 : (int)fminf((m - s) * per_bucket, (float)(kBuckets - 1)); }
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
    using T4 = T __attribute__((ext_vector_type(4), aligned(sizeof(T)), may_alias));
    const T *p = (const T *)row + v;
    if (v + 4 <= end) {
        const T4 x = *(const T4 *)p;
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = logit((float)x[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) s[j] = v + j < end ? logit((float)p[j]) : -__builtin_inff();
    }
}
template <int VF> __device__ __forceinline__ void probs4(void *row, int32_t v, int32_t end, const float *x) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4), aligned(sizeof(T)), may_alias));
    T *p = (T *)row + v;
    if (v + 4 <= end) {
        T4 y;
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = (T)x[j];
        *(T4 *)p = y;
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
    unsigned long long units[kBuckets], low, high, found, found_units, base_units, part_units[16];
    uint32_t counts[kBuckets], part_counts[16];
    uint32_t bin, bin_count, base_count, listed;
    int32_t token;
    float part_max[16];
};

// Sum over the threads below this one; *total: of all.
__device__ __forceinline__ uint64_t block_before(SampleShared &sh, uint64_t v, uint64_t *total) {
    const int wave = threadIdx.x >> 6;
    uint64_t before = before_in_wave(v), all = 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) sh.part_units[wave] = before + v;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        const uint64_t p = sh.part_units[w];
        if (w < wave) before += p;
        all += p;
    }
    *total = all;
    return before;
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
    cb += sh.base_count;
    ub += sh.base_units;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        if (BY_COUNT) cb += w < wave ? sh.part_counts[w] : 0;
        if (UNITS) ub += w < wave ? sh.part_units[w] : 0;
    }
    __syncthreads();                                           // (base_* are read)
    if (BY_COUNT ? cb < target && cb + c >= target : ub < target && ub + u >= target) {   // one thread, or none
        sh.bin = tid;
        sh.bin_count = c;
        sh.base_count = cb;
        sh.base_units = ub;
    }
    __syncthreads();
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

// Where what is kept of a row ends: the last token's place (0: nothing is cut).  sh.units and sh.counts hold the row's histogram.
template <typename Tokens>
__device__ __forceinline__ uint64_t end_of_kept(SampleShared &sh, const SampleRow &row, Tokens &tokens) {
    const int tid = threadIdx.x;
    const uint32_t c = sh.counts[tid];
    const uint64_t u = sh.units[tid];
    auto restore = [&] {                                       // the histogram again (a search uses its place), from the start
        __syncthreads();
        sh.counts[tid] = c;
        sh.units[tid] = u;
        if (tid == 0) { sh.base_count = 0; sh.base_units = 0; sh.bin = kBuckets; }
        __syncthreads();
    };
    restore();
    uint64_t end = 0, units;
    block_before(sh, u, &units);
    if (row.k) {
        find_bin<true>(sh, (uint64_t)row.k);
        if (sh.bin < kBuckets) {                               // (uniform) else fewer tokens than k have units
            tokens.gather((int)sh.bin);
            find_token<true>(sh, (uint64_t)row.k, tokens);
            end = sh.found;
            units = sh.found_units;
        }
    }
    if (row.p < 1u << 24) {
        const uint64_t part = part_of(units, row.p), target = part ? part : 1;
        restore();
        find_bin<false>(sh, target);
        if (sh.bin < kBuckets) {
            tokens.gather((int)sh.bin);
            find_token<false>(sh, target, tokens);
            end = sh.found;
        }
    }
    return end;
}

// ---- reading a row, four tokens at a time: -infinity behind its end ------------------------------------------------------------------------
template <int VF> struct RowInMemory {
    const void *p;
    int32_t vocab;
    __device__ __forceinline__ void operator()(int32_t v, float *s) const { logits4<VF>(p, v, vocab, s); }
};
template <int VF> struct RowInLds {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    const T *p;
    int32_t vocab;                             // (rounded up to four: the rest holds -infinity)
    __device__ __forceinline__ void operator()(int32_t v, float *s) const {
        if (v < vocab) {
            const T4 x = *(const T4 *)(p + v);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = logit((float)x[j]);
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
// Tokens of a row in the buckets from `low` to `high`, in a list in LDS in any order; sh.listed: how many there are, which may be more than the list holds.
template <typename Read>
__device__ __forceinline__ void list_tokens(SampleShared &sh, const SampleRow &row, const Read &read, int32_t vocab, int low, int high, uint64_t *list) {
    __syncthreads();
    if (threadIdx.x == 0) sh.listed = 0;
    __syncthreads();
#pragma unroll 1
    for (int32_t v0 = 0; v0 < vocab; v0 += 16384) {
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) read(v0 + 4096 * i + 4 * (int)threadIdx.x, s[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int b = row.bucket(s[i / 4][i % 4]);
            if (b >= low && b <= high) {
                const uint32_t n = atomicAdd(&sh.listed, 1u);
                if (n < (uint32_t)kListMost) list[n] = place(s[i / 4][i % 4], v0 + 4096 * (i / 4) + 4 * threadIdx.x + i % 4);
            }
        }
    }
    __syncthreads();
}

// The tokens of one bucket: from the list, or from the row each time where it does not hold them.
template <typename Read> struct BucketTokens {
    SampleShared &sh;
    const SampleRow &row;
    const Read &read;
    int32_t vocab;
    uint64_t *list;
    int bucket;
    __device__ __forceinline__ void gather(int b) {
        bucket = b;
        list_tokens(sh, row, read, vocab, b, b, list);
    }
    template <typename Take> __device__ __forceinline__ void each(Take take) const {
        if (sh.listed <= (uint32_t)kListMost) {                // (uniform)
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

// Units of a token of a row whose kept end at `end`.
__device__ __forceinline__ double kept_units(const SampleRow &row, float s, int32_t v, uint64_t end) {
    if (place(s, (uint32_t)v) < end) return 0.0;
    const double w = row.weight(s);
    return w < row.least ? 0.0 : w;
}

struct Kept { uint64_t end, total; int32_t token; };   // the last token's place, units of all, the token drawn (all threads have them)

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
    return {sh.found, all, sh.token};
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

// A row by one workgroup of 1024 threads.  Wavefront w draws from the `per` tokens from w per on, 256 at a time.
template <typename Read>
__device__ __forceinline__ Kept draw_alone(SampleShared &sh, const SampleRow &row, const Read &read, int32_t vocab, uint64_t *list, uint32_t number) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t end = 0;
    if (row.cut()) {
        __syncthreads();
        sh.counts[tid] = 0;
        sh.units[tid] = 0;
        __syncthreads();
#pragma unroll 1
        for (int32_t v = 4 * tid; v < vocab; v += 4096) {
            float s[4];
            read(v, s);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = row.bucket(s[j]);
                if (b < kBuckets - 1) {
                    if (row.k) atomicAdd(&sh.counts[b], 1u);
                    atomicAdd(&sh.units[b], (unsigned long long)whole(row.weight(s[j])));
                }
            }
        }
        __syncthreads();
        BucketTokens<Read> tokens{sh, row, read, vocab, list, 0};
        end = end_of_kept(sh, row, tokens);
    }
    const int32_t per = (vocab + 4095) / 4096 * 256, first = wave * per, stop = min(first + per, vocab);
    uint64_t mine = 0;
#pragma unroll 1
    for (int32_t v = first + 4 * lane; v < stop; v += 256) {
        float s[4];
        read(v, s);
        double here = 0.0;
#pragma unroll
        for (int j = 0; j < 4; ++j) here += kept_units(row, s[j], v + j, end);
        mine += whole(here);
    }
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
                u[j] = whole(kept_units(row, s[j], v0 + 4 * lane + j, end));
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
    return {end, all, sh.token};
}

// The distribution's entries from v on.
template <int VF>
__device__ __forceinline__ void probs_of(const SampleRow &row, void *to, int32_t v, int32_t vocab, const float *s, uint64_t end, double per) {
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = per > 0.0 ? (float)(kept_units(row, s[j], v + j, end) * per) : 0.0f;
    probs4<VF>(to, v, vocab, x);
}

template <int VF, int BYTES>
__global__ __launch_bounds__(1024) void sample_small_kernel(const SampleDev a) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    using T4_any = T __attribute__((ext_vector_type(4), aligned(sizeof(T)), may_alias));
    __shared__ SampleShared sh;
    __shared__ uint64_t list[kListMost];
    __shared__ T4 held[BYTES / sizeof(T4)];
    const int number = blockIdx.x, tid = threadIdx.x;
    const T *from = (const T *)a.logits + (int64_t)number * a.ld;
    float largest = -__builtin_inff();                         // of the thread's tokens
#pragma unroll
    for (int i = 0; i < BYTES / (int)sizeof(T4) / 1024; ++i) {
        const int32_t v = 4 * tid + 4096 * i;
        if (v < a.vocab) {
            T4 x;
            if (v + 4 <= a.vocab) x = *(const T4_any *)(from + v);
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = v + j < a.vocab ? from[v + j] : (T)-__builtin_inff();
            }
            held[v / 4] = x;
#pragma unroll
            for (int j = 0; j < 4; ++j) largest = fmaxf(largest, logit((float)x[j]));
        }
    }
    const float m = block_max(sh, largest);                    // (the barrier is for the row too)
    const SampleRow row(a, number, m);
    const RowInLds<VF> read{(const T *)held, a.vocab};
    const uint32_t r = a.tokens ? draw_number(a.r[number]) : 0;
    Kept kept{0, 0, -1};
    if (m > -__builtin_inff()) {                               // (uniform, as all that follows)
        bool few = false;
        if (row.k && row.k <= kFewest) {
            const int b = bucket_of_first(sh, row, [&](auto take) { take(largest); });
            list_tokens(sh, row, read, a.vocab, 0, b, list);
            few = sh.listed <= (uint32_t)kFewMost;
        }
        kept = few ? draw_of_few(sh, row, list, sh.listed, r) : draw_alone(sh, row, read, a.vocab, list, r);
    }
    if (a.tokens && tid == 0) a.tokens[number] = kept.token;
    if (a.probs) {
        void *to = (T *)a.probs + (int64_t)number * a.ldp;
        const double per = kept.total ? 1.0 / (double)kept.total : 0.0;
#pragma unroll 1
        for (int32_t v = 4 * tid; v < a.vocab; v += 4096) {
            float s[4];
            read(v, s);
            probs_of<VF>(row, to, v, a.vocab, s, kept.end, per);
        }
    }
}

// ---- larger rows: a workgroup of 1024 threads a chunk, sixteen tokens a thread ---------------------------------------------------------------
__device__ __forceinline__ float max_of_row(SampleShared &sh, const SampleDev &a, int row) {
    return block_max(sh, (int)threadIdx.x < a.chunks ? a.maxes[(int64_t)row * a.chunks + threadIdx.x] : -__builtin_inff());
}
// Sixteen tokens of a chunk that starts at `first`: numbers first + 4096 (i / 4) + 4 tid + i % 4.
template <int VF> __device__ __forceinline__ void chunk_tokens(const SampleDev &a, int row, int32_t first, float (*s)[4]) {
    const void *from = (const typename Elem<VF>::T *)a.logits + (int64_t)row * a.ld;
#pragma unroll
    for (int i = 0; i < 4; ++i) logits4<VF>(from, first + 4096 * i + 4 * (int)threadIdx.x, a.vocab, s[i]);
}
__device__ __forceinline__ int32_t chunk_number(int32_t first, int i) { return first + 4096 * (i / 4) + 4 * (int)threadIdx.x + i % 4; }

template <int VF>
__global__ __launch_bounds__(1024) void sample_max_kernel(const SampleDev a) {
    __shared__ SampleShared sh;
    const int row = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    float s[4][4], m = -__builtin_inff();
    chunk_tokens<VF>(a, row, c * kChunk, s);
#pragma unroll
    for (int i = 0; i < 16; ++i) m = fmaxf(m, s[i / 4][i % 4]);
    a.groups[(int64_t)blockIdx.x * 1024 + tid] = m;
    m = block_max(sh, m);
    if (tid == 0) a.maxes[blockIdx.x] = m;
    if (c == 0) {                                              // the row's histogram starts empty
        a.counts[(int64_t)row * kBuckets + tid] = 0;
        a.units[(int64_t)row * kBuckets + tid] = 0;
        if (tid == 0) a.listed[row] = 0;
    }
}

// Few tokens by the row's first workgroup; the histogram, or the chunk's units where nothing is cut, by all.
template <int VF>
__global__ __launch_bounds__(1024) void sample_first_kernel(const SampleDev a) {
    __shared__ SampleShared sh;
    __shared__ uint64_t list[kListMost];
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    const float m = max_of_row(sh, a, number);
    const SampleRow row(a, number, m);
    const bool any = m > -__builtin_inff();
    if (any && row.k && row.k <= kFewest) {                    // (uniform)
        if (c) return;
        const float *groups = a.groups + (int64_t)number * a.chunks * 1024;
        const int b = bucket_of_first(sh, row, [&](auto take) {
#pragma unroll 8
            for (int i = tid; i < a.chunks * 1024; i += 1024) take(groups[i]);
        });
        // the groups that have tokens up to that bucket, then their tokens, four to a thread
        uint32_t *hits = (uint32_t *)list + kListMost;         // (the list's second half)
        if (tid == 0) { sh.listed = 0; sh.bin_count = 0; }
        __syncthreads();
#pragma unroll 8
        for (int i = tid; i < a.chunks * 1024; i += 1024)
            if (row.bucket(groups[i]) <= b) {
                const uint32_t n = atomicAdd(&sh.bin_count, 1u);
                if (n < (uint32_t)kFewMost) hits[n] = i;
            }
        __syncthreads();
        const uint32_t n = sh.bin_count;
        if (n <= (uint32_t)kFewMost) {
            const void *from = (const typename Elem<VF>::T *)a.logits + (int64_t)number * a.ld;
            for (uint32_t i = tid; i < n * 4; i += 1024) {
                const uint32_t g = hits[i / 4];
                const int32_t v = (int32_t)(g >> 10) * kChunk + 4096 * (int32_t)(i & 3) + 4 * (int32_t)(g & 1023);
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
        const bool few = n <= (uint32_t)kFewMost && sh.listed <= (uint32_t)kFewMost;
        if (few) {
            const Kept kept = draw_of_few(sh, row, list, sh.listed, a.tokens ? draw_number(a.r[number]) : 0);
            if (tid == 0) {
                if (a.tokens) a.tokens[number] = kept.token;
                a.ends[number] = kept.end;
                a.totals[number] = kept.total;
            }
        }
        if (tid == 0) a.state[number] = few ? ROW_DONE : ROW_ALONE;
        return;
    }
    // (one of the two ends: of both the second is known when the first is)
    const uint32_t state = !any ? ROW_DONE : !row.cut() ? ROW_WHOLE : row.k && row.p < 1u << 24 ? ROW_ALONE : ROW_CUT;
    if (c == 0 && tid == 0) {
        a.state[number] = state;
        if (!any) {
            if (a.tokens) a.tokens[number] = -1;
            a.ends[number] = a.totals[number] = 0;
        }
    }
    if (state == ROW_DONE || state == ROW_ALONE) return;
    float s[4][4];
    chunk_tokens<VF>(a, number, c * kChunk, s);
    if (state == ROW_WHOLE) {
        double here = 0.0;                                     // (16 weights: exact)
#pragma unroll
        for (int i = 0; i < 16; ++i) here += kept_units(row, s[i / 4][i % 4], chunk_number(c * kChunk, i), 0);
        uint64_t all;
        block_before(sh, whole(here), &all);
        if (tid == 0) a.sums[blockIdx.x] = all;
        return;
    }
    sh.counts[tid] = 0;
    sh.units[tid] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float x = s[i / 4][i % 4];
        const int b = row.bucket(x);
        if (b < kBuckets - 1) {
            if (row.k) atomicAdd(&sh.counts[b], 1u);
            atomicAdd(&sh.units[b], (unsigned long long)whole(row.weight(x)));
        }
    }
    __syncthreads();
    if (sh.units[tid] || sh.counts[tid]) {
        if (row.k) atomicAdd(&a.counts[(int64_t)number * kBuckets + tid], sh.counts[tid]);
        atomicAdd(&a.units[(int64_t)number * kBuckets + tid], sh.units[tid]);
    }
}

// The row's histogram in LDS, and the bucket in which what is kept ends (kBuckets: nothing is cut); sh.base_*: what lies before it.  *target: of find_bin.
__device__ __forceinline__ int bucket_of_row(SampleShared &sh, const SampleDev &a, int number, const SampleRow &row, uint64_t *target) {
    const int tid = threadIdx.x;
    __syncthreads();
    sh.counts[tid] = a.counts[(int64_t)number * kBuckets + tid];
    const uint64_t u = sh.units[tid] = a.units[(int64_t)number * kBuckets + tid];
    if (tid == 0) { sh.base_count = 0; sh.base_units = 0; sh.bin = kBuckets; }
    uint64_t all;
    block_before(sh, u, &all);
    if (row.k) find_bin<true>(sh, *target = (uint64_t)row.k);
    else {
        const uint64_t part = part_of(all, row.p);
        find_bin<false>(sh, *target = part ? part : 1);
    }
    return (int)sh.bin;
}

// Rows that are cut: the tokens of the bucket in which what is kept ends, in any order, and the units of the chunk before it.
template <int VF>
__global__ __launch_bounds__(1024) void sample_bucket_kernel(const SampleDev a) {
    __shared__ SampleShared sh;
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    if (a.state[number] != ROW_CUT) return;
    float s[4][4];
    chunk_tokens<VF>(a, number, c * kChunk, s);
    const float m = max_of_row(sh, a, number);
    const SampleRow row(a, number, m);
    uint64_t target;
    const int bucket = bucket_of_row(sh, a, number, row, &target);
    double here = 0.0;
    uint32_t mine = 0;                                         // which of the sixteen are the bucket's
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const float x = s[i / 4][i % 4];
        const int b = row.bucket(x);
        if (b < bucket) here += kept_units(row, x, 0, 0);
        else if (b == bucket) mine |= 1u << i;
    }
    uint64_t total;
    uint32_t at = (uint32_t)block_before(sh, (uint64_t)__builtin_popcount(mine), &total);
    if (tid == 0) sh.listed = total ? atomicAdd(&a.listed[number], (uint32_t)total) : 0;     // a place for the workgroup's
    __syncthreads();
    at += sh.listed;
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (mine >> i & 1) {
            if (at < (uint32_t)kListMost) a.list[(int64_t)number * kListMost + at] = place(s[i / 4][i % 4], chunk_number(c * kChunk, i));
            ++at;
        }
    uint64_t all;
    block_before(sh, whole(here), &all);
    if (tid == 0) a.sums[blockIdx.x] = all;
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
    __shared__ uint64_t list[kListMost];
    __shared__ unsigned long long sums[kMaxChunks];
    const int number = blockIdx.x, tid = threadIdx.x;
    const uint32_t state = a.state[number];
    if (state == ROW_DONE) return;
    const float m = max_of_row(sh, a, number);
    const SampleRow row(a, number, m);
    const uint32_t r = a.tokens ? draw_number(a.r[number]) : 0;
    const uint32_t listed = state == ROW_CUT ? a.listed[number] : 0;
    if (state == ROW_ALONE || listed > (uint32_t)kListMost) {
        const RowInMemory<VF> read{(const typename Elem<VF>::T *)a.logits + (int64_t)number * a.ld, a.vocab};
        const Kept kept = draw_alone(sh, row, read, a.vocab, list, r);
        if (tid == 0) {
            if (a.tokens) a.tokens[number] = kept.token;
            a.ends[number] = kept.end;
            a.totals[number] = kept.total;
        }
        return;
    }
    uint64_t end = 0;
    sums[tid] = tid < a.chunks ? a.sums[(int64_t)number * a.chunks + tid] : 0;
    if (state == ROW_CUT) {
        for (uint32_t i = tid; i < listed; i += 1024) list[i] = a.list[(int64_t)number * kListMost + i];
        uint64_t target;
        const int bucket = bucket_of_row(sh, a, number, row, &target);
        if (bucket < kBuckets) {
            const ListedTokens tokens{row, list, listed};
            if (row.k) find_token<true>(sh, target, tokens);
            else find_token<false>(sh, target, tokens);
            end = sh.found;
            for (uint32_t i = tid; i < listed; i += 1024)
                if (list[i] >= end) {
                    const uint32_t v = 0xffffffffu - (uint32_t)list[i];
                    atomicAdd(&sums[v / kChunk], (unsigned long long)whole(kept_units(row, logit_at(list[i]), v, end)));
                }
        }
    }
    __syncthreads();
    uint64_t all;
    const uint64_t here = sums[tid], before = block_before(sh, here, &all), limit = part_of(all, r);
    if (tid == 0) {
        a.ends[number] = end;
        a.totals[number] = all;
    }
    if (!a.tokens) return;
    if (tid == 0) { sh.bin = kMaxChunks; sh.token = -1; }
    __syncthreads();
    if (before <= limit && limit < before + here) { sh.bin = tid; sh.base_units = before; }
    __syncthreads();
    const uint32_t c = sh.bin;
    if (c < (uint32_t)kMaxChunks) {                            // (any weight)
        uint64_t from = sh.base_units;
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {                          // 4096 tokens by number, four a thread
            const int32_t v = (int32_t)c * kChunk + 4096 * i + 4 * tid;
            float s[4];
            uint64_t u[4], sum = 0, part;
            logits4<VF>((const typename Elem<VF>::T *)a.logits + (int64_t)number * a.ld, v, a.vocab, s);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                u[j] = whole(kept_units(row, s[j], v + j, end));
                sum += u[j];
            }
            uint64_t at = from + block_before(sh, sum, &part);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (at <= limit && limit < at + u[j]) sh.token = v + j;
                at += u[j];
            }
            from += part;
            if (limit < from) break;                           // (uniform)
        }
    }
    __syncthreads();
    if (tid == 0) a.tokens[number] = sh.token;
}

template <int VF>
__global__ __launch_bounds__(1024) void sample_probs_kernel(const SampleDev a) {
    __shared__ SampleShared sh;
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks;
    float s[4][4];
    chunk_tokens<VF>(a, number, c * kChunk, s);
    const float m = max_of_row(sh, a, number);
    const SampleRow row(a, number, m);
    const uint64_t end = a.ends[number], all = a.totals[number];
    const double per = all ? 1.0 / (double)all : 0.0;
    void *to = (typename Elem<VF>::T *)a.probs + (int64_t)number * a.ldp;
#pragma unroll
    for (int i = 0; i < 4; ++i) probs_of<VF>(row, to, chunk_number(c * kChunk, 4 * i), a.vocab, s[i], end, per);
}

struct SamplePlaces { size_t maxes, groups, units, sums, counts, listed, state, ends, totals, list, bytes; };
static SamplePlaces sample_places(int64_t rows, int64_t chunks) {
    SamplePlaces p{};
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    p.units = take((size_t)rows * kBuckets * 8);
    p.list = take((size_t)rows * kListMost * 8);
    p.sums = take((size_t)rows * chunks * 8);
    p.ends = take((size_t)rows * 8);
    p.totals = take((size_t)rows * 8);
    p.counts = take((size_t)rows * kBuckets * 4);
    p.groups = take((size_t)rows * chunks * 1024 * 4);
    p.maxes = take((size_t)rows * chunks * 4);
    p.listed = take((size_t)rows * 4);
    p.state = take((size_t)rows * 4);
    p.bytes = at;
    return p;
}
static int32_t sample_chunks(int32_t vocab) { return (vocab + kChunk - 1) / kChunk; }       // (at most kMaxChunks)

static bool one_workgroup(const SampleDev &d, int64_t bytes) { return bytes <= kRowSmall || (bytes <= kRowMost && d.top_k); }

template <int VF>
static void launch_sample(const SampleDev &d, hipStream_t st) {
    const int64_t bytes = (int64_t)d.vocab * (VF == CSB_VAL_F32 ? 4 : 2);
    const dim3 block(1024), rows((uint32_t)d.rows), grid((uint32_t)d.rows * (uint32_t)d.chunks);
    if (bytes <= kRowSmall) {
        hipLaunchKernelGGL((sample_small_kernel<VF, kRowSmall>), rows, block, 0, st, d);
        return;
    }
    // one workgroup a row: where few tokens are asked for it takes half as long as several launches; where their share is, its exponentials take
    // longer than those of many workgroups (165 rows of 32003, top-p and the distribution: 79 us instead of 45)
    if (one_workgroup(d, bytes)) {
        hipLaunchKernelGGL((sample_small_kernel<VF, kRowMost>), rows, block, 0, st, d);
        return;
    }
    hipLaunchKernelGGL(sample_max_kernel<VF>, grid, block, 0, st, d);
    hipLaunchKernelGGL(sample_first_kernel<VF>, grid, block, 0, st, d);
    if (d.top_k || d.top_p || d.temperature)                   // (a temperature of zero cuts too)
        hipLaunchKernelGGL(sample_bucket_kernel<VF>, grid, block, 0, st, d);
    hipLaunchKernelGGL(sample_draw_kernel<VF>, rows, block, 0, st, d);
    if (d.probs) hipLaunchKernelGGL(sample_probs_kernel<VF>, grid, block, 0, st, d);
}

}  // namespace csb

extern "C" size_t csb_sample_workspace_bytes(int32_t n_rows, int32_t vocab) {
    if (n_rows <= 0 || vocab <= csb::kRowSmall / 4) return 0;
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
    if (((uintptr_t)d_logits | (uintptr_t)d_probs) % (uintptr_t)type_size(type) ||
        ((uintptr_t)d_temperature | (uintptr_t)d_top_k | (uintptr_t)d_top_p | (uintptr_t)d_min_p | (uintptr_t)d_r | (uintptr_t)d_tokens) % 4)
        return fail(CSB_EINVAL, "misaligned pointer");
    SampleDev d{};
    d.logits = d_logits; d.ld = ld; d.temperature = d_temperature; d.top_k = d_top_k; d.top_p = d_top_p; d.min_p = d_min_p; d.r = d_r;
    d.rows = n_rows; d.vocab = vocab; d.tokens = d_tokens; d.probs = d_probs; d.ldp = ldprobs;
    d.chunks = sample_chunks(vocab);
    if (n_rows > 1 << 21 || (int64_t)n_rows * d.chunks > kMaxWorkgroups / 4) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    if (!one_workgroup(d, (int64_t)vocab * type_size(type))) {
        if (!d_ws) return fail(CSB_EINVAL, "NULL workspace");
        if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
        const SamplePlaces p = sample_places(n_rows, d.chunks);
        char *ws = (char *)d_ws;
        d.units = (unsigned long long *)(ws + p.units); d.sums = (unsigned long long *)(ws + p.sums); d.list = (uint64_t *)(ws + p.list);
        d.ends = (uint64_t *)(ws + p.ends); d.totals = (uint64_t *)(ws + p.totals); d.counts = (uint32_t *)(ws + p.counts);
        d.groups = (float *)(ws + p.groups); d.maxes = (float *)(ws + p.maxes); d.listed = (uint32_t *)(ws + p.listed); d.state = (uint32_t *)(ws + p.state);
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
