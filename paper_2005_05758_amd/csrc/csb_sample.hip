// Sampling from logits with temperature, top-k, top-p and min-p (csb_sample).
//
// A token's weight is a whole number of units, floor(2^38 e^((logit - max) / T)), so sums of units are the same in any order, and what is kept and
// drawn depends on nothing but the row and its numbers.  Top-k and top-p keep a beginning of the order by (logit, number); where it ends
// is searched for without sorting: a histogram of 1024 buckets of (max - logit) / T holds how many tokens and units each has, sums over it
// find the bucket, and the tokens of that one bucket are split again by their place in the order, 1024 parts at a time, until the part has
// one token: mostly one or two turns.  (A place is the logit's bits and the token's number in 64 bits, so places differ and ties need no care.)
// Buckets end where weights are no whole unit: tokens behind them are counted nowhere, they cannot be drawn.
//
// Exponentials are binary64, which this card does as fast as binary32: a unit is 2^-38 of the largest weight.
//
// Vocabularies up to kSampleSmall: one launch, a workgroup a row, its logits and weights in registers.  Larger ones: maxima of chunks; the
// histogram; the end of what is kept, a workgroup a row, over the tokens of the buckets in question; units of the kept by chunk; the draw.
#include <algorithm>
#include <new>

#include "csb_layer.hpp"

namespace csb {

constexpr int kSampleBlocks = 6, kSampleSmall = 16 * 256 * kSampleBlocks;
constexpr int kBuckets = 1024, kMaxChunks = 1024, kListMost = 4096;
constexpr double kUnit = 274877906944.0;       // 2^38

struct SampleDev {
    const void *logits;
    const float *temperature, *top_p, *min_p, *r;
    const int32_t *top_k;
    int32_t *tokens;
    void *probs;
    int64_t ld, ldp;
    int32_t rows, vocab, chunks, chunk;
    // workspace: [rows][chunks], [rows][kBuckets], [rows], [rows][chunks]
    float *maxes;
    unsigned long long *units;
    uint32_t *counts;
    uint64_t *cuts, *sums;
};

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
        double e = 4.4455382718708110e-10;                              // (ln 2)^i / i!: e^(f ln 2), |f| <= 1/2, to 2^-42
        e = __builtin_fma(e, f, 7.0549116208011233e-09);
        e = __builtin_fma(e, f, 1.0178086009239699e-07);
        e = __builtin_fma(e, f, 1.3215486790144309e-06);
        e = __builtin_fma(e, f, 1.5252733804059840e-05);
        e = __builtin_fma(e, f, 1.5403530393381609e-04);
        e = __builtin_fma(e, f, 1.3333558146428443e-03);
        e = __builtin_fma(e, f, 9.6181291076284772e-03);
        e = __builtin_fma(e, f, 5.5504108664821580e-02);
        e = __builtin_fma(e, f, 2.4022650695910071e-01);
        e = __builtin_fma(e, f, 6.9314718055994531e-01);
        e = __builtin_fma(e, f, 1.0);
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

template <typename N> __device__ __forceinline__ N sum_of_wave(N v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
// Sum over the lanes below this one.
template <typename N> __device__ __forceinline__ N before_in_wave(N v) {
    N upto = v;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const N o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    return upto - v;
}

// A workgroup's memory for the searches of a row.
struct SampleShared {
    unsigned long long units[kBuckets], low, high, found, found_units, base_units, part_units[16];
    uint32_t counts[kBuckets], part_counts[16];
    uint32_t bin, bin_count, base_count, listed;
    float part_max[16];
};

// The bin, of counts and units in LDS by thread, in which what is kept ends: of `target` tokens (BY_COUNT), or of those with fewer
// than `target` units before them; counted from what sh.base_* hold, which is moved up to the bin.  1024 threads, all of them.
template <bool BY_COUNT> __device__ __forceinline__ void find_bin(SampleShared &sh, uint64_t target) {
    const int tid = threadIdx.x, wave = tid >> 6;
    const uint32_t c = sh.counts[tid];
    const uint64_t u = sh.units[tid];
    uint32_t cb = before_in_wave(c);
    uint64_t ub = before_in_wave(u);
    if ((tid & 63) == 63) { sh.part_counts[wave] = cb + c; sh.part_units[wave] = ub + u; }
    __syncthreads();
    cb += sh.base_count;
    ub += sh.base_units;
    for (int w = 0; w < wave; ++w) { cb += sh.part_counts[w]; ub += sh.part_units[w]; }
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
    if (low <= high) { atomicMin(&sh.low, (unsigned long long)low); atomicMax(&sh.high, (unsigned long long)high); }
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
    find_bin<false>(sh, ~0ull);                                // (no bin: part_units are of use)
    units = 0;
    for (int w = 0; w < 16; ++w) units += sh.part_units[w];
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

// The tokens of a row's bucket: from a list of them in LDS, or from the row each time where there are more than the list holds.
template <int VF> struct BucketTokens {
    SampleShared &sh;
    const SampleRow &row;
    const void *from;
    uint64_t *list;
    int32_t vocab;
    int bucket;
    template <typename Take> __device__ __forceinline__ void scan(Take take) const {
#pragma unroll 1
        for (int32_t v0 = 0; v0 < vocab; v0 += 16384) {
            float s[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) logits4<VF>(from, v0 + 4096 * i + 4 * (int)threadIdx.x, vocab, s[i]);
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (row.bucket(s[i / 4][i % 4]) == bucket) take(place(s[i / 4][i % 4], v0 + 4096 * (i / 4) + 4 * (int)threadIdx.x + i % 4));
        }
    }
    __device__ __forceinline__ void gather(int b) {
        bucket = b;
        if (threadIdx.x == 0) sh.listed = 0;
        __syncthreads();
        scan([&](uint64_t at) {
            const uint32_t i = atomicAdd(&sh.listed, 1u);
            if (i < (uint32_t)kListMost) list[i] = at;
        });
        __syncthreads();
    }
    template <typename Take> __device__ __forceinline__ void each(Take take) const {
        if (sh.listed <= (uint32_t)kListMost)                  // (uniform)
            for (uint32_t i = threadIdx.x; i < sh.listed; i += 1024) take(list[i], row.weight(logit_at(list[i])));
        else scan([&](uint64_t at) { take(at, row.weight(logit_at(at))); });
    }
};

// Units of a token of a row whose kept end at `end`.
__device__ __forceinline__ double kept_units(const SampleRow &row, float s, int32_t v, uint64_t end) {
    if (place(s, (uint32_t)v) < end) return 0.0;
    const double w = row.weight(s);
    return w < row.least ? 0.0 : w;
}

// A row in one workgroup: wavefront w has the `blocks` times 256 tokens from w * blocks * 256 on, four to a lane and block.  The row is read again by
// every phase, from the caches.  Sums of units are whole numbers of binary64: at most 2^15 of 2^38 each.
template <int VF>
__global__ __launch_bounds__(1024) void sample_small_kernel(const SampleDev a, const int32_t blocks) {
    using T = typename Elem<VF>::T;
    __shared__ SampleShared sh;
    __shared__ uint64_t list[kListMost];
    __shared__ double sums[16];
    __shared__ int32_t token;
    const int number = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const void *from = (const T *)a.logits + (int64_t)number * a.ld;
    const int32_t first = wave * blocks * 256 + 4 * lane;
    float m = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kSampleBlocks; ++i)
        if (i < blocks) {
            float s[4];
            logits4<VF>(from, first + 256 * i, a.vocab, s);
            m = fmaxf(fmaxf(fmaxf(m, s[0]), fmaxf(s[1], s[2])), s[3]);
        }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if (lane == 0) sh.part_max[wave] = m;
    sh.counts[tid] = 0;
    sh.units[tid] = 0;
    if (tid == 0) token = -1;
    __syncthreads();
    for (int w = 0; w < 16; ++w) m = fmaxf(m, sh.part_max[w]);
    const SampleRow row(a, number, m);
    const bool any = m > -__builtin_inff();                    // (uniform)
    uint64_t end = 0;
    if (any && row.cut()) {
#pragma unroll 1
        for (int i = 0; i < blocks; ++i) {
            float s[4];
            logits4<VF>(from, first + 256 * i, a.vocab, s);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = row.bucket(s[j]);
                if (b < kBuckets - 1) {
                    atomicAdd(&sh.counts[b], 1u);
                    atomicAdd(&sh.units[b], (unsigned long long)whole(row.weight(s[j])));
                }
            }
        }
        __syncthreads();
        BucketTokens<VF> tokens{sh, row, from, list, a.vocab, 0};
        end = end_of_kept(sh, row, tokens);
    }
    auto weights = [&](int i, double *w) {
        float s[4];
        logits4<VF>(from, first + 256 * i, a.vocab, s);
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = any ? kept_units(row, s[j], first + 256 * i + j, end) : 0.0;
    };
    double mine = 0.0;
#pragma unroll 1
    for (int i = 0; i < blocks; ++i) {
        double w[4];
        weights(i, w);
        mine += w[0] + w[1] + w[2] + w[3];
    }
    mine = sum_of_wave(mine);
    if (lane == 0) sums[wave] = mine;
    __syncthreads();
    double all = 0.0, before = 0.0;
    for (int v = 0; v < 16; ++v) {
        if (v < wave) before += sums[v];
        all += sums[v];
    }
    if (a.tokens) {
        const double limit = (double)part_of((uint64_t)all, draw_number(a.r[number]));
        if (before <= limit && limit < before + mine) {        // one wavefront, if there is any weight
            double upto = before;
#pragma unroll 1
            for (int i = 0; i < blocks; ++i) {
                double w[4];
                weights(i, w);
                double at = upto + before_in_wave(w[0] + w[1] + w[2] + w[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (at <= limit && limit < at + w[j]) token = first + 256 * i + j;
                    at += w[j];
                }
                upto = __shfl(at, 63);
            }
        }
        __syncthreads();
        if (tid == 0) a.tokens[number] = token;
    }
    if (a.probs) {
        void *to = (T *)a.probs + (int64_t)number * a.ldp;
        const double per = all > 0.0 ? 1.0 / all : 0.0;
#pragma unroll 1
        for (int i = 0; i < blocks; ++i) {
            double w[4];
            float x[4];
            weights(i, w);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = (float)(w[j] * per);
            probs4<VF>(to, first + 256 * i, a.vocab, x);
        }
    }
}

// ---- larger vocabularies: a workgroup of 256 threads a chunk, sixteen tokens a thread at a time --------------------------------------------
constexpr int kChunkLeast = 4096;

__device__ __forceinline__ float max_of_row(const SampleDev &a, int row, float *part) {          // by all of 256 or 1024 threads
    float m = -__builtin_inff();
    for (int i = threadIdx.x; i < a.chunks; i += blockDim.x) m = fmaxf(m, a.maxes[(int64_t)row * a.chunks + i]);
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    for (int w = 0; w < (int)blockDim.x / 64; ++w) m = fmaxf(m, part[w]);
    return m;
}

template <int VF>
__global__ __launch_bounds__(256) void sample_max_kernel(const SampleDev a) {
    using T = typename Elem<VF>::T;
    __shared__ float part[4];
    const int row = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    const void *from = (const T *)a.logits + (int64_t)row * a.ld;
    const int32_t first = c * a.chunk, end = min(first + a.chunk, a.vocab);
    float m = -__builtin_inff();
    for (int32_t v = first; v < end; v += kChunkLeast) {
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) logits4<VF>(from, v + 1024 * i + 4 * tid, end, s[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, s[i / 4][i % 4]);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    if ((tid & 63) == 0) part[tid >> 6] = m;
    __syncthreads();
    if (tid == 0) a.maxes[blockIdx.x] = fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
    for (int i = c * 256 + tid; i < kBuckets; i += a.chunks * 256) {             // the row's histogram starts empty
        a.counts[(int64_t)row * kBuckets + i] = 0;
        a.units[(int64_t)row * kBuckets + i] = 0;
    }
}

template <int VF>
__global__ __launch_bounds__(256) void sample_histogram_kernel(const SampleDev a) {
    using T = typename Elem<VF>::T;
    __shared__ unsigned long long units[kBuckets];
    __shared__ uint32_t counts[kBuckets];
    __shared__ float part[4];
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    const float m = max_of_row(a, number, part);
    const SampleRow row(a, number, m);
    if (!row.cut() || !(m > -__builtin_inff())) return;        // (uniform)
    for (int i = tid; i < kBuckets; i += 256) { counts[i] = 0; units[i] = 0; }
    __syncthreads();
    const void *from = (const T *)a.logits + (int64_t)number * a.ld;
    const int32_t first = c * a.chunk, end = min(first + a.chunk, a.vocab);
    for (int32_t v = first; v < end; v += kChunkLeast) {
        float s[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) logits4<VF>(from, v + 1024 * i + 4 * tid, end, s[i]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float x = s[i / 4][i % 4];
            const int b = row.bucket(x);
            if (b < kBuckets - 1) {
                atomicAdd(&counts[b], 1u);
                atomicAdd(&units[b], (unsigned long long)whole(row.weight(x)));
            }
        }
    }
    __syncthreads();
    for (int i = tid; i < kBuckets; i += 256)
        if (counts[i]) {
            atomicAdd(&a.counts[(int64_t)number * kBuckets + i], counts[i]);
            atomicAdd(&a.units[(int64_t)number * kBuckets + i], units[i]);
        }
}

template <int VF>
__global__ __launch_bounds__(1024) void sample_cut_kernel(const SampleDev a) {
    using T = typename Elem<VF>::T;
    __shared__ SampleShared sh;
    __shared__ uint64_t list[kListMost];
    const int number = blockIdx.x, tid = threadIdx.x;
    const float m = max_of_row(a, number, sh.part_max);
    const SampleRow row(a, number, m);
    if (!row.cut() || !(m > -__builtin_inff())) {              // (uniform)
        if (tid == 0) a.cuts[number] = 0;
        return;
    }
    sh.counts[tid] = a.counts[(int64_t)number * kBuckets + tid];
    sh.units[tid] = a.units[(int64_t)number * kBuckets + tid];
    __syncthreads();
    BucketTokens<VF> tokens{sh, row, (const T *)a.logits + (int64_t)number * a.ld, list, a.vocab, 0};
    const uint64_t end = end_of_kept(sh, row, tokens);
    if (tid == 0) a.cuts[number] = end;
}

template <int VF>
__global__ __launch_bounds__(256) void sample_sums_kernel(const SampleDev a, const bool cut) {
    using T = typename Elem<VF>::T;
    __shared__ float part[4];
    __shared__ uint64_t parts[4];
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
    const float m = max_of_row(a, number, part);
    const SampleRow row(a, number, m);
    const uint64_t last = cut ? a.cuts[number] : 0;
    const void *from = (const T *)a.logits + (int64_t)number * a.ld;
    const int32_t first = c * a.chunk, end = min(first + a.chunk, a.vocab);
    uint64_t sum = 0;
    if (m > -__builtin_inff())                                 // (uniform)
        for (int32_t v = first; v < end; v += kChunkLeast) {
            float s[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) logits4<VF>(from, v + 1024 * i + 4 * tid, end, s[i]);
            double here = 0.0;                                 // (16 weights: exact)
#pragma unroll
            for (int i = 0; i < 16; ++i) here += kept_units(row, s[i / 4][i % 4], v + 1024 * (i / 4) + 4 * tid + i % 4, last);
            sum += whole(here);
        }
    sum = sum_of_wave(sum);
    if ((tid & 63) == 0) parts[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) a.sums[blockIdx.x] = parts[0] + parts[1] + parts[2] + parts[3];
}

// The draw in the chunk that the number falls into, and the distribution, chunk by chunk (a workgroup each).
template <int VF>
__global__ __launch_bounds__(256) void sample_draw_kernel(const SampleDev a, const bool cut) {
    using T = typename Elem<VF>::T;
    __shared__ float part[4];
    __shared__ uint64_t all_parts[4], before_parts[4];
    const int number = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint64_t all = 0, before = 0;
    for (int i = tid; i < a.chunks; i += 256) {
        const uint64_t s = a.sums[(int64_t)number * a.chunks + i];
        all += s;
        if (i < c) before += s;
    }
    all = sum_of_wave(all);
    before = sum_of_wave(before);
    if (lane == 0) { all_parts[wave] = all; before_parts[wave] = before; }
    __syncthreads();
    all = all_parts[0] + all_parts[1] + all_parts[2] + all_parts[3];
    before = before_parts[0] + before_parts[1] + before_parts[2] + before_parts[3];
    const uint64_t here = a.sums[blockIdx.x], limit = a.tokens ? part_of(all, draw_number(a.r[number])) : 0;
    const bool mine = a.tokens && before <= limit && limit < before + here;      // (uniform)
    if (a.tokens && c == 0 && all == 0 && tid == 0) a.tokens[number] = -1;
    if (!mine && !a.probs) return;
    const float m = max_of_row(a, number, part);
    const SampleRow row(a, number, m);
    const bool any = m > -__builtin_inff();
    const uint64_t last = cut ? a.cuts[number] : 0;
    const double per = all ? 1.0 / (double)all : 0.0;
    const void *from = (const T *)a.logits + (int64_t)number * a.ld;
    void *to = (T *)a.probs + (int64_t)number * a.ldp;
    const int32_t first = c * a.chunk, end = min(first + a.chunk, a.vocab);
    for (int32_t v0 = first; v0 < end; v0 += 1024) {           // four tokens a thread
        const int32_t v = v0 + 4 * tid;
        float s[4], x[4];
        double w[4], sum = 0.0;
        logits4<VF>(from, v, end, s);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = any ? kept_units(row, s[j], v + j, last) : 0.0;
            sum += w[j];
            x[j] = (float)(w[j] * per);
        }
        if (a.probs) probs4<VF>(to, v, end, x);
        if (mine) {
            const uint64_t own = whole(sum);
            uint64_t at = before + before_in_wave(own);
            __syncthreads();
            if (lane == 63) all_parts[wave] = at - before + own;
            __syncthreads();
            for (int k = 0; k < 4; ++k) {
                if (k < wave) at += all_parts[k];
                before += all_parts[k];
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint64_t u = whole(w[j]);
                if (at <= limit && limit < at + u) a.tokens[number] = v + j;
                at += u;
            }
        }
    }
}

// Tokens of a chunk: kChunkLeast, or more where that would make more than kMaxChunks.
static void sample_chunks(int32_t vocab, int32_t *chunks, int32_t *chunk) {
    int64_t c = kChunkLeast;
    while ((vocab + c - 1) / c > kMaxChunks) c *= 2;
    *chunk = (int32_t)c;
    *chunks = (int32_t)((vocab + c - 1) / c);
}

struct SamplePlaces { size_t maxes, units, counts, cuts, sums, bytes; };
static SamplePlaces sample_places(int64_t rows, int64_t chunks) {
    SamplePlaces p{};
    size_t at = 0;
    const auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    p.units = take((size_t)rows * kBuckets * 8);
    p.sums = take((size_t)rows * chunks * 8);
    p.cuts = take((size_t)rows * 8);
    p.counts = take((size_t)rows * kBuckets * 4);
    p.maxes = take((size_t)rows * chunks * 4);
    p.bytes = at;
    return p;
}

template <int VF>
static void launch_sample(const SampleDev &d, hipStream_t st) {
    if (d.vocab <= kSampleSmall) {
        hipLaunchKernelGGL(sample_small_kernel<VF>, dim3((uint32_t)d.rows), dim3(1024), 0, st, d, (d.vocab + 4095) / 4096);
        return;
    }
    const dim3 grid((uint32_t)d.rows * (uint32_t)d.chunks), block(256);
    const bool cut = d.top_k || d.top_p || d.temperature;      // (a temperature of zero cuts too)
    hipLaunchKernelGGL(sample_max_kernel<VF>, grid, block, 0, st, d);
    if (cut) {
        hipLaunchKernelGGL(sample_histogram_kernel<VF>, grid, block, 0, st, d);
        hipLaunchKernelGGL(sample_cut_kernel<VF>, dim3((uint32_t)d.rows), dim3(1024), 0, st, d);
    }
    hipLaunchKernelGGL(sample_sums_kernel<VF>, grid, block, 0, st, d, cut);
    hipLaunchKernelGGL(sample_draw_kernel<VF>, grid, block, 0, st, d, cut);
}

}  // namespace csb

extern "C" size_t csb_sample_workspace_bytes(int32_t n_rows, int32_t vocab) {
    if (n_rows <= 0 || vocab <= csb::kSampleSmall) return 0;
    int32_t chunks, chunk;
    csb::sample_chunks(vocab, &chunks, &chunk);
    return csb::sample_places(n_rows, chunks).bytes;
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
    sample_chunks(vocab, &d.chunks, &d.chunk);
    if (n_rows > 1 << 21 || (int64_t)n_rows * d.chunks > kMaxWorkgroups) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    if (vocab > kSampleSmall) {
        if (!d_ws) return fail(CSB_EINVAL, "NULL workspace");
        if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
        const SamplePlaces p = sample_places(n_rows, d.chunks);
        char *ws = (char *)d_ws;
        d.units = (unsigned long long *)(ws + p.units); d.sums = (uint64_t *)(ws + p.sums); d.cuts = (uint64_t *)(ws + p.cuts);
        d.counts = (uint32_t *)(ws + p.counts); d.maxes = (float *)(ws + p.maxes);
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
