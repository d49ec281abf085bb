// The selective state space scan (csb_selective_scan).
//
// Per channel c, with a state h of n numbers: h[j] <- exp(s A[j]) h[j] + s x B[j], y = sum_j C[j] h[j] + D x.  The issue of vector instructions binds: an
// exponential (8.4 clocks of a SIMD), two products (2.4) and two fused ones (4.2) a (token, channel, number), and 45 instructions a (token, channel) around them: 16384
// tokens of 4096 channels of 16 numbers take 448 us, the card's SIMDs busy all the time.  (s x B is a product of a number of the channel's and one of the
// group's: matrix instructions of 4 x 4 numbers made it and its sum with the decayed state in binary32, but each token waited for its own, 632 us instead of
// the 548 that it took then.)
// A channel's numbers lie with four lanes, K each, in registers from the first token to the last; a workgroup has 64 channels of one group, whose B and C come
// through LDS once for all of them.  What is a token's and channel's alone (its step s through softplus, s x, the gate, types) is made once by
// the lanes together, eight channels of a token each, and handed over through LDS; outputs come back in the same places.
//
// Few long sequences are split into chunks of 2^shift tokens: the decays of a chunk are exp(A sum s), so a chunk's effect is that factor and
// the state that it leaves from zero.  The first launch makes these for all chunks but the last (and keeps the state in front of the first,
// which the second launch replaces while others still need it), the second starts every chunk from the combination of those before it.
#include <algorithm>
#include <new>

#include "csb_layer.hpp"

namespace csb {

constexpr int kScanTile = 32, kScanCols = 64, kScanRow = 2 * kScanCols + 32;      // tokens and channels in LDS; floats of a token's row there
constexpr int kScanMany = 1024;                // workgroups that are enough for the card
// Tokens a sequence, on average, up to which wavefronts work alone: 64 sequences of 4096 channels, 8 tokens each: 21 us, 33 in tiles; 16: 31 and 37; 32: 51 and 46.
// All that the host knows is the mean: 255 single tokens and a prompt of 2048 (4096 channels, n = 16) are 1900 us in one call, 34 and 76 in two; and sequences
// that are enough for the card are not split: 47 prompts of 100 tokens and one of 8192 are 1050 us, 99 and 246 in two.
constexpr int kScanFew = 16;

struct ScanDev {
    const void *x, *dt, *z, *B, *C;
    const float *A, *D, *bias;
    const int32_t *start, *len, *slot;
    const float *s_in;
    float *s_out;
    void *out;
    float *begin, *sums;                       // [tiles][channels][n], [tiles][channels]
    int64_t ldx, lddt, ldz, ldB, ldC, ldo, n_tokens, each;
    int32_t channels, per_group, n, n_seq, n_states, softplus, shift, group_tiles, col_tiles;
};

// A decay as the exponentials of base 2 take it.  From -2.36e38 down, -infinity among them, it counts as the lowest number: steps of zero, which the places behind a
// sequence's end have too, keep the state then (their products with -infinity would be NaN).
__device__ __forceinline__ float decay_of(float A) {
    const float d = A * 1.44269502162933349609375f;
    return d < -0x1.fffffep127f ? -0x1.fffffep127f : d;        // (NaN stays)
}

// Lane q 16 + c gets the sum over the lanes c, 16 + c, 32 + c, 48 + c of y[q].
__device__ __forceinline__ float sum_of_rows(const float *y) {
    const auto even = [](float a, float b) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(a), __float_as_uint(b), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    };
    const float low = even(y[0], y[1]), high = even(y[2], y[3]);
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(low), __float_as_uint(high), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// OUT: outputs and last states; else what the chunks before the last leave.  FULL: n is 4 K.
template <int VF, int K, bool FULL, bool OUT>
__global__ __launch_bounds__(256) void selective_scan_kernel(const ScanDev a) {
    using T = typename Elem<VF>::T;
    using Run = Run8<VF>;
    __shared__ __attribute__((aligned(16))) float steps[kScanTile * kScanRow];   // s and s x of a token's channels, then y in place of s
    __shared__ __attribute__((aligned(16))) float Bs[kScanTile * 4 * K];
    __shared__ __attribute__((aligned(16))) float Cs[OUT ? kScanTile * 4 * K : 4];
    const int tid = threadIdx.x;
    const int64_t tile = blockIdx.x / a.col_tiles;
    const int seq = tile_sequence(a.start, a.n_seq, a.n_tokens, a.shift, tile, a.each);
    if (seq < 0) return;
    int64_t first, end;
    sequence_range(a.start, seq, a.each, a.n_tokens, &first, &end);
    const int64_t tile0 = (first >> a.shift) + seq, number = tile - tile0;
    if (a.len) end = first + clamp64(a.len[seq], 0, end - first);
    const int64_t count = end - first, t0 = number << a.shift, each = (int64_t)1 << a.shift;
    const bool last = t0 + each >= count;
    if (number < 0 || (number > 0 && t0 >= count) || (!OUT && last)) return;     // (uniform)
    const int32_t s = a.slot ? a.slot[seq] : seq;
    const bool known = s >= 0 && s < a.n_states;
    const int ct = (int)(blockIdx.x % a.col_tiles), group = ct / a.group_tiles;
    const int col0 = (ct % a.group_tiles) * kScanCols, cols = min(kScanCols, a.per_group - col0);   // the workgroup's channels in its group
    const int64_t base = (int64_t)group * a.per_group + col0;                    // its first channel

    // a lane's numbers of a channel
    const int q = (tid >> 4) & 3, c = (tid >> 6) * 16 + (tid & 15), j0 = q * K;
    const bool mine = c < cols;
    auto have = [&](int k) { return FULL || j0 + k < a.n; };
    const int64_t channel = base + (mine ? c : 0);
    float A[K], h[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        A[k] = have(k) ? decay_of(a.A[channel * a.n + j0 + k]) : 0.0f;
        h[k] = 0.0f;
    }
    auto get = [&](const float *p) {
#pragma unroll
        for (int k = 0; k < K; ++k) h[k] = have(k) ? p[channel * a.n + j0 + k] : 0.0f;
    };
    auto put = [&](float *p) {
        if (!mine) return;
#pragma unroll
        for (int k = 0; k < K; ++k) if (have(k)) p[channel * a.n + j0 + k] = h[k];
    };
    const int64_t state = (int64_t)a.channels * a.n;
    if (number == 0) {
        if (OUT && !last) get(a.begin + tile * state);         // (kept by the first launch: the last chunk may have replaced it)
        else if (a.s_in && known) get(a.s_in + s * state);
        if (!OUT) put(a.begin + tile * state);
    } else if (OUT) {
        get(a.begin + (tile0 + 1) * state);
#pragma unroll 4
        for (int64_t i = tile0 + 1; i < tile; ++i) {
            const float sum = a.sums[i * a.channels + channel];
            const float *p = a.begin + (i + 1) * state;
#pragma unroll
            for (int k = 0; k < K; ++k) h[k] = fmaf(__builtin_amdgcn_exp2f(sum * A[k]), h[k], have(k) ? p[channel * a.n + j0 + k] : 0.0f);
        }
    }

    // Two channels of a token, 16 bytes, lie together in LDS, those of eight channels turned by `turn`, so that neighbouring threads' are in banks of their own:
    // of sixteen threads eight have the even token's, eight the odd one's, whose row is 32 banks on.
    using f32x4 = float __attribute__((ext_vector_type(4)));
    using f32x2 = float __attribute__((ext_vector_type(2)));
    const auto pair = [](int channel, int token) { return (channel >> 3 << 4) + (((channel >> 1) + (channel >> 5) + 2 * token) & 3) * 4; };
    const int even = pair(c, 0) + 2 * (c & 1), odd = pair(c, 1) + 2 * (c & 1);
    // the same thread makes what eight channels of a token need, and their outputs
    const int sc = (tid & 7) * 8, st = tid >> 3, there = cols - sc;
    float bias[8], D[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        bias[i] = a.bias && i < there ? a.bias[base + sc + i] : 0.0f;
        D[i] = OUT && a.D && i < there ? a.D[base + sc + i] : 0.0f;
    }
    const int64_t stop = count < t0 + each ? count : t0 + each;
    Run x, z, next_x, next_dt, next_z;                         // a tile's operands are requested while the one before is worked on
    T next_B[K / 2], next_C[K / 2];
    // whole: all 64 channels, and all of a tile's tokens: nothing to ask for each thread
    const bool wide = FULL && cols == kScanCols;
    const int bt = tid / (4 * K), bj = tid % (4 * K);
    constexpr int STEP = 256 / (4 * K);                        // tokens of B and C that the workgroup loads at a time
    const int64_t from = first + t0 + st, from_b = first + t0 + bt, at_b = (int64_t)group * a.n + bj;
    const T *px = (const T *)a.x + from * a.ldx + base + sc, *pdt = (const T *)a.dt + from * a.lddt + base + sc;
    const T *pz = OUT && a.z ? (const T *)a.z + from * a.ldz + base + sc : nullptr;
    const T *pB = (const T *)a.B + from_b * a.ldB + at_b, *pC = (const T *)a.C + from_b * a.ldC + at_b;
    T *po = (T *)a.out + from * a.ldo + base + sc;
    auto load = [&](int64_t t) {
        if (wide && t + kScanTile <= stop) {
            next_x.load(px, 8);
            next_dt.load(pdt, 8);
            if (OUT && a.z) next_z.load(pz, 8);
#pragma unroll
            for (int i = 0; i < K / 2; ++i) {
                next_B[i] = pB[i * STEP * a.ldB];
                if (OUT) next_C[i] = pC[i * STEP * a.ldC];
            }
        } else {
            next_x.v = next_dt.v = next_z.v = typename Run::T8{};
            if (t + st < stop && there > 0) {
                next_x.load(px, there);
                next_dt.load(pdt, there);
                if (OUT && a.z) next_z.load(pz, there);
            }
#pragma unroll
            for (int i = 0; i < K / 2; ++i) {
                const bool in = t + bt + i * STEP < stop && bj < a.n;
                next_B[i] = in ? pB[i * STEP * a.ldB] : (T)0.0f;
                if (OUT) next_C[i] = in ? pC[i * STEP * a.ldC] : (T)0.0f;
            }
        }
        px += kScanTile * a.ldx;
        pdt += kScanTile * a.lddt;
        pB += kScanTile * a.ldB;
        if (OUT) { pz += kScanTile * a.ldz; pC += kScanTile * a.ldC; }
    };
    double total = 0.0;
    load(t0);
    for (int64_t t = t0; t < stop; t += kScanTile) {
        const int live = (int)(stop - t < kScanTile ? stop - t : kScanTile);
        float *row = steps + st * kScanRow;
        x = next_x;
        z = next_z;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float d[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                d[k] = next_dt[i + k] + bias[i + k];
                if (a.softplus) d[k] = softplus_from<VF>(d[k]);
            }
            if (live < kScanTile && st >= live) d[0] = d[1] = 0.0f;              // (past the end: nothing decays, nothing comes in)
            *(f32x4 *)(row + pair(sc + i, st)) = f32x4{d[0], d[0] * x[i], d[1], d[1] * x[i + 1]};
        }
#pragma unroll
        for (int i = 0; i < K / 2; ++i) {
            Bs[tid + 256 * i] = (float)next_B[i];
            if (OUT) Cs[tid + 256 * i] = (float)next_C[i];
        }
        if (t + kScanTile < stop) load(t + kScanTile);
        __syncthreads();
        float sum = 0.0f;
        float *e = steps + even, *o = steps + odd, *to = steps + q * kScanRow + (q & 1 ? odd : even) + (q >> 1);
        const float *b = Bs + j0, *cc = Cs + j0;
        for (int i = 0; i < live; i += 4) {
            float y[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float *d = (u & 1 ? o : e) + u * kScanRow;
                const f32x2 both = *(const f32x2 *)d;
                const float step = both[0], in = both[1];
                y[u] = 0.0f;
                f32x4 bu[K / 4], cu[K / 4];
#pragma unroll
                for (int k = 0; k < K / 4; ++k) {
                    bu[k] = *(const f32x4 *)(b + u * 4 * K + 4 * k);
                    if (OUT) cu[k] = *(const f32x4 *)(cc + u * 4 * K + 4 * k);
                }
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    h[k] = fmaf(__builtin_amdgcn_exp2f(step * A[k]), h[k], in * bu[k / 4][k % 4]);
                    if (!FULL) h[k] = have(k) ? h[k] : 0.0f;   // (infinite inputs make NaN of zeros)
                    if (OUT) y[u] = fmaf(cu[k / 4][k % 4], h[k], y[u]);
                }
                if (!OUT) sum += step;
            }
            // of token i + q, in place of the step, or of its product: other banks for the third and fourth
            if (OUT) *to = sum_of_rows(y);
            e += 4 * kScanRow;
            o += 4 * kScanRow;
            to += 4 * kScanRow;
            b += 16 * K;
            cc += 16 * K;
        }
        total += sum;
        __syncthreads();
        if (OUT && (live == kScanTile || st < live) && (wide || there > 0)) {
            Run o;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const f32x4 from = *(const f32x4 *)(row + pair(sc + i, st));
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    float y = fmaf(D[i + k], x[i + k], st & 2 ? from[2 * k + 1] : from[2 * k]);
                    if (a.z) y *= silu<VF>(z[i + k]);
                    o.set(i + k, y);
                }
            }
            o.store(po, wide ? 8 : there);
        }
        if (OUT) po += kScanTile * a.ldo;
    }
    if (OUT) {
        if (last && a.s_out && known) put(a.s_out + s * state);
    } else {
        put(a.begin + (tile + 1) * state);
        if (mine && q == 0) a.sums[tile * a.channels + channel] = (float)total;
    }
}

// The value of lane `lane ^ N` of a lane's four neighbours.
template <int N> __device__ __forceinline__ float quad_xor(float v) {
    constexpr int order = N == 1 ? 0xb1 : 0x4e;
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), order, 0xf, 0xf, false));
}

// The same for the few tokens of a decoding step: P lanes a channel, K numbers each, a wavefront 64 / P channels by itself, without LDS and barriers.
// The next token's operands are on their way while one is worked on.  (Four lanes a channel, as above, make its step and gate four times: 64
// requests of one token, 4096 channels of 16 numbers, 13.8 us instead of 11.9.)
template <int VF, int K, int P, bool FULL>
__global__ __launch_bounds__(256) void selective_scan_few_kernel(const ScanDev a, const uint32_t waves) {
    using T = typename Elem<VF>::T;
    using Run = Run8<VF>;
    using f32x4 = float __attribute__((ext_vector_type(4)));
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (wave >= waves) return;                                 // (no barrier in this kernel)
    const int seq = (int)(wave / (uint32_t)a.col_tiles), ct = (int)(wave % (uint32_t)a.col_tiles), group = ct / a.group_tiles;
    int64_t first, end;
    sequence_range(a.start, seq, a.each, a.n_tokens, &first, &end);
    if (a.len) end = first + clamp64(a.len[seq], 0, end - first);
    const int32_t s = a.slot ? a.slot[seq] : seq;
    const bool known = s >= 0 && s < a.n_states;
    const int64_t c = (int64_t)(ct % a.group_tiles) * (64 / P) + lane / P;
    const int j0 = (int)(lane % P) * K;
    const bool mine = c < a.per_group;
    const int64_t channel = (int64_t)group * a.per_group + (mine ? c : 0);
    const int there = FULL ? K : a.n - j0;                     // of the lane's K numbers
    struct Token { Run b[K / 8], c[K / 8]; T x, dt, z; };
    auto load = [&](int64_t t, Token &w) {
        const T *b = (const T *)a.B + t * a.ldB + (int64_t)group * a.n + j0, *cc = (const T *)a.C + t * a.ldC + (int64_t)group * a.n + j0;
#pragma unroll
        for (int i = 0; i < K / 8; ++i) {
            w.b[i].load(b + 8 * i, FULL ? 8 : there - 8 * i);
            w.c[i].load(cc + 8 * i, FULL ? 8 : there - 8 * i);
        }
        w.x = ((const T *)a.x)[t * a.ldx + channel];
        w.dt = ((const T *)a.dt)[t * a.lddt + channel];
        w.z = a.z ? ((const T *)a.z)[t * a.ldz + channel] : (T)0.0f;
    };
    auto numbers = [&](const float *p, float *v) {
#pragma unroll
        for (int i = 0; i < K / 4; ++i) {
            if (FULL || 4 * i + 4 <= there) {
                const f32x4 x = load_any<f32x4>(p + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * i + j] = x[j];
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[4 * i + j] = 4 * i + j < there ? p[4 * i + j] : 0.0f;
            }
        }
    };
    Token now{}, next{};
    if (first < end) load(first, now);
    float A[K], h[K];
    const int64_t state = (int64_t)s * a.channels * a.n + channel * a.n + j0;
    if (a.s_in && known) numbers(a.s_in + state, h);           // (uniform)
    else {
#pragma unroll
        for (int k = 0; k < K; ++k) h[k] = 0.0f;
    }
    numbers(a.A + channel * a.n + j0, A);
    const float bias = a.bias ? a.bias[channel] : 0.0f, D = a.D ? a.D[channel] : 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) A[k] = decay_of(A[k]);
    for (int64_t t = first; t < end; ++t) {
        if (t + 1 < end) load(t + 1, next);
        const float x = (float)now.x;
        float step = (float)now.dt + bias, y = 0.0f;
        if (a.softplus) step = softplus_from<VF>(step);
        const float in = step * x;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            h[k] = fmaf(__builtin_amdgcn_exp2f(step * A[k]), h[k], in * now.b[k / 8][k % 8]);
            if (!FULL) h[k] = k < there ? h[k] : 0.0f;         // (infinite inputs make NaN of zeros)
            y = fmaf(now.c[k / 8][k % 8], h[k], y);
        }
        if constexpr (P > 1) y += quad_xor<1>(y);
        if constexpr (P > 2) y += quad_xor<2>(y);
        if constexpr (P > 4) y += __shfl_xor(y, 4);
        y = fmaf(D, x, y);
        if (a.z) y *= silu<VF>((float)now.z);
        if (mine && lane % P == 0) ((T *)a.out)[t * a.ldo + channel] = (T)y;
        now = next;
    }
    if (a.s_out && known && mine)
#pragma unroll
        for (int i = 0; i < K / 4; ++i) {
            float *p = a.s_out + state + 4 * i;
            if (FULL || 4 * i + 4 <= there) store_any(p, f32x4{h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]});
            else {
#pragma unroll
                for (int j = 0; j < 4; ++j) if (4 * i + j < there) p[j] = h[4 * i + j];
            }
        }
}

// Chunks of a call, as a power of two of tokens (31: whole sequences).  Sequences and channels that give every CU four workgroups are not split (a split costs
// the chunks' own states beside the outputs: twice the exponentials).  Others are, as finely as makes that many, but no finer than 128 chunks
// a sequence, whose states every later chunk combines (16384 tokens of 64 channels in 512 chunks 86 us, in 128 52), and no coarser than 512 tokens
// (16384 tokens of 4096 channels take 6 % longer in 16 chunks than in 32).
static int scan_shift(const csb_scan_args *a, int64_t col_tiles) {
    const int64_t mean = a->n_tokens / a->n_seq, tiles = a->n_seq * col_tiles;
    if (tiles >= kScanMany || mean < 2 * kScanTile) return 31;
    int shift = 5;
    while ((mean >> shift) > 128 || (shift < 9 && (mean >> shift) * tiles > kScanMany)) ++shift;
    return mean >> shift < 2 ? 31 : shift;
}

static int scan_lanes(int32_t n) { return n <= 16 ? 1 : n <= 32 ? 2 : n <= 64 ? 4 : 8; }     // a channel, of the kernel for few tokens

struct ScanPlan { int32_t group_tiles; int64_t col_tiles, tiles; int shift; bool few; size_t begin, bytes; };
static Refusal scan_plan(const csb_scan_args *a, ScanPlan *p) {
    if (!a) return {CSB_EINVAL, "NULL arguments"};
    if (!known_type(a->type)) return {CSB_EINVAL, "unknown type"};
    if (a->n_seq < 0 || a->n_tokens < 0 || a->channels < 1 || a->groups < 1 || a->n < 1) return {CSB_EINVAL, "bad size"};
    if (a->channels % a->groups) return {CSB_EINVAL, "channels is no multiple of groups"};
    if (a->n > 128) return {CSB_EUNSUPPORTED, "n above 128 (a channel's numbers are held in the registers of 4 lanes)"};
    if (a->n_tokens > 0x7fffffff) return {CSB_EUNSUPPORTED, "offsets are 32-bit: more than 2^31 - 1 tokens"};
    *p = ScanPlan{};
    if (a->n_seq == 0) return {CSB_OK, nullptr};
    p->few = a->n_tokens / a->n_seq <= kScanFew;
    const int cols = p->few ? 64 / scan_lanes(a->n) : kScanCols;
    p->group_tiles = (int32_t)(((int64_t)a->channels / a->groups + cols - 1) / cols);      // (32 bits do not hold cols more than the most channels)
    p->col_tiles = (int64_t)p->group_tiles * a->groups;
    p->shift = p->few ? 31 : scan_shift(a, p->col_tiles);
    p->tiles = p->few ? a->n_seq : tile_numbers(a->n_tokens, a->n_seq, p->shift);
    if (p->tiles * p->col_tiles > kMaxWorkgroups) return {CSB_EUNSUPPORTED, "more workgroups than a launch takes"};
    if (p->shift < 31) {
        p->begin = ((size_t)p->tiles * a->channels * a->n * 4 + 255) / 256 * 256;
        p->bytes = p->begin + ((size_t)p->tiles * a->channels * 4 + 255) / 256 * 256;
    }
    return {CSB_OK, nullptr};
}

template <int VF, int K, int P>
static void launch_scan_few(const ScanDev &d, uint32_t waves, hipStream_t st) {
    if (d.n == K * P) hipLaunchKernelGGL((selective_scan_few_kernel<VF, K, P, true>), dim3((waves + 3) / 4), dim3(256), 0, st, d, waves);
    else hipLaunchKernelGGL((selective_scan_few_kernel<VF, K, P, false>), dim3((waves + 3) / 4), dim3(256), 0, st, d, waves);
}
template <int VF, int K, bool FULL>
static void launch_scan(const ScanDev &d, dim3 grid, hipStream_t st) {
    if (d.shift < 31) hipLaunchKernelGGL((selective_scan_kernel<VF, K, FULL, false>), grid, dim3(256), 0, st, d);
    hipLaunchKernelGGL((selective_scan_kernel<VF, K, FULL, true>), grid, dim3(256), 0, st, d);
}
template <int VF, int K>
static void launch_scan(const ScanDev &d, dim3 grid, hipStream_t st) {
    if (d.n == 4 * K) launch_scan<VF, K, true>(d, grid, st);
    else launch_scan<VF, K, false>(d, grid, st);
}
template <int VF>
static void launch_scan(const ScanDev &d, bool few, dim3 grid, hipStream_t st) {
    if (few) {
        switch (scan_lanes(d.n)) {
            case 1: d.n <= 8 ? launch_scan_few<VF, 8, 1>(d, grid.x, st) : launch_scan_few<VF, 16, 1>(d, grid.x, st); break;
            case 2: launch_scan_few<VF, 16, 2>(d, grid.x, st); break;
            case 4: launch_scan_few<VF, 16, 4>(d, grid.x, st); break;
            default: launch_scan_few<VF, 16, 8>(d, grid.x, st); break;
        }
        return;
    }
    if (d.n <= 16) launch_scan<VF, 4>(d, grid, st);
    else if (d.n <= 32) launch_scan<VF, 8>(d, grid, st);
    else if (d.n <= 64) launch_scan<VF, 16>(d, grid, st);
    else launch_scan<VF, 32>(d, grid, st);
}

}  // namespace csb

extern "C" size_t csb_scan_workspace_bytes(const csb_scan_args *args) {
    csb::ScanPlan p;
    return csb::scan_plan(args, &p).code == CSB_OK ? p.bytes : 0;
}

extern "C" int csb_selective_scan(const csb_scan_args *a, void *d_ws, void *stream) {
    using namespace csb;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_selective_scan: ") + what); return code; };
    ScanPlan p;
    const Refusal sizes = scan_plan(a, &p);
    if (sizes.code != CSB_OK) return fail(sizes.code, sizes.what);
    if (!a->d_A || (a->n_tokens && (!a->d_x || !a->d_dt || !a->d_B || !a->d_C || !a->d_out))) return fail(CSB_EINVAL, "NULL pointer");
    const int64_t w = a->channels, wn = (int64_t)a->groups * a->n;
    if (a->ldx < w || a->lddt < w || a->ldo < w || (a->d_z && a->ldz < w) || a->ldB < wn || a->ldC < wn)
        return fail(CSB_EINVAL, "a leading dimension below the width of its rows");
    if (a->n_tokens && ((a->d_out == a->d_x && a->ldo != a->ldx) || (a->d_out == a->d_dt && a->ldo != a->lddt) || (a->d_out == a->d_z && a->ldo != a->ldz) ||
                        a->d_out == a->d_B || a->d_out == a->d_C))
        return fail(CSB_EINVAL, "out in place of x, dt or z at another leading dimension, or of B or C");
    if (!a->d_start && a->n_seq && a->n_tokens % a->n_seq) return fail(CSB_EINVAL, "n_tokens is no multiple of n_seq (and there are no offsets)");
    if ((a->d_state_in || a->d_state_out) && a->n_states < 1) return fail(CSB_EINVAL, "states without room for one");
    if (((uintptr_t)a->d_x | (uintptr_t)a->d_dt | (uintptr_t)a->d_z | (uintptr_t)a->d_B | (uintptr_t)a->d_C | (uintptr_t)a->d_out) % (uintptr_t)type_size(a->type) ||
        ((uintptr_t)a->d_A | (uintptr_t)a->d_D | (uintptr_t)a->d_dt_bias | (uintptr_t)a->d_state_in | (uintptr_t)a->d_state_out |
         (uintptr_t)a->d_start | (uintptr_t)a->d_len | (uintptr_t)a->d_slot) % 4)
        return fail(CSB_EINVAL, "misaligned pointer");
    if (a->n_seq == 0) return CSB_OK;
    if (p.bytes) {
        if (!d_ws) return fail(CSB_EINVAL, "NULL workspace");
        if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
        try {
            static const char scan_user = 0;                   // this entry point as a user of workspaces
            workspace_changed_hands(d_ws, &scan_user);
        } catch (const std::bad_alloc &) {
            return fail(CSB_ENOMEM, "out of host memory");
        }
    }
    ScanDev d{};
    d.x = a->d_x; d.dt = a->d_dt; d.z = a->d_z; d.B = a->d_B; d.C = a->d_C;
    d.A = a->d_A; d.D = a->d_D; d.bias = a->d_dt_bias;
    d.start = a->d_start; d.len = a->d_len; d.slot = a->d_slot; d.s_in = a->d_state_in; d.s_out = a->d_state_out; d.out = a->d_out;
    d.begin = (float *)d_ws; d.sums = (float *)((char *)d_ws + p.begin);
    d.ldx = a->ldx; d.lddt = a->lddt; d.ldz = a->ldz; d.ldB = a->ldB; d.ldC = a->ldC; d.ldo = a->ldo;
    d.n_tokens = a->n_tokens; d.each = a->n_tokens / a->n_seq;
    d.channels = a->channels; d.per_group = a->channels / a->groups; d.n = a->n; d.n_seq = a->n_seq; d.n_states = a->n_states;
    d.softplus = a->softplus; d.shift = p.shift; d.group_tiles = p.group_tiles; d.col_tiles = (int32_t)p.col_tiles;
    const dim3 grid((uint32_t)(p.tiles * p.col_tiles));
    hipStream_t st = (hipStream_t)stream;
    switch (a->type) {
        case CSB_VAL_F32: launch_scan<CSB_VAL_F32>(d, p.few, grid, st); break;
        case CSB_VAL_F16: launch_scan<CSB_VAL_F16>(d, p.few, grid, st); break;
        default: launch_scan<CSB_VAL_BF16>(d, p.few, grid, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(CSB_EDEVICE, hipGetErrorString(e));
    return CSB_OK;
}
