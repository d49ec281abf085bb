// Norms around a block (csb_block_norm): r = x + scale s norm_after(y gate), out = norm_before(r), one pass over memory.
//
// Bound by HBM: a token's entries are read once, stay in registers over both norms, and are written once.  L lanes share a row (a token, or a
// group of one), NV runs of eight entries each.  Where all operands are row by row a row's lanes are neighbours; where one is column by column
// (a product's operand) neighbouring lanes are neighbouring tokens, eight of them, so that columns are read and written 16 or 32
// bytes at a time, and the workgroups of neighbouring tokens share an XCD, whose L2 puts these pieces together: their number bounds those calls.
// (16411 tokens of 16 heads of 128, gated, binary16, row by row: 45 us, 4.5 TB/s; 2048 tokens of 8192 entries between products: 58, of which 24 are the
// 33 MB that are written 16 bytes at a time.)
//
// Sums are binary64, as fast here as binary32: entries of 1e20 have squares there, and the variance may be taken from sums of v - v[0] and its
// square, in one pass.
#include <algorithm>

#include "csb_layer.hpp"

namespace csb {

struct NormOperand { const void *d; int64_t ld; int32_t type, columns; };
struct NormDev {
    NormOperand y, gate, x, r, out;
    const float *aw, *ab, *s, *bw, *bb;
    int64_t tokens, tiles;                     // tiles: of tokens, where lanes are tokens
    int32_t width, groups, after, before, sigmoid, gate_first;   // width: of a group
    int32_t plain_gate, plain_scale, past;     // results are rounded to 16 bits; nothing is scaled; x and r go past the caches
    float scale;
    double eps, per;                           // per: 1 / width
};

struct Raw8 { uint32_t w[8]; };                // eight entries as they are stored: one a word, or two of 16 bits in each of the first four (rows)

// Eight entries of one token.  NEAR: columns lie within a window of 2^31 bytes from the workgroup's first token on, so that an entry's
// place is one 32-bit number; else 64-bit addresses, eight for each run.  WHOLE: eight entries are there or none.  ROWS_ONLY: no columns.
template <bool NEAR, bool WHOLE, bool ROWS_ONLY> struct NormAccess {
    const NormOperand &o;
    int64_t t;
    window_t w;
    uint32_t at, step;
    // token t = t0 + off of `tokens`, t0 the same for all lanes; live: whether it is one
    __device__ __forceinline__ NormAccess(const NormOperand &operand, int64_t t0, int off, bool live, int64_t tokens, int64_t width) : o(operand), t(t0 + off) {
        if constexpr (NEAR) {
            const uint32_t size = o.type == CSB_VAL_F32 ? 4 : 2;
            w = window((const char *)o.d + t0 * size, (uint32_t)(((width - 1) * o.ld + tokens - t0) * size));
            step = (uint32_t)o.ld * size;
            at = live ? (uint32_t)off * size : kOutside;
        }
    }
    __device__ __forceinline__ bool by_columns() const { return !ROWS_ONLY && o.columns; }
    // entries j .. j + 7, the first `there` of them
    __device__ __forceinline__ Raw8 load(int64_t j, int there) const {
        using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
        Raw8 r{};
        const bool half = o.type != CSB_VAL_F32;               // (uniform, as the order)
        if (WHOLE && there <= 0) return r;
        if (NEAR && by_columns()) {
            const uint32_t from = at + (uint32_t)j * step;
            if (half) {
#pragma unroll
                for (int i = 0; i < 8; ++i) r.w[i] = window_load<_Float16>(w, WHOLE || i < there ? from + i * step : kOutside);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) r.w[i] = window_load<float>(w, WHOLE || i < there ? from + i * step : kOutside);
            }
        } else if (by_columns()) {
            if (half) {
                const uint16_t *p = (const uint16_t *)o.d + j * o.ld + t;
#pragma unroll
                for (int i = 0; i < 8; ++i) if (WHOLE || i < there) r.w[i] = p[i * o.ld];
            } else {
                const uint32_t *p = (const uint32_t *)o.d + j * o.ld + t;
#pragma unroll
                for (int i = 0; i < 8; ++i) if (WHOLE || i < there) r.w[i] = p[i * o.ld];
            }
        } else if (half) {
            const uint16_t *p = (const uint16_t *)o.d + t * o.ld + j;
            if (WHOLE || there >= 8) {
                const u32x4 v = load_any<u32x4>(p);
#pragma unroll
                for (int i = 0; i < 4; ++i) r.w[i] = v[i];
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i) if (i < there) r.w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
            }
        } else {
            const uint32_t *p = (const uint32_t *)o.d + t * o.ld + j;
            if (WHOLE || there >= 8) {
                const u32x4 v = load_any<u32x4>(p), u = load_any<u32x4>(p + 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) { r.w[i] = v[i]; r.w[4 + i] = u[i]; }
            } else {
#pragma unroll
                for (int i = 0; i < 7; ++i) if (i < there) r.w[i] = p[i];
            }
        }
        return r;
    }
    __device__ __forceinline__ void widen(const Raw8 &r, float *v) const {
        if (o.type == CSB_VAL_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, r.w[i]);
        } else if (by_columns() && o.type == CSB_VAL_BF16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, r.w[i] << 16);
        } else if (by_columns()) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)r.w[i]);
        } else if (o.type == CSB_VAL_BF16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2] & 0xffff));
        }
    }
    __device__ __forceinline__ void store(int64_t j, int there, const float *v) const {
        using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
        if (WHOLE && there <= 0) return;
        const bool half = o.type != CSB_VAL_F32;
        uint32_t b[8];
        if (o.type == CSB_VAL_F32) {
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = __builtin_bit_cast(uint32_t, v[i]);
        } else if (o.type == CSB_VAL_BF16) {
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = __builtin_bit_cast(uint16_t, (__bf16)v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) b[i] = __builtin_bit_cast(uint16_t, (_Float16)v[i]);
        }
        if (NEAR && by_columns()) {
            const uint32_t to = at + (uint32_t)j * step;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t here = WHOLE || i < there ? to + i * step : kOutside;
                if (half) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)b[i], w, (int)here, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b32(b[i], w, (int)here, 0, 0);
            }
            return;
        }
        const bool columns = by_columns();
        const int64_t from = columns ? j * o.ld + t : t * o.ld + j, by = columns ? o.ld : 1;
        if (half) {
            uint16_t *p = (uint16_t *)o.d + from;
            if (!columns && (WHOLE || there >= 8)) store_any(p, u32x4{b[0] | b[1] << 16, b[2] | b[3] << 16, b[4] | b[5] << 16, b[6] | b[7] << 16});
            else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (WHOLE || i < there) p[i * by] = (uint16_t)b[i];
            }
        } else {
            uint32_t *p = (uint32_t *)o.d + from;
            if (!columns && (WHOLE || there >= 8)) {
                store_any(p, u32x4{b[0], b[1], b[2], b[3]});
                store_any(p + 4, u32x4{b[4], b[5], b[6], b[7]});
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) if (WHOLE || i < there) p[i * by] = b[i];
            }
        }
    }
};
// Eight factors: `fill` where there is no vector of them; zeros behind the row's end, so that what is not there stays zero.
template <bool WHOLE> __device__ __forceinline__ void norm_factors(const float *p, int64_t j, int there, float fill, float *v) {
    using f32x4 = float __attribute__((ext_vector_type(4)));
    if (WHOLE ? there > 0 : there >= 8) {
        if (p) {
            const f32x4 a = load_any<f32x4>(p + j), b = load_any<f32x4>(p + j + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = fill;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = WHOLE || i >= there ? 0.0f : p ? p[j + i] : fill;
    }
}

// Eight factors of a gate.
template <typename Access> __device__ __forceinline__ void gate_factors(const NormDev &a, const Access &gate, const Raw8 &raw, float *g) {
    gate.widen(raw, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float x = g[j], s = a.plain_gate ? sigmoid_for<CSB_VAL_BF16>(x) : sigmoid_within(x);
        g[j] = a.sigmoid ? (x != x ? x : s) : x * s;
    }
}

// The rows of a workgroup of THREADS, L lanes each.  TOKENS: its rows are neighbouring lanes, else a row's lanes are.
template <int L, int THREADS, bool TOKENS> struct NormRows {
    static constexpr int ROWS = THREADS / L, WAVES = THREADS / 64, STEP = TOKENS ? ROWS : 1;
    struct Shared { double sums[2][2][WAVES * STEP]; float head[ROWS]; };
    Shared &sh;
    int64_t t0;                                // token: t0 + off
    int off, lane, group, turn;
    bool there;                                // whether the workgroup has any
    __device__ __forceinline__ NormRows(const NormDev &a, Shared &shared) : sh(shared), turn(0), there(true) {
        const int tid = threadIdx.x;
        if constexpr (TOKENS) {
            // the tiles that an XCD gets, one after the other, are neighbours
            const int64_t per = (a.tiles + 7) / 8, tile = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8 % per;
            group = (int)(blockIdx.x / (8 * per));
            there = tile < a.tiles;
            t0 = tile * ROWS;
            off = tid % ROWS;
            lane = tid / ROWS;
        } else {
            const int64_t row = (int64_t)blockIdx.x * ROWS + tid / L;
            t0 = row / a.groups;                               // (no columns here: not the same for all lanes)
            off = 0;
            group = (int)(row % a.groups);
            lane = tid % L;
        }
    }
    // sum over a row's lanes, in every one of them (a fixed order)
    template <int N> static __device__ __forceinline__ double other(double v) {
        const uint64_t b = __builtin_bit_cast(uint64_t, v);
        const uint32_t low = (uint32_t)b, high = (uint32_t)(b >> 32);
        if constexpr (N == 16) {
            // (both halves of a swap hold one of the two: their sum is the same)
            const auto l = __builtin_amdgcn_permlane16_swap(low, low, false, false), h = __builtin_amdgcn_permlane16_swap(high, high, false, false);
            return __builtin_bit_cast(double, (uint64_t)h[0] << 32 | l[0]) + __builtin_bit_cast(double, (uint64_t)h[1] << 32 | l[1]);
        } else if constexpr (N == 32) {
            const auto l = __builtin_amdgcn_permlane32_swap(low, low, false, false), h = __builtin_amdgcn_permlane32_swap(high, high, false, false);
            return __builtin_bit_cast(double, (uint64_t)h[0] << 32 | l[0]) + __builtin_bit_cast(double, (uint64_t)h[1] << 32 | l[1]);
        } else {
            // neighbours by 1 and 2; then fours, whose lanes agree, by the mirror of eight lanes; then eights, by a turn of sixteen
            constexpr int order = N == 1 ? 0xb1 : N == 2 ? 0x4e : N == 4 ? 0x141 : 0x128;
            const uint32_t l = (uint32_t)__builtin_amdgcn_mov_dpp((int)low, order, 0xf, 0xf, false), h = (uint32_t)__builtin_amdgcn_mov_dpp((int)high, order, 0xf, 0xf, false);
            return v + __builtin_bit_cast(double, (uint64_t)h << 32 | l);
        }
    }
    __device__ __forceinline__ double sum_in_wave(double v) const {
        if constexpr (TOKENS) {
#pragma unroll
            for (int d = STEP; d < 64; d *= 2) v += __shfl_xor(v, d);
        } else {
            v = other<1>(v);
            v = other<2>(v);
            v = other<4>(v);
            if constexpr (L > 8) v = other<8>(v);
            if constexpr (L > 16) { v = other<16>(v); v = other<32>(v); }
        }
        return v;
    }
    __device__ __forceinline__ void sum(int kind, double &p, double &q) {
        const int wave = threadIdx.x >> 6;
        q = sum_in_wave(q);
        if (kind == CSB_NORM_MEAN) p = sum_in_wave(p);
        if constexpr (TOKENS || L > 64) {
            double(*to)[WAVES * STEP] = sh.sums[turn];
            turn ^= 1;
            const int own = TOKENS ? threadIdx.x % ROWS : 0;
            if ((threadIdx.x & 63) < STEP) { to[0][wave * STEP + own] = p; to[1][wave * STEP + own] = q; }
            __syncthreads();
            q = 0.0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) q += to[1][w * STEP + own];
            if (kind == CSB_NORM_MEAN) {
                p = 0.0;
#pragma unroll
                for (int w = 0; w < WAVES; ++w) p += to[0][w * STEP + own];
            }
        }
    }
    // a row's first entry, which lane 0 has
    __device__ __forceinline__ float first(float v) {
        if constexpr (!TOKENS && L <= 64) return __shfl(v, 0, L);
        __syncthreads();                                       // (the last one has been read)
        const int row = TOKENS ? threadIdx.x % ROWS : threadIdx.x / L;
        if (lane == 0) sh.head[row] = v;
        __syncthreads();
        return sh.head[row];
    }
};

// A row's norm: sums of v - shift and of its square, then what its entries are taken off and multiplied by.
struct RowNorm {
    double shift = 0.0, p = 0.0, q = 0.0, mean = 0.0;
    float one = 1.0f, factor = 1.0f;
    // (entries that are not there are zeros) without a shift in binary32, eight squares at a time, where they and their sum are normal numbers
    template <bool WHOLE> __device__ __forceinline__ void add(int kind, const float *v, int there) {
        if (kind != CSB_NORM_MEAN) {
            float most = 0.0f, sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                most = fmaxf(most, fabsf(v[j]));
                sum = fmaf(v[j], v[j], sum);
            }
            const bool fine = most == 0.0f ? sum == 0.0f : most > 0x1p-50f && most < 0x1p60f;
            if (__builtin_expect(fine, 1)) { q += sum; return; }       // (each lane as if alone: a token does not depend on others of its wavefront)
        }
        auto one_more = [&](float x) {
            const double d = (double)x - shift;
            p += d;
            q = __builtin_fma(d, d, q);
        };
        if (WHOLE ? there > 0 : there >= 8) {
#pragma unroll
            for (int j = 0; j < 8; ++j) one_more(v[j]);
        } else if (!WHOLE) {
#pragma unroll
            for (int j = 0; j < 7; ++j) if (j < there) one_more(v[j]);
        }
    }
    __device__ __forceinline__ void finish(int kind, double per, double eps) {
        double square = q * per;
        if (kind == CSB_NORM_MEAN) {
            mean = p * per;
            square = __builtin_fmax(square - mean * mean, 0.0) + (p - p);        // (NaN where a sum is not finite: a maximum drops it)
            mean += shift;
        }
        const double e = square + eps;
        double y = __builtin_amdgcn_rsq(e);                    // two steps of Newton's: all digits of binary32, and more
        y = y * __builtin_fma(-0.5 * e * y, y, 1.5);
        y = y * __builtin_fma(-0.5 * e * y, y, 1.5);
        one = 1.0f;
        if (__builtin_expect(e > 0x1p150, 0)) {                // a factor below binary32's normal numbers: in two parts
            one = 0x1p-80f;
            y = e == __builtin_inf() ? 0.0 : y * 0x1p80;       // (of zero a step makes NaN: infinity times it)
        }
        factor = (float)y;
    }
    // eight entries (without the branch where the loads of many runs are to be in flight beside it)
    __device__ __forceinline__ float of(int kind, float v) const { return (kind == CSB_NORM_MEAN ? (float)(((double)v - mean) * one) : v * one) * factor; }
    __device__ __forceinline__ void of(int kind, float *v) const {
        if (kind == CSB_NORM_MEAN) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = (float)(((double)v[j] - mean) * one) * factor;
        } else if (__all(one == 1.0f)) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= factor;
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = v[j] * one * factor;
        }
    }
};

// NV runs of eight entries a lane, in registers from the first load to the last store; everything is requested at once.
template <int L, int NV, int THREADS, bool TOKENS, bool NEAR, bool WHOLE>
__global__ __launch_bounds__(THREADS) void block_norm_kernel(const NormDev a) {
    using Rows = NormRows<L, THREADS, TOKENS>;
    __shared__ typename Rows::Shared shared;
    Rows rows(a, shared);
    if (!rows.there) return;
    const int64_t base = (int64_t)rows.group * a.width, width = (int64_t)a.width * a.groups;
    const bool live = rows.t0 + rows.off < a.tokens;
    using Access = NormAccess<NEAR, WHOLE, !TOKENS>;
    const Access ya(a.y, rows.t0, rows.off, live, a.tokens, width), ga(a.gate, rows.t0, rows.off, live, a.tokens, width),
        xa(a.x, rows.t0, rows.off, live, a.tokens, width), ra(a.r, rows.t0, rows.off, live, a.tokens, width), oa(a.out, rows.t0, rows.off, live, a.tokens, width);
    auto at = [&](int i) { return (i * L + rows.lane) * 8; };
    auto entries = [&](int i) { return live ? a.width - at(i) : 0; };
    float v[NV][8];
    auto normed = [&](int kind, const float *weight, const float *bias) {
        RowNorm n;
        if (kind == CSB_NORM_MEAN) n.shift = rows.first(v[0][0]);
#pragma unroll
        for (int i = 0; i < NV; ++i) n.add<WHOLE>(kind, v[i], a.width - at(i));
        rows.sum(kind, n.p, n.q);
        n.finish(kind, a.per, a.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float w[8], b[8];
            n.of(kind, v[i]);
            norm_factors<WHOLE>(weight, base + at(i), a.width - at(i), 1.0f, w);
            norm_factors<WHOLE>(bias, base + at(i), a.width - at(i), 0.0f, b);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], w[j], b[j]);
        }
    };
    Raw8 y[NV], g[NV], x[NV];
    if (a.y.d)
#pragma unroll
        for (int i = 0; i < NV; ++i) y[i] = ya.load(base + at(i), entries(i));
    if (a.gate.d)
#pragma unroll
        for (int i = 0; i < NV; ++i) g[i] = ga.load(base + at(i), entries(i));
    if (a.x.d)
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = xa.load(base + at(i), entries(i));
    if (a.y.d) {
        float f[8];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            ya.widen(y[i], v[i]);
            if (a.gate.d && a.gate_first) {
                gate_factors(a, ga, g[i], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= f[j];
            }
        }
        if (a.after) normed(a.after, a.aw, a.ab);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (a.gate.d && !a.gate_first) {
                gate_factors(a, ga, g[i], f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= f[j];
            }
            if (!a.plain_scale) {
                norm_factors<WHOLE>(a.s, base + at(i), a.width - at(i), 1.0f, f);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] *= a.scale * f[j];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (a.x.d) {
            float f[8];
            xa.widen(x[i], f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = a.y.d ? f[j] + v[i][j] : f[j];
        }
        if (a.r.d) ra.store(base + at(i), entries(i), v[i]);
    }
    if (!a.before) return;
    normed(a.before, a.bw, a.bb);
#pragma unroll
    for (int i = 0; i < NV; ++i) oa.store(at(i), entries(i), v[i]);
}

// Rows that do not fit: once for each norm's sums, and once for the results, from the caches.  (One copy of the code for all three.)
template <int L, int THREADS, bool TOKENS, bool NEAR, bool WHOLE>
__global__ __launch_bounds__(THREADS) void block_norm_long_kernel(const NormDev a) {
    using Rows = NormRows<L, THREADS, TOKENS>;
    __shared__ typename Rows::Shared shared;
    Rows rows(a, shared);
    if (!rows.there) return;
    const int64_t base = (int64_t)rows.group * a.width, width = (int64_t)a.width * a.groups;
    const bool live = rows.t0 + rows.off < a.tokens;
    using Access = NormAccess<NEAR, WHOLE, !TOKENS>;
    const Access ya(a.y, rows.t0, rows.off, live, a.tokens, width), ga(a.gate, rows.t0, rows.off, live, a.tokens, width),
        xa(a.x, rows.t0, rows.off, live, a.tokens, width), ra(a.r, rows.t0, rows.off, live, a.tokens, width), oa(a.out, rows.t0, rows.off, live, a.tokens, width);
    RowNorm after, before;
    float v[8], f[8];
    enum { AFTER, BEFORE, RESULTS };
#pragma unroll 1
    for (int phase = a.after ? AFTER : a.before ? BEFORE : RESULTS; phase <= RESULTS; phase += phase == AFTER && !a.before ? 2 : 1) {
        const int norm = phase == AFTER ? a.after : phase == BEFORE ? a.before : 0;
        const bool gated = a.gate.d && (phase != AFTER || a.gate_first);
        bool shifted = norm != CSB_NORM_MEAN;
#pragma unroll 1
        for (int j0 = rows.lane * 8; j0 < a.width || !shifted; j0 += 8 * L) {    // (lanes behind a row's end take part in its first turn)
            const int there = live ? a.width - j0 : 0;
            if (a.y.d) {
                ya.widen(ya.load(base + j0, there), v);
                if (gated) {
                    gate_factors(a, ga, ga.load(base + j0, there), f);
                    if (a.gate_first)
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] *= f[j];
                }
            }
            if (phase != AFTER) {
                if (a.y.d) {
                    float w[8];
                    if (a.after) {
                        float b[8];
                        after.of(a.after, v);
                        norm_factors<WHOLE>(a.aw, base + j0, there, 1.0f, w);
                        norm_factors<WHOLE>(a.ab, base + j0, there, 0.0f, b);
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j], w[j], b[j]);
                    }
                    norm_factors<WHOLE>(a.s, base + j0, there, 1.0f, w);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        if (a.gate.d && !a.gate_first) v[j] *= f[j];
                        v[j] *= a.scale * w[j];
                    }
                }
                if (a.x.d) {
                    xa.widen(xa.load(base + j0, there), f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = a.y.d ? f[j] + v[j] : f[j];
                }
            }
            if (!shifted) {
                (phase == AFTER ? after : before).shift = rows.first(v[0]);
                shifted = true;
            }
            if (phase == AFTER) after.add<WHOLE>(norm, v, a.width - j0);
            else if (phase == BEFORE) before.add<WHOLE>(norm, v, a.width - j0);
            else {
                if (a.r.d) ra.store(base + j0, there, v);
                if (a.before) {
                    float w[8];
                    before.of(a.before, v);
                    norm_factors<WHOLE>(a.bw, j0, there, 1.0f, w);
                    norm_factors<WHOLE>(a.bb, j0, there, 0.0f, f);
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j], w[j], f[j]);
                    oa.store(j0, there, v);
                }
            }
        }
        if (phase == AFTER) {
            rows.sum(norm, after.p, after.q);
            after.finish(a.after, a.per, a.eps);
        } else if (phase == BEFORE) {
            rows.sum(norm, before.p, before.q);
            before.finish(a.before, a.per, a.eps);
        }
    }
}

// What stands between two products: y binary32 and the result column by column, x and r of one type and order, no gate; whole runs.  TB tokens
// side by side, a row in the registers of 1024 / TB lanes, up to eight runs each.
template <int VFX, bool XCOLS, int VFN, int TB>
__global__ __launch_bounds__(1024) void block_norm_product_kernel(const NormDev a) {
    constexpr int L = 1024 / TB, NV = 8;
    using Rows = NormRows<L, 1024, true>;
    using X = typename Elem<VFX>::T;
    using N = typename Elem<VFN>::T;
    __shared__ typename Rows::Shared shared;
    Rows rows(a, shared);
    if (!rows.there) return;
    const int64_t left = a.tokens - rows.t0;
    const bool live = rows.off < left;
    auto columns = [&](const NormOperand &o, int size) { return window((const char *)o.d + rows.t0 * size, (uint32_t)(((int64_t)(a.width - 1) * o.ld + left) * size)); };
    // the place of entry j of the lane's token in a window
    auto at = [&](const NormOperand &o, int size, int j) { return live && j < a.width ? ((uint32_t)j * (uint32_t)o.ld + (uint32_t)rows.off) * (uint32_t)size : kOutside; };
    auto first = [&](int i) { return (i * L + rows.lane) * 8; };
    float v[NV][8];
    {
        const window_t w = columns(a.y, 4);
        const uint32_t step = (uint32_t)a.y.ld * 4;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const uint32_t from = at(a.y, 4, first(i));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = i * L * 8 < a.width ? __builtin_bit_cast(float, window_load<float>(w, from + j * step)) : 0.0f;
        }
    }
    auto sums = [&](int kind, RowNorm &n) {
        if (kind == CSB_NORM_MEAN) n.shift = rows.first(v[0][0]);
#pragma unroll
        for (int i = 0; i < NV; ++i) if (i * L * 8 < a.width) n.add<true>(kind, v[i], a.width - first(i));
        rows.sum(kind, n.p, n.q);
        n.finish(kind, a.per, a.eps);
    };
    RowNorm after, before;
    if (a.after) sums(a.after, after);
    const window_t xw = columns(a.x, sizeof(X)), rw = columns(a.r, sizeof(X));
    const X *xp = (const X *)a.x.d + (rows.t0 + (live ? rows.off : 0)) * a.x.ld;
    X *rp = (X *)a.r.d + (rows.t0 + (live ? rows.off : 0)) * a.r.ld;
    const uint32_t x_step = (uint32_t)a.x.ld * sizeof(X), r_step = (uint32_t)a.r.ld * sizeof(X);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * L * 8 < a.width) {
            const int j0 = first(i), there = live ? a.width - j0 : 0;
            Run8<VFX> run;
            float f[8], b[8], s[8];
            if (a.x.d) {
                if constexpr (XCOLS) {
                    const uint32_t from = at(a.x, sizeof(X), j0);
#pragma unroll
                    for (int j = 0; j < 8; ++j) run.v[j] = __builtin_bit_cast(X, window_load<X>(xw, from + j * x_step));
                } else if (there > 0) {
                    if (a.past) run.v = __builtin_nontemporal_load((const typename Run8<VFX>::T8 *)(xp + j0));
                    else run.v = load_any<typename Run8<VFX>::T8>(xp + j0);
                }
            }
            norm_factors<true>(a.s, j0, a.width - j0, 1.0f, s);
            if (a.after) {
                norm_factors<true>(a.aw, j0, a.width - j0, 1.0f, f);
                norm_factors<true>(a.ab, j0, a.width - j0, 0.0f, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = fmaf(after.of(a.after, v[i][j]), f[j], b[j]);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[i][j] *= a.scale * s[j];
                if (a.x.d) v[i][j] += there > 0 ? run[j] : 0.0f;
            }
            if (a.r.d) {
#pragma unroll
                for (int j = 0; j < 8; ++j) run.set(j, v[i][j]);
                if constexpr (XCOLS) {
                    const uint32_t to = at(a.r, sizeof(X), j0);
#pragma unroll
                    for (int j = 0; j < 8; ++j) window_store<X>(rw, to + j * r_step, run.v[j]);
                } else if (there > 0) {
                    if (a.past) __builtin_nontemporal_store(run.v, (typename Run8<VFX>::T8 *)(rp + j0));
                    else store_any(rp + j0, run.v);
                }
            }
        }
    if (!a.before) return;
    sums(a.before, before);
    const window_t w = columns(a.out, sizeof(N));
    const uint32_t step = (uint32_t)a.out.ld * sizeof(N);
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (i * L * 8 < a.width) {
            const int j0 = first(i);
            float f[8], b[8];
            norm_factors<true>(a.bw, j0, a.width - j0, 1.0f, f);
            norm_factors<true>(a.bb, j0, a.width - j0, 0.0f, b);
            const uint32_t to = at(a.out, sizeof(N), j0);
#pragma unroll
            for (int j = 0; j < 8; ++j) window_store<N>(w, to + j * step, (N)fmaf(before.of(a.before, v[i][j]), f[j], b[j]));
        }
}

constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1024;

// NV 0: rows that do not fit
template <int L, int NV, int THREADS, bool TOKENS, bool NEAR, bool WHOLE>
static bool launch_norm(NormDev &d, hipStream_t st) {
    constexpr int64_t ROWS = THREADS / L;
    int64_t blocks;
    if (TOKENS) {
        d.tiles = (d.tokens + ROWS - 1) / ROWS;
        blocks = (d.tiles + 7) / 8 * 8;
        if (blocks > kMaxThreads / THREADS / d.groups) return false;
        blocks *= d.groups;
    } else {
        if (d.tokens > kMaxThreads / d.groups) return false;
        blocks = (d.tokens * d.groups + ROWS - 1) / ROWS;
    }
    if (blocks > kMaxThreads / THREADS) return false;
    if constexpr (NV == 0) hipLaunchKernelGGL((block_norm_long_kernel<L, THREADS, TOKENS, NEAR, WHOLE>), dim3((uint32_t)blocks), dim3(THREADS), 0, st, d);
    else hipLaunchKernelGGL((block_norm_kernel<L, NV, THREADS, TOKENS, NEAR, WHOLE>), dim3((uint32_t)blocks), dim3(THREADS), 0, st, d);
    return true;
}
template <int ROWS, bool NEAR>
static bool launch_norm_tokens(NormDev &d, hipStream_t st) {
    constexpr int L = 1024 / ROWS;
    if (d.width <= 8 * L) return launch_norm<L, 1, 1024, true, NEAR, false>(d, st);
    if (d.width <= 16 * L) return launch_norm<L, 2, 1024, true, NEAR, false>(d, st);
    return launch_norm<L, 0, 1024, true, NEAR, false>(d, st);
}

template <int VFX, bool XCOLS, int VFN, int TB>
static bool launch_norm_product(NormDev &d, hipStream_t st) {
    d.tiles = (d.tokens + TB - 1) / TB;
    const int64_t blocks = (d.tiles + 7) / 8 * 8;
    if (blocks > kMaxThreads / 1024) return false;
    hipLaunchKernelGGL((block_norm_product_kernel<VFX, XCOLS, VFN, TB>), dim3((uint32_t)blocks), dim3(1024), 0, st, d);
    return true;
}
template <int VFX, bool XCOLS, int VFN>
static bool launch_norm_product(NormDev &d, hipStream_t st) {
    // x and r row by row, read and written once, of as many bytes as the L2 caches hold (32 MiB) and more take the place of the columns' pieces there, which are put together
    // from several workgroups'; smaller ones are found there by what comes next.  Through the caches and past them, operands of 16 bits that change from call to call:
    // 1024 tokens of 8192 entries 31 and 32 us, 4096 of 4088 51 and 55, 4096 of 4096 51 and 50, 2048 of 8192 60 and 56 (without norm_before 44 and 33), 2560 99 and 96 (73 and 51).
    // (The other way round for the same operands again and again, 2048 of 8192 39 and 46; tall ones of 24 MiB gain already, 1536 of 8192 52 and 42.)
    const auto whole = [](const NormOperand &o) { return !o.d || ((uintptr_t)o.d % 16 == 0 && o.ld % 8 == 0); };
    d.past = !XCOLS && d.tokens * d.width * (int64_t)sizeof(typename Elem<VFX>::T) >= 32 << 20 && whole(d.x) && whole(d.r);
    // tokens side by side: as many as leave every CU a workgroup, and as registers hold (2048 tokens of 8192 entries by eights 58 us, by fours 79; of 8191 by the kernel for any operands 107)
    int tb = 1;
    while (tb < 16 && d.tokens > 256 * tb && (int64_t)d.width * tb * 2 <= 65536) tb *= 2;
    switch (tb) {
        case 1: return launch_norm_product<VFX, XCOLS, VFN, 1>(d, st);
        case 2: return launch_norm_product<VFX, XCOLS, VFN, 2>(d, st);
        case 4: return launch_norm_product<VFX, XCOLS, VFN, 4>(d, st);
        case 8: return launch_norm_product<VFX, XCOLS, VFN, 8>(d, st);
        default: return launch_norm_product<VFX, XCOLS, VFN, 16>(d, st);
    }
}
// Whether the call is the products' (above): *ok: whether it was launched.
static bool norm_of_products(NormDev &d, hipStream_t st, bool *ok) {
    if (d.groups > 1 || d.width % 8 || d.gate.d || !d.y.d || !d.y.columns || d.y.type != CSB_VAL_F32) return false;
    if (d.before && !d.out.columns) return false;
    const NormOperand &x = d.x.d ? d.x : d.r;
    if (!x.d || (d.x.d && d.r.d && (d.x.type != d.r.type || d.x.columns != d.r.columns))) return false;
    const int n = d.before ? d.out.type : x.type;
    const auto is = [&](int vfx, bool columns, int vfn) { return x.type == vfx && (x.columns != 0) == columns && n == vfn; };
    if (is(CSB_VAL_BF16, false, CSB_VAL_BF16)) *ok = launch_norm_product<CSB_VAL_BF16, false, CSB_VAL_BF16>(d, st);
    else if (is(CSB_VAL_F16, false, CSB_VAL_F16)) *ok = launch_norm_product<CSB_VAL_F16, false, CSB_VAL_F16>(d, st);
    else if (is(CSB_VAL_F32, false, CSB_VAL_F32)) *ok = launch_norm_product<CSB_VAL_F32, false, CSB_VAL_F32>(d, st);
    else if (is(CSB_VAL_F32, false, CSB_VAL_BF16)) *ok = launch_norm_product<CSB_VAL_F32, false, CSB_VAL_BF16>(d, st);
    else if (is(CSB_VAL_F32, false, CSB_VAL_F16)) *ok = launch_norm_product<CSB_VAL_F32, false, CSB_VAL_F16>(d, st);
    else if (is(CSB_VAL_F32, true, CSB_VAL_F32)) *ok = launch_norm_product<CSB_VAL_F32, true, CSB_VAL_F32>(d, st);
    else if (is(CSB_VAL_F32, true, CSB_VAL_BF16)) *ok = launch_norm_product<CSB_VAL_F32, true, CSB_VAL_BF16>(d, st);
    else if (is(CSB_VAL_F32, true, CSB_VAL_F16)) *ok = launch_norm_product<CSB_VAL_F32, true, CSB_VAL_F16>(d, st);
    else return false;
    return true;
}

template <bool WHOLE>
static bool launch_norm_rows(NormDev &d, hipStream_t st) {
    const int w = d.width;
    if (w <= 64) return launch_norm<8, 1, 256, false, false, WHOLE>(d, st);
    if (w <= 128) return launch_norm<16, 1, 256, false, false, WHOLE>(d, st);
    if (w <= 512) return launch_norm<64, 1, 256, false, false, WHOLE>(d, st);
    if (w <= 2048) return launch_norm<256, 1, 256, false, false, WHOLE>(d, st);
    if (w <= 4096) return launch_norm<256, 2, 256, false, false, WHOLE>(d, st);
    if (w <= 8192) return launch_norm<1024, 1, 1024, false, false, WHOLE>(d, st);
    if (w <= 16384) return launch_norm<1024, 2, 1024, false, false, WHOLE>(d, st);
    return launch_norm<1024, 0, 1024, false, false, WHOLE>(d, st);
}

static bool launch_norm(NormDev &d, bool columns, bool far, hipStream_t st) {
    if (!columns) return d.width % 8 ? launch_norm_rows<false>(d, st) : launch_norm_rows<true>(d, st);
    if (far) return launch_norm_tokens<1, false>(d, st);
    bool ok;
    if (norm_of_products(d, st, &ok)) return ok;
    if (d.width <= 256) return launch_norm<32, 1, 256, true, true, false>(d, st);
    const int64_t rows = d.tokens * d.groups;                  // (as above)
    if (rows <= 256) return launch_norm_tokens<1, true>(d, st);
    if (rows <= 512) return launch_norm_tokens<2, true>(d, st);
    if (rows <= 1024) return launch_norm_tokens<4, true>(d, st);
    if (rows <= 2048) return launch_norm_tokens<8, true>(d, st);
    return launch_norm_tokens<16, true>(d, st);
}

}  // namespace csb

extern "C" int csb_block_norm(const csb_norm_args *a, void *stream) {
    using namespace csb;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_block_norm: ") + what); return code; };
    if (!a) return fail(CSB_EINVAL, "NULL arguments");
    if (a->n_tokens < 0 || a->width < 1 || a->groups < 1) return fail(CSB_EINVAL, "bad size");
    if (a->width % a->groups) return fail(CSB_EINVAL, "width is no multiple of groups");
    for (int kind : {a->after, a->before})
        if (kind != CSB_NORM_NONE && kind != CSB_NORM_RMS && kind != CSB_NORM_MEAN) return fail(CSB_EINVAL, "unknown norm");
    if (a->gate_kind != CSB_GATE_SILU && a->gate_kind != CSB_GATE_SIGMOID) return fail(CSB_EINVAL, "unknown gate");
    if (!(a->eps >= 0.0f && a->eps <= 0x1.fffffep127f)) return fail(CSB_EINVAL, "eps below zero or not finite");
    if (a->width / a->groups > 32768) return fail(CSB_EUNSUPPORTED, "more than 32768 entries under one norm");
    if (a->before && a->groups > 1) return fail(CSB_EUNSUPPORTED, "norm_before with several groups");
    if (a->n_tokens == 0) return CSB_OK;
    if (!a->y.d && !a->x.d) return fail(CSB_EINVAL, "NULL pointer: neither y nor x");
    if (!a->y.d && (a->gate.d || a->after)) return fail(CSB_EINVAL, "a gate or norm_after without y");
    if (a->before ? !a->out.d : !a->r.d) return fail(CSB_EINVAL, "NULL pointer: no output");
    if (a->before && a->r.d == a->out.d) return fail(CSB_EINVAL, "both outputs in one place");
    NormDev d{};
    bool columns = false, far = false;                         // far: columns of 2^31 bytes and more
    const csb_norm_operand *from[5] = {&a->y, &a->gate, &a->x, &a->r, &a->out};
    NormOperand *to[5] = {&d.y, &d.gate, &d.x, &d.r, &d.out};
    for (int i = 0; i < 5; ++i) {
        const csb_norm_operand &o = *from[i];
        if (!o.d || (i == 4 && !a->before)) continue;
        if (!known_type(o.type)) return fail(CSB_EINVAL, "unknown type");
        if (o.ld < (o.columns ? a->n_tokens : (int64_t)a->width)) return fail(CSB_EINVAL, "a leading dimension below the width of its rows");
        if ((uintptr_t)o.d % (uintptr_t)type_size(o.type)) return fail(CSB_EINVAL, "misaligned pointer");
        *to[i] = {o.d, o.ld, o.type, o.columns != 0};
        columns |= o.columns != 0;
        far |= o.columns && o.ld > 0x7fffffff / type_size(o.type) / a->width;
    }
    for (int i = 0; i < 3; ++i)
        for (int o = 3; o < 5; ++o)
            if (to[i]->d && to[i]->d == to[o]->d && (to[i]->ld != to[o]->ld || to[i]->type != to[o]->type || to[i]->columns != to[o]->columns))
                return fail(CSB_EINVAL, "an output in place of an input of another type, order or leading dimension");
    for (const float *p : {a->d_after_w, a->d_after_b, a->d_scale, a->d_before_w, a->d_before_b})
        if ((uintptr_t)p % 4) return fail(CSB_EINVAL, "misaligned pointer");
    d.aw = a->d_after_w; d.ab = a->d_after_b; d.s = a->d_scale; d.bw = a->d_before_w; d.bb = a->d_before_b;
    d.tokens = a->n_tokens; d.width = a->width / a->groups; d.groups = a->groups;
    d.after = a->after; d.before = a->before; d.sigmoid = a->gate_kind == CSB_GATE_SIGMOID; d.gate_first = a->gate_first;
    d.scale = a->scale; d.eps = a->eps; d.per = 1.0 / d.width;
    d.plain_scale = !a->d_scale && a->scale == 1.0f;
    d.plain_gate = (!d.r.d || d.r.type != CSB_VAL_F32) && (!d.out.d || d.out.type != CSB_VAL_F32);
    if (!launch_norm(d, columns, far, (hipStream_t)stream)) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(CSB_EDEVICE, hipGetErrorString(e));
    return CSB_OK;
}
