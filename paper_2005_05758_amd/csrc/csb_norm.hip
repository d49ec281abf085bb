// Norms around a block (csb_block_norm): r = x + scale s norm_after(y gate), out = norm_before(r), one pass over memory.
//
// Bound by HBM: a token's entries are read once, stay in registers over both norms, and are written once.  L lanes share a row (a token, or a
// group of one), NV runs of eight entries each.  Where all operands are row by row a row's lanes are neighbours; where one is column by column
// (a product's operand) neighbouring lanes are neighbouring tokens, eight of them, so that columns are read and written 16 or 32
// bytes at a time, and the workgroups of neighbouring tokens share an XCD, whose L2 puts these pieces together.
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
    float scale;
    double eps;
};

struct Raw8 { uint32_t w[8]; };                // eight entries as they are stored: 16 bits each in the first four words, or 32

// Entries j .. j + 7 of token t, the first `there` of them.
__device__ __forceinline__ Raw8 norm_load(const NormOperand &o, int64_t t, int64_t j, int there) {
    using u32x4 = uint32_t __attribute__((ext_vector_type(4), aligned(2), may_alias));
    Raw8 r{};
    const bool half = o.type != CSB_VAL_F32;                   // (uniform, as the order)
    if (o.columns) {
        if (half) {
            const uint16_t *p = (const uint16_t *)o.d + j * o.ld + t;
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < there) r.w[i / 2] |= (uint32_t)p[i * o.ld] << (16 * (i & 1));
        } else {
            const uint32_t *p = (const uint32_t *)o.d + j * o.ld + t;
#pragma unroll
            for (int i = 0; i < 8; ++i) if (i < there) r.w[i] = p[i * o.ld];
        }
    } else if (half) {
        const uint16_t *p = (const uint16_t *)o.d + t * o.ld + j;
        if (there >= 8) {
            const u32x4 v = *(const u32x4 *)p;
#pragma unroll
            for (int i = 0; i < 4; ++i) r.w[i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i) if (i < there) r.w[i / 2] |= (uint32_t)p[i] << (16 * (i & 1));
        }
    } else {
        const uint32_t *p = (const uint32_t *)o.d + t * o.ld + j;
        if (there >= 8) {
            const u32x4 v = *(const u32x4 *)p, w = *(const u32x4 *)(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) { r.w[i] = v[i]; r.w[4 + i] = w[i]; }
        } else {
#pragma unroll
            for (int i = 0; i < 7; ++i) if (i < there) r.w[i] = p[i];
        }
    }
    return r;
}
__device__ __forceinline__ void norm_widen(const Raw8 &r, int type, float *v) {
    if (type == CSB_VAL_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, r.w[i]);
    } else if (type == CSB_VAL_BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = __builtin_bit_cast(float, i & 1 ? r.w[i / 2] & 0xffff0000u : r.w[i / 2] << 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(i & 1 ? r.w[i / 2] >> 16 : r.w[i / 2] & 0xffff));
    }
}
template <typename T> __device__ __forceinline__ uint16_t bits16(float v) { return __builtin_bit_cast(uint16_t, (T)v); }
__device__ __forceinline__ void norm_store(const NormOperand &o, int64_t t, int64_t j, int there, const float *v) {
    using u32x4 = uint32_t __attribute__((ext_vector_type(4), aligned(2), may_alias));
    const bool half = o.type != CSB_VAL_F32;
    uint32_t w[8];
    if (o.type == CSB_VAL_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = __builtin_bit_cast(uint32_t, v[i]);
    } else if (o.type == CSB_VAL_BF16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = bits16<__bf16>(v[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = bits16<_Float16>(v[i]);
    }
    if (half) {
        uint16_t *p = (uint16_t *)o.d + (o.columns ? j * o.ld + t : t * o.ld + j);
        if (!o.columns && there >= 8) {
            *(u32x4 *)p = u32x4{w[0] | w[1] << 16, w[2] | w[3] << 16, w[4] | w[5] << 16, w[6] | w[7] << 16};
            return;
        }
        const int64_t step = o.columns ? o.ld : 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < there) p[i * step] = (uint16_t)w[i];
    } else {
        uint32_t *p = (uint32_t *)o.d + (o.columns ? j * o.ld + t : t * o.ld + j);
        if (!o.columns && there >= 8) {
            *(u32x4 *)p = u32x4{w[0], w[1], w[2], w[3]};
            *(u32x4 *)(p + 4) = u32x4{w[4], w[5], w[6], w[7]};
            return;
        }
        const int64_t step = o.columns ? o.ld : 1;
#pragma unroll
        for (int i = 0; i < 8; ++i) if (i < there) p[i * step] = w[i];
    }
}
__device__ __forceinline__ void norm_factors(const float *p, int64_t j, int there, float fill, float *v) {
    using f32x4 = float __attribute__((ext_vector_type(4), aligned(4), may_alias));
    if (p && there >= 8) {
        const f32x4 a = *(const f32x4 *)(p + j), b = *(const f32x4 *)(p + j + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = p && i < there ? p[j + i] : fill;
    }
}

// L lanes a row, NV runs of eight entries a lane, THREADS a workgroup.  TOKENS: a workgroup's rows are neighbouring lanes, else a row's lanes are.
template <int L, int NV, int THREADS, bool TOKENS>
__global__ __launch_bounds__(THREADS) void block_norm_kernel(const NormDev a) {
    constexpr int ROWS = THREADS / L, WAVES = THREADS / 64;
    __shared__ double sums[2][2][WAVES * (TOKENS ? ROWS : 1)];
    const int tid = threadIdx.x, wave = tid >> 6;
    int64_t t;
    int lane, group;
    if constexpr (TOKENS) {
        // the tiles that an XCD gets, one after the other, are neighbours
        const int64_t per = (a.tiles + 7) / 8, tile = (int64_t)(blockIdx.x % 8) * per + blockIdx.x / 8 % per;
        group = (int)(blockIdx.x / (8 * per));
        if (tile >= a.tiles) return;
        t = tile * ROWS + tid % ROWS;
        lane = tid / ROWS;
    } else {
        const int64_t row = (int64_t)blockIdx.x * ROWS + tid / L;
        t = row / a.groups;
        group = (int)(row % a.groups);
        lane = tid % L;
    }
    const bool live = t < a.tokens;
    const int64_t base = (int64_t)group * a.width;

    // sums over a row's lanes, in every one of them (a fixed order)
    int turn = 0;
    auto row_sums = [&](double &p, double &q) {
        constexpr int LOW = TOKENS ? ROWS : 1, HIGH = TOKENS ? 64 : L < 64 ? L : 64;
#pragma unroll
        for (int d = LOW; d < HIGH; d *= 2) {
            p += __shfl_xor(p, d);
            q += __shfl_xor(q, d);
        }
        if constexpr (TOKENS || L > 64) {
            double(*to)[WAVES * (TOKENS ? ROWS : 1)] = sums[turn];
            turn ^= 1;
            const int own = TOKENS ? tid % ROWS : 0;
            constexpr int STEP = TOKENS ? ROWS : 1;
            if ((tid & 63) < STEP) { to[0][wave * STEP + own] = p; to[1][wave * STEP + own] = q; }
            __syncthreads();
            p = q = 0.0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { p += to[0][w * STEP + own]; q += to[1][w * STEP + own]; }
        }
    };
    float v[NV][8];
    // v <- norm(v), w and b still to come
    auto normed = [&](int kind) {
        double p = 0.0, q = 0.0, shift = 0.0;
        if (kind == CSB_NORM_MEAN) {                           // v[0] of the row: lane 0's
            if constexpr (TOKENS) {
                __shared__ float head[ROWS];
                if (lane == 0) head[tid] = v[0][0];
                __syncthreads();
                shift = head[tid % ROWS];
            } else if constexpr (L <= 64) {
                shift = __shfl(v[0][0], 0, L);
            } else {
                __shared__ float head;
                if (tid == 0) head = v[0][0];
                __syncthreads();
                shift = head;
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if ((i * L + lane) * 8 + j < a.width) {
                    const double d = (double)v[i][j] - shift;
                    p += d;
                    q = __builtin_fma(d, d, q);
                }
        row_sums(p, q);
        double mean = 0.0, square = q / a.width;
        if (kind == CSB_NORM_MEAN) {
            mean = p / a.width;
            square = __builtin_fmax(square - mean * mean, 0.0);
            mean += shift;
            if (p != p) square = p;
        }
        const double e = square + a.eps;
        double y = __builtin_amdgcn_rsq(e);                    // two steps of Newton's: all digits of binary32, and more
        y = y * __builtin_fma(-0.5 * e * y, y, 1.5);
        y = y * __builtin_fma(-0.5 * e * y, y, 1.5);
        const bool large = e > 0x1p150;                        // a factor below binary32's normal numbers: in two parts
        const float one = large ? 0x1p-80f : 1.0f, f = (float)(large ? y * 0x1p80 : y);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float c = kind == CSB_NORM_MEAN ? (float)(((double)v[i][j] - mean) * one) : v[i][j] * one;
                v[i][j] = c * f;
            }
    };
    auto entries = [&](int i) { return live ? a.width - (i * L + lane) * 8 : 0; };
    float gate[NV][8];
    if (a.y.d) {
        Raw8 y[NV], g[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            y[i] = norm_load(a.y, t, base + (i * L + lane) * 8, entries(i));
            if (a.gate.d) g[i] = norm_load(a.gate, t, base + (i * L + lane) * 8, entries(i));
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            norm_widen(y[i], a.y.type, v[i]);
            if (a.gate.d) {
                norm_widen(g[i], a.gate.type, gate[i]);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float x = gate[i][j], s = sigmoid_within(x);
                    gate[i][j] = a.sigmoid ? (x != x ? x : s) : x * s;
                    if (a.gate_first) v[i][j] *= gate[i][j];
                }
            }
        }
        if (a.after) {
            normed(a.after);
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float w[8], b[8];
                norm_factors(a.aw, base + (i * L + lane) * 8, entries(i), 1.0f, w);
                norm_factors(a.ab, base + (i * L + lane) * 8, entries(i), 0.0f, b);
#pragma unroll
                for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], w[j], b[j]);
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float s[8];
            norm_factors(a.s, base + (i * L + lane) * 8, entries(i), 1.0f, s);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (a.gate.d && !a.gate_first) v[i][j] *= gate[i][j];
                v[i][j] *= a.scale * s[j];
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.0f;
    }
    if (a.x.d) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float x[8];
            norm_widen(norm_load(a.x, t, base + (i * L + lane) * 8, entries(i)), a.x.type, x);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = a.y.d ? x[j] + v[i][j] : x[j];
        }
    }
    if (a.r.d)
#pragma unroll
        for (int i = 0; i < NV; ++i) norm_store(a.r, t, base + (i * L + lane) * 8, entries(i), v[i]);
    if (!a.before) return;
    normed(a.before);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float w[8], b[8];
        norm_factors(a.bw, (i * L + lane) * 8, entries(i), 1.0f, w);
        norm_factors(a.bb, (i * L + lane) * 8, entries(i), 0.0f, b);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = fmaf(v[i][j], w[j], b[j]);
        norm_store(a.out, t, (i * L + lane) * 8, entries(i), v[i]);
    }
}

constexpr int64_t kMaxThreads = ((int64_t)1 << 32) - 1024;

template <int L, int NV, int THREADS, bool TOKENS>
static bool launch_norm(NormDev &d, hipStream_t st) {
    constexpr int64_t ROWS = THREADS / L;
    int64_t blocks;
    if (TOKENS) {
        d.tiles = (d.tokens + ROWS - 1) / ROWS;
        blocks = (d.tiles + 7) / 8 * 8 * d.groups;
    } else {
        if (d.tokens > ((int64_t)1 << 40) / d.groups) return false;
        blocks = (d.tokens * d.groups + ROWS - 1) / ROWS;
    }
    if (blocks > kMaxThreads / THREADS) return false;
    hipLaunchKernelGGL((block_norm_kernel<L, NV, THREADS, TOKENS>), dim3((uint32_t)blocks), dim3(THREADS), 0, st, d);
    return true;
}

static bool launch_norm(NormDev &d, bool tokens, hipStream_t st) {
    const int w = d.width;
    if (tokens) {
        if (w <= 256) return launch_norm<32, 1, 256, true>(d, st);
        if (w <= 1024) return launch_norm<128, 1, 1024, true>(d, st);
        if (w <= 2048) return launch_norm<128, 2, 1024, true>(d, st);
        if (w <= 4096) return launch_norm<128, 4, 1024, true>(d, st);
        if (w <= 8192) return launch_norm<256, 4, 1024, true>(d, st);
        if (w <= 16384) return launch_norm<512, 4, 1024, true>(d, st);
        return launch_norm<1024, 4, 1024, true>(d, st);
    }
    if (w <= 64) return launch_norm<8, 1, 256, false>(d, st);
    if (w <= 128) return launch_norm<16, 1, 256, false>(d, st);
    if (w <= 512) return launch_norm<64, 1, 256, false>(d, st);
    if (w <= 2048) return launch_norm<256, 1, 256, false>(d, st);
    if (w <= 4096) return launch_norm<256, 2, 256, false>(d, st);
    if (w <= 8192) return launch_norm<1024, 1, 1024, false>(d, st);
    if (w <= 16384) return launch_norm<1024, 2, 1024, false>(d, st);
    return launch_norm<1024, 4, 1024, false>(d, st);
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
    if (!(a->eps >= 0.0f)) return fail(CSB_EINVAL, "eps below zero");
    if (a->width / a->groups > 32768) return fail(CSB_EUNSUPPORTED, "more than 32768 entries under one norm (a row stays in a workgroup's registers)");
    if (a->before && a->groups > 1) return fail(CSB_EUNSUPPORTED, "norm_before with several groups");
    if (a->n_tokens == 0) return CSB_OK;
    if (!a->y.d && !a->x.d) return fail(CSB_EINVAL, "NULL pointer: neither y nor x");
    if (!a->y.d && (a->gate.d || a->after)) return fail(CSB_EINVAL, "a gate or norm_after without y");
    if (a->before ? !a->out.d : !a->r.d) return fail(CSB_EINVAL, "NULL pointer: no output");
    if (a->before && a->r.d == a->out.d) return fail(CSB_EINVAL, "both outputs in one place");
    NormDev d{};
    bool columns = false;
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
    }
    for (const float *p : {a->d_after_w, a->d_after_b, a->d_scale, a->d_before_w, a->d_before_b})
        if ((uintptr_t)p % 4) return fail(CSB_EINVAL, "misaligned pointer");
    d.aw = a->d_after_w; d.ab = a->d_after_b; d.s = a->d_scale; d.bw = a->d_before_w; d.bb = a->d_before_b;
    d.tokens = a->n_tokens; d.width = a->width / a->groups; d.groups = a->groups;
    d.after = a->after; d.before = a->before; d.sigmoid = a->gate_kind == CSB_GATE_SIGMOID; d.gate_first = a->gate_first;
    d.scale = a->scale; d.eps = a->eps;
    if (!launch_norm(d, columns, (hipStream_t)stream)) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(CSB_EDEVICE, hipGetErrorString(e));
    return CSB_OK;
}
