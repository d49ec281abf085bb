// The short causal convolution in front of a recurrence (csb_short_conv): out[t, c] = act(b[c] + sum_j w[c][j] x[t - (W - 1) + j, c]), with
// the inputs before a sequence's first token from its state.
//
// Bound by HBM: every input is read once, every output written once; the W - 1 inputs before a tile come from the caches (48 packed prompts, 16411 tokens of 4096
// bfloat16 channels, width 4: 62 us, 4.3 TB/s; a call among others 68).  A thread has eight channels (their W weights in registers) and walks down kConvRun tokens with the last W - 1
// inputs in registers, kConvAhead tokens requested together (one by one that call took 97 us, four together 80; the weights in 16-byte words and runs of 32 tokens
// took it to 68).  The first tile of a sequence also makes its new state: it alone reads the old one, so a state may be replaced in place while later tiles run.
#include <algorithm>
#include <type_traits>

#include "csb_layer.hpp"

namespace csb {

constexpr int kConvRun = 32, kConvAhead = 4;

struct ConvDev {
    const void *x;
    const float *w, *bias;
    const int32_t *start, *len, *slot;
    const void *s_in;
    void *s_out, *out;
    int64_t ldx, ldo, n_tokens, each;
    int32_t channels, n_seq, n_states, silu, lanes, shift, col_tiles;   // lanes: threads side by side on a token's channels, a power of two
};

template <int VF, int W>
__global__ __launch_bounds__(256) void short_conv_kernel(const ConvDev a) {
    using T = typename Elem<VF>::T;
    using Run = Run8<VF>;
    const int64_t tile = blockIdx.x / a.col_tiles;
    const int seq = tile_sequence(a.start, a.n_seq, a.n_tokens, a.shift, tile, a.each);
    if (seq < 0) return;
    int64_t first, end;
    sequence_range(a.start, seq, a.each, a.n_tokens, &first, &end);
    const int64_t number = tile - ((first >> a.shift) + seq);  // of this tile in its sequence
    if (a.len) end = first + clamp64(a.len[seq], 0, end - first);
    const int64_t count = end - first;
    if (number < 0 || (number > 0 && (number << a.shift) >= count)) return;
    const int lane = threadIdx.x & (a.lanes - 1), row = threadIdx.x / a.lanes;
    const int64_t c = ((int64_t)(blockIdx.x % a.col_tiles) * a.lanes + lane) * 8;
    if (c >= a.channels) return;
    const int there = a.channels - (int)c;
    const int32_t s = a.slot ? a.slot[seq] : seq;
    const bool known = s >= 0 && s < a.n_states;
    const T *x = (const T *)a.x + first * a.ldx + c;
    const T *old = a.s_in && known ? (const T *)a.s_in + (int64_t)s * (W - 1) * a.channels + c : nullptr;
    // input `at` of the sequence, the state's for -1 and before
    auto input = [&](int64_t at) {
        Run r;
        if (at >= 0) r.load(x + at * a.ldx, there);
        else if (old) r.load(old + (at + W - 1) * a.channels, there);
        else r.v = typename Run::T8{};
        return r;
    };
    const int64_t t0 = (number << a.shift) + row * kConvRun, t1 = t0 + kConvRun < count ? t0 + kConvRun : count;
    if (t0 < count) {
        float w[W][8], bias[8], v[W][8];
        const float *wp = a.w + c * W;
        if (there >= 8) {
            using f32x4 = float __attribute__((ext_vector_type(4)));
#pragma unroll
            for (int k = 0; k < 2 * W; ++k) {
                const f32x4 x = load_any<f32x4>(wp + 4 * k);
#pragma unroll
                for (int e = 0; e < 4; ++e) w[(4 * k + e) % W][(4 * k + e) / W] = x[e];
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4 x = a.bias ? load_any<f32x4>(a.bias + c + 4 * k) : f32x4{};
#pragma unroll
                for (int e = 0; e < 4; ++e) bias[4 * k + e] = x[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                bias[i] = a.bias && i < there ? a.bias[c + i] : 0.0f;
#pragma unroll
                for (int j = 0; j < W; ++j) w[j][i] = i < there ? wp[i * W + j] : 0.0f;
            }
        }
        auto widen = [&](const Run &r, float *to) {
#pragma unroll
            for (int i = 0; i < 8; ++i) to[i] = r[i];
        };
#pragma unroll
        for (int j = 0; j < W - 1; ++j) widen(input(t0 - (W - 1) + j), v[j]);
        const T *from = x + t0 * a.ldx;
        T *out = (T *)a.out + (first + t0) * a.ldo + c;
        const int n = (int)(t1 - t0);
        // kConvAhead tokens are requested together
        auto tokens = [&](auto whole, int count) {
            Run in[kConvAhead];
#pragma unroll
            for (int k = 0; k < kConvAhead; ++k)
                if (whole || k < count) in[k].load(from + k * a.ldx, there);
#pragma unroll
            for (int k = 0; k < kConvAhead; ++k)
                if (whole || k < count) {
                    widen(in[k], v[W - 1]);
                    Run o;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float y = bias[i];
#pragma unroll
                        for (int j = 0; j < W; ++j) y = fmaf(w[j][i], v[j][i], y);
                        o.set(i, a.silu ? silu<VF>(y) : y);
                    }
                    o.store(out + k * a.ldo, there);
#pragma unroll
                    for (int j = 0; j < W - 1; ++j)
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[j][i] = v[j + 1][i];
                }
            from += kConvAhead * a.ldx;
            out += kConvAhead * a.ldo;
        };
        int t = 0;
        for (; t + kConvAhead <= n; t += kConvAhead) tokens(std::true_type{}, kConvAhead);
        if (t < n) tokens(std::false_type{}, n - t);
    }
    if (W > 1 && number == 0 && row == 0 && a.s_out && known) {
        Run v[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) v[j] = input(count - (W - 1) + j);     // all read before one is written
        T *to = (T *)a.s_out + (int64_t)s * (W - 1) * a.channels + c;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) v[j].store(to + (int64_t)j * a.channels, there);
    }
}

template <int VF>
static void launch_conv(const ConvDev &d, int width, dim3 grid, dim3 block, hipStream_t st) {
    switch (width) {
        case 1: hipLaunchKernelGGL((short_conv_kernel<VF, 1>), grid, block, 0, st, d); break;
        case 2: hipLaunchKernelGGL((short_conv_kernel<VF, 2>), grid, block, 0, st, d); break;
        case 3: hipLaunchKernelGGL((short_conv_kernel<VF, 3>), grid, block, 0, st, d); break;
        case 4: hipLaunchKernelGGL((short_conv_kernel<VF, 4>), grid, block, 0, st, d); break;
        case 5: hipLaunchKernelGGL((short_conv_kernel<VF, 5>), grid, block, 0, st, d); break;
        case 6: hipLaunchKernelGGL((short_conv_kernel<VF, 6>), grid, block, 0, st, d); break;
        case 7: hipLaunchKernelGGL((short_conv_kernel<VF, 7>), grid, block, 0, st, d); break;
        default: hipLaunchKernelGGL((short_conv_kernel<VF, 8>), grid, block, 0, st, d); break;
    }
}

}  // namespace csb

extern "C" int csb_short_conv(const csb_conv_args *a, void *stream) {
    using namespace csb;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_short_conv: ") + what); return code; };
    if (!a) return fail(CSB_EINVAL, "NULL arguments");
    if (!known_type(a->type)) return fail(CSB_EINVAL, "unknown type");
    if (a->n_seq < 0 || a->n_tokens < 0 || a->channels < 1 || a->width < 1) return fail(CSB_EINVAL, "bad size");
    if (a->width > 8) return fail(CSB_EUNSUPPORTED, "width above 8 (a thread holds the weights of eight channels in registers)");
    if (a->n_tokens > 0x7fffffff) return fail(CSB_EUNSUPPORTED, "offsets are 32-bit: more than 2^31 - 1 tokens");
    if (!a->d_w || (a->n_tokens && (!a->d_x || !a->d_out))) return fail(CSB_EINVAL, "NULL pointer");
    if (a->n_tokens && a->d_x == a->d_out) return fail(CSB_EINVAL, "out is x (tokens behind read what would be overwritten)");
    if (a->ldx < a->channels || a->ldo < a->channels) return fail(CSB_EINVAL, "a leading dimension below the width of its rows");
    if (!a->d_start && a->n_seq && a->n_tokens % a->n_seq) return fail(CSB_EINVAL, "n_tokens is no multiple of n_seq (and there are no offsets)");
    if ((a->d_state_in || a->d_state_out) && a->n_states < 1) return fail(CSB_EINVAL, "states without room for one");
    if (((uintptr_t)a->d_x | (uintptr_t)a->d_out | (uintptr_t)a->d_state_in | (uintptr_t)a->d_state_out) % (uintptr_t)type_size(a->type) ||
        ((uintptr_t)a->d_w | (uintptr_t)a->d_bias | (uintptr_t)a->d_start | (uintptr_t)a->d_len | (uintptr_t)a->d_slot) % 4)
        return fail(CSB_EINVAL, "misaligned pointer");
    if (a->n_seq == 0) return CSB_OK;
    ConvDev d{};
    d.x = a->d_x; d.w = a->d_w; d.bias = a->d_bias; d.start = a->d_start; d.len = a->d_len; d.slot = a->d_slot;
    d.s_in = a->d_state_in; d.s_out = a->d_state_out; d.out = a->d_out;
    d.ldx = a->ldx; d.ldo = a->ldo; d.n_tokens = a->n_tokens; d.each = a->n_tokens / a->n_seq;
    d.channels = a->channels; d.n_seq = a->n_seq; d.n_states = a->n_states; d.silu = a->silu;
    const int64_t runs = ((int64_t)a->channels + 7) / 8;       // of eight channels
    d.lanes = 64;
    while (d.lanes > 1 && d.lanes / 2 >= runs) d.lanes /= 2;
    // rows of threads on runs of tokens one behind the other: four, or one where a sequence has no more than a run on average, and a wavefront at least (the
    // workgroup looks for its sequence with all of its threads: 4096 sequences of 64 tokens, 8 channels, 64 us, by four threads 500)
    const int rows = std::max(64 / d.lanes, a->n_tokens / a->n_seq <= kConvRun ? 1 : 4);
    d.col_tiles = (int32_t)((runs + d.lanes - 1) / d.lanes);
    d.shift = 0;
    while ((1 << d.shift) < rows * kConvRun) ++d.shift;
    const int64_t groups = tile_numbers(a->n_tokens, a->n_seq, d.shift) * d.col_tiles;
    if (groups > kMaxWorkgroups) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    const dim3 grid((uint32_t)groups), block((uint32_t)(rows * d.lanes));
    hipStream_t st = (hipStream_t)stream;
    switch (a->type) {
        case CSB_VAL_F32: launch_conv<CSB_VAL_F32>(d, a->width, grid, block, st); break;
        case CSB_VAL_F16: launch_conv<CSB_VAL_F16>(d, a->width, grid, block, st); break;
        default: launch_conv<CSB_VAL_BF16>(d, a->width, grid, block, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(CSB_EDEVICE, hipGetErrorString(e));
    return CSB_OK;
}
