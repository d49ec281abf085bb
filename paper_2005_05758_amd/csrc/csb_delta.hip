// The gated delta rule token by token (csb_delta_recurrent), and the checks of its arguments.
//
// Per value head, with the state S in binary32:  S <- e^g S;  u = beta (v - S^T k);  S <- S + k u^T;
// o = scale S^T q.  The columns of S do not depend on each other, so a wavefront takes 32 of them with
// all their rows and keeps them in registers from the first token to the last: a state is read once and
// written once however many tokens a call brings.  Both products are taken from the decayed state before
// the update, o = scale (S^T q + (k.q) u): one reduction per token instead of two that wait for each other.
// Bound by HBM where requests are many: 64 of them, one token, 32 heads of 128 x 128, 268 MB: 58 us, 4.6 TB/s (43 where
// the caches hold part of it); by the latency of a launch and one trip to memory for one request (5.4 us; 4.8 replayed from a graph).
#include "csb_delta.hpp"

namespace csb {

// Sum over the 8 lanes with the same lane % 8, in every one of them (a fixed order).
__device__ __forceinline__ float column_sum(float v) {
    v += row_rotated<8>(v);
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Lane (x = lane % 8, y = lane / 8) holds the 4 columns from 4 x on of the rows y JN .. y JN + JN - 1: eight lanes read 128
// consecutive bytes of a row.  (16 lanes on 16 rows, 64 bytes of each, were 122 us instead of 43 on 64 requests, 32 heads of 128 x 128.)
// VEC: operands that are aligned to 4 elements, widths that are multiples of 4.  Else the same words at any element, and element by element where a
// row ends inside one (32 requests, 96 tokens, 16 heads of 121 x 121: 23 us a call instead of 35; of 124 x 124 17).
template <int VF, int JN, bool VEC>
__global__ __launch_bounds__(256) void delta_recurrent_kernel(const DeltaDev a, const uint32_t tiles, const uint32_t waves) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    using f32x4 = float __attribute__((ext_vector_type(4)));
    using T4_any = T __attribute__((ext_vector_type(4), aligned(sizeof(T)), may_alias));
    using f32x4_any = float __attribute__((ext_vector_type(4), aligned(4), may_alias));
    const uint32_t lane = threadIdx.x & 63u, x = lane & 7u, y = lane >> 3;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * (blockDim.x >> 6) + (threadIdx.x >> 6));
    if (wave >= waves) return;                                 // (no barrier in this kernel)
    const uint32_t rest = wave / tiles, h = rest % a.hv, seq = rest / a.hv;
    const uint32_t col = (wave % tiles) * 32 + 4 * x, row = y * JN, DK = a.dk, DV = a.dv;
    int64_t first, end, slot;
    delta_sequence(a, (int)seq, &first, &end, &slot);
    const size_t state = ((size_t)(slot < 0 ? 0 : slot) * a.hv + h) * DK * DV;
    struct Token { T4 k[JN / 4], q[JN / 4], v; float g, beta; };
    const uint32_t kh = h / a.group;
    auto load4 = [&](const T *p, uint32_t at, uint32_t most) {                // p[0 .. 3] as far as at + j < most
        T4 v{};
        if constexpr (VEC) {
            if (at < most) v = *(const T4 *)p;
        } else if (at + 4 <= most) v = *(const T4_any *)p;
        else {
#pragma unroll
            for (int j = 0; j < 4; ++j) if (at + j < most) v[j] = p[j];
        }
        return v;
    };
    auto load = [&](int64_t t, Token &w) {
        const T *kp = (const T *)a.k + t * a.ldk + (size_t)kh * DK + row, *qp = (const T *)a.q + t * a.ldq + (size_t)kh * DK + row;
#pragma unroll
        for (int j = 0; j < JN / 4; ++j) {
            w.k[j] = load4(kp + 4 * j, row + 4 * j, DK);
            w.q[j] = load4(qp + 4 * j, row + 4 * j, DK);
        }
        w.v = load4((const T *)a.v + t * a.ldv + (size_t)h * DV + col, col, DV);
        w.g = a.g[t * a.ldg + h];
        w.beta = a.beta[t * a.ldb + h];
    };
    Token now{}, next{};
    if (first < end) load(first, now);
    f32x4 S[JN];
#pragma unroll
    for (int j = 0; j < JN; ++j) S[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (a.s_in && slot >= 0) {                                 // uniform
        const float *p = a.s_in + state + (size_t)row * DV + col;
        if (VEC ? col < DV : col + 4 <= DV) {
#pragma unroll
            for (int j = 0; j < JN; ++j)
                if (row + j < DK) {
                    if constexpr (VEC) S[j] = *(const f32x4 *)(p + (size_t)j * DV);
                    else S[j] = *(const f32x4_any *)(p + (size_t)j * DV);
                }
        } else if constexpr (!VEC) {
#pragma unroll
            for (int j = 0; j < JN; ++j)
                if (row + j < DK)
#pragma unroll
                    for (int c = 0; c < 3; ++c) if (col + c < DV) S[j][c] = p[(size_t)j * DV + c];
        }
    }
    for (int64_t t = first; t < end; ++t) {
        if (t + 1 < end) load(t + 1, next);
        const float decay = __builtin_amdgcn_exp2f((float)((double)now.g * 1.4426950408889634));   // (the argument rounded once)
        f32x4 pk{0.0f, 0.0f, 0.0f, 0.0f}, pq = pk;
        float kq = 0.0f;
#pragma unroll
        for (int j = 0; j < JN; ++j) {
            const float k = (float)now.k[j / 4][j % 4], q = (float)now.q[j / 4][j % 4];
            S[j] *= decay;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                pk[c] = fmaf(S[j][c], k, pk[c]);
                pq[c] = fmaf(S[j][c], q, pq[c]);
            }
            kq = fmaf(k, q, kq);
        }
        kq = column_sum(kq);
        f32x4 u, o;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            u[c] = now.beta * ((float)now.v[c] - column_sum(pk[c]));
            o[c] = a.scale * fmaf(kq, u[c], column_sum(pq[c]));
        }
#pragma unroll
        for (int j = 0; j < JN; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) S[j][c] = fmaf((float)now.k[j / 4][j % 4], u[c], S[j][c]);
        if (y == 0) {
            T *op = (T *)a.out + t * a.ldo + (size_t)h * DV + col;
            if constexpr (VEC) {
                T4 oo;
#pragma unroll
                for (int c = 0; c < 4; ++c) oo[c] = (T)o[c];
                if (col < DV) *(T4 *)op = oo;
            } else {
#pragma unroll
                for (int c = 0; c < 4; ++c) if (col + c < DV) op[c] = (T)o[c];
            }
        }
        now = next;
    }
    if (!a.s_out || slot < 0) return;
    float *p = a.s_out + state + (size_t)row * DV + col;
    if (VEC ? col < DV : col + 4 <= DV) {
#pragma unroll
        for (int j = 0; j < JN; ++j)
            if (row + j < DK) {
                if constexpr (VEC) *(f32x4 *)(p + (size_t)j * DV) = S[j];
                else *(f32x4_any *)(p + (size_t)j * DV) = S[j];
            }
    } else if constexpr (!VEC) {
#pragma unroll
        for (int j = 0; j < JN; ++j)
            if (row + j < DK)
#pragma unroll
                for (int c = 0; c < 3; ++c) if (col + c < DV) p[(size_t)j * DV + c] = S[j][c];
    }
}

Refusal delta_sizes(const csb_delta_args *a) {
    if (!a) return {CSB_EINVAL, "NULL arguments"};
    if (!known_type(a->type)) return {CSB_EINVAL, "unknown type"};
    if (a->n_seq < 0 || a->n_tokens < 0 || a->heads_k < 1 || a->heads_v < 1 || a->dk < 1 || a->dv < 1) return {CSB_EINVAL, "bad size"};
    if (a->heads_v % a->heads_k) return {CSB_EINVAL, "heads_v is no multiple of heads_k"};
    if (a->dk > 256) return {CSB_EUNSUPPORTED, "dk above 256 (a state's rows are held in the registers of 8 lanes)"};
    if (a->n_tokens > 0x7fffffff) return {CSB_EUNSUPPORTED, "offsets are 32-bit: more than 2^31 - 1 tokens"};
    return {CSB_OK, nullptr};
}

int check_delta(const char *who, const csb_delta_args *a) {
    const auto fail = [&](int code, const char *what) { set_error(std::string(who) + ": " + what); return code; };
    const Refusal sizes = delta_sizes(a);
    if (sizes.code != CSB_OK) return fail(sizes.code, sizes.what);
    if (a->n_tokens && (!a->d_q || !a->d_k || !a->d_v || !a->d_g || !a->d_beta || !a->d_out)) return fail(CSB_EINVAL, "NULL pointer");
    const int64_t wk = (int64_t)a->heads_k * a->dk, wv = (int64_t)a->heads_v * a->dv;
    if (a->ldq < wk || a->ldk < wk || a->ldv < wv || a->ldo < wv || a->ldg < a->heads_v || a->ldbeta < a->heads_v)
        return fail(CSB_EINVAL, "a leading dimension below the width of its rows");
    if (!a->d_start && a->n_seq && a->n_tokens % a->n_seq) return fail(CSB_EINVAL, "n_tokens is no multiple of n_seq (and there are no offsets)");
    if ((a->d_state_in || a->d_state_out) && a->n_states < 1) return fail(CSB_EINVAL, "states without room for one");
    if (((uintptr_t)a->d_state_in | (uintptr_t)a->d_state_out | (uintptr_t)a->d_g | (uintptr_t)a->d_beta) % 4) return fail(CSB_EINVAL, "misaligned pointer");
    if (((uintptr_t)a->d_q | (uintptr_t)a->d_k | (uintptr_t)a->d_v | (uintptr_t)a->d_out) % type_size(a->type)) return fail(CSB_EINVAL, "misaligned pointer");
    return CSB_OK;
}

DeltaDev delta_dev(const csb_delta_args *a) {
    DeltaDev d{};
    d.q = a->d_q; d.k = a->d_k; d.v = a->d_v; d.g = a->d_g; d.beta = a->d_beta;
    d.start = a->d_start; d.len = a->d_len; d.slot = a->d_slot;
    d.s_in = a->d_state_in; d.s_out = a->d_state_out; d.out = a->d_out;
    d.ldq = a->ldq; d.ldk = a->ldk; d.ldv = a->ldv; d.ldg = a->ldg; d.ldb = a->ldbeta; d.ldo = a->ldo;
    d.n_tokens = a->n_tokens;
    d.each = a->n_seq ? a->n_tokens / a->n_seq : 0;
    d.hk = a->heads_k; d.hv = a->heads_v; d.group = a->heads_v / a->heads_k;
    d.dk = a->dk; d.dv = a->dv; d.n_seq = a->n_seq; d.n_states = a->n_states;
    d.scale = a->scale;
    return d;
}

template <int VF, int JN>
static void launch_recurrent(const DeltaDev &d, bool vec, uint32_t tiles, uint32_t waves, hipStream_t st) {
    const uint32_t threads = waves < 1024 ? 64 : 256;          // (few wavefronts: a CU each)
    const dim3 grid((waves * 64 + threads - 1) / threads);
    if (vec) hipLaunchKernelGGL((delta_recurrent_kernel<VF, JN, true>), grid, dim3(threads), 0, st, d, tiles, waves);
    else hipLaunchKernelGGL((delta_recurrent_kernel<VF, JN, false>), grid, dim3(threads), 0, st, d, tiles, waves);
}

template <int VF>
static void launch_recurrent(const DeltaDev &d, bool vec, uint32_t tiles, uint32_t waves, hipStream_t st) {
    if (d.dk <= 64) launch_recurrent<VF, 8>(d, vec, tiles, waves, st);
    else if (d.dk <= 128) launch_recurrent<VF, 16>(d, vec, tiles, waves, st);
    else launch_recurrent<VF, 32>(d, vec, tiles, waves, st);
}

int launch_delta_recurrent(const csb_delta_args *a, hipStream_t st) {
    const int64_t tiles = ((int64_t)a->dv + 31) / 32;          // 32 columns of a state each: a wavefront's
    if (tiles * a->heads_v > kMaxWorkgroups || tiles * a->heads_v * a->n_seq > kMaxWorkgroups) {
        set_error("csb_delta: more wavefronts than a launch takes");
        return CSB_EUNSUPPORTED;
    }
    const DeltaDev d = delta_dev(a);
    const uintptr_t four = 4 * (uintptr_t)type_size(a->type);
    const bool vec = a->dk % 4 == 0 && a->dv % 4 == 0 && a->ldq % 4 == 0 && a->ldk % 4 == 0 && a->ldv % 4 == 0 && a->ldo % 4 == 0 &&
                     ((uintptr_t)a->d_q | (uintptr_t)a->d_k | (uintptr_t)a->d_v | (uintptr_t)a->d_out) % four == 0 &&
                     ((uintptr_t)a->d_state_in | (uintptr_t)a->d_state_out) % 16 == 0;
    const uint32_t waves = (uint32_t)(tiles * a->heads_v * a->n_seq);
    switch (a->type) {
        case CSB_VAL_F32: launch_recurrent<CSB_VAL_F32>(d, vec, (uint32_t)tiles, waves, st); break;
        case CSB_VAL_F16: launch_recurrent<CSB_VAL_F16>(d, vec, (uint32_t)tiles, waves, st); break;
        default: launch_recurrent<CSB_VAL_BF16>(d, vec, (uint32_t)tiles, waves, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error(std::string("csb_delta: ") + hipGetErrorString(e)); return CSB_EDEVICE; }
    return CSB_OK;
}

}  // namespace csb

extern "C" int csb_delta_recurrent(const csb_delta_args *args, void *stream) {
    const int rc = csb::check_delta("csb_delta_recurrent", args);
    if (rc != CSB_OK || args->n_seq == 0) return rc;
    return csb::launch_delta_recurrent(args, (hipStream_t)stream);
}
