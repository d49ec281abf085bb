// The gated delta rule chunk by chunk (csb_delta_chunked).
//
// With G_i the sum of g over a chunk's tokens up to i, and S the state before the chunk, the chunk's
// u_i obey  u_i = beta_i (v_i - e^G_i S^T k_i - sum_{j<i} e^(G_i - G_j) (k_i.k_j) u_j),  so with
// T_ij = beta_i e^(G_i - G_j) k_i.k_j below the diagonal and M = (1 + T)^-1 diag(beta)
//     R = V - diag(e^G) K S,   U = M R,
//     O = scale (diag(e^G) Q S + P U),   P_ij = e^(G_i - G_j) q_i.k_j on and below the diagonal,
//     S <- e^G_64 S + K^T diag(e^(G_64 - G_j)) U:
// matrix products for the matrix cores instead of 64 dependent steps.  Two launches.  The first makes M and P
// of every chunk at once; the second takes the chunks of a sequence one after the other, S in registers.
//
// Precision: state, M, R and U have 24 bits.  A binary32 number is the exact sum of three bfloat16
// numbers (8 bits each), so a product of the matrix cores' 16-bit form takes as many passes as its
// operands have parts (bfloat16 inputs one, binary16 two, binary32 three), without the ones below 2^-24; that
// is 16 / 6 to 16 / 3 of the rate of their binary32 form.  What only the output sees has two parts where the output has 16 bits.
//
// Not finite: an entry of a later token must not reach an earlier one through a zero of M or P.  R and
// U are looked at once per chunk; from its first token that is not finite on a column of them is taken out of
// the products and everything it would have reached is set to NaN.
#include <algorithm>
#include <new>

#include "csb_delta.hpp"
#include "csb_kernels.hpp"

namespace csb {

constexpr int kChunk = 64, kChunkShift = 6;
constexpr uint32_t kFrag = 1024;               // bytes of a 16 x 32 operand of 16-bit numbers: 16 per lane
constexpr uint32_t kLower = 6;                 // operands that cover the lower triangle of 64 x 64 (see lower_frag)

using f32x4 = float __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

// Parts that a number has in a product, and a chunk's block of the workspace: M's operands, P's, then
// e^G_i and e^(G_64 - G_i).  binary32 operands lie there whole (they are split when read: parts would not fit the LDS).
template <int VF> struct Parts {
    static constexpr int in = VF == CSB_VAL_BF16 ? 1 : VF == CSB_VAL_F16 ? 2 : 3;      // of q and k
    static constexpr int out = VF == CSB_VAL_F32 ? 3 : 2;                              // of what only the output sees
    static constexpr bool whole = VF == CSB_VAL_F32;
    static constexpr uint32_t m_bytes = kLower * (whole ? 2 : 3) * kFrag, p_bytes = kLower * 2 * kFrag;
    static constexpr uint32_t bytes = m_bytes + p_bytes + 512;
};

// Operand numbers.  Rows come in pairs of tiles: tile (p, t) has the rows 32 p + 2 m + t (m = 0 .. 15), so that the
// results of a pair leave a lane with eight consecutive rows -- which is how the next product wants them as its other operand.
__device__ __forceinline__ constexpr uint32_t lower_frag(int p, int t, int ks) { return p == 0 ? t : 2 + 2 * t + ks; }

__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }   // a's in the low half
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// x as N bfloat16 numbers, each the nearest to what is left: exact for N = 3 (8 bits and a sign each), to 2^-18 for N = 2.
template <int N>
__device__ __forceinline__ void split8(const float *x, u32x4 *part) {
    using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 near = {(__bf16)rest[2 * i], (__bf16)rest[2 * i + 1]};
            const uint32_t two = __builtin_bit_cast(uint32_t, near);
            part[n][i] = two;
            if (n + 1 < N) {
                rest[2 * i] -= __uint_as_float(two << 16);
                rest[2 * i + 1] -= __uint_as_float(two & 0xffff0000u);
            }
        }
}

// d += a b, over the parts whose product is not below 2^(-8 MOST); the small ones first.
template <int NA, int NB, int MOST>
__device__ __forceinline__ f32x4 mma(const u32x4 *a, const u32x4 *b, f32x4 d) {
#pragma unroll
    for (int s = NA + NB - 2; s >= 0; --s) {
        if (s > MOST) continue;
#pragma unroll
        for (int i = 0; i < NA; ++i) {
            const int j = s - i;
            if (j < 0 || j >= NB) continue;
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[j]), d, 0, 0, 0);
        }
    }
    return d;
}

// ---- first launch: M and P -----------------------------------------------------------------------
// A wavefront takes one chunk of one value head.

// Eight numbers of a row of q or k from element d on, as they are stored (zeros past dk).
template <int VF, bool VEC> struct Row8 {
    using T = typename Elem<VF>::T;
    static constexpr int words = VF == CSB_VAL_F32 ? 2 : 1;
    u32x4 w[words];
    __device__ __forceinline__ void load(const T *row, int d, int dk) {
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < words; ++i) {
                w[i] = u32x4{0, 0, 0, 0};
                if (d + 8 / words * i < dk) w[i] = *(const u32x4 *)(row + d + 8 / words * i);
            }
        } else {
            T e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = d + i < dk ? row[d + i] : (T)0.0f;
            __builtin_memcpy(w, e, sizeof(e));
        }
    }
};

// d += a b^T over 32 elements of the rows, exact products, sums in binary32.
template <int VF, bool VEC>
__device__ __forceinline__ f32x4 row_dot(const Row8<VF, VEC> &a, const Row8<VF, VEC> &b, f32x4 d) {
    if constexpr (VF == CSB_VAL_BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.w[0]), __builtin_bit_cast(bf16x8, b.w[0]), d, 0, 0, 0);
    else if constexpr (VF == CSB_VAL_F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a.w[0]), __builtin_bit_cast(f16x8, b.w[0]), d, 0, 0, 0);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) d = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w[i / 4][i % 4]), __uint_as_float(b.w[i / 4][i % 4]), d, 0, 0, 0);
        return d;
    }
}

// Orders a wavefront's LDS accesses: what its other lanes wrote before is there behind it.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

constexpr int kLdT = 68;                       // words of a row of a 64 x 64 matrix in LDS: rows stay 16-byte aligned

// The lower triangle in LDS as operands in the workspace: 3 or 2 parts, or whole.
template <int NP, bool WHOLE>
__device__ __forceinline__ void store_lower(const float (*m)[kLdT], uint8_t *to, uint32_t lane) {
    const uint32_t g = lane >> 4, i = lane & 15u;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int ks = 0; ks <= p; ++ks) {
                const float *row = &m[32 * p + 2 * i + t][32 * ks + 8 * g];
                float x[8];
                *(f32x4 *)x = *(const f32x4 *)row;
                *(f32x4 *)(x + 4) = *(const f32x4 *)(row + 4);
                u32x4 part[3];
                if constexpr (WHOLE) {
                    part[0] = *(u32x4 *)x;
                    part[1] = *(u32x4 *)(x + 4);
                } else split8<NP>(x, part);
                constexpr int n = WHOLE ? 2 : NP;
#pragma unroll
                for (int k = 0; k < n; ++k) *(u32x4 *)(to + (lower_frag(p, t, ks) * n + k) * kFrag + lane * 16) = part[k];
            }
}

template <int VF, bool VEC>
__global__ __launch_bounds__(256) void delta_prepare_kernel(const DeltaDev a, uint8_t *ws, const uint32_t head_groups) {
    using T = typename Elem<VF>::T;
    __shared__ __align__(16) float mat[4][kChunk][kLdT];
    __shared__ double sums[4][kChunk];
    __shared__ float betas[4][kChunk];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15u;
    const int64_t number = blockIdx.x / head_groups;
    const int seq = tile_sequence(a.start, a.n_seq, a.n_tokens, kChunkShift, number, a.each);
    if (seq < 0) return;                                       // uniform
    int64_t first, end, slot;
    delta_sequence(a, seq, &first, &end, &slot);
    const int64_t base = first + (number - (first >> kChunkShift) - seq) * kChunk;
    if (base < first || base >= end) return;                   // (before it: offsets that do not ascend)
    const int h = (int)(blockIdx.x % head_groups) * 4 + (int)wave;
    if (h >= a.hv) return;                                     // (no barrier below: a wavefront keeps to its own LDS)
    uint8_t *block = ws + ((size_t)number * a.hv + h) * Parts<VF>::bytes;
    const int kh = h / a.group, n = (int)min((int64_t)kChunk, end - base);

    // sums of g in 64 bits: differences of large sums count (a token that forgets, then tokens that hardly do)
    double G = 0.0;
    float beta = 0.0f;
    if ((int)lane < n) {
        const float gv = a.g[(base + lane) * a.ldg + h];
        G = gv < -1e4f ? -1e4 : (double)gv;                    // e^-10000 is zero; sums stay finite
        beta = a.beta[(base + lane) * a.ldb + h];
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(G, d);
        if ((int)lane >= d) G += o;
    }
    const double all = __shfl(G, 63);
    constexpr double log2e = 1.4426950408889634;
    float *decay = (float *)(block + Parts<VF>::m_bytes + Parts<VF>::p_bytes);
    decay[lane] = __builtin_amdgcn_exp2f((float)(G * log2e));
    decay[64 + lane] = __builtin_amdgcn_exp2f((float)((all - G) * log2e));
    sums[wave][lane] = G;
    betas[wave][lane] = beta;

    f32x4 kk[4][4], qk[4][4];                                  // tiles on and below the diagonal
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y <= x; ++y) kk[x][y] = qk[x][y] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int d = 0; d < a.dk; d += 32) {
        Row8<VF, VEC> kr[4], qr[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int64_t t = min(base + 16 * x + (int64_t)i, end - 1);    // (past the end beta is zero)
            kr[x].load((const T *)a.k + t * a.ldk + (size_t)kh * a.dk, d + 8 * (int)g, a.dk);
            qr[x].load((const T *)a.q + t * a.ldq + (size_t)kh * a.dk, d + 8 * (int)g, a.dk);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y <= x; ++y) {
                kk[x][y] = row_dot(kr[x], kr[y], kk[x][y]);
                qk[x][y] = row_dot(qr[x], kr[y], qk[x][y]);
            }
    }
    wave_sync();
    float (*m)[kLdT] = mat[wave];
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y <= x; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * x + 4 * (int)g + r, col = 16 * y + (int)i;
                const float e = __builtin_amdgcn_exp2f((float)((sums[wave][row] - sums[wave][col]) * log2e));
                m[row][col] = row > col ? betas[wave][row] * e * kk[x][y][r] : 0.0f;
                qk[x][y][r] = row >= col ? e * qk[x][y][r] : 0.0f;
            }
    wave_sync();
    // (1 + T)^-1 by forward substitution, a column per lane, its entries in registers
    float inv[kChunk];
#pragma unroll
    for (int r = 0; r < kChunk; ++r) {
        float s0 = r == (int)lane ? 1.0f : 0.0f, s1 = 0.0f;
#pragma unroll
        for (int j = 0; j < r; j += 4) {
            const f32x4 t = *(const f32x4 *)&m[r][j];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (j + c < r) {
                    if (c & 1) s1 = fmaf(-t[c], inv[j + c], s1);
                    else s0 = fmaf(-t[c], inv[j + c], s0);
                }
        }
        inv[r] = r >= (int)lane ? s0 + s1 : 0.0f;              // (zero also where a row of T is not finite)
    }
    wave_sync();
#pragma unroll
    for (int r = 0; r < kChunk; ++r) m[r][lane] = r >= (int)lane ? inv[r] * beta : 0.0f;
    wave_sync();
    store_lower<3, Parts<VF>::whole>(m, block, lane);
    wave_sync();
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y <= (x | 1); ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) m[16 * x + 4 * g + r][16 * y + i] = y <= x ? qk[x][y <= x ? y : 0][r] : 0.0f;
    wave_sync();
    store_lower<2, Parts<VF>::whole>(m, block + Parts<VF>::m_bytes, lane);
}

// ---- second launch: the chunks of a sequence one after the other ---------------------------------

typedef const __attribute__((address_space(1))) void glb_void_t;
typedef __attribute__((address_space(3))) void lds_void_t;
__device__ __forceinline__ void to_lds16(const void *g, uint32_t at) {         // lane l's 16 bytes land at `at` + 16 l
    __builtin_amdgcn_global_load_lds((glb_void_t *)g, (lds_void_t *)(uintptr_t)at, 16, 0, 0);
}
__device__ __forceinline__ u32x4 lds16(uint32_t at) { return *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)at; }
__device__ __forceinline__ uint32_t lds4(uint32_t at) { return *(const __attribute__((address_space(3))) uint32_t *)(uintptr_t)at; }
__device__ __forceinline__ f32x4 lds_f4(uint32_t at) { return __builtin_bit_cast(f32x4, lds16(at)); }

// LDS of a chunk: K's operands, Q's (kDP * 4 each), then the chunk's block of the workspace.
template <int VF, int DP> struct ChunkLds {
    static constexpr uint32_t half = VF == CSB_VAL_F32 ? 2 : 1;               // 16-byte words of a lane's eight numbers
    static constexpr uint32_t frag = half * kFrag, q = 4 * DP * frag, m = 2 * q;
    static constexpr uint32_t bytes = m + (Parts<VF>::bytes + kFrag - 1) / kFrag * kFrag;
};

// An operand of K or Q lies in LDS with lane (g, m)'s numbers -- row 2 m + t of its 32 tokens, elements 8 g to 8 g + 7 of its 32 --
// at place 16 g + (m + g) % 16: the transposed reads below, 4 bytes from 16 places with m % 4 alike, then hit 16 different banks' words.
__device__ __forceinline__ uint32_t place(uint32_t g, uint32_t m) { return (g * 16 + ((m + g) & 15u)) * 16; }

// The parts of an operand of K or Q (rows of tokens).
template <int VF>
__device__ __forceinline__ void row_parts(uint32_t at, u32x4 *part) {
    if constexpr (VF == CSB_VAL_BF16) part[0] = lds16(at);
    else {
        float x[8];
        if constexpr (VF == CSB_VAL_F16) {
            const f16x8 v = __builtin_bit_cast(f16x8, lds16(at));
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
        } else {
            *(u32x4 *)x = lds16(at);
            *(u32x4 *)(x + 4) = lds16(at + kFrag);
        }
        split8<Parts<VF>::in>(x, part);
    }
}

// The parts of K^T for elements 32 dp + 2 m + t (t = 0, 1: part[t]) of the tokens 32 ks + 8 g .. + 7.
template <int VF, int DP>
__device__ __forceinline__ void column_parts(uint32_t k_at, int dp, int ks, uint32_t g, uint32_t m, u32x4 part[2][3]) {
    using L = ChunkLds<VF, DP>;
    if constexpr (VF == CSB_VAL_F32) {
        float x[2][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t at = k_at + ((2 * ks + (j & 1)) * DP + dp) * L::frag + place(m >> 2, 4 * g + (j >> 1)) + ((m >> 1) & 1u) * kFrag + (m & 1u) * 8;
            x[0][j] = __uint_as_float(lds4(at));
            x[1][j] = __uint_as_float(lds4(at + 4));
        }
        split8<3>(x[0], part[0]);
        split8<3>(x[1], part[1]);
    } else {
        u32x4 both[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t at = k_at + (2 * ks * DP + dp) * L::frag + place(m >> 2, 4 * g + j) + (m & 3u) * 4;
            const uint32_t even = lds4(at), odd = lds4(at + DP * L::frag);     // tokens 2 j and 2 j + 1
            both[0][j] = low_halves(even, odd);
            both[1][j] = high_halves(even, odd);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            if constexpr (VF == CSB_VAL_BF16) part[t][0] = both[t];
            else {
                const f16x8 v = __builtin_bit_cast(f16x8, both[t]);
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
                split8<2>(x, part[t]);
            }
        }
    }
}

// The parts of an operand of M (N = 3) or P.
template <int VF, int N>
__device__ __forceinline__ void lower_parts(uint32_t at, uint32_t f, uint32_t lane, u32x4 *part) {
    if constexpr (Parts<VF>::whole) {
        float x[8];
        *(u32x4 *)x = lds16(at + 2 * f * kFrag + lane * 16);
        *(u32x4 *)(x + 4) = lds16(at + (2 * f + 1) * kFrag + lane * 16);
        split8<3>(x, part);
    } else {
#pragma unroll
        for (int n = 0; n < N; ++n) part[n] = lds16(at + (f * N + n) * kFrag + lane * 16);
    }
}

__device__ __forceinline__ bool any_not_finite(const float (*x)[8]) {
    float z = 0.0f;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) z = fmaf(x[p][e], 0.0f, z);
    return __ballot(z != 0.0f) != 0;                           // (NaN is not 0 either)
}

// The first token with a number in x that is not finite, over the lanes of a column (at most `before`); x is zero from it on.
__device__ __forceinline__ int take_out(float (*x)[8], int before, uint32_t g) {
    int bad = before;
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (!(fabsf(x[p][e]) < __builtin_inff())) bad = min(bad, 32 * p + 8 * (int)g + e);
    bad = min(bad, __shfl_xor(bad, 16));
    bad = min(bad, __shfl_xor(bad, 32));
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (32 * p + 8 * (int)g + e >= bad) x[p][e] = 0.0f;
    return bad;
}

// A wavefront takes 16 columns of the state of one sequence and value head, NW of them share the chunk's operands in LDS.
// Lane (g = lane / 16, m = lane % 16) has column m; of every 32 rows of a matrix with 16 columns (S, R, U) it has 8 g .. 8 g + 7.
// DP: 32s of dk.  VEC: rows of q and k in aligned 16-byte words.
template <int VF, int DP, int NW, bool VEC>
__global__ __launch_bounds__(64 * NW, 1) void delta_scan_kernel(const DeltaDev a, const uint8_t *ws, const uint32_t tiles) {
    using T = typename Elem<VF>::T;
    using L = ChunkLds<VF, DP>;
    using P = Parts<VF>;
    constexpr bool ahead = VEC && 2 * L::bytes <= 160 * 1024;                  // the next chunk is fetched during this one
    constexpr int S2 = P::out;
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, m = lane & 15u;
    // workgroups of one sequence and head run on one XCD (they are dealt out by their number modulo 8): its L2 has their operands once
    const uint32_t pair = blockIdx.x / (8 * tiles) * 8 + blockIdx.x % 8, tile = blockIdx.x / 8 % tiles;
    if (pair >= (uint32_t)a.n_seq * a.hv) return;
    const uint32_t h = pair % a.hv, seq = pair / a.hv, kh = h / a.group;
    const int DK = a.dk, DV = a.dv, col = (int)((tile * NW + wave) * 16 + m);
    const bool mine = col < DV;
    int64_t first, end, slot;
    delta_sequence(a, (int)seq, &first, &end, &slot);
    const size_t state = (((size_t)(slot < 0 ? 0 : slot) * a.hv + h) * DK) * DV;
    f32x4 S[DP][2];                                            // [dp][t][r]: row 32 dp + 8 g + 2 r + t
#pragma unroll
    for (int dp = 0; dp < DP; ++dp)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 32 * dp + 8 * (int)g + 2 * r + t;
                S[dp][t][r] = a.s_in && slot >= 0 && mine && d < DK ? a.s_in[state + (size_t)d * DV + col] : 0.0f;
            }
    const int chunks = (int)((end - first + kChunk - 1) >> kChunkShift);
    const int64_t number0 = (first >> kChunkShift) + seq;

    // Offsets within a chunk fit 32 bits (leading dimensions below 2^24): an address is a chunk's base and a lane's offset.
    const uint32_t ldk = (uint32_t)(a.ldk * sizeof(T)), ldq = (uint32_t)(a.ldq * sizeof(T)), ldv = (uint32_t)(a.ldv * sizeof(T)), ldo = (uint32_t)(a.ldo * sizeof(T));
    // a chunk's operands into LDS; VEC: requested only (the wavefront's count of outstanding operations covers them)
    auto stage = [&](int c, uint32_t at) {
        const int64_t base = first + ((int64_t)c << kChunkShift);
        const uint8_t *block = ws + ((size_t)(number0 + c) * a.hv + h) * P::bytes;
        const uint8_t *kb = (const uint8_t *)((const T *)a.k + base * a.ldk + (size_t)kh * DK);
        const uint8_t *qb = (const uint8_t *)((const T *)a.q + base * a.ldq + (size_t)kh * DK);
        const uint32_t last = (uint32_t)min((int64_t)kChunk, end - base) - 1;  // (past the end M and P have zeros)
        constexpr uint32_t extra = (P::bytes + kFrag - 1) / kFrag;
#pragma unroll 1
        for (uint32_t k = 0; k < 4 / NW; ++k) {
            const uint32_t pt = wave + k * NW;                 // tile (p, t) = (pt / 2, pt % 2)
            const uint32_t row = min(32 * (pt >> 1) + 2 * ((m - g) & 15u) + (pt & 1u), last);
#pragma unroll
            for (uint32_t dp = 0; dp < DP; ++dp) {
                const uint32_t to = at + (pt * DP + dp) * L::frag;
                const int d = (int)(32 * dp + 8 * g);
                if constexpr (VEC) {                           // past dk the first elements again (the state's rows there are zeros)
#pragma unroll
                    for (uint32_t i = 0; i < L::half; ++i) {
                        const uint32_t e = (uint32_t)(d + (int)i * 4 < DK ? d + (int)i * 4 : 0) * (uint32_t)sizeof(T);
                        to_lds16(kb + (row * ldk + e), to + i * kFrag);
                        to_lds16(qb + (row * ldq + e), to + L::q + i * kFrag);
                    }
                } else {
                    Row8<VF, false> kv, qv;
                    kv.load((const T *)(kb + row * ldk), d, DK);
                    qv.load((const T *)(qb + row * ldq), d, DK);
#pragma unroll
                    for (uint32_t i = 0; i < L::half; ++i) {
                        *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)(to + i * kFrag + lane * 16) = kv.w[i];
                        *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)(to + L::q + i * kFrag + lane * 16) = qv.w[i];
                    }
                }
            }
        }
#pragma unroll 4
        for (uint32_t k = 0; k < (extra + NW - 1) / NW; ++k) {
            const uint32_t u = wave + k * NW;
            if (u * kFrag + lane * 16 < P::bytes) to_lds16(block + u * kFrag + lane * 16, at + L::m + u * kFrag);
        }
    };
    T v_next[2][8];                                            // of the next chunk (past the end the last token's)
    const uint32_t v_col = ((uint32_t)h * DV + min(col, DV - 1)) * (uint32_t)sizeof(T), o_col = ((uint32_t)h * DV + col) * (uint32_t)sizeof(T);
    auto load_v = [&](int c) {
        const int64_t base = first + ((int64_t)c << kChunkShift);
        const uint8_t *vb = (const uint8_t *)((const T *)a.v + base * a.ldv);
        const uint32_t last = (uint32_t)min((int64_t)kChunk, end - base) - 1;
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) v_next[p][e] = *(const T *)(vb + (min(32 * p + 8 * g + e, last) * ldv + v_col));
    };
    u32x4 Sp[DP][3];
    auto split_state = [&]() {
#pragma unroll
        for (int dp = 0; dp < DP; ++dp) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = S[dp][e & 1][e >> 1];
            split8<3>(x, Sp[dp]);
        }
    };
    split_state();
    if (chunks > 0) {
        load_v(0);
        if (ahead) stage(0, lds0);
    }
    for (int c = 0; c < chunks; ++c) {
        const uint32_t at = ahead ? lds0 + (c & 1) * L::bytes : lds0;
        if (!ahead) {
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");    // the chunk before is done with
            stage(c, at);
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        float v[2][8];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[p][e] = (float)v_next[p][e];
        const int64_t base = first + ((int64_t)c << kChunkShift);
        const int count = (int)min((int64_t)kChunk, end - base);
        if (c + 1 < chunks) {
            load_v(c + 1);
            if (ahead) stage(c + 1, lds0 + ((c + 1) & 1) * L::bytes);
        }
        const uint32_t decay = at + L::m + P::m_bytes + P::p_bytes;

        f32x4 ks[2][2], o[2][2];
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int t = 0; t < 2; ++t) ks[p][t] = o[p][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int dp = 0; dp < DP; ++dp)
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    u32x4 part[3];
                    const uint32_t f = at + ((2 * p + t) * DP + dp) * L::frag + place(g, m);
                    row_parts<VF>(f, part);
                    ks[p][t] = mma<P::in, 3, 2>(part, Sp[dp], ks[p][t]);
                    row_parts<VF>(f + L::q, part);
                    o[p][t] = mma<P::in, S2, S2 - 1>(part, Sp[dp], o[p][t]);
                }
        float R[2][8];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            float eg[8];
            *(f32x4 *)eg = lds_f4(decay + (32 * p + 8 * g) * 4);
            *(f32x4 *)(eg + 4) = lds_f4(decay + (32 * p + 8 * g) * 4 + 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                R[p][e] = v[p][e] - eg[e] * ks[p][e & 1][e >> 1];
                o[p][e & 1][e >> 1] *= eg[e];
            }
        }
        int bad = kChunk;
        if (any_not_finite(R)) bad = take_out(R, bad, g);      // uniform
        u32x4 Rp[2][3];
        split8<3>(R[0], Rp[0]);
        split8<3>(R[1], Rp[1]);
        float U[2][8];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                f32x4 u{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int s = 0; s <= p; ++s) {
                    u32x4 part[3];
                    lower_parts<VF, 3>(at + L::m, lower_frag(p, t, s), lane, part);
                    u = mma<3, 3, 2>(part, Rp[s], u);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) U[p][2 * r + t] = u[r];
            }
        }
        if (any_not_finite(U) || bad < kChunk) bad = take_out(U, bad, g);
        {
            u32x4 Up[2][3];
            split8<S2>(U[0], Up[0]);
            split8<S2>(U[1], Up[1]);
            uint8_t *ob = (uint8_t *)((T *)a.out + base * a.ldo);
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int t = 0; t < 2; ++t) {
#pragma unroll
                    for (int s = 0; s <= p; ++s) {
                        u32x4 part[3];
                        lower_parts<VF, 2>(at + L::m + P::m_bytes, lower_frag(p, t, s), lane, part);
                        o[p][t] = mma<S2, S2, S2 - 1>(part, Up[s], o[p][t]);
                    }
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int row = 32 * p + 8 * (int)g + 2 * r + t;
                        o[p][t][r] = row >= bad ? __builtin_nanf("") : a.scale * o[p][t][r];
                    }
                }
            if (mine) {
                if (count == kChunk) {
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int e = 0; e < 8; ++e) *(T *)(ob + ((32 * p + 8 * g + e) * ldo + o_col)) = (T)o[p][e & 1][e >> 1];
                } else {
#pragma unroll
                    for (int p = 0; p < 2; ++p)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (32 * p + 8 * (int)g + e < count) *(T *)(ob + ((32 * p + 8 * g + e) * ldo + o_col)) = (T)o[p][e & 1][e >> 1];
                }
            }
        }
        u32x4 Up[2][3];
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            float left[8];
            *(f32x4 *)left = lds_f4(decay + 256 + (32 * p + 8 * g) * 4);
            *(f32x4 *)(left + 4) = lds_f4(decay + 256 + (32 * p + 8 * g) * 4 + 16);
#pragma unroll
            for (int e = 0; e < 8; ++e) left[e] *= U[p][e];
            split8<3>(left, Up[p]);
        }
        const float keep = __uint_as_float(lds4(decay + 63 * 4));
#pragma unroll
        for (int dp = 0; dp < DP; ++dp) {
            S[dp][0] *= keep;
            S[dp][1] *= keep;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                u32x4 part[2][3];
                column_parts<VF, DP>(at, dp, s, g, m, part);
                S[dp][0] = mma<P::in, 3, 2>(part[0], Up[s], S[dp][0]);
                S[dp][1] = mma<P::in, 3, 2>(part[1], Up[s], S[dp][1]);
            }
        }
        if (DK < 32 * DP || bad < kChunk) {
#pragma unroll
            for (int dp = 0; dp < DP; ++dp)
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        if (32 * dp + 8 * (int)g + 2 * r + t >= DK) S[dp][t][r] = 0.0f;
                        else if (bad < kChunk) S[dp][t][r] = __builtin_nanf("");
                    }
        }
        split_state();
    }
    if (!a.s_out || slot < 0 || !mine) return;
    int dk = DK;
    asm volatile("" : "+v"(dk));                               // compared again here: the masks of the first loads would be kept in registers till now
#pragma unroll
    for (int dp = 0; dp < DP; ++dp)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = 32 * dp + 8 * (int)g + 2 * r + t;
                if (d < dk) a.s_out[state + (size_t)d * DV + col] = S[dp][t][r];
            }
}

static size_t chunk_block(int32_t type) {
    return type == CSB_VAL_F32 ? Parts<CSB_VAL_F32>::bytes : Parts<CSB_VAL_BF16>::bytes;
}

template <int VF, int DP, int NW, bool VEC>
static hipError_t launch_scan(const DeltaDev &d, uint8_t *ws, hipStream_t st) {
    using L = ChunkLds<VF, DP>;
    const size_t lds = VEC && 2 * L::bytes <= 160 * 1024 ? 2 * L::bytes : L::bytes;
    static_assert(L::bytes <= 160 * 1024, "a chunk's operands fit the LDS");
    const uint32_t tiles = (uint32_t)((d.dv + 16 * NW - 1) / (16 * NW)), pairs = (uint32_t)d.n_seq * (uint32_t)d.hv;
    const auto kern = delta_scan_kernel<VF, DP, NW, VEC>;
    const hipError_t e = ensure_dynamic_lds((const void *)kern, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((pairs + 7) / 8 * 8 * tiles), dim3(64 * NW), lds, st, d, (const uint8_t *)ws, tiles);
    return hipGetLastError();
}

template <int VF, bool VEC>
static hipError_t launch_chunked(const DeltaDev &d, uint8_t *ws, int64_t numbers, bool one, hipStream_t st) {
    const uint32_t head_groups = (uint32_t)(d.hv + 3) / 4;
    if (d.n_tokens > 0) {
        hipLaunchKernelGGL((delta_prepare_kernel<VF, VEC>), dim3((uint32_t)numbers * head_groups), dim3(256), 0, st, d, ws, head_groups);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (d.dk <= 64) return one ? launch_scan<VF, 2, 1, VEC>(d, ws, st) : launch_scan<VF, 2, 4, VEC>(d, ws, st);
    if (d.dk <= 128) return one ? launch_scan<VF, 4, 1, VEC>(d, ws, st) : launch_scan<VF, 4, 4, VEC>(d, ws, st);
    return one ? launch_scan<VF, 8, 1, VEC>(d, ws, st) : launch_scan<VF, 8, 4, VEC>(d, ws, st);
}

}  // namespace csb

extern "C" size_t csb_delta_workspace_bytes(const csb_delta_args *args) {
    using namespace csb;
    if (!args || !known_type(args->type) || args->heads_v < 1 || args->n_seq < 1 || args->n_tokens < 1) return 0;
    return ((size_t)tile_numbers(args->n_tokens, args->n_seq, kChunkShift) * (size_t)args->heads_v * chunk_block(args->type) + 255) / 256 * 256;
}

extern "C" int csb_delta_chunked(const csb_delta_args *args, void *d_ws, void *stream) {
    using namespace csb;
    const int rc = check_delta("csb_delta_chunked", args);
    if (rc != CSB_OK || args->n_seq == 0) return rc;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_delta_chunked: ") + what); return code; };
    if (args->n_tokens && !d_ws) return fail(CSB_EINVAL, "NULL pointer");
    if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
    const int64_t most = 0xffffffffll / (4 * kChunk);          // a chunk's offsets are 32-bit, in bytes
    if (args->n_tokens && (args->ldq > most || args->ldk > most || args->ldv > most || args->ldo > most))
        return fail(CSB_EUNSUPPORTED, "more than 2^24 - 1 elements from one token to the next");
    const int64_t numbers = tile_numbers(args->n_tokens, args->n_seq, kChunkShift);
    const int64_t pairs = ((int64_t)args->n_seq * args->heads_v + 7) / 8 * 8, wide = ((int64_t)args->dv + 63) / 64, narrow = ((int64_t)args->dv + 15) / 16;
    if (pairs > kMaxWorkgroups || pairs * narrow > kMaxWorkgroups || numbers * ((args->heads_v + 3) / 4) > kMaxWorkgroups)
        return fail(CSB_EUNSUPPORTED, "more than 2^24 workgroups");
    if (d_ws) {
        try {
            static const char delta_user = 0;                  // this entry point as a user of workspaces
            workspace_changed_hands(d_ws, &delta_user);
        } catch (const std::bad_alloc &) {
            return fail(CSB_ENOMEM, "out of host memory");
        }
    }
    const DeltaDev d = delta_dev(args);
    const int64_t word = 16 / type_size(args->type);           // elements of an aligned 16-byte word
    const bool vec = args->dk % 8 == 0 && args->ldq % word == 0 && args->ldk % word == 0 && ((uintptr_t)args->d_q | (uintptr_t)args->d_k) % 16 == 0;
    const bool one = pairs * wide < 256;                       // wavefronts on CUs of their own while there are such
    hipStream_t st = (hipStream_t)stream;
    uint8_t *ws = (uint8_t *)d_ws;
    hipError_t e;
    switch (args->type) {
        case CSB_VAL_F32: e = vec ? launch_chunked<CSB_VAL_F32, true>(d, ws, numbers, one, st) : launch_chunked<CSB_VAL_F32, false>(d, ws, numbers, one, st); break;
        case CSB_VAL_F16: e = vec ? launch_chunked<CSB_VAL_F16, true>(d, ws, numbers, one, st) : launch_chunked<CSB_VAL_F16, false>(d, ws, numbers, one, st); break;
        default: e = vec ? launch_chunked<CSB_VAL_BF16, true>(d, ws, numbers, one, st) : launch_chunked<CSB_VAL_BF16, false>(d, ws, numbers, one, st); break;
    }
    if (e != hipSuccess) { set_error(std::string("csb_delta_chunked: ") + hipGetErrorString(e)); return CSB_EDEVICE; }
    return CSB_OK;
}
