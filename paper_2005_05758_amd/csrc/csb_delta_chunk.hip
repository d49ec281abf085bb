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
// Precision: state, M, P, R and U have 24 bits.  A binary32 number is the exact sum of three bfloat16
// numbers (8 bits each), so a product of the matrix cores' 16-bit form takes as many passes as its
// operands have parts (bfloat16 inputs one, binary16 two, binary32 three), without the ones below 2^-24; that
// is 16 / 6 to 16 / 3 of the rate of their binary32 form.
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
constexpr uint32_t kLower = 6;                 // operands that cover the lower triangle of 64 x 64 

using f32x4 = float __attribute__((ext_vector_type(4)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
using u32x4_any = uint32_t __attribute__((ext_vector_type(4), aligned(2), may_alias));     // at any element
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));

// Parts that a number has in a product, and a chunk's block of the workspace: M's operands, P's, then
// e^G_i and e^(G_64 - G_i).  binary32 operands lie there whole (they are split when read: parts would not fit the LDS).
template <int VF> struct Parts {
    static constexpr int in = VF == CSB_VAL_BF16 ? 1 : VF == CSB_VAL_F16 ? 2 : 3;      // of q and k
    static constexpr bool whole = VF == CSB_VAL_F32;
    static constexpr uint32_t m_bytes = kLower * (whole ? 2 : 3) * kFrag, p_bytes = m_bytes;
    static constexpr uint32_t bytes = m_bytes + p_bytes + 512;
};

// Operand numbers.  The 64 tokens of a chunk are four tiles (p, t) of 16 rows: row m of a tile is token
// 32 p + 8 (m / 4) + 4 t + m % 4.  A product leaves a lane with four consecutive tokens of a column then, which are one half
// of the eight consecutive ones that the next product wants from a lane of its other operand.
__device__ __forceinline__ uint32_t tile_token(uint32_t pt, uint32_t m) { return 32 * (pt >> 1) + 8 * (m >> 2) + 4 * (pt & 1u) + (m & 3u); }
// operand of tile pt and the 32 columns ks of a lower triangle (pt 0, 1: ks 0 only): 0, 1, then 2 pt - 2 + ks

__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }   // a's in the low half
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }

// E numbers as N bfloat16 numbers each, every part the nearest to what is left: exact for N = 3 (8 bits and a sign each), and for
// N = 2 where they have 16 bits or fewer (binary16 numbers).  From 3.3962e38 on the nearest bfloat16 number is infinity: the first of three parts is the largest one
// there, and what is left fits the other two.
template <int N, int E, typename Words>
__device__ __forceinline__ void split(const float *x, Words *part) {
    using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));
    float rest[E];
#pragma unroll
    for (int i = 0; i < E; ++i) rest[i] = x[i];
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
        for (int i = 0; i < E / 2; ++i) {
            const auto most = [n](float v) { return N == 3 && n == 0 ? __builtin_amdgcn_fmed3f(v, -kMostBf16, kMostBf16) : v; };
            const bf16x2 near = {(__bf16)most(rest[2 * i]), (__bf16)most(rest[2 * i + 1])};
            const uint32_t two = __builtin_bit_cast(uint32_t, near);
            part[n][i] = two;
            if (n + 1 < N) {
                rest[2 * i] -= __uint_as_float(two << 16);
                rest[2 * i + 1] -= __uint_as_float(two & 0xffff0000u);
            }
        }
}

__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 d) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), d, 0, 0, 0);
}

// f(i, j) for the pairs of parts whose product is not below 2^(-8 MOST), the small ones first.
template <int NA, int NB, int MOST, typename F>
__device__ __forceinline__ void part_pairs(const F &f) {
#pragma unroll
    for (int s = MOST; s >= 0; --s)
#pragma unroll
        for (int i = 0; i < NA; ++i)
            if (s - i >= 0 && s - i < NB) f(i, s - i);
}

// An operand of K or Q is read from memory with four neighbouring lanes on 64 consecutive bytes of a row (a lane for each of the
// multiplication's (g, m) would touch 64 pieces of 16 bytes: the path to the caches takes them one by one) and turned over in LDS.
// Its 16-byte word of row m, elements 8 g to 8 g + 7, lies at place 16 (m % 4) + 4 (m / 4) + (g ^ m % 4): the multiplication's lanes and
// the transposed reads below (4 bytes from all g and m / 4 with m % 4 alike) hit every bank once.
__device__ __forceinline__ uint32_t place(uint32_t g, uint32_t m) { return (16 * (m & 3u) + 4 * (m >> 2) + (g ^ (m & 3u))) * 16; }
__device__ __forceinline__ uint32_t loaded_row(uint32_t lane) { return ((lane >> 2) & 3u) * 4 + (lane >> 4); }          // what lane's place holds
__device__ __forceinline__ uint32_t loaded_part(uint32_t lane) { return (lane & 3u) ^ (lane >> 4); }

__device__ __forceinline__ u32x4 lds16(uint32_t at) { return *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)at; }
__device__ __forceinline__ uint32_t lds4(uint32_t at) { return *(const __attribute__((address_space(3))) uint32_t *)(uintptr_t)at; }
__device__ __forceinline__ void to_lds(uint32_t at, u32x4 v) { *(__attribute__((address_space(3))) u32x4 *)(uintptr_t)at = v; }
__device__ __forceinline__ void to_lds(uint32_t at, u32x2 v) { *(__attribute__((address_space(3))) u32x2 *)(uintptr_t)at = v; }
__device__ __forceinline__ void to_lds(uint32_t at, uint32_t v) { *(__attribute__((address_space(3))) uint32_t *)(uintptr_t)at = v; }

// ---- first launch: M and P -----------------------------------------------------------------------
// A wavefront takes one chunk of one value head.  Bound by its own latency where chunks are few (13 us for 64 tokens or for 16 short
// prompts: loads, the products, then the inverse's dependent steps), by the wait for loads where they are many (512 chunks of 16 heads, 128
// elements each: 95 us, of which wavefronts wait 44 %; 280 chunks of 48 prompts and 16 heads: 77 us).

// Eight numbers of a row of q or k from element d on, as they are stored (zeros past dk).  VEC: 16-byte words that are aligned and never cut by
// the row's end.  Else they lie at any element, and the last one of a row is read from dk - per on and moved into place when it is used
// (4096 tokens of 8 sequences, 8 heads of 121 x 121: 59 us, of 124 x 124 50, aligned ones of 128 x 128 47; element by element they were 149, 189 and 49).
template <int VF, bool VEC> struct Row8 {
    using T = typename Elem<VF>::T;
    static constexpr int words = VF == CSB_VAL_F32 ? 2 : 1, per = 8 / words;
    u32x4 w[words];
    static __device__ __forceinline__ int first_of(int e, int dk) { return VEC ? e : min(e, dk - per); }
    __device__ __forceinline__ void load(const T *row, int d, int dk) {
#pragma unroll
        for (int i = 0; i < words; ++i) {
            const int e = d + per * i;
            w[i] = u32x4{0, 0, 0, 0};
            if (e < dk) {
                if constexpr (VEC) w[i] = *(const u32x4 *)(row + e);
                else w[i] = *(const u32x4_any *)(row + first_of(e, dk));
            }
        }
    }
    // the same from a window, the row at byte `at` of it
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, uint32_t at, int d, int dk);
    // to the lane's place of an operand in LDS, and from there as a multiplication wants it
    __device__ __forceinline__ void put(uint32_t at, uint32_t lane, int d, int dk) const {
#pragma unroll
        for (int i = 0; i < words; ++i) {
            u32x4 v = w[i];
            if constexpr (!VEC) {
                const int e = d + per * i, bits = e < dk ? (e - first_of(e, dk)) * (int)sizeof(T) * 8 : 0;     // towards the word's start
                if (bits & 64) v = u32x4{v[2], v[3], 0, 0};
                if (bits & 32) v = u32x4{v[1], v[2], v[3], 0};
                if (sizeof(T) == 2 && (bits & 16)) v = u32x4{v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
            }
            to_lds(at + i * kFrag + lane * 16, v);
        }
    }
    __device__ __forceinline__ void get(uint32_t at, uint32_t g, uint32_t m) {
#pragma unroll
        for (int i = 0; i < words; ++i) w[i] = lds16(at + i * kFrag + place(g, m));
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

// The lower triangle in LDS as operands in the workspace: 3 parts, or whole.  (A loop, like all that may be one here: a launch of
// few chunks waits for its code from memory, some 0.4 us a KiB.)
template <bool WHOLE>
__device__ __forceinline__ void store_lower(const float (*m)[kLdT], uint8_t *to, uint32_t lane) {
    const uint32_t g = lane >> 4, i = lane & 15u;
#pragma unroll 1
    for (uint32_t f = 0; f < kLower; ++f) {
        const uint32_t pt = f < 2 ? f : (f + 2) / 2, ks = f < 2 ? 0 : f & 1u;          // the operand's tile and columns
        const float *row = &m[tile_token(pt, i)][32 * ks + 8 * g];
        float x[8];
        *(f32x4 *)x = *(const f32x4 *)row;
        *(f32x4 *)(x + 4) = *(const f32x4 *)(row + 4);
        u32x4 part[3];
        if constexpr (WHOLE) {
            part[0] = *(u32x4 *)x;
            part[1] = *(u32x4 *)(x + 4);
        } else split<3, 8>(x, part);
        constexpr int n = WHOLE ? 2 : 3;
#pragma unroll
        for (int k = 0; k < n; ++k) *(u32x4 *)(to + (f * n + k) * kFrag + lane * 16) = part[k];
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
    const uint32_t stage = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) float *)&mat[wave][0][0];
    constexpr uint32_t frag = Row8<VF, VEC>::words * kFrag;
    static_assert(8 * frag <= sizeof(mat[0]), "K and Q of 32 elements fit");
    Row8<VF, VEC> next[8];
    auto request = [&](int d) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int64_t t = min(base + 16 * x + (int64_t)loaded_row(lane), end - 1);    // (past the end the last one's, with a beta of zero)
            next[x].load((const T *)a.k + t * a.ldk + (size_t)kh * a.dk, d + 8 * (int)loaded_part(lane), a.dk);
            next[4 + x].load((const T *)a.q + t * a.ldq + (size_t)kh * a.dk, d + 8 * (int)loaded_part(lane), a.dk);
        }
    };
    request(0);
    for (int d = 0; d < a.dk; d += 32) {
        Row8<VF, VEC> kr[4], qr[4];
#pragma unroll
        for (int x = 0; x < 8; ++x) next[x].put(stage + x * frag, lane, d + 8 * (int)loaded_part(lane), a.dk);
        wave_sync();
        if (d + 32 < a.dk) request(d + 32);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            kr[x].get(stage + x * frag, g, i);
            qr[x].get(stage + (4 + x) * frag, g, i);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int y = 0; y <= x; ++y) {
                kk[x][y] = row_dot(kr[x], kr[y], kk[x][y]);
                qk[x][y] = row_dot(qr[x], kr[y], qk[x][y]);
            }
        wave_sync();
    }
    float (*m)[kLdT] = mat[wave];
    float strange = 0.0f;                                      // NaN when T has an entry that is not finite
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y <= x; ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * x + 4 * (int)g + r, col = 16 * y + (int)i;
                const float e = __builtin_amdgcn_exp2f((float)((sums[wave][row] - sums[wave][col]) * log2e));
                const float t = row > col ? betas[wave][row] * e * kk[x][y][r] : 0.0f;
                strange = fmaf(t, 0.0f, strange);
                m[row][col] = t;
                qk[x][y][r] = row >= col ? e * qk[x][y][r] : 0.0f;
            }
    wave_sync();
    // A row of T that is not finite must not reach the rows before it through the zeros of (1 + T)^-1: from the first one on T is taken
    // as zero here, and M's rows become NaN.  Rows past the end are zero: only a product of the last key with itself can have made them anything else.
    int bad = kChunk;
    if (__builtin_expect(__ballot(strange != 0.0f) != 0, 0)) {
        float z = 0.0f;                                        // a row per lane
        for (int c = 0; c < (int)lane; ++c) z = fmaf(m[lane][c], 0.0f, z);
        const uint64_t rows = __ballot(z != 0.0f && (int)lane < n);
        bad = rows ? __builtin_ctzll(rows) : kChunk;
        for (int r = min(bad, n); r < kChunk; ++r) m[r][lane] = 0.0f;
        wave_sync();
    }
    // (1 + T)^-1 in blocks of 16.  On the diagonal by forward substitution, lane (g, i) column i of block g; ...
    {
        float inv[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            float s0 = r == (int)i ? 1.0f : 0.0f, s1 = 0.0f;
#pragma unroll
            for (int j = 0; j < r; j += 4) {
                const f32x4 t = *(const f32x4 *)&m[16 * g + r][16 * g + j];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (j + c < r) {
                        if (c & 1) s1 = fmaf(-t[c], inv[j + c], s1);
                        else s0 = fmaf(-t[c], inv[j + c], s0);
                    }
            }
            inv[r] = s0 + s1;
        }
        wave_sync();
#pragma unroll
        for (int r = 0; r < 16; ++r) m[16 * g + r][16 * g + i] = inv[r];
        wave_sync();
    }
    // ... below it  A_xy = -A_xx sum over y <= k < x of T_xk A_ky,  on the matrix cores in binary32.  A product leaves lane (g, i) with rows
    // 4 g + r of column i, which is what it takes of its right-hand operand when step r runs over columns 4 g + r of the left one.
    f32x4 inv[4][4];
    auto left_of = [&](int x, int y) { return *(const f32x4 *)&m[16 * x + i][16 * y + 4 * g]; };
    auto product = [&](f32x4 left, f32x4 right, f32x4 d) {
#pragma unroll
        for (int r = 0; r < 4; ++r) d = __builtin_amdgcn_mfma_f32_16x16x4f32(left[r], right[r], d, 0, 0, 0);
        return d;
    };
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int r = 0; r < 4; ++r) inv[x][x][r] = m[16 * x + 4 * g + r][16 * x + i];
#pragma unroll
    for (int apart = 1; apart < 4; ++apart)
#pragma unroll
        for (int x = apart; x < 4; ++x) {
            const int y = x - apart;
            f32x4 d{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = y; k < x; ++k) d = product(left_of(x, k), inv[k][y], d);
            inv[x][y] = product(-left_of(x, x), d, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
        }
    wave_sync();
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y <= (x | 1); ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int row = 16 * x + 4 * (int)g + r, col = 16 * y + (int)i;
                float v = 0.0f;
                if (y <= x) {
                    v = row >= bad ? __builtin_nanf("") : inv[x][y <= x ? y : 0][r] * betas[wave][col];
                    if (y == x && row < col) v = 0.0f;         // (also where beta is not finite)
                }
                m[row][col] = v;
            }
    wave_sync();
    store_lower<Parts<VF>::whole>(m, block, lane);
    wave_sync();
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y <= (x | 1); ++y)
#pragma unroll
            for (int r = 0; r < 4; ++r) m[16 * x + 4 * g + r][16 * y + i] = y <= x ? qk[x][y <= x ? y : 0][r] : 0.0f;
    wave_sync();
    store_lower<Parts<VF>::whole>(m, block + Parts<VF>::m_bytes, lane);
}

// ---- second launch: the chunks of a sequence one after the other ---------------------------------

// All that the wavefront wrote to LDS is there, for the whole workgroup.  (Global loads stay in flight: __syncthreads would wait for them.)
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

template <int VF, bool VEC>
__device__ __forceinline__ void Row8<VF, VEC>::load(window_t from, uint32_t at, int d, int dk) {
#pragma unroll
    for (int i = 0; i < words; ++i) {
        const int e = d + per * i;
        w[i] = __builtin_amdgcn_raw_buffer_load_b128(from, (int)(e < dk ? at + first_of(e, dk) * (uint32_t)sizeof(T) : kOutside), 0, 0);
    }
}

// LDS of a workgroup: K of a chunk (NG = 2: and of the next), Q, e^G_i and e^(G_64 - G_i) of a chunk and of the next, then per 16
// columns the parts of S, the four wavefronts' sums of K S, R's parts, U's and e^(G_64 - G) U's, and what tells of numbers that
// are not finite.
template <int VF, int DP, int NG> struct ScanLds {
    static constexpr uint32_t half = VF == CSB_VAL_F32 ? 2 : 1;               // 16-byte words of a lane's eight numbers of K
    static constexpr uint32_t frag = half * kFrag, k = 4 * DP * frag, q_at = NG * k, decay = q_at + k, groups_at = decay + 1024;
    static constexpr uint32_t sums = 3 * DP * kFrag, r = sums + 16 * kFrag, u = r + 6 * kFrag, flags = u + 12 * kFrag, told = flags + 32,
                              group = told + 2 * 4 * 16 * 4;
    static constexpr uint32_t bytes = groups_at + NG * group;
};

// The parts of an operand of K or Q from its numbers.
template <int VF, bool VEC>
__device__ __forceinline__ void row_parts(const Row8<VF, VEC> &row, u32x4 *part) {
    if constexpr (VF == CSB_VAL_BF16) part[0] = row.w[0];
    else {
        float x[8];
        if constexpr (VF == CSB_VAL_F16) {
            const f16x8 v = __builtin_bit_cast(f16x8, row.w[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
        } else {
            *(u32x4 *)x = row.w[0];
            *(u32x4 *)(x + 4) = row.w[1];
        }
        split<Parts<VF>::in, 8>(x, part);
    }
}

// The parts of K^T for elements 32 dp + 2 m + t (t = 0, 1: part[t]) of the tokens 32 ks + 8 g .. + 7.
template <int VF, int DP>
__device__ __forceinline__ void column_parts(uint32_t k_at, int dp, int ks, uint32_t g, uint32_t m, u32x4 part[2][Parts<VF>::in]) {
    using L = ScanLds<VF, DP, 1>;                              // (an operand's size)
    // row 4 g + c of a tile, c = 0 .. 3, elements from 8 (m / 4) on: place(m / 4, 4 g + c)
    const uint32_t word = m >> 2, low = 4 * g * 16;
    if constexpr (VF == CSB_VAL_F32) {
        float x[2][8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t at = k_at + ((2 * ks + (j >> 2)) * DP + dp) * L::frag + low + (j & 3) * 256 + (word ^ (j & 3)) * 16 + ((m >> 1) & 1u) * kFrag + (m & 1u) * 8;
            x[0][j] = __uint_as_float(lds4(at));
            x[1][j] = __uint_as_float(lds4(at + 4));
        }
        split<3, 8>(x[0], part[0]);
        split<3, 8>(x[1], part[1]);
    } else {
        u32x4 both[2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {                          // tokens 2 j and 2 j + 1
            const uint32_t at = k_at + ((2 * ks + (j >> 1)) * DP + dp) * L::frag + (m & 3u) * 4 + low;
            const uint32_t c = 2 * (j & 1);
            const uint32_t even = lds4(at + c * 256 + (word ^ c) * 16), odd = lds4(at + (c + 1) * 256 + (word ^ (c + 1)) * 16);
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
                split<2, 8>(x, part[t]);
            }
        }
    }
}

// An operand of M or P as it lies in the workspace, and its parts.
template <int VF> struct Lower {
    static constexpr int words = Parts<VF>::whole ? 2 : 3;
    u32x4 w[words];
    __device__ __forceinline__ void load(const uint8_t *from, uint32_t f, uint32_t lane) {
#pragma unroll
        for (int i = 0; i < words; ++i) w[i] = *(const u32x4 *)(from + (f * words + i) * kFrag + lane * 16);
    }
    __device__ __forceinline__ void parts(u32x4 *part) const {
        if constexpr (Parts<VF>::whole) {
            float x[8];
            *(u32x4 *)x = w[0];
            *(u32x4 *)(x + 4) = w[1];
            split<3, 8>(x, part);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i) part[i] = w[i];
        }
    }
};

// Takes numbers that are not finite out of a lane's four (tokens from `token` on) and says so: told[column] = the column's first
// such token of the wavefront's, or kChunk.  Returns whether there were any.
__device__ __forceinline__ bool take_out(float *x, int token, uint32_t told, uint32_t g, uint32_t m) {
    bool any = false;
#pragma unroll
    for (int r = 0; r < 4; ++r) any |= __builtin_amdgcn_classf(x[r], 0x207);  // (infinite or NaN)
    if (__builtin_expect(__ballot(any) == 0, 1)) return false;
    int first = kChunk;
#pragma unroll
    for (int r = 3; r >= 0; --r)
        if (!(fabsf(x[r]) < __builtin_inff())) { first = token + r; x[r] = 0.0f; }
    first = min(first, __shfl_xor(first, 16));
    first = min(first, __shfl_xor(first, 32));
    if (g == 0) to_lds(told + m * 4, (uint32_t)first);
    return true;
}

// The column's first token that is not finite in a chunk's R or U, kChunk if none: from what the four wavefronts that made them have told.
__device__ __forceinline__ int first_bad(u32x4 in_r, u32x4 in_u, uint32_t told, uint32_t m) {
    int bad = kChunk;
    if (__builtin_expect(__ballot((in_r[0] | in_r[1] | in_r[2] | in_r[3] | in_u[0] | in_u[1] | in_u[2] | in_u[3]) != 0) != 0, 0)) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (in_r[w]) bad = min(bad, (int)lds4(told + w * 64 + m * 4));
            if (in_u[w]) bad = min(bad, (int)lds4(told + 256 + w * 64 + m * 4));
        }
    }
    return bad;
}

// Eight wavefronts take 16 columns of the state of one sequence and value head; NG such groups share a chunk's K and Q in LDS.  Wavefronts
// 0 to 3 carry the state: number pt holds its rows 32 dp .. 32 dp + 31 for dp = pt, pt + 4, multiplies all of K with them (the four
// sums are added up where R is made: S itself would be three parts for each of them to read), and makes the rows of tile pt = 2 p + t of R and
// U = M R.  Wavefronts 4 to 7 make the output's tiles, Q S and P U, a step behind, and fetch K and Q.  What one makes and others multiply
// with goes through LDS, three barriers a chunk.  M and P go from memory to the registers of the wavefront that multiplies with them,
// requested when it has used the chunk's before.
// Lane (g = lane / 16, m = lane % 16) has column m; of a tile over tokens the four from 8 g + 4 t on, of 32 rows of the state 8 g .. 8 g + 7.
// DP: 32s of dk.  VEC: rows of q and k in aligned 16-byte words.
// Bound by what follows on what: K S, R, U and the state wait for each other chunk after chunk, three times through LDS.  32768 tokens
// of one sequence, 16 heads of 128 x 128: 512 chunks of 1.8 us each, 915 us.  48 prompts, 16411 tokens, 16 heads, two workgroups a CU: 270 us,
// in which LDS is busy 45 % of the time, the vector issue 49 and the matrix cores 23, and wavefronts wait for 36 (one sequence: 40, 39, 21; 36).  A sequence's chunks are not split over workgroups: a part would need its
// product of the chunks' matrices besides, dk columns more beside the state's dv, and a second pass, three times the work, and a full card does
// 1.9 times the chunks a second that this one sequence does.
// bfloat16 with rows of 65 to 128 is held to 128 registers, with which a CU takes two workgroups (140 without: 48 prompts 401 us a call instead of
// 337, 32768 tokens of one sequence 980 instead of 1010).
template <int VF, int DP, int NG, bool VEC>
__global__ __launch_bounds__(512 * NG, VF == CSB_VAL_BF16 && DP == 4 ? 4 : 2 * NG) void delta_scan_kernel(const DeltaDev a, const uint8_t *ws, const uint32_t tiles) {
    using T = typename Elem<VF>::T;
    using L = ScanLds<VF, DP, NG>;
    using P = Parts<VF>;
    constexpr int own = (DP + 3) / 4;
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, m = lane & 15u;
    const uint32_t pt = wave & 3u, group = wave >> 3;
    const bool carries = (wave & 4u) == 0;
    const uint32_t k_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    const uint32_t group_at = k_at + L::groups_at + group * L::group, flags = group_at + L::flags, told = group_at + L::told;
    // workgroups of one sequence and head run on one XCD (they are dealt out by their number modulo 8): its L2 has their operands once
    const uint32_t pair = blockIdx.x / (8 * tiles) * 8 + blockIdx.x % 8, tile = blockIdx.x / 8 % tiles;
    if (pair >= (uint32_t)a.n_seq * a.hv) return;
    const uint32_t h = pair % a.hv, seq = pair / a.hv, kh = h / a.group;
    const int DK = a.dk, DV = a.dv, col = (int)((tile * NG + group) * 16 + m);
    const bool mine = col < DV;
    int64_t first_, end_, slot;
    delta_sequence(a, (int)seq, &first_, &end_, &slot);
    const int first = __builtin_amdgcn_readfirstlane((int)first_), end = __builtin_amdgcn_readfirstlane((int)end_);
    const int chunks = (int)(((uint32_t)(end - first) + kChunk - 1) >> kChunkShift);
    const uint8_t *block0 = ws + ((size_t)((uint32_t)(first >> kChunkShift) + seq) * a.hv + h) * P::bytes;
    auto block = [&](int c) { return block0 + (size_t)c * a.hv * P::bytes; };
    auto decay = [&](int c) { return (const float *)(block(c) + P::m_bytes + P::p_bytes); };
    const int token = 32 * (int)(pt >> 1) + 8 * (int)g + 4 * (int)(pt & 1u);   // the first of the lane's four
    const uint32_t row = tile_token(pt, loaded_row(lane));                     // the row of K or Q that the lane reads, and its element of 32
    const int element = 8 * (int)loaded_part(lane);
    constexpr int each = DP / NG;                              // operands of K or Q that a wavefront reads: those of tile pt, dp from each * group on
    const int dp0 = each * (int)group;
    const uint32_t f0 = pt < 2 ? pt : 2 * pt - 2, f1 = pt < 2 ? pt : 2 * pt - 1;   // its operands of M or P: one for the first 32 tokens, else two
    auto window_of = [&](const void *base, int64_t ld, size_t head, int c, int width) {    // the chunk's tokens, `width` elements of each
        const int before = c << kChunkShift, count = min(kChunk, end - first - before);   // (offsets below 2^31: leading dimensions below 2^23)
        const uint32_t ldb = (uint32_t)(ld * sizeof(T));
        return window((const T *)base + (size_t)(first + before) * ld + head, (uint32_t)(count - 1) * ldb + (uint32_t)width * (uint32_t)sizeof(T));
    };
    // Behind the last chunk its operands are requested again: what is in flight is known at every wait only if nothing is requested sometimes.
    auto next_of = [&](int c) { return min(c + 1, chunks - 1); };

    if (!carries) {
        const uint32_t ldq = (uint32_t)(a.ldq * sizeof(T)), ldo = (uint32_t)(a.ldo * sizeof(T)), o_at = mine ? token * ldo + col * (uint32_t)sizeof(T) : kOutside;
        const uint32_t ldk = (uint32_t)(a.ldk * sizeof(T));
        Row8<VF, VEC> qr[each], kr[each];
        Lower<VF> pr[2];
        const bool puts_decay = wave == 4;                     // (one wavefront's: 32 lanes hold a chunk's 128 numbers)
        f32x4 dk;
        auto load_decay = [&](int c) { if (puts_decay && lane < 32) dk = *(const f32x4 *)(decay(c) + 4 * lane); };
        auto put_decay = [&](int c) { if (puts_decay && lane < 32) to_lds(k_at + L::decay + (c & 1) * 512 + lane * 16, __builtin_bit_cast(u32x4, dk)); };
        auto load_q = [&](int c) {                             // (tokens past the end: zeros)
            const window_t qw = window_of(a.q, a.ldq, (size_t)kh * DK, c, DK);
#pragma unroll
            for (int i = 0; i < each; ++i) qr[i].load(qw, row * ldq, 32 * (dp0 + i) + element, DK);
        };
        auto load_k = [&](int c) {
            const window_t kw = window_of(a.k, a.ldk, (size_t)kh * DK, c, DK);
#pragma unroll
            for (int i = 0; i < each; ++i) kr[i].load(kw, row * ldk, 32 * (dp0 + i) + element, DK);
        };
        auto put_q = [&]() {
#pragma unroll
            for (int i = 0; i < each; ++i) qr[i].put(k_at + L::q_at + (pt * DP + dp0 + i) * L::frag, lane, 32 * (dp0 + i) + element, DK);
        };
        auto put_k = [&](int c) {
#pragma unroll
            for (int i = 0; i < each; ++i) kr[i].put(k_at + (c % NG) * L::k + (pt * DP + dp0 + i) * L::frag, lane, 32 * (dp0 + i) + element, DK);
        };
        auto load_p = [&](int c) {
            pr[0].load(block(c) + P::m_bytes, f0, lane);
            pr[1].load(block(c) + P::m_bytes, f1, lane);
        };
        if (chunks > 0) {
            load_decay(0);
            load_k(0);
            put_decay(0);
            put_k(0);
            if (NG == 2) load_k(next_of(0));
            in_order();
            load_q(0);
            in_order();
            if (NG == 1) load_k(next_of(0));
            in_order();
            load_decay(next_of(0));
            in_order();
            load_p(0);
            lds_barrier();                                     // the first K is there
        }
        const uint32_t here = group_at + lane * 16;
        for (int c = 0; c < chunks; ++c) {
            lds_barrier();                                     // Q of the chunk before is done with (NG = 2: and its K)
            if constexpr (NG == 2) {
                put_k(c + 1);
                load_k(next_of(c + 1));
                in_order();
            }
            put_q();
            load_q(next_of(c));
            in_order();
            lds_barrier();                                     // S and Q are there (NG = 1: K is done with)
            if constexpr (NG == 1) {
                put_k(c + 1);
                load_k(next_of(c + 1));
                in_order();
            }
            put_decay(c + 1);
            load_decay(next_of(c + 1));
            in_order();
            const f32x4 eg = __builtin_bit_cast(f32x4, lds16(k_at + L::decay + (c & 1) * 512 + token * 4));
            f32x4 o[3];
#pragma unroll
            for (int n = 0; n < 3; ++n) o[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int dp = 0; dp < DP; ++dp) {
                Row8<VF, VEC> rows;
                u32x4 sp[3], part[3];
                rows.get(k_at + L::q_at + (pt * DP + dp) * L::frag, g, m);
#pragma unroll
                for (int n = 0; n < 3; ++n) sp[n] = lds16(here + (dp * 3 + n) * kFrag);
                row_parts<VF, VEC>(rows, part);
                part_pairs<P::in, 3, 2>([&](int i, int j) { o[j] = mfma16(part[i], sp[j], o[j]); });
            }
            f32x4 out = o[0];
#pragma unroll
            for (int n = 1; n < 3; ++n) out += o[n];
            out *= eg;
            lds_barrier();                                     // U is there, Q done with
            const u32x4 r0 = lds16(flags), u0 = lds16(flags + 16);
            f32x4 more[3];
#pragma unroll
            for (int n = 0; n < 3; ++n) more[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (s == 0 || pt >= 2) {
                    u32x4 up[3], part[3];
                    pr[s].parts(part);
#pragma unroll
                    for (int n = 0; n < 3; ++n) up[n] = lds16(here + L::u + (2 * n + s) * kFrag);
                    part_pairs<3, 3, 2>([&](int i, int j) { more[j] = mfma16(part[i], up[j], more[j]); });
                }
#pragma unroll
            for (int n = 0; n < 3; ++n) out += more[n];
            const int bad = first_bad(r0, u0, told, m);
            const window_t ow = window_of(a.out, a.ldo, (size_t)h * DV, c, DV);
#pragma unroll
            for (int r = 0; r < 4; ++r) window_store<T>(ow, o_at + r * ldo, (T)(token + r >= bad ? __builtin_nanf("") : a.scale * out[r]));
            load_p(next_of(c));
        }
        return;
    }

    const uint32_t ldv = (uint32_t)(a.ldv * sizeof(T)), v_at = mine ? token * ldv + col * (uint32_t)sizeof(T) : kOutside;
    const size_t state = (((size_t)(slot < 0 ? 0 : slot) * a.hv + h) * DK) * DV;
    const uint32_t state_bytes = (uint32_t)DK * (uint32_t)DV * 4;              // (below 2^31: dv at most 2^20)
    auto state_at = [&](int w, int t, int r) {
        const int d = 32 * ((int)pt + 4 * w) + 8 * (int)g + 2 * r + t;
        return mine && d < DK ? ((uint32_t)d * (uint32_t)DV + (uint32_t)col) * 4 : kOutside;
    };
    f32x4 S[own][2];                                           // [dp / 4][t][r]: row 32 dp + 8 g + 2 r + t
    {
        const window_t from = a.s_in && slot >= 0 ? window(a.s_in + state, state_bytes) : window(a.g, 0);   // (none: zeros)
#pragma unroll
        for (int w = 0; w < own; ++w)
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) S[w][t][r] = __uint_as_float(window_load<float>(from, state_at(w, t, r)));
    }
    raw_t<T> v_0, v_1, v_2, v_3;                               // (an array of them would be packed, two to a register, as soon as they are loaded)
    Lower<VF> mr[2];
    auto load_v = [&](int c) {
        const window_t vw = window_of(a.v, a.ldv, (size_t)h * DV, c, DV);
        v_0 = window_load<T>(vw, v_at);
        v_1 = window_load<T>(vw, v_at + ldv);
        v_2 = window_load<T>(vw, v_at + 2 * ldv);
        v_3 = window_load<T>(vw, v_at + 3 * ldv);
    };
    auto load_m = [&](int c) {
        mr[0].load(block(c), f0, lane);
        mr[1].load(block(c), f1, lane);
    };
    u32x4 Sp[own][3];                                          // the parts of the wavefront's rows of S
    auto split_state = [&]() {
#pragma unroll
        for (int w = 0; w < own; ++w) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = S[w][e & 1][e >> 1];
            split<3, 8>(x, Sp[w]);
        }
    };
    const bool rows_mine = DP >= 4 || (int)pt < DP;
    // K S over the wavefront's rows of S, for the chunk whose K is at `at`
    auto share_sums = [&](uint32_t at) {
        if (!rows_mine) return;                                // uniform
        f32x4 ks[4];
#pragma unroll
        for (int n = 0; n < 4; ++n) ks[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < own; ++w) {
            u32x4 part[4][P::in];
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                Row8<VF, VEC> rows;
                rows.get(at + (n * DP + pt + 4 * w) * L::frag, g, m);
                row_parts<VF, VEC>(rows, part[n]);
            }
            part_pairs<P::in, 3, 2>([&](int i, int j) {
#pragma unroll
                for (int n = 0; n < 4; ++n) ks[n] = mfma16(part[n][i], Sp[w][j], ks[n]);   // (four sums side by side: none waits for the one before)
            });
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) to_lds(group_at + L::sums + (n * 4 + pt) * kFrag + lane * 16, __builtin_bit_cast(u32x4, ks[n]));
    };
    // K^T for the state: waits for nobody; with one K it is read before the next one takes its place
    u32x4 kt[own][2][2][P::in];
    auto transpose_k = [&](uint32_t at) {
        if (rows_mine)
#pragma unroll
            for (int w = 0; w < own; ++w)
#pragma unroll
                for (int s = 0; s < 2; ++s) column_parts<VF, DP>(at, (int)pt + 4 * w, s, g, m, kt[w][s]);
    };
    // where a lane's four tokens go in an operand over tokens: half (pt & 1) of the place of lane (g, m) of the 32 tokens pt >> 1
    const uint32_t quad = (pt >> 1) * kFrag + lane * 16 + (pt & 1u) * 8;

    if (chunks > 0) {
        load_v(0);
        in_order();
        load_m(0);
        in_order();
        split_state();
        lds_barrier();                                         // the first K is there
        share_sums(k_at);
    }
    for (int c = 0; c < chunks; ++c) {
        const uint32_t k_here = k_at + (c % NG) * L::k, k_there = k_at + ((c + 1) % NG) * L::k;
        const uint32_t decays = k_at + L::decay + (c & 1) * 512;
        lds_barrier();                                         // K S is there
        const f32x4 eg = __builtin_bit_cast(f32x4, lds16(decays + token * 4));
        f32x4 ks[4];
#pragma unroll
        for (int n = 0; n < (DP < 4 ? DP : 4); ++n) ks[n] = __builtin_bit_cast(f32x4, lds16(group_at + L::sums + (pt * 4 + n) * kFrag + lane * 16));
        if (rows_mine)                                         // S for the output
#pragma unroll
            for (int w = 0; w < own; ++w)
#pragma unroll
                for (int n = 0; n < 3; ++n) to_lds(group_at + ((pt + 4 * w) * 3 + n) * kFrag + lane * 16, Sp[w][n]);
        if constexpr (DP < 4) ks[0] += ks[1];
        else ks[0] = (ks[0] + ks[1]) + (ks[2] + ks[3]);
        float R[4];
        const raw_t<T> v[4] = {v_0, v_1, v_2, v_3};
#pragma unroll
        for (int r = 0; r < 4; ++r) R[r] = fmaf(-eg[r], ks[0][r], (float)__builtin_bit_cast(T, v[r]));
        const bool bad_r = take_out(R, token, told + pt * 64, g, m);
        {
            u32x2 part[3];
            split<3, 4>(R, part);
#pragma unroll
            for (int n = 0; n < 3; ++n) to_lds(group_at + L::r + n * 2 * kFrag + quad, part[n]);
        }
        if (lane == 0) to_lds(flags + pt * 4, (uint32_t)bad_r);
        if constexpr (NG == 1) transpose_k(k_here);
        load_v(next_of(c));
        lds_barrier();                                         // R is there
        f32x4 u[3];
#pragma unroll
        for (int n = 0; n < 3; ++n) u[n] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        const f32x4 left = __builtin_bit_cast(f32x4, lds16(decays + 256 + token * 4));
        u32x4 rp[2][3];
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s == 0 || pt >= 2)
#pragma unroll
                for (int n = 0; n < 3; ++n) rp[s][n] = lds16(group_at + L::r + (2 * n + s) * kFrag + lane * 16);
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (s == 0 || pt >= 2) {
                u32x4 part[3];
                mr[s].parts(part);
                part_pairs<3, 3, 2>([&](int i, int j) { u[i] = mfma16(part[i], rp[s][j], u[i]); });
            }
        float U[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) U[r] = u[0][r] + (u[1][r] + u[2][r]);
        const bool bad_u = take_out(U, token, told + 256 + pt * 64, g, m);
        {
            u32x2 part[3];
            float l[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) l[r] = U[r] * left[r];
            split<3, 4>(l, part);
#pragma unroll
            for (int n = 0; n < 3; ++n) to_lds(group_at + L::u + (3 + n) * 2 * kFrag + quad, part[n]);
            split<3, 4>(U, part);
#pragma unroll
            for (int n = 0; n < 3; ++n) to_lds(group_at + L::u + n * 2 * kFrag + quad, part[n]);
        }
        if (lane == 0) to_lds(flags + 16 + pt * 4, (uint32_t)bad_u);
        if constexpr (NG == 2) transpose_k(k_here);            // (before R, it would be in registers that there are not)
        load_m(next_of(c));
        in_order();
        lds_barrier();                                         // U is there
        const u32x4 r0 = lds16(flags), u0 = lds16(flags + 16);
        const float keep = __uint_as_float(lds4(decays + 63 * 4));
#pragma unroll
        for (int w = 0; w < own; ++w)
            if (rows_mine) {
                f32x4 more[2];                                 // (the second 32 tokens' sums: none waits for the one before)
                more[0] = more[1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                S[w][0] *= keep;
                S[w][1] *= keep;
                u32x4 lp[2][3];
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int n = 0; n < 3; ++n) lp[s][n] = lds16(group_at + L::u + ((3 + n) * 2 + s) * kFrag + lane * 16);
                part_pairs<P::in, 3, 2>([&](int i, int j) {
                    S[w][0] = mfma16(kt[w][0][0][i], lp[0][j], S[w][0]);
                    S[w][1] = mfma16(kt[w][0][1][i], lp[0][j], S[w][1]);
                    more[0] = mfma16(kt[w][1][0][i], lp[1][j], more[0]);
                    more[1] = mfma16(kt[w][1][1][i], lp[1][j], more[1]);
                });
                S[w][0] += more[0];
                S[w][1] += more[1];
            }
        if (first_bad(r0, u0, told, m) < kChunk) {
#pragma unroll
            for (int w = 0; w < own; ++w) S[w][0] = S[w][1] = f32x4{__builtin_nanf(""), __builtin_nanf(""), __builtin_nanf(""), __builtin_nanf("")};
        }
        split_state();
        share_sums(k_there);                                // (behind the last chunk nobody reads it)
    }
    if (!a.s_out || slot < 0) return;                          // uniform
    const window_t to = window(a.s_out + state, state_bytes);
#pragma unroll
    for (int w = 0; w < own; ++w)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) window_store<float>(to, state_at(w, t, r), S[w][t][r]);
}

static size_t chunk_block(int32_t type) {
    return type == CSB_VAL_F32 ? Parts<CSB_VAL_F32>::bytes : Parts<CSB_VAL_BF16>::bytes;
}

template <int VF, int DP, int NG, bool VEC>
static hipError_t launch_scan(const DeltaDev &d, uint8_t *ws, hipStream_t st) {
    constexpr size_t lds = ScanLds<VF, DP, NG>::bytes;
    static_assert(lds <= 160 * 1024, "LDS of a workgroup");
    const uint32_t tiles = (uint32_t)((d.dv + 16 * NG - 1) / (16 * NG)), pairs = (uint32_t)d.n_seq * (uint32_t)d.hv;
    const auto kern = delta_scan_kernel<VF, DP, NG, VEC>;
    const hipError_t e = ensure_dynamic_lds((const void *)kern, lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kern, dim3((pairs + 7) / 8 * 8 * tiles), dim3(512 * NG), lds, st, d, (const uint8_t *)ws, tiles);
    return hipGetLastError();
}

template <int VF, bool VEC>
static hipError_t launch_chunked(const DeltaDev &d, uint8_t *ws, int64_t numbers, bool few, hipStream_t st) {
    const uint32_t head_groups = (uint32_t)(d.hv + 3) / 4;
    if (d.n_tokens > 0) {
        hipLaunchKernelGGL((delta_prepare_kernel<VF, VEC>), dim3((uint32_t)numbers * head_groups), dim3(256), 0, st, d, ws, head_groups);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    // 16 columns a workgroup, of which a CU takes two with bfloat16 rows of up to 128 (16411 tokens, 8 heads of 128 x 128: 174 us; 32 columns 182).
    // binary16 has one part of K and Q more and the registers for one only: 32 columns a workgroup where CUs have enough of them (232 us against
    // 270, though it keeps 16 registers of a lane in memory then).  Rows of 64 gain nothing by that (157 against 143), wider ones have not the LDS.
    if (d.dk <= 64) return launch_scan<VF, 2, 1, VEC>(d, ws, st);
    if (d.dk <= 128) {
        if constexpr (VF == CSB_VAL_F16)
            if (!few) return launch_scan<VF, 4, 2, VEC>(d, ws, st);
        return launch_scan<VF, 4, 1, VEC>(d, ws, st);
    }
    if constexpr (VF != CSB_VAL_F32) return launch_scan<VF, 8, 1, VEC>(d, ws, st);
    return hipErrorInvalidValue;                               // (not reached: csb_delta_chunked)
}

// binary32 rows wider than 128 do not fit the LDS beside the rest, rows of less than 16 bytes no word: token by token
static bool delta_by_token(const csb_delta_args *a) {
    return (a->type == CSB_VAL_F32 && a->dk > 128) || a->dk * type_size(a->type) < 16;
}

// Sizes that only the chunks refuse.
static Refusal chunk_sizes(const csb_delta_args *a) {
    if (a->dv > 1 << 20) return {CSB_EUNSUPPORTED, "dv above 2^20"};
    const int64_t pairs = ((int64_t)a->n_seq * a->heads_v + 7) / 8 * 8, narrow = ((int64_t)a->dv + 15) / 16;
    const int64_t numbers = tile_numbers(a->n_tokens, a->n_seq, kChunkShift);
    if (pairs > kMaxWorkgroups || pairs * narrow > kMaxWorkgroups / 4 || numbers * (((int64_t)a->heads_v + 3) / 4) > kMaxWorkgroups)
        return {CSB_EUNSUPPORTED, "more workgroups than a launch takes"};
    return {CSB_OK, nullptr};
}

}  // namespace csb

extern "C" size_t csb_delta_workspace_bytes(const csb_delta_args *args) {
    using namespace csb;
    if (delta_sizes(args).code != CSB_OK || args->n_seq < 1 || args->n_tokens < 1 || delta_by_token(args) || chunk_sizes(args).code != CSB_OK) return 0;
    return ((size_t)tile_numbers(args->n_tokens, args->n_seq, kChunkShift) * (size_t)args->heads_v * chunk_block(args->type) + 255) / 256 * 256;
}

extern "C" int csb_delta_chunked(const csb_delta_args *args, void *d_ws, void *stream) {
    using namespace csb;
    const int rc = check_delta("csb_delta_chunked", args);
    if (rc != CSB_OK || args->n_seq == 0) return rc;
    if (delta_by_token(args)) return launch_delta_recurrent(args, (hipStream_t)stream);
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_delta_chunked: ") + what); return code; };
    if (args->n_tokens && !d_ws) return fail(CSB_EINVAL, "NULL pointer");
    if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
    const int64_t most = (1 << 23) - 1;                        // (a chunk's offsets in bytes are below 2^31)
    if (args->n_tokens && (args->ldq > most || args->ldk > most || args->ldv > most || args->ldo > most))
        return fail(CSB_EUNSUPPORTED, "2^23 or more elements from one token to the next");
    const Refusal sizes = chunk_sizes(args);
    if (sizes.code != CSB_OK) return fail(sizes.code, sizes.what);
    const int64_t numbers = tile_numbers(args->n_tokens, args->n_seq, kChunkShift);
    const int64_t pairs = ((int64_t)args->n_seq * args->heads_v + 7) / 8 * 8, wide = ((int64_t)args->dv + 63) / 64;
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
    const bool few = pairs * wide < 256;                       // CUs idle with workgroups of more columns
    hipStream_t st = (hipStream_t)stream;
    uint8_t *ws = (uint8_t *)d_ws;
    hipError_t e;
    switch (args->type) {
        case CSB_VAL_F32: e = vec ? launch_chunked<CSB_VAL_F32, true>(d, ws, numbers, few, st) : launch_chunked<CSB_VAL_F32, false>(d, ws, numbers, few, st); break;
        case CSB_VAL_F16: e = vec ? launch_chunked<CSB_VAL_F16, true>(d, ws, numbers, few, st) : launch_chunked<CSB_VAL_F16, false>(d, ws, numbers, few, st); break;
        default: e = vec ? launch_chunked<CSB_VAL_BF16, true>(d, ws, numbers, few, st) : launch_chunked<CSB_VAL_BF16, false>(d, ws, numbers, few, st); break;
    }
    if (e != hipSuccess) { set_error(std::string("csb_delta_chunked: ") + hipGetErrorString(e)); return CSB_EDEVICE; }
    return CSB_OK;
}
