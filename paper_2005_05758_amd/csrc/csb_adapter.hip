// Low-rank adapters of many requests beside a shared projection (csb_adapter_add):
//     Y[:, n] += scale_a B_a (A_a X[:, n]),  a the adapter of the request that column n belongs to.
//
// Two launches.  The first takes A X, the long sums (over `cols`), split over the grid and over the wavefronts of
// a workgroup; each split leaves its partial sums in the workspace.  The second adds the splits up and takes B
// times that, the short sums (over the rank), into Y: it moves 8 bytes per entry of Y and is bound by that.
// Both work on tiles of 32 columns, at multiples of 32.  A tile has as many adapters as its columns ask for, one in a
// long request, up to 32 where every column is a request of its own: for each of them the product is made for all 32 columns and
// kept in its own, so that X and Y are read and written in whole rows of a tile whatever the requests are, and an adapter that several
// requests of a tile share is read once for them.
#include <algorithm>
#include <new>

#include "csb_lm.hpp"

namespace csb {

constexpr int kAdapterTile = 32, kAdapterMaxRank = 128;

struct AdapterDev {
    const void *X, *A, *B;
    float *Y, *t;                              // t [splits][max_rank][batch]: partial sums of A X
    const int32_t *rank, *start, *id;
    const float *scale;
    int64_t ldx, ldy, rows, cols;
    int32_t batch, n_adapters, max_rank, n_seg, splits;
    int32_t k_wave;                            // columns of A that a wavefront of the first launch takes
    int32_t row_group;                         // rows of Y that a workgroup of the second takes
};

// Tiles of the launch's first dimension: neighbours on the same XCD (workgroups are dealt out by their number modulo 8), whose L2 then
// has whole lines of X and longer pieces of Y's rows.  A multiple of 8 workgroups; -1 for the ones too many.
__device__ __forceinline__ int32_t tile_here(int32_t batch) {
    const int32_t tiles = (batch + kAdapterTile - 1) / kAdapterTile, x = (int32_t)blockIdx.x;
    if (tiles < 16) return x;
    const int32_t k = x % 8, at = x / 8, each = tiles / 8, more = tiles % 8;
    return at < each + (k < more) ? k * each + min(k, more) + at : -1;
}

using f32x2 = float __attribute__((ext_vector_type(2)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using u16x8 = uint16_t __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));
// the same at any element
using u32_any = uint32_t __attribute__((aligned(2), may_alias));
using u32x4_any = uint32_t __attribute__((ext_vector_type(4), aligned(2), may_alias));
using f32x2_any = float __attribute__((ext_vector_type(2), aligned(4), may_alias));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

// 16 bytes of T from p on, at any element; zeros from element n > 0 on, which are not read.
template <typename T> __device__ __forceinline__ u32x4 any_words(const T *p, int n) {
    if (n >= (int)(16 / sizeof(T))) return *(const u32x4_any *)p;
    u32x4 w{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < (int)(16 / sizeof(T)); ++j) if (j < n) {
        if constexpr (sizeof(T) == 4) w[j] = __float_as_uint(p[j]);
        else w[j / 2] |= (uint32_t)((const uint16_t *)p)[j] << 16 * (j % 2);
    }
    return w;
}

// The adapters of a tile's columns, each once, with the columns that they have (a bit each) and the ranks they use.
struct AdapterList {
    int32_t of[kAdapterTile];                  // of a column, -1: none
    int32_t id[kAdapterTile], rank[kAdapterTile];
    uint32_t columns[kAdapterTile];
    int32_t n;
};
// Filled by the whole workgroup, for columns base .. base + 31.  (Offsets that do not ascend may name a column twice: one of the two is taken.)
__device__ __forceinline__ void list_adapters(const AdapterDev &a, int32_t base, AdapterList &w) {
    if (threadIdx.x < kAdapterTile) {
        const int32_t col = base + (int32_t)threadIdx.x;
        w.of[threadIdx.x] = !a.start && col < a.batch ? a.id[col] : -1;
    }
    if (a.start) {
        __syncthreads();
        for (int32_t s = (int32_t)threadIdx.x; s < a.n_seg; s += (int32_t)blockDim.x) {
            const int32_t first = min(max(a.start[s], 0), a.batch), end = min(max(a.start[s + 1], first), a.batch);
            if (first < base + kAdapterTile && end > base)
                for (int32_t c = max(first, base), id = a.id[s]; c < min(end, base + kAdapterTile); ++c) w.of[c - base] = id;
        }
    }
    __syncthreads();
    if (threadIdx.x < 64) {                    // a lane a column; the first of those with one adapter speaks for all
        int32_t id = threadIdx.x < kAdapterTile ? w.of[threadIdx.x] : -1;
        int32_t rank = 0;
        if (id >= 0 && id < a.n_adapters) rank = a.rank ? min(max(a.rank[id], 0), a.max_rank) : a.max_rank;
        if (rank == 0) id = -1;
        uint32_t mine = 0;
        for (int c = 0; c < kAdapterTile; ++c) {
            const uint32_t same = (uint32_t)__ballot(id == __builtin_amdgcn_readlane(id, c));
            if (c == (int)threadIdx.x) mine = same;
        }
        const bool speaks = id >= 0 && (int)__builtin_ctz(mine) == (int)threadIdx.x;
        const uint64_t speakers = __ballot(speaks);
        if (speaks) {
            const int at = __popcll(speakers & ((1ull << threadIdx.x) - 1));
            w.id[at] = id;
            w.rank[at] = rank;
            w.columns[at] = mine;
        }
        if (threadIdx.x == 0) w.n = __popcll(speakers);
    }
    __syncthreads();
}

// t = A X for one tile: 16 x 16 products on the matrix cores, RT sixteens of ranks by the 32 columns.  A wavefront takes
// k_wave consecutive columns of A, 32 (16 for binary32) at a time; lane (g = lane / 16, i = lane % 16) holds row i of A at
// 8 (4) columns from 8 g (4 g) on.  16-bit operands: X comes as pairs of neighbouring columns of Y, so that the first product takes the
// even and the second the odd ones, and no lane needs another's data to have its 8 consecutive rows of X.
// AV: rows of A in aligned 16-byte words, none of them cut by the row's end.  XV: pairs of X in aligned 4-byte words.  Else the same words at any
// element (2999 columns of A instead of 3008, rank 40, 776 columns of X: 16 us instead of 11.5; element by element it was 44).
// MANY: the adapters of a tile are dealt out to gridDim.z workgroups, and a wavefront keeps its part of X (k_wave at most kStay) in registers
// for all of them; else the steps over X are outermost (a tile of one adapter, rarely two).
constexpr int kStay = 128;
template <int VF, int RT, bool AV, bool XV, bool MANY>
__global__ __launch_bounds__(256) void adapter_down_kernel(const AdapterDev a) {
    using T = typename Elem<VF>::T;
    constexpr int step = VF == CSB_VAL_F32 ? 16 : 32, per = step / 4;          // columns of A a step, of a lane
    __shared__ float part[4][RT * 16][kAdapterTile];
    __shared__ AdapterList list;
    const int32_t tile = tile_here(a.batch), base = tile * kAdapterTile;
    if (tile < 0) return;
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15u;
    const int64_t k0 = ((int64_t)blockIdx.y * 4 + wave) * a.k_wave, k1 = min(k0 + a.k_wave, a.cols);
    const T *X = (const T *)a.X;
    // X's operands of one step: binary32 columns i and 16 + i, 16-bit 2 i and 2 i + 1
    const int32_t n0 = base + (VF == CSB_VAL_F32 ? (int32_t)i : 2 * (int32_t)i), n1 = n0 + (VF == CSB_VAL_F32 ? 16 : 1);
    const bool in0 = n0 < a.batch, in1 = n1 < a.batch;
    struct Right { u32x4 w[2]; };
    auto load_x = [&](int64_t k) {
        const int64_t kg = k + per * g;
        Right x;
        if constexpr (VF == CSB_VAL_F32) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x.w[0][j] = in0 && kg + j < k1 ? __float_as_uint(X[(kg + j) * a.ldx + n0]) : 0u;
                x.w[1][j] = in1 && kg + j < k1 ? __float_as_uint(X[(kg + j) * a.ldx + n1]) : 0u;
            }
        } else {
            uint32_t v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint16_t *p = (const uint16_t *)X + (kg + j) * a.ldx + n0;
                v[j] = 0;
                if (kg + j < k1) {
                    if (in1) {
                        if constexpr (XV) v[j] = *(const uint32_t *)p;
                        else v[j] = *(const u32_any *)p;
                    } else if (in0) v[j] = p[0];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x.w[0][j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], 0x05040100u);
                x.w[1][j] = __builtin_amdgcn_perm(v[2 * j + 1], v[2 * j], 0x07060302u);
            }
        }
        return x;
    };
    auto load_a = [&](const T *A, int rank, int r, int64_t k) {
        const int64_t kg = k + per * g;
        const int32_t row = 16 * r + (int32_t)i;
        const T *p = A + (size_t)row * a.cols + kg;
        u32x4 v{0, 0, 0, 0};
        if constexpr (AV) {
            if (row < rank && kg < k1) v = *(const u32x4 *)p;
        } else if (row < rank && kg < k1) v = any_words<T>(p, (int)min(k1 - kg, (int64_t)per));
        return v;
    };
    auto multiply = [&](u32x4 l, const Right &x, f32x4 *d) {
        using T8 = T __attribute__((ext_vector_type(16 / sizeof(T))));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (VF == CSB_VAL_F32) {
#pragma unroll
                for (int j = 0; j < 4; ++j) d[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(l[j]), __uint_as_float(x.w[h][j]), d[h], 0, 0, 0);
            } else if constexpr (VF == CSB_VAL_F16)
                d[h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(T8, l), __builtin_bit_cast(T8, x.w[h]), d[h], 0, 0, 0);
            else d[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(T8, l), __builtin_bit_cast(T8, x.w[h]), d[h], 0, 0, 0);
        }
    };
    const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f};
    f32x4 acc[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r][0] = acc[r][1] = zero;
    uint32_t done = 0;                                         // the columns that this workgroup's adapters have
    const uint32_t bit0 = 1u << (n0 - base), bit1 = 1u << (n1 - base);
    if constexpr (MANY) {
        constexpr int steps = kStay / step;
        Right x[steps];
#pragma unroll
        for (int s = 0; s < steps; ++s) x[s] = load_x(k0 + s * step);          // (requested before the adapters are known)
        list_adapters(a, base, list);
        auto fetch = [&](int e, u32x4 v[RT][steps]) {
            const T *A = (const T *)a.A + (size_t)list.id[e] * a.max_rank * a.cols;
            const int rank = list.rank[e];
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int s = 0; s < steps; ++s) v[r][s] = load_a(A, rank, r, k0 + s * step);
        };
        u32x4 v[RT][steps], w[RT][steps];
        int e = (int)blockIdx.z;
        if (e < list.n) fetch(e, v);
        for (; e < list.n; e += (int)gridDim.z) {
            const int after = e + (int)gridDim.z;
            if (after < list.n) fetch(after, w);               // the next one's while this one's are multiplied
            const uint32_t columns = list.columns[e];
            done |= columns;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                f32x4 d[2] = {zero, zero};
#pragma unroll
                for (int s = 0; s < steps; ++s) multiply(v[r][s], x[s], d);
                if (columns & bit0) acc[r][0] = d[0];
                if (columns & bit1) acc[r][1] = d[1];
            }
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int s = 0; s < steps; ++s) v[r][s] = w[r][s];
        }
    } else {
        list_adapters(a, base, list);
        for (int e = 0; e < list.n; ++e) {
            const T *A = (const T *)a.A + (size_t)list.id[e] * a.max_rank * a.cols;
            const uint32_t columns = list.columns[e];
            const int rank = list.rank[e];
            done |= columns;
            f32x4 d[RT][2];
#pragma unroll
            for (int r = 0; r < RT; ++r) d[r][0] = d[r][1] = zero;
            Right x = load_x(k0);
            u32x4 v[RT];
#pragma unroll
            for (int r = 0; r < RT; ++r) v[r] = load_a(A, rank, r, k0);
            for (int64_t k = k0; k < k1; k += step) {          // the next step's operands while this one's are multiplied
                const Right x_next = load_x(k + step);
                u32x4 v_next[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) v_next[r] = load_a(A, rank, r, k + step);
#pragma unroll
                for (int r = 0; r < RT; ++r) multiply(v[r], x, d[r]);
                x = x_next;
#pragma unroll
                for (int r = 0; r < RT; ++r) v[r] = v_next[r];
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                if (columns & bit0) acc[r][0] = d[r][0];
                if (columns & bit1) acc[r][1] = d[r][1];
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < 4; ++c) part[wave][16 * r + 4 * g + c][(h ? n1 : n0) - base] = acc[r][h][c];
    __syncthreads();
    const uint32_t n = threadIdx.x & 31u;
    if (!(done >> n & 1u)) return;
    for (int32_t r = threadIdx.x >> 5; r < a.max_rank; r += 8)  // (past an adapter's ranks: zeros)
        a.t[((size_t)blockIdx.y * a.max_rank + r) * a.batch + base + n] = (part[0][r][n] + part[1][r][n]) + (part[2][r][n] + part[3][r][n]);
}

// E numbers as 3 bfloat16 numbers each, every part the nearest to what is left: exact (8 bits and a sign each).  LARGE: binary32 numbers, of which
// the nearest to those from 3.3962e38 on is infinity: the first part is the largest number there, and what is left fits the other two.
template <int E, bool LARGE>
__device__ __forceinline__ void three_parts(const float *x, uint16_t (*part)[E]) {
#pragma unroll
    for (int e = 0; e < E; ++e) {
        float rest = x[e];
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            const __bf16 near = (__bf16)(LARGE && n == 0 ? __builtin_amdgcn_fmed3f(rest, -kMostBf16, kMostBf16) : rest);
            part[n][e] = __builtin_bit_cast(uint16_t, near);
            rest -= (float)near;
        }
    }
}

// Y += B t for one tile and row_group rows.  t, its splits added up and scaled, goes through LDS into the operands of the matrix cores:
// tile column h of lane i is column 2 i + h, so that a lane has two neighbouring columns of Y and 16 lanes a whole row of the tile.
// 16-bit B: t as three bfloat16 parts (24 bits), 3 / 16 of the time of the binary32 form; binary16 B as two.  binary32 B: the binary32 form.
// 8192 rows x 2048 columns of rank 64: 34 us, 4 TB/s, bound by HBM and what starts before it (the adapters' list, t).  With loads that lanes take part
// in or not, as the edges have them, every wait is for all that is in flight: 48 us.  (Three wavefronts a SIMD up to rank 64, at which 16-bit B of ranks 33
// to 64 keeps 2 registers of a lane in memory: the call 72 us instead of 74 with two.)
// Wavefronts share the rows; of groups below 64 rows, where a tile has 4 adapters or more, the adapters (each column has one, so nothing is added up).
// BV: rows of B in aligned words of 8 (binary32: 4) elements.  YV: pairs of Y in aligned 8-byte words.  Else words at any element.
template <int VF, int KS, bool BV, bool YV>
__global__ __launch_bounds__(256, KS == 1 || (KS == 2 && VF != CSB_VAL_F32) ? 3 : 2) void adapter_up_kernel(const AdapterDev a) {
    using T = typename Elem<VF>::T;
    constexpr int per = VF == CSB_VAL_F32 ? 4 : 8, step = 4 * per;             // ranks of a lane, of a step
    __shared__ AdapterList list;
    __shared__ float t[KS * 32][kAdapterTile];
    __shared__ float many[4][16][kAdapterTile];
    __shared__ u32x4 tp[VF == CSB_VAL_F32 ? 1 : 6 * KS][64];
    const int32_t tile = tile_here(a.batch), base = tile * kAdapterTile;
    if (tile < 0) return;
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, i = lane & 15u;
    const int64_t first = (int64_t)blockIdx.y * a.row_group, last = min(first + a.row_group, a.rows);
    const int32_t col = base + 2 * (int32_t)i;
    const bool there0 = col < a.batch, there1 = col + 1 < a.batch;
    auto load_y = [&](int64_t row0, f32x2 *y) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t row = row0 + 4 * g + c;
            const float *p = a.Y + row * a.ldy + col;
            y[c] = f32x2{0.0f, 0.0f};
            if (row < last) {
                if (there1) {
                    if constexpr (YV) y[c] = *(const f32x2 *)p;
                    else y[c] = *(const f32x2_any *)p;
                } else if (there0) y[c][0] = p[0];
            }
        }
    };
    // What needs no adapter's number is requested before those are known: the first rows of Y, and t, of which a thread adds up ranks r0, r0 + 8,
    // ... of one column, 16 loads in flight together.  (t of columns that have no adapter was not written: not used.)
    // STREAM: rows of Y and the operands of B are requested `depth` steps of 64 rows ahead, through windows, where the tile allows it.
    constexpr bool STREAM = BV && YV;
    constexpr int words = VF == CSB_VAL_F32 ? 2 * KS : KS, depth = KS == 4 ? 2 : 3;
    struct Left { u32x4 w[words]; };
    struct Ahead { f32x2 y[4]; Left b[2]; } ahead_of[STREAM ? depth : 1];
    const bool near = a.ldy < 1 << 25;                         // (offsets in 16 rows of Y stay below 2^31 bytes)
    const uint32_t y_row = (uint32_t)a.ldy * 4;
    uint32_t y_at = there1 ? 4 * g * y_row + 8 * i : kOutside;
    auto y_window = [&](int64_t row0) {                        // of the tile's columns in 16 rows
        const int n = (int)max(min(last - row0, (int64_t)16), (int64_t)0);
        return window(a.Y + row0 * a.ldy + base, n ? (uint32_t)(n - 1) * y_row + 4 * min(kAdapterTile, a.batch - base) : 0);
    };
    auto request_y = [&](Ahead &to, int64_t row0) {
        const window_t w = y_window(row0);
#pragma unroll
        for (int c = 0; c < 4; ++c) to.y[c] = __builtin_bit_cast(f32x2, __builtin_amdgcn_raw_buffer_load_b64(w, (int)(y_at + c * y_row), 0, 0));
    };
    const int64_t row_first = first + 16 * wave;
    f32x2 y[4];
    if (STREAM && near) request_y(ahead_of[0], row_first);
    else load_y(row_first, y);
    const uint32_t tn = threadIdx.x & 31u, r0 = threadIdx.x >> 5;
    constexpr int turns = 4 / KS;
    float sum[4 * KS];
    {
#pragma unroll
        for (int k = 0; k < 4 * KS; ++k) sum[k] = 0.0f;
        const float *p = a.t + min(base + (int32_t)tn, a.batch - 1);
        const size_t split = (size_t)a.max_rank * a.batch;
        for (int32_t s = 0; s < a.splits; s += turns) {
            float v[turns][4 * KS];
#pragma unroll
            for (int q = 0; q < turns; ++q)
#pragma unroll
                for (int k = 0; k < 4 * KS; ++k) v[q][k] = p[min(s + q, a.splits - 1) * split + (size_t)min((int32_t)r0 + 8 * k, a.max_rank - 1) * a.batch];
#pragma unroll
            for (int q = 0; q < turns; ++q)
#pragma unroll
                for (int k = 0; k < 4 * KS; ++k) sum[k] += s + q < a.splits ? v[q][k] : 0.0f;
        }
    }
    list_adapters(a, base, list);
    if (list.n == 0) return;                                   // uniform
    uint32_t all = 0;
    for (int e = 0; e < list.n; ++e) all |= list.columns[e];
    const uint32_t bit0 = 1u << (2 * i), bit1 = 2u << (2 * i);
    const bool in0 = all & bit0, in1 = all & bit1;             // (columns of no adapter are not written)
    {
        const bool in = all >> tn & 1u;
        const float scale = in && a.scale ? a.scale[list.of[tn]] : 1.0f;
#pragma unroll
        for (int k = 0; k < 4 * KS; ++k) t[r0 + 8 * k][tn] = in && (int32_t)r0 + 8 * k < a.max_rank ? sum[k] * scale : 0.0f;
    }
    __syncthreads();
    // t as right-hand operands, made once for all rows: lane (g, i) has ranks 32 s + 8 g .. + 7 of columns 2 i + h.  They stay in LDS
    // (their registers would halve the wavefronts of a CU, and with them the rows of Y in flight).
    if constexpr (VF != CSB_VAL_F32) {
        for (uint32_t f = wave; f < 2 * KS; f += 4) {
            const uint32_t s = f / 2, h = f % 2;
            float x[8];
            uint16_t p[3][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = t[32 * s + 8 * g + j][2 * i + h];
            three_parts<8, true>(x, p);
#pragma unroll
            for (int n = 0; n < 3; ++n) __builtin_memcpy(&tp[f * 3 + n][lane], p[n], 16);
        }
        __syncthreads();
    }
    const f32x4 zero{0.0f, 0.0f, 0.0f, 0.0f};
    auto load_b = [&](int e, int64_t row, int64_t last) {      // the lane's part of row `row` (zeros past the adapter's ranks: what is stored there is not used)
        const T *p = (const T *)a.B + ((size_t)list.id[e] * a.rows + row) * a.max_rank;
        const int rank = list.rank[e];
        Left l;
#pragma unroll
        for (int s = 0; s < words; ++s) {
            const int r = step * s + per * (int)g;
            T v[per];
            u32x4 w{0, 0, 0, 0};
            if constexpr (BV) {
                if (row < last && r < rank) w = *(const u32x4 *)(p + r);
                if (r + per > rank) {
                    __builtin_memcpy(v, &w, 16);
#pragma unroll
                    for (int j = 0; j < per; ++j) if (r + j >= rank) v[j] = (T)0.0f;
                    __builtin_memcpy(&w, v, 16);
                }
            } else if (row < last && r < rank) w = any_words<T>(p + r, rank - r);
            l.w[s] = w;
        }
        return l;
    };
    auto multiply = [&](const Left &l, f32x4 *d) {
#pragma unroll
        for (int s = 0; s < words; ++s) {
            if constexpr (VF == CSB_VAL_F32) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x2 two = *(const f32x2 *)&t[16 * s + 4 * g + j][2 * i];
#pragma unroll
                    for (int h = 0; h < 2; ++h) d[h] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(l.w[s][j]), two[h], d[h], 0, 0, 0);
                }
            } else {
                u32x4 parts[2];
                constexpr int np = VF == CSB_VAL_F16 ? 2 : 1;
                if constexpr (VF == CSB_VAL_F16) {             // 11 bits: two parts are exact
                    float x[8];
                    uint16_t q[3][8];
                    const auto v = __builtin_bit_cast(_Float16 __attribute__((ext_vector_type(8))), l.w[s]);
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = (float)v[j];
                    three_parts<8, false>(x, q);
                    __builtin_memcpy(&parts[0], q[0], 16);
                    __builtin_memcpy(&parts[1], q[1], 16);
                } else parts[0] = l.w[s];
#pragma unroll
                for (int n = 2; n >= 0; --n)
#pragma unroll
                    for (int b = 0; b < np; ++b)
                        if (n + b <= 2) {
#pragma unroll
                            for (int h = 0; h < 2; ++h)
                                d[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, parts[b]), __builtin_bit_cast(bf16x8, tp[(2 * s + h) * 3 + n][lane]), d[h], 0, 0, 0);
                        }
            }
        }
    };
    auto store_y = [&](int64_t row0, const f32x2 *y) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t row = row0 + 4 * g + c;
            float *p = a.Y + row * a.ldy + col;
            if (row < last) {
                if (in0 && in1) {
                    if constexpr (YV) *(f32x2 *)p = y[c];
                    else *(f32x2_any *)p = y[c];
                } else {
                    if (in0) p[0] = y[c][0];
                    if (in1) p[1] = y[c][1];
                }
            }
        }
    };
    if constexpr (STREAM) {
        // One or two adapters, pairs of columns with both or neither in an adapter: a stream.
        int id[2], rank[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            id[e] = __builtin_amdgcn_readfirstlane(list.id[e < list.n ? e : 0]);
            rank[e] = __builtin_amdgcn_readfirstlane(e < list.n ? list.rank[e] : 0);
        }
        const bool stream = near && list.n <= 2 && !__ballot(in0 != in1);
        auto request_b = [&](Ahead &to, int64_t row0) {
            const uint32_t n = (uint32_t)max(min(last - row0, (int64_t)16), (int64_t)0), row = (uint32_t)(a.max_rank * sizeof(T));
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const window_t w = window((const T *)a.B + ((size_t)id[e] * a.rows + row0) * a.max_rank, n * row);
#pragma unroll
                for (int s = 0; s < words; ++s) {
                    const int r = step * s + per * (int)g;
                    to.b[e].w[s] = __builtin_amdgcn_raw_buffer_load_b128(w, (int)(r < rank[e] ? i * row + r * (uint32_t)sizeof(T) : kOutside), 0, 0);
                }
            }
        };
        if (stream) {                                          // uniform
#pragma unroll
            for (int d = 0; d < depth; ++d) {
                if (d) request_y(ahead_of[d], row_first + 64 * d);
                request_b(ahead_of[d], row_first + 64 * d);
                in_order();
            }
            u32x4 kept[2];                                     // of the word in which the adapter's ranks end (what is stored past them is not used)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int ranks = rank[e] % step - per * (int)g;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    kept[e][j] = VF == CSB_VAL_F32 ? (j < ranks ? ~0u : 0) : (2 * j < ranks ? 0xffffu : 0) | (2 * j + 1 < ranks ? 0xffff0000u : 0);
            }
            auto cut = [&](Left &l, int e) {
#pragma unroll
                for (int s = 0; s < words; ++s) if (s == rank[e] / step) l.w[s] &= kept[e];
            };
            y_at = in0 ? y_at : kOutside;
            const uint32_t columns1 = list.n > 1 ? list.columns[1] : 0;
            for (int64_t row0 = row_first; row0 < last; row0 += 64 * depth)   // (past `last` the windows are empty)
#pragma unroll
                for (int d = 0; d < depth; ++d) {
                    const int64_t row = row0 + 64 * d;
                    Ahead &now = ahead_of[d];
                    f32x4 sum[2] = {zero, zero};
                    cut(now.b[0], 0);
                    multiply(now.b[0], sum);
                    if (list.n > 1) {
                        f32x4 more[2] = {zero, zero};
                        cut(now.b[1], 1);
                        multiply(now.b[1], more);
                        if (columns1 & bit0) sum[0] = more[0];
                        if (columns1 & bit1) sum[1] = more[1];
                    }
                    const window_t w = y_window(row);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
                        const f32x2 v = now.y[c] + f32x2{sum[0][c], sum[1][c]};
                        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, v), w, (int)(y_at + c * y_row), 0, 0);
                    }
                    in_order();
                    request_y(now, row + 64 * depth);
                    request_b(now, row + 64 * depth);
                    in_order();
                }
            return;
        }
        if (near) {
            if ((a.batch & 1) && base + kAdapterTile > a.batch) load_y(row_first, y);    // (the last column alone was not requested)
            else {
#pragma unroll
                for (int c = 0; c < 4; ++c) y[c] = ahead_of[0].y[c];
            }
        }
    }
    if (list.n < 4 || a.row_group >= 64) {                     // uniform: wavefronts share the rows
        f32x2 y_next[4];
        Left l, l_next;
        int64_t row0 = row_first;
        if (row0 < last) l = load_b(0, row0 + i, last);
        for (; row0 < last; row0 += 64) {
            if (row0 + 64 < last) load_y(row0 + 64, y_next);   // the next rows while these are multiplied
            f32x4 sum[2] = {zero, zero};
            in_order();                                        // (t's operands are read where they are used)
            for (int e = 0; e < list.n; ++e) {
                const bool more = e + 1 < list.n;              // the next adapter's part of B, or of the next rows, while this one is multiplied
                if (more || row0 + 64 < last) l_next = load_b(more ? e + 1 : 0, row0 + (more ? 0 : 64) + i, last);
                f32x4 d[2] = {zero, zero};
                multiply(l, d);
                const uint32_t columns = list.columns[e];
                if (columns & bit0) sum[0] = d[0];
                if (columns & bit1) sum[1] = d[1];
                l = l_next;
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) y[c] += f32x2{sum[0][c], sum[1][c]};
            store_y(row0, y);
#pragma unroll
            for (int c = 0; c < 4; ++c) y[c] = y_next[c];
        }
        return;
    }
    for (int64_t row0 = first; row0 < last; row0 += 16) {      // wavefronts share the adapters
        if (wave == 0 && row0 > first) load_y(row0, y);
        f32x4 sum[2] = {zero, zero};
        int e = (int)wave;
        Left l, l_next;
        if (e < list.n) l = load_b(e, row0 + i, last);
        for (; e < list.n; e += 4) {
            if (e + 4 < list.n) l_next = load_b(e + 4, row0 + i, last);
            f32x4 d[2] = {zero, zero};
            multiply(l, d);
            const uint32_t columns = list.columns[e];
            if (columns & bit0) sum[0] = d[0];
            if (columns & bit1) sum[1] = d[1];
            l = l_next;
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < 4; ++c) many[wave][4 * g + c][2 * i + h] = sum[h][c];      // (zero where another wavefront's adapter is)
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int c = 0; c < 4; ++c)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t r = 4 * g + c, n = 2 * i + h;
                    y[c][h] += (many[0][r][n] + many[1][r][n]) + (many[2][r][n] + many[3][r][n]);
                }
            store_y(row0, y);
        }
        __syncthreads();
    }
}

// Below 32 columns a request MANY (ranks up to 64, which the registers hold): k_wave = kStay, at most 64 splits.  64 requests of one column beside
// 4096 x 4096, rank 16: 17 us instead of 106; 2048 columns beside 8192 x 8192 in requests of 16, rank 16, 49 instead of 55, of 32 44 instead of
// 45, of 32 and rank 64 64 instead of 63; beside 3001 x 2999, rank 13, requests of 9 21 instead of 27, of 31 23 instead of 24.  Else at most 8 splits
// (the second launch reads what each leaves), k_wave a multiple of 32.
static bool adapter_many(int64_t cols, int32_t batch, int32_t n_seg, int32_t rank) {
    return batch < 32ll * n_seg && rank <= 64 && cols <= 64 * 4 * kStay;
}
static void adapter_split(int64_t cols, int32_t batch, bool many, int32_t *splits, int32_t *k_wave) {
    const int64_t tiles = ((int64_t)batch + kAdapterTile - 1) / kAdapterTile;
    if (many) *k_wave = kStay;
    else {
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>(8, 512 / std::max<int64_t>(1, tiles)));
        *k_wave = (int32_t)std::max<int64_t>(32, ((cols + want * 4 - 1) / (want * 4) + 31) / 32 * 32);
    }
    *splits = (int32_t)((cols + 4ll * *k_wave - 1) / (4ll * *k_wave));
}

template <int VF, bool AV, bool XV, bool MANY>
static void launch_down(const AdapterDev &d, dim3 grid, hipStream_t st) {
    if (d.max_rank <= 16) hipLaunchKernelGGL((adapter_down_kernel<VF, 1, AV, XV, MANY>), grid, dim3(256), 0, st, d);
    else if (d.max_rank <= 32) hipLaunchKernelGGL((adapter_down_kernel<VF, 2, AV, XV, MANY>), grid, dim3(256), 0, st, d);
    else if (MANY || d.max_rank <= 64) hipLaunchKernelGGL((adapter_down_kernel<VF, 4, AV, XV, MANY>), grid, dim3(256), 0, st, d);
    else if constexpr (!MANY) hipLaunchKernelGGL((adapter_down_kernel<VF, 8, AV, XV, MANY>), grid, dim3(256), 0, st, d);
}
template <int VF, bool BV, bool YV>
static void launch_up(const AdapterDev &d, dim3 grid, hipStream_t st) {
    if (d.max_rank <= 32) hipLaunchKernelGGL((adapter_up_kernel<VF, 1, BV, YV>), grid, dim3(256), 0, st, d);
    else if (d.max_rank <= 64) hipLaunchKernelGGL((adapter_up_kernel<VF, 2, BV, YV>), grid, dim3(256), 0, st, d);
    else hipLaunchKernelGGL((adapter_up_kernel<VF, 4, BV, YV>), grid, dim3(256), 0, st, d);
}

template <int VF>
static void launch_adapter(const AdapterDev &d, bool av, bool xv, bool bv, bool yv, bool many, dim3 down, dim3 up, hipStream_t st) {
    const bool fast = av && xv;
    if (many && fast) launch_down<VF, true, true, true>(d, down, st);
    else if (many) launch_down<VF, false, false, true>(d, down, st);
    else if (fast) launch_down<VF, true, true, false>(d, down, st);
    else launch_down<VF, false, false, false>(d, down, st);
    if (bv && yv) launch_up<VF, true, true>(d, up, st);
    else launch_up<VF, false, false>(d, up, st);
}

}  // namespace csb

extern "C" size_t csb_adapter_workspace_bytes(int64_t cols, int32_t batch, int32_t n_seg, int32_t rank) {
    if (cols <= 0 || batch <= 0 || n_seg <= 0 || rank <= 0 || rank > csb::kAdapterMaxRank) return 0;
    int32_t splits, k_wave;
    csb::adapter_split(cols, batch, csb::adapter_many(cols, batch, n_seg, rank), &splits, &k_wave);
    return ((size_t)splits * (size_t)rank * (size_t)batch * sizeof(float) + 255) / 256 * 256;
}

extern "C" int csb_adapter_add(int32_t type, const void *d_X, int64_t ldx, float *d_Y, int64_t ldy, int64_t rows,
                               int64_t cols, int32_t batch, const void *d_A, const void *d_B, int32_t n_adapters,
                               int32_t rank, const int32_t *d_rank, const float *d_scale, int32_t n_seg,
                               const int32_t *d_start, const int32_t *d_id, void *d_ws, void *stream) {
    using namespace csb;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_adapter_add: ") + what); return code; };
    if (!known_type(type)) return fail(CSB_EINVAL, "unknown type");
    if (rows <= 0 || cols <= 0 || batch < 0 || n_seg < 0 || n_adapters < 1 || rank < 1) return fail(CSB_EINVAL, "bad size");
    if (rank > kAdapterMaxRank) return fail(CSB_EUNSUPPORTED, "rank above 128 (a tile's sums are held in registers)");
    if (batch > 1 << 30 || rows > 0x7fffffff || cols > 0x7fffffff) return fail(CSB_EUNSUPPORTED, "more than 2^30 columns of X, or 2^31 - 1 rows or columns of a projection");
    if (ldx < batch || ldy < batch) return fail(CSB_EINVAL, "a leading dimension below batch");
    if (!d_start && n_seg != batch) return fail(CSB_EINVAL, "n_seg is not batch (and there are no offsets)");
    if (batch == 0 || n_seg == 0) return CSB_OK;
    if (!d_X || !d_Y || !d_A || !d_B || !d_id || !d_ws) return fail(CSB_EINVAL, "NULL pointer");
    if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
    const uintptr_t size = (uintptr_t)type_size(type);
    if (((uintptr_t)d_X | (uintptr_t)d_A | (uintptr_t)d_B) % size || (uintptr_t)d_Y % 4) return fail(CSB_EINVAL, "misaligned pointer");
    const int64_t tiles = ((int64_t)batch + kAdapterTile - 1) / kAdapterTile;
    AdapterDev d{};
    d.X = d_X; d.A = d_A; d.B = d_B; d.Y = d_Y; d.t = (float *)d_ws;
    d.rank = d_rank; d.start = d_start; d.id = d_id; d.scale = d_scale;
    d.ldx = ldx; d.ldy = ldy; d.rows = rows; d.cols = cols;
    d.batch = batch; d.n_adapters = n_adapters; d.max_rank = rank; d.n_seg = n_seg;
    const uintptr_t per = type == CSB_VAL_F32 ? 4 : 8;         // elements of a 16-byte word
    const bool av = cols % per == 0 && (uintptr_t)d_A % 16 == 0;
    const bool xv = type == CSB_VAL_F32 || (ldx % 2 == 0 && (uintptr_t)d_X % 4 == 0);
    const bool bv = rank % per == 0 && (uintptr_t)d_B % 16 == 0;
    const bool yv = ldy % 2 == 0 && (uintptr_t)d_Y % 8 == 0;
    const bool many = adapter_many(cols, batch, n_seg, rank);
    adapter_split(cols, batch, many, &d.splits, &d.k_wave);
    int64_t group = many ? 16 : 64;                            // rows of a workgroup: enough workgroups, and t read by few of them
    while (group < 2048 && tiles * ((rows + 2 * group - 1) / (2 * group)) >= 512) group *= 2;
    while ((rows + group - 1) / group > 65535) group *= 2;     // (a launch's second dimension)
    d.row_group = (int32_t)group;
    const int64_t row_groups = (rows + group - 1) / group;
    // adapters of a tile over several workgroups while CUs are idle
    const int64_t deal = many ? std::max<int64_t>(1, std::min<int64_t>(8, 512 / (tiles * d.splits))) : 1;
    if ((tiles + 7) * std::max<int64_t>(row_groups, deal * d.splits) > kMaxWorkgroups) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    try {
        static const char adapter_user = 0;                    // this entry point as a user of workspaces
        workspace_changed_hands(d_ws, &adapter_user);
    } catch (const std::bad_alloc &) {
        return fail(CSB_ENOMEM, "out of host memory");
    }
    const uint32_t across = (uint32_t)(tiles < 16 ? tiles : (tiles + 7) / 8 * 8);
    const dim3 down(across, (uint32_t)d.splits, (uint32_t)deal), up(across, (uint32_t)row_groups);
    hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case CSB_VAL_F32: launch_adapter<CSB_VAL_F32>(d, av, xv, bv, yv, many, down, up, st); break;
        case CSB_VAL_F16: launch_adapter<CSB_VAL_F16>(d, av, xv, bv, yv, many, down, up, st); break;
        default: launch_adapter<CSB_VAL_BF16>(d, av, xv, bv, yv, many, down, up, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error(std::string("csb_adapter_add: ") + hipGetErrorString(e)); return CSB_EDEVICE; }
    return CSB_OK;
}
