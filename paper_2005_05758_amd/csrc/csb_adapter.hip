// Low-rank adapters of many requests beside a shared projection (csb_adapter_add):
//     Y[:, n] += scale_a B_a (A_a X[:, n]),  a the adapter of the request that column n belongs to.
//
// Two launches.  The first takes A X, the long sums (over `cols`), split over the grid and over the wavefronts of
// a workgroup; each split leaves its partial sums in the workspace.  The second adds the splits up and takes B
// times that, the short sums (over the rank), into Y: it moves 8 bytes per entry of Y and is bound by that.
// Both work on tiles of 32 columns, at multiples of 32, of one request: a tile has one adapter, and a column
// that a neighbour request has too in the same tile is left to that request's own tile.
#include <algorithm>
#include <new>

#include "csb_lm.hpp"

namespace csb {

constexpr int kAdapterTile = 32, kAdapterShift = 5, kAdapterMaxRank = 128;

struct AdapterDev {
    const void *X, *A, *B;
    float *Y, *t;                              // t [splits][rank][batch]: partial sums of A X
    const int32_t *rank, *start, *id;
    const float *scale;
    int64_t ldx, ldy, rows, cols;
    int32_t batch, n_adapters, max_rank, n_seg, splits;
    int32_t k_wave;                            // columns of A that a wavefront of the first launch takes
    int32_t row_group;                         // rows of Y that a workgroup of the second takes
};

// The columns [c0, c1) of this workgroup's tile that belong to its request, the tile's first column, and the
// adapter (negative: nothing to do).
struct AdapterTile {
    int32_t base, c0, c1, adapter, rank;
};
__device__ __forceinline__ AdapterTile adapter_tile(const AdapterDev &a, uint32_t number) {
    AdapterTile w{0, 0, 0, -1, 0};
    int64_t first, end, base;
    int s;
    if (a.start) {
        s = tile_sequence(a.start, a.n_seg, a.batch, kAdapterShift, number);
        if (s < 0) return w;
        sequence_range(a.start, s, 0, a.batch, &first, &end);
        base = ((first >> kAdapterShift) + ((int64_t)number - (first >> kAdapterShift) - s)) << kAdapterShift;
    } else {                                   // one column each: no search
        s = (int)number;
        first = number;
        end = first + 1;
        base = first & ~(int64_t)(kAdapterTile - 1);
    }
    if (base >= end) return w;
    const int32_t id = a.id[s];
    if (id < 0 || id >= a.n_adapters) return w;
    w.base = (int32_t)base;
    w.c0 = (int32_t)(first > base ? first : base);
    w.c1 = (int32_t)(end < base + kAdapterTile ? end : base + kAdapterTile);
    w.rank = a.rank ? min(max(a.rank[id], 0), a.max_rank) : a.max_rank;
    if (w.c0 < w.c1 && w.rank > 0) w.adapter = id;
    return w;
}

using f32x4 = float __attribute__((ext_vector_type(4)));
using u16x8 = uint16_t __attribute__((ext_vector_type(8)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

// t = A X for one tile: 16 x 16 products on the matrix cores, RT sixteens of ranks by the 32 columns.  A wavefront takes
// k_wave consecutive columns of A, 32 (16 for binary32) at a time; lane (g = lane / 16, i = lane % 16) holds row i of A at
// 8 (4) columns from 8 g (4 g) on.  16-bit operands: X comes as pairs of neighbouring columns of Y, so that the first product takes the
// even and the second the odd ones, and no lane needs another's data to have its 8 consecutive rows of X.
// AV: rows of A in aligned 16-byte words.  XV: pairs of X in aligned 4-byte words.
template <int VF, int RT, bool AV, bool XV>
__global__ __launch_bounds__(256) void adapter_down_kernel(const AdapterDev a) {
    using T = typename Elem<VF>::T;
    __shared__ float part[4][RT * 16][kAdapterTile];
    const AdapterTile w = adapter_tile(a, blockIdx.x);
    if (w.adapter < 0) return;                 // uniform
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15u;
    const int64_t k0 = ((int64_t)blockIdx.y * 4 + wave) * a.k_wave, k1 = min(k0 + a.k_wave, a.cols);
    const T *A = (const T *)a.A + (size_t)w.adapter * a.max_rank * a.cols, *X = (const T *)a.X;
    f32x4 acc[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r) acc[r][0] = acc[r][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (VF == CSB_VAL_F32) {
        const int32_t n0 = w.base + (int32_t)i, n1 = n0 + 16;
        const bool in0 = n0 >= w.c0 && n0 < w.c1, in1 = n1 >= w.c0 && n1 < w.c1;
        for (int64_t k = k0; k < k1; k += 16) {
            const int64_t kg = k + 4 * g;
            float x0[4], x1[4], v[RT][4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x0[j] = in0 && kg + j < k1 ? X[(kg + j) * a.ldx + n0] : 0.0f;
                x1[j] = in1 && kg + j < k1 ? X[(kg + j) * a.ldx + n1] : 0.0f;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int32_t row = 16 * r + (int32_t)i;
                const float *p = A + (size_t)row * a.cols + kg;
                if constexpr (AV) {
                    f32x4 q{0.0f, 0.0f, 0.0f, 0.0f};
                    if (row < w.rank && kg < k1) q = *(const f32x4 *)p;
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[r][j] = q[j];
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[r][j] = row < w.rank && kg + j < k1 ? p[j] : 0.0f;
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    acc[r][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][j], x0[j], acc[r][0], 0, 0, 0);
                    acc[r][1] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][j], x1[j], acc[r][1], 0, 0, 0);
                }
        }
    } else {
        const int32_t n0 = w.base + 2 * (int32_t)i, n1 = n0 + 1;
        const bool in0 = n0 >= w.c0 && n0 < w.c1, in1 = n1 >= w.c0 && n1 < w.c1;
        const uint16_t *Xb = (const uint16_t *)X, *Ab = (const uint16_t *)A;
        for (int64_t k = k0; k < k1; k += 32) {
            const int64_t kg = k + 8 * g;
            uint32_t x[8];
            u32x4 v[RT];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint16_t *p = Xb + (kg + j) * a.ldx + n0;
                x[j] = 0;
                if (kg + j < k1) {
                    if (XV && in0 && in1) x[j] = *(const uint32_t *)p;
                    else {
                        if (in0) x[j] = p[0];
                        if (in1) x[j] |= (uint32_t)p[1] << 16;
                    }
                }
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const int32_t row = 16 * r + (int32_t)i;
                const uint16_t *p = Ab + (size_t)row * a.cols + kg;
                v[r] = u32x4{0, 0, 0, 0};
                if constexpr (AV) {
                    if (row < w.rank && kg < k1) v[r] = *(const u32x4 *)p;
                } else if (row < w.rank) {
                    u16x8 q{0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (kg + j < k1) q[j] = p[j];
                    v[r] = __builtin_bit_cast(u32x4, q);
                }
            }
            u32x4 even, odd;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                even[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x05040100u);
                odd[j] = __builtin_amdgcn_perm(x[2 * j + 1], x[2 * j], 0x07060302u);
            }
            using T8 = T __attribute__((ext_vector_type(8)));
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const T8 av = __builtin_bit_cast(T8, v[r]), e = __builtin_bit_cast(T8, even), o = __builtin_bit_cast(T8, odd);
                if constexpr (VF == CSB_VAL_F16) {
                    acc[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, e, acc[r][0], 0, 0, 0);
                    acc[r][1] = __builtin_amdgcn_mfma_f32_16x16x32_f16(av, o, acc[r][1], 0, 0, 0);
                } else {
                    acc[r][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, e, acc[r][0], 0, 0, 0);
                    acc[r][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, o, acc[r][1], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                part[wave][16 * r + 4 * g + c][VF == CSB_VAL_F32 ? 16 * h + i : 2 * i + h] = acc[r][h][c];
    __syncthreads();
    const uint32_t n = threadIdx.x & 31u;
    const int32_t col = w.base + (int32_t)n;
    if (col < w.c0 || col >= w.c1) return;
    for (int32_t r = threadIdx.x >> 5; r < w.rank; r += 8)
        a.t[((size_t)blockIdx.y * a.max_rank + r) * a.batch + col] = (part[0][r][n] + part[1][r][n]) + (part[2][r][n] + part[3][r][n]);
}

// Y += B t for one tile and row_group rows: t, its splits added up and scaled, sits in LDS; a wavefront takes 16 rows of B at
// a time.  binary32 products on the matrix cores: t keeps its 24 bits.
// BV: rows of B in aligned words of 4 elements.
template <int VF, bool BV>
__global__ __launch_bounds__(256) void adapter_up_kernel(const AdapterDev a) {
    using T = typename Elem<VF>::T;
    using T4 = T __attribute__((ext_vector_type(4)));
    __shared__ float t[kAdapterMaxRank][kAdapterTile + 1];
    const AdapterTile w = adapter_tile(a, blockIdx.x);
    if (w.adapter < 0) return;                 // uniform
    const float scale = a.scale ? a.scale[w.adapter] : 1.0f;
    const int32_t steps = (w.rank + 15) / 16;
    {
        const uint32_t n = threadIdx.x & 31u;
        const int32_t col = w.base + (int32_t)n;
        const bool in = col >= w.c0 && col < w.c1;
        for (int32_t r = threadIdx.x >> 5; r < 16 * steps; r += 8) {
            float s = 0.0f;
            if (in && r < w.rank)
                for (int32_t p = 0; p < a.splits; ++p) s += a.t[((size_t)p * a.max_rank + r) * a.batch + col];
            t[r][n] = s * scale;
        }
    }
    __syncthreads();
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6, g = lane >> 4, i = lane & 15u;
    const T *B = (const T *)a.B + (size_t)w.adapter * a.rows * a.max_rank;
    const int32_t n0 = w.base + (int32_t)i, n1 = n0 + 16;
    const bool in0 = n0 >= w.c0 && n0 < w.c1, in1 = n1 >= w.c0 && n1 < w.c1;
    const int64_t first = (int64_t)blockIdx.y * a.row_group, last = min(first + a.row_group, a.rows);
    for (int64_t row0 = first + 16 * wave; row0 < last; row0 += 64) {
        float y0[4], y1[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t row = row0 + 4 * g + c;
            y0[c] = in0 && row < last ? a.Y[row * a.ldy + n0] : 0.0f;
            y1[c] = in1 && row < last ? a.Y[row * a.ldy + n1] : 0.0f;
        }
        f32x4 d0{0.0f, 0.0f, 0.0f, 0.0f}, d1 = d0;
        const T *p = B + (row0 + i) * a.max_rank;
        for (int32_t s = 0; s < steps; ++s) {
            const int32_t r = 16 * s + 4 * (int32_t)g;
            T4 b{};
            if (row0 + i < last) {
                if constexpr (BV) {
                    if (r < w.rank) b = *(const T4 *)(p + r);
#pragma unroll
                    for (int j = 0; j < 4; ++j) if (r + j >= w.rank) b[j] = (T)0.0f;   // what is stored past the rank is not used
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) if (r + j < w.rank) b[j] = p[r + j];
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                d0 = __builtin_amdgcn_mfma_f32_16x16x4f32((float)b[j], t[r + j][i], d0, 0, 0, 0);
                d1 = __builtin_amdgcn_mfma_f32_16x16x4f32((float)b[j], t[r + j][16 + i], d1, 0, 0, 0);
            }
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int64_t row = row0 + 4 * g + c;
            if (in0 && row < last) a.Y[row * a.ldy + n0] = y0[c] + d0[c];
            if (in1 && row < last) a.Y[row * a.ldy + n1] = y1[c] + d1[c];
        }
    }
}

// How the long sums are split: parts of the grid (at most 16) and columns per wavefront, a multiple of 32.
static void adapter_split(int64_t cols, int64_t tiles, int32_t *splits, int32_t *k_wave) {
    const int64_t want = std::max<int64_t>(1, std::min<int64_t>(16, 1024 / std::max<int64_t>(1, tiles)));
    const int64_t per = std::max<int64_t>(32, ((cols + want * 4 - 1) / (want * 4) + 31) / 32 * 32);
    *k_wave = (int32_t)per;
    *splits = (int32_t)((cols + 4 * per - 1) / (4 * per));
}

static int64_t adapter_tiles(int32_t batch, int32_t n_seg, bool offsets) {
    return offsets ? tile_numbers(batch, n_seg, kAdapterShift) : n_seg;
}

template <int VF, bool AV, bool XV>
static void launch_down(const AdapterDev &d, dim3 grid, hipStream_t st) {
    if (d.max_rank <= 16) hipLaunchKernelGGL((adapter_down_kernel<VF, 1, AV, XV>), grid, dim3(256), 0, st, d);
    else if (d.max_rank <= 32) hipLaunchKernelGGL((adapter_down_kernel<VF, 2, AV, XV>), grid, dim3(256), 0, st, d);
    else if (d.max_rank <= 64) hipLaunchKernelGGL((adapter_down_kernel<VF, 4, AV, XV>), grid, dim3(256), 0, st, d);
    else hipLaunchKernelGGL((adapter_down_kernel<VF, 8, AV, XV>), grid, dim3(256), 0, st, d);
}

template <int VF>
static void launch_adapter(const AdapterDev &d, bool av, bool xv, bool bv, dim3 down, dim3 up, hipStream_t st) {
    if (av && xv) launch_down<VF, true, true>(d, down, st);
    else if (av) launch_down<VF, true, false>(d, down, st);
    else launch_down<VF, false, false>(d, down, st);
    if (bv) hipLaunchKernelGGL((adapter_up_kernel<VF, true>), up, dim3(256), 0, st, d);
    else hipLaunchKernelGGL((adapter_up_kernel<VF, false>), up, dim3(256), 0, st, d);
}

}  // namespace csb

extern "C" size_t csb_adapter_workspace_bytes(int64_t cols, int32_t batch, int32_t n_seg, int32_t rank) {
    if (cols <= 0 || batch <= 0 || n_seg <= 0 || rank <= 0 || rank > csb::kAdapterMaxRank) return 0;
    int32_t splits, k_wave, most = 1;                          // (with offsets there are more tiles and never more splits)
    csb::adapter_split(cols, csb::adapter_tiles(batch, n_seg, true), &splits, &k_wave);
    most = std::max(most, splits);
    csb::adapter_split(cols, csb::adapter_tiles(batch, n_seg, false), &splits, &k_wave);
    most = std::max(most, splits);
    return ((size_t)most * (size_t)rank * (size_t)batch * sizeof(float) + 255) / 256 * 256;
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
    if (batch > 1 << 30) return fail(CSB_EUNSUPPORTED, "more than 2^30 columns of X");
    if (ldx < batch || ldy < batch) return fail(CSB_EINVAL, "a leading dimension below batch");
    if (!d_start && n_seg != batch) return fail(CSB_EINVAL, "n_seg is not batch (and there are no offsets)");
    if (batch == 0 || n_seg == 0) return CSB_OK;
    if (!d_X || !d_Y || !d_A || !d_B || !d_id || !d_ws) return fail(CSB_EINVAL, "NULL pointer");
    if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
    const uintptr_t size = (uintptr_t)type_size(type);
    if (((uintptr_t)d_X | (uintptr_t)d_A | (uintptr_t)d_B) % size || (uintptr_t)d_Y % 4) return fail(CSB_EINVAL, "misaligned pointer");
    const int64_t tiles = adapter_tiles(batch, n_seg, d_start != nullptr);
    AdapterDev d{};
    d.X = d_X; d.A = d_A; d.B = d_B; d.Y = d_Y; d.t = (float *)d_ws;
    d.rank = d_rank; d.start = d_start; d.id = d_id; d.scale = d_scale;
    d.ldx = ldx; d.ldy = ldy; d.rows = rows; d.cols = cols;
    d.batch = batch; d.n_adapters = n_adapters; d.max_rank = rank; d.n_seg = n_seg;
    adapter_split(cols, tiles, &d.splits, &d.k_wave);
    int64_t group = 64;                                        // rows of a workgroup: enough workgroups, and t read by few of them
    while (group < 512 && tiles * ((rows + 2 * group - 1) / (2 * group)) >= 2048) group *= 2;
    d.row_group = (int32_t)group;
    const int64_t row_groups = (rows + group - 1) / group;
    if (tiles * std::max<int64_t>(row_groups, d.splits) > kMaxWorkgroups || row_groups > 65535) return fail(CSB_EUNSUPPORTED, "more than 2^24 workgroups");
    try {
        static const char adapter_user = 0;                    // this entry point as a user of workspaces
        workspace_changed_hands(d_ws, &adapter_user);
    } catch (const std::bad_alloc &) {
        return fail(CSB_ENOMEM, "out of host memory");
    }
    const uintptr_t per = type == CSB_VAL_F32 ? 4 : 8;         // elements of a 16-byte word
    const bool av = cols % per == 0 && (uintptr_t)d_A % 16 == 0;
    const bool xv = ldx % 2 == 0 && (uintptr_t)d_X % 4 == 0;
    const bool bv = rank % 4 == 0 && (uintptr_t)d_B % (4 * size) == 0;
    const dim3 down((uint32_t)tiles, (uint32_t)d.splits), up((uint32_t)tiles, (uint32_t)row_groups);
    hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case CSB_VAL_F32: launch_adapter<CSB_VAL_F32>(d, av, true, bv, down, up, st); break;
        case CSB_VAL_F16: launch_adapter<CSB_VAL_F16>(d, av, xv, bv, down, up, st); break;
        default: launch_adapter<CSB_VAL_BF16>(d, av, xv, bv, down, up, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error(std::string("csb_adapter_add: ") + hipGetErrorString(e)); return CSB_EDEVICE; }
    return CSB_OK;
}
