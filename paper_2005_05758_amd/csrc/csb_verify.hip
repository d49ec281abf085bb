// Verification of drafted tokens (csb_verify_drafts).
//
// Draft x of row i is accepted if u q_i(x) < p_i(x); behind the first one refused the next token is drawn from
// max(p - q, 0), so that what comes out is distributed as the target's own samples.  Of all rows given only the
// one (and its draft's) where the drafts end is read in full: that is what the operator is bound by.  Weights are
// whole units of 2^-38, so the sum of a row, the place of a random number in it and with it the token are the same however
// the row is split over workgroups.
//
// Vocabularies up to kVerifySmall: one launch, a workgroup a request (one request over 20011 tokens 7.6 us instead of 8.7, over 24000 8.4
// instead of 8.7, over 32768 11.4 instead of 8.4; a call from the host saves a launch besides).  Larger ones: two launches, the
// first adds up the units of the row in chunks, the second finds the chunk that the number falls into and the token in it
// (64 requests over 131072 tokens, 67 MB: 17 us, 3.9 TB/s, and 4.7).
#include <algorithm>
#include <new>

#include "csb_lm.hpp"

namespace csb {

constexpr float kUnits = 274877906944.0f;      // 2^38
constexpr int kVerifyMaxChunks = 1024, kVerifyBlocks = 6, kVerifySmall = 16 * 256 * kVerifyBlocks;

struct VerifyDev {
    const void *p, *q;
    const int32_t *draft, *count;
    const float *u, *r;
    int64_t *sums;                             // [n_req][chunks][2]: units of the weights, and of p itself
    int32_t *accepted_ws, *tokens, *accepted;
    int64_t ldp, ldq;
    int32_t n_req, n_draft, vocab, chunks, chunk;
};

__device__ __forceinline__ int64_t units(float w) { return w > 0.0f ? (int64_t)(fminf(w, 1.0f) * kUnits) : 0; }

__device__ __forceinline__ int drafts_of(const VerifyDev &a, int b) {
    return a.count ? min(max(a.count[b], 0), a.n_draft) : a.n_draft;
}

// Number of accepted drafts of request b, by one wavefront: a lane looks at one draft.
template <int VF>
__device__ __forceinline__ int accepted_drafts(const VerifyDev &a, int b, int lane) {
    using T = typename Elem<VF>::T;
    const int n = drafts_of(a, b);
    for (int base = 0; base < n; base += 64) {
        const int i = base + lane;
        bool ok = false;
        if (i < n) {
            const int32_t x = a.draft[(int64_t)b * a.n_draft + i];
            if (x >= 0 && x < a.vocab) {
                const float p = (float)((const T *)a.p)[((int64_t)b * (a.n_draft + 1) + i) * a.ldp + x];
                const float q = a.q ? (float)((const T *)a.q)[((int64_t)b * a.n_draft + i) * a.ldq + x] : 1.0f;
                ok = a.u[(int64_t)b * a.n_draft + i] * q < p;
            }
        }
        const uint64_t refused = ~__ballot(ok);
        const int first = refused ? base + __builtin_ctzll(refused) : base + 64;
        if (first < base + 64) return min(first, n);
    }
    return n;
}

// The row that the next token comes from, and the weight of a token in it.
template <int VF> struct VerifyRow {
    using T = typename Elem<VF>::T;
    const T *p, *q;                            // q null: nothing is taken off, but for `x`
    int32_t x;                                 // >= 0: the refused draft without probabilities, which had all of the mass
    __device__ __forceinline__ VerifyRow(const VerifyDev &a, int b, int accepted) {
        const bool refused = accepted < drafts_of(a, b);
        p = (const T *)a.p + ((int64_t)b * (a.n_draft + 1) + accepted) * a.ldp;
        q = refused && a.q ? (const T *)a.q + ((int64_t)b * a.n_draft + accepted) * a.ldq : nullptr;
        x = refused && !a.q ? a.draft[(int64_t)b * a.n_draft + accepted] : -1;
    }
    // four tokens from v on (zeros past `end`): the weights, p - q (p - 1 at x), and p itself
    __device__ __forceinline__ void at(int32_t v, int32_t end, float *left, float *own) const {
        using T4 = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));  // (rows start at any element)
        T4 pv{}, qv{};
        if (v + 4 <= end) {
            pv = *(const T4 *)(p + v);
            if (q) qv = *(const T4 *)(q + v);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (v + j < end) {
                    pv[j] = p[v + j];
                    if (q) qv[j] = q[v + j];
                }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float off = q ? (float)qv[j] : v + j == x ? 1.0f : 0.0f;
            own[j] = (float)pv[j];
            left[j] = own[j] - off;
        }
    }
    __device__ __forceinline__ void at(int32_t v, int32_t end, int64_t *left, int64_t *own) const {        // ... in units
        float l[4], o[4];
        at(v, end, l, o);
#pragma unroll
        for (int j = 0; j < 4; ++j) { left[j] = units(l[j]); own[j] = units(o[j]); }
    }
};

template <typename N>
__device__ __forceinline__ N wave_sum(N v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// floor(all * floor(r 2^24) / 2^24), which is below `all`: the units that lie before the token drawn.
__device__ __forceinline__ int64_t units_before(int64_t all, float r) {
    const int64_t m = r > 0.0f ? min((int64_t)(fminf(r, 1.0f) * 16777216.0f), (int64_t)16777215) : 0;
    return (all >> 24) * m + (((all & 0xffffff) * m) >> 24);
}

// A wavefront adds up one chunk, 1024 tokens at a time: sixteen to a lane, all of their loads in flight.
template <int VF>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyDev a) {
    const int lane = threadIdx.x & 63;
    const int number = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    const int b = number / a.chunks, c = number % a.chunks;
    if (b >= a.n_req) return;
    const int accepted = accepted_drafts<VF>(a, b, lane);
    const VerifyRow<VF> row(a, b, accepted);
    const int32_t first = c * a.chunk, end = min(first + a.chunk, a.vocab);
    int64_t left = 0, own = 0;
    for (int32_t v = first; v < end; v += 1024) {
        int64_t l[16], o[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) row.at(v + 256 * i + 4 * lane, end, l + 4 * i, o + 4 * i);
#pragma unroll
        for (int i = 0; i < 16; ++i) { left += l[i]; own += o[i]; }
    }
    left = wave_sum(left);
    own = wave_sum(own);
    if (lane == 0) {
        int64_t *to = a.sums + ((int64_t)b * a.chunks + c) * 2;
        to[0] = left;
        to[1] = own;
        if (c == 0) a.accepted_ws[b] = accepted;
    }
}

// Exclusive sum over the workgroup's 256 threads, in thread order; *total: of all.
__device__ __forceinline__ int64_t block_before(int64_t v, int64_t *total, int64_t (*part)) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t upto = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int64_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    __syncthreads();
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += part[w];
        all += part[w];
    }
    *total = all;
    return before + upto - v;
}

template <int VF>
__global__ __launch_bounds__(256) void verify_draw_kernel(const VerifyDev a) {
    __shared__ int64_t part[4], found_before;
    __shared__ int32_t found_chunk, found_token;
    const int b = blockIdx.x, tid = threadIdx.x;
    const int accepted = a.accepted_ws[b];
    const int64_t *sums = a.sums + (int64_t)b * a.chunks * 2;
    const int per = (a.chunks + 255) / 256, c0 = tid * per;    // chunks of this thread
    int64_t mine[2] = {0, 0}, total[2], before[2];
    for (int c = c0; c < min(c0 + per, a.chunks); ++c) { mine[0] += sums[2 * c]; mine[1] += sums[2 * c + 1]; }
    if (tid == 0) { found_chunk = -1; found_token = -1; }
    before[0] = block_before(mine[0], &total[0], part);
    before[1] = block_before(mine[1], &total[1], part);
    const int kind = total[0] > 0 ? 0 : 1;                     // no weight left: p's own
    const int64_t limit = units_before(total[kind], a.r[b]);
    __syncthreads();
    if (before[kind] <= limit && limit < before[kind] + mine[kind]) {          // one thread, if any weight is there
        int64_t s = before[kind];
        for (int c = c0; c < min(c0 + per, a.chunks); ++c) {
            const int64_t w = sums[2 * c + kind];
            if (limit < s + w) { found_chunk = c; found_before = s; break; }
            s += w;
        }
    }
    __syncthreads();
    if (found_chunk >= 0) {                                    // uniform
        const VerifyRow<VF> row(a, b, accepted);
        const int32_t first = found_chunk * a.chunk, end = min(first + a.chunk, a.vocab);
        int64_t before_v = found_before;
        for (int32_t v0 = first; v0 < end; v0 += 1024) {       // four tokens a thread
            const int32_t v = v0 + 4 * tid;
            int64_t w[2][4], all_of_it, sum = 0;
            row.at(v, end, w[0], w[1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                w[0][j] = kind ? w[1][j] : w[0][j];
                sum += w[0][j];
            }
            int64_t s = before_v + block_before(sum, &all_of_it, part);
            if (s <= limit && limit < s + sum)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (s <= limit && limit < s + w[0][j]) found_token = v + j;
                    s += w[0][j];
                }
            before_v += all_of_it;
            if (limit < before_v) break;                       // uniform
        }
        __syncthreads();
    }
    for (int i = tid; i <= a.n_draft; i += 256)
        a.tokens[(int64_t)b * (a.n_draft + 1) + i] = i < accepted ? a.draft[(int64_t)b * a.n_draft + i] : i == accepted ? found_token : -1;
    if (tid == 0) a.accepted[b] = accepted;
}

// One launch for a request: wavefront w of 16 has the `blocks` times 256 tokens from w * blocks * 256 on, four to a lane and block.
// Units are added up as whole numbers of binary64: at most 2^15 of 2^38 each, so every sum is exact (and the code half as long: a launch
// this short waits for its code).
__device__ __forceinline__ double small_units(float w) { return w > 0.0f ? (double)truncf(fminf(w, 1.0f) * kUnits) : 0.0; }
template <int VF>
__global__ __launch_bounds__(1024) void verify_small_kernel(const VerifyDev a, const int32_t blocks) {
    __shared__ double sums[2][16];
    __shared__ int32_t token;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float r = a.r[b];
    const int accepted = accepted_drafts<VF>(a, b, lane);
    const VerifyRow<VF> row(a, b, accepted);
    const int32_t first = wave * blocks * 256 + 4 * lane;
    if (tid == 0) token = -1;
    // the wavefront's units, and all of the workgroup's and those before it
    double mine, all, before;
    auto share = [&](double units, double *sums) {
        mine = wave_sum(units);
        if (lane == 0) sums[wave] = mine;
        __syncthreads();
        all = before = 0.0;
#pragma unroll 4
        for (int v = 0; v < 16; ++v) {
            if (v < wave) before += sums[v];
            all += sums[v];
        }
    };
    {
        float w[kVerifyBlocks][4], own[4];
#pragma unroll
        for (int i = 0; i < kVerifyBlocks; ++i) {              // all loads in flight (four blocks at a time: 11.0 us instead of 8.7 at 20011 tokens)
#pragma unroll
            for (int j = 0; j < 4; ++j) w[i][j] = 0.0f;
            if (i < blocks) row.at(first + 256 * i, a.vocab, w[i], own);
        }
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kVerifyBlocks; ++i)
            if (i < blocks)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += small_units(w[i][j]);
        share(sum, sums[0]);
    }
    const bool own = all <= 0.0;                               // uniform: no weight left, so p's own
    if (own) {
        double sum = 0.0;
#pragma unroll 1
        for (int i = 0; i < blocks; ++i) {
            float l[4], o[4];
            row.at(first + 256 * i, a.vocab, l, o);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += small_units(o[j]);
        }
        share(sum, sums[1]);
    }
    const double limit = (double)units_before((int64_t)all, r), here = mine;
    double s = before;
    if (s <= limit && limit < s + here) {                      // one wavefront, if any weight is there
#pragma unroll 1
        for (int i = 0; i < blocks; ++i) {                     // its blocks once more: they are near
            float l[4], o[4];
            double x[4], sum = 0.0;
            row.at(first + 256 * i, a.vocab, l, o);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] = small_units(own ? o[j] : l[j]);
                sum += x[j];
            }
            double upto = sum;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const double v = __shfl_up(upto, d);
                if (lane >= d) upto += v;
            }
            double at = s + upto - sum;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (at <= limit && limit < at + x[j]) token = first + 256 * i + j;
                at += x[j];
            }
            s += __shfl(upto, 63);
            if (limit < s) break;
        }
    }
    __syncthreads();
    for (int i = tid; i <= a.n_draft; i += 1024)
        a.tokens[(int64_t)b * (a.n_draft + 1) + i] = i < accepted ? a.draft[(int64_t)b * a.n_draft + i] : i == accepted ? token : -1;
    if (tid == 0) a.accepted[b] = accepted;
}

// Tokens of a row that a wavefront of the first launch adds up: 1024, or more where that would make more
// than kVerifyMaxChunks chunks.
static void verify_chunks(int32_t vocab, int32_t *chunks, int32_t *chunk) {
    int64_t c = 1024;
    while ((vocab + c - 1) / c > kVerifyMaxChunks) c *= 2;
    *chunk = (int32_t)c;
    *chunks = (int32_t)((vocab + c - 1) / c);
}

template <int VF>
static void launch_verify(const VerifyDev &d, hipStream_t st) {
    if (d.vocab <= kVerifySmall) {
        hipLaunchKernelGGL(verify_small_kernel<VF>, dim3((uint32_t)d.n_req), dim3(1024), 0, st, d, (d.vocab + 4095) / 4096);
        return;
    }
    hipLaunchKernelGGL(verify_sums_kernel<VF>, dim3(((uint32_t)d.n_req * (uint32_t)d.chunks + 3) / 4), dim3(256), 0, st, d);
    hipLaunchKernelGGL(verify_draw_kernel<VF>, dim3((uint32_t)d.n_req), dim3(256), 0, st, d);
}

}  // namespace csb

extern "C" size_t csb_verify_workspace_bytes(int32_t n_req, int32_t vocab) {
    if (n_req <= 0 || vocab <= 0) return 0;
    int32_t chunks, chunk;
    csb::verify_chunks(vocab, &chunks, &chunk);
    return ((size_t)n_req * ((size_t)chunks * 16 + 4) + 255) / 256 * 256;
}

extern "C" int csb_verify_drafts(int32_t type, const void *d_p, int64_t ldp, const void *d_q, int64_t ldq,
                                 const int32_t *d_draft, const float *d_u, const float *d_r, const int32_t *d_count,
                                 int32_t n_req, int32_t n_draft, int32_t vocab, int32_t *d_tokens, int32_t *d_accepted,
                                 void *d_ws, void *stream) {
    using namespace csb;
    const auto fail = [](int code, const char *what) { set_error(std::string("csb_verify_drafts: ") + what); return code; };
    if (!known_type(type)) return fail(CSB_EINVAL, "unknown type");
    if (n_req < 0 || n_draft < 0 || vocab < 1) return fail(CSB_EINVAL, "bad size");
    if (vocab > 1 << 24) return fail(CSB_EUNSUPPORTED, "vocabulary above 2^24 (its units would pass 63 bits)");
    if (ldp < vocab || (d_q && ldq < vocab)) return fail(CSB_EINVAL, "a leading dimension below the vocabulary");
    if (n_req == 0) return CSB_OK;
    if (!d_p || !d_r || !d_tokens || !d_accepted || !d_ws || (n_draft && (!d_draft || !d_u))) return fail(CSB_EINVAL, "NULL pointer");
    if ((uintptr_t)d_ws % 256) return fail(CSB_EINVAL, "workspace not 256-byte aligned");
    if (((uintptr_t)d_p | (uintptr_t)d_q) % (uintptr_t)type_size(type)) return fail(CSB_EINVAL, "misaligned pointer");
    VerifyDev d{};
    d.p = d_p; d.q = n_draft ? d_q : nullptr; d.draft = d_draft; d.count = d_count; d.u = d_u; d.r = d_r;
    d.ldp = ldp; d.ldq = ldq; d.n_req = n_req; d.n_draft = n_draft; d.vocab = vocab;
    d.tokens = d_tokens; d.accepted = d_accepted;
    verify_chunks(vocab, &d.chunks, &d.chunk);
    if (n_req > 1 << 21 || (int64_t)n_req * d.chunks > kMaxWorkgroups) return fail(CSB_EUNSUPPORTED, "more workgroups than a launch takes");
    d.sums = (int64_t *)d_ws;
    d.accepted_ws = (int32_t *)(d.sums + (size_t)n_req * d.chunks * 2);
    try {
        static const char verify_user = 0;                     // this entry point as a user of workspaces
        workspace_changed_hands(d_ws, &verify_user);
    } catch (const std::bad_alloc &) {
        return fail(CSB_ENOMEM, "out of host memory");
    }
    hipStream_t st = (hipStream_t)stream;
    switch (type) {
        case CSB_VAL_F32: launch_verify<CSB_VAL_F32>(d, st); break;
        case CSB_VAL_F16: launch_verify<CSB_VAL_F16>(d, st); break;
        default: launch_verify<CSB_VAL_BF16>(d, st); break;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) { set_error(std::string("csb_verify_drafts: ") + hipGetErrorString(e)); return CSB_EDEVICE; }
    return CSB_OK;
}
