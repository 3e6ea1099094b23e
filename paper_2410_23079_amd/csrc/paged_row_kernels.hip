// Rows of queries, keys and values on their way: norm and position rotation, into and out of the pages of a paged cache.
//
// What bounds these kernels: every row is read once and written once, some ten operations per element in between:
// memory.  What they have to arrange is that the rest stays small beside that:
//   - angles: one sine and cosine per position and pair, in 64 bits up to the reduction to one turn, shared by all
//     heads.  A block works on 16 positions and several heads, and keeps them in LDS;
//   - a row is handled by as many lanes as it has 16-byte pieces: mean and maximum are sums over neighbouring lanes,
//     and the other half of a pair is a lane away (rot_dim is a multiple of 16, so a piece lies in one half);
//   - values turn around on their way into a page ([row / g][dim][g]): 16 positions are gathered in LDS and leave as
//     whole 16-byte pieces where all g rows of one are new, as single elements where they are not.  Tiles are aligned
//     to 16 positions of the sequence, so that a piece and a page belong to one block, and its page is one number.
#include <math.h>

#include "paged_internal.h"

namespace buzz {
namespace {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTile = kPagedTileTokens, kThreads = 256;

template <int DT> struct Elem;
template <> struct Elem<BUZZ_FP32> { using vec = f32x4; using one = float; };
template <> struct Elem<BUZZ_FP16> { using vec = f16x8_t; using one = _Float16; };
template <> struct Elem<BUZZ_BF16> { using vec = bf16x8_t; using one = __bf16; };

// A lane's 16 bytes of a row as fp32, and back (rounded to nearest even).
template <int DT> struct Piece {
    static constexpr int EB = DT == BUZZ_FP32 ? 4 : 2, N = 16 / EB;
    float x[N];
    __device__ inline void load(const void* p)
    {
        const auto v = *(const typename Elem<DT>::vec*)p;
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)v[i];
    }
    __device__ inline void store(void* p) const
    {
        typename Elem<DT>::vec v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (typename Elem<DT>::one)x[i];
        *(typename Elem<DT>::vec*)p = v;
    }
    // e4m3 codes, 4 to a dword
    __device__ inline void store_codes(void* p, float by) const
    {
        int w[N / 4];
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(finite(x[4 * i]) * by, finite(x[4 * i + 1]) * by, 0, false);
            w[i] = __builtin_amdgcn_cvt_pk_fp8_f32(finite(x[4 * i + 2]) * by, finite(x[4 * i + 3]) * by, w[i], true);
        }
        if constexpr (N == 8) *(i32x2*)p = i32x2{w[0], w[1]};
        else *(int*)p = w[0];
    }
    __device__ inline void load_codes(const void* p, float by)
    {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const int w = ((const int*)p)[i];
            x[4 * i] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * by;
            x[4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * by;
            x[4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * by;
            x[4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * by;
        }
    }
    // the type has no infinity: an infinite value becomes NaN
    __device__ static inline float finite(float v) { return fabsf(v) <= 3.4028234663852886e38f ? v : __builtin_nanf(""); }
};

template <int LPR> __device__ inline float row_sum(float v)
{
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) v += __shfl_xor(v, o);
    return v;
}
template <int LPR> __device__ inline float row_max(float v)
{
#pragma unroll
    for (int o = 1; o < LPR; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

// The exponent byte of a row whose largest finite value is `top`: the least e, 1 .. 254, with top <= 448 * 2^(e - 127).
// 448 = 1.75 * 2^8: the exponent of top less 8, one more if its fraction exceeds 0.75.
__device__ inline int exponent_for(float top)
{
    const unsigned u = __float_as_uint(top);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return e < 1 ? 1 : e;
}
__device__ inline float scale_of(int e) { return __uint_as_float((unsigned)e << 23); }     // 2^(e - 127), e 1 .. 254

template <int DT> __device__ inline float largest_finite(const Piece<DT>& p)
{
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < Piece<DT>::N; ++i) {
        const float v = fabsf(p.x[i]);
        top = fmaxf(top, v <= 3.4028234663852886e38f ? v : 0.f);
    }
    return top;
}

// Sine and cosine of position * inv_freq.  The product and its reduction to [-1/2, 1/2] turns take 64 bits: 2^28 radians
// are right to 2^-25.
__device__ inline float2 turn(int64_t pos, double inv_freq)
{
    const double turns = (double)pos * (inv_freq * 0.15915494309189535);
    float s, c;
    sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
    return make_float2(c, s);
}

// Norm and rotation of a lane's piece of one row: elements e0 .. e0 + N - 1 of D; cs: the position's (cosine, sine) pairs.
template <int DT, int D>
__device__ inline void norm_rotate(const RotateArgs& a, const Piece<DT>& w, bool norm, const float2* cs, int l, Piece<DT>& p)
{
    constexpr int N = Piece<DT>::N, LPR = D / N;
    const int e0 = l * N;
    if (norm) {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) ss = fmaf(p.x[i], p.x[i], ss);
        const float r = 1.0f / sqrtf(row_sum<LPR>(ss) * (1.0f / D) + a.eps);
#pragma unroll
        for (int i = 0; i < N; ++i) p.x[i] = p.x[i] * r * w.x[i];
    }
    if (a.half == 0) return;
    if (a.interleaved) {
        if (e0 < 2 * a.half) {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const float2 t = cs[(e0 + i) / 2];
                const float x = p.x[i], y = p.x[i + 1];
                p.x[i] = x * t.x - y * t.y;
                p.x[i + 1] = y * t.x + x * t.y;
            }
        }
    } else {
        const bool low = e0 < a.half, in = e0 < 2 * a.half;
        const int away = a.half / N, lane = threadIdx.x & 63, other = in ? (low ? lane + away : lane - away) : lane;
        float y[N];
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = __shfl(p.x[i], other);
        if (in) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float2 t = cs[(low ? e0 : e0 - a.half) + i];
                p.x[i] = low ? p.x[i] * t.x - y[i] * t.y : p.x[i] * t.x + y[i] * t.y;
            }
        }
    }
}

// One block: the rows of 16 positions (those of them that are there) of some heads of q, of k or of v.
// E4M3: the pages hold 8 bits.  PAGED: keys and values go to pages.
template <int DT, int D, bool E4M3, bool PAGED>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const RotateArgs a)
{
    using P = Piece<DT>;
    constexpr int N = P::N, LPR = D / N, RPB = kThreads / LPR, PB = E4M3 ? 1 : P::EB, KG = 16 / PB;   // page: bytes of an element, rows of a piece
    constexpr size_t kTurns = kTile * (D / 2) * sizeof(float2), kValues = PAGED ? kTile * D * PB : 0;
    __shared__ alignas(16) char lds[kTurns > kValues ? kTurns : kValues];
    const int tid = threadIdx.x, b = blockIdx.z, l = tid % LPR;
    const Span span = row_span(a.start, a.count, b, a.n_rows);
    const int64_t p0 = (span.start / kTile + blockIdx.x) * kTile;
    const int64_t lo = span.lo > p0 ? span.lo : p0, hi = span.hi < p0 + kTile ? span.hi : p0 + kTile;
    if (lo >= hi) return;
    const int n = (int)(hi - lo);

    // the block's page, and whether there is one
    int64_t page_row = 0;
    bool stored = true;
    const int job = blockIdx.y;
    const bool is_q = job < a.q_jobs, is_v = job >= a.q_jobs + a.k_jobs;
    if constexpr (PAGED) {
        if (!is_q) {
            stored = false;
            if (p0 < (int64_t)a.pages.cols * a.pages.rows) {
                const int pg = page_of(a.pages.table + (int64_t)b * a.pages.cols, p0, a.pages.rows_log2, a.pages.n_pages);
                stored = pg >= 0;
                page_row = (int64_t)pg * a.pages.heads * a.pages.rows + (p0 & (a.pages.rows - 1));   // of head 0
            }
            if (!stored) return;
        }
    }

    if (PAGED && is_v) {
        const int h0 = (job - a.q_jobs - a.k_jobs) * a.kv_chunk, h1 = min(h0 + a.kv_chunk, a.Hkv);
        for (int h = h0; h < h1; ++h) {
            const char* src = a.v.data + (int64_t)b * a.v.seq + (int64_t)h * a.v.head;
            const int64_t at = page_row + (int64_t)h * a.pages.rows;                 // page row of position p0
            for (int r = tid / LPR; r < n; r += RPB) {
                P p;
                p.load(src + (lo - span.start + r) * a.v.row + l * 16);
                char* to = lds + ((int)(lo - p0) + r) * (D * PB) + l * N * PB;
                if constexpr (E4M3) {
                    const int e = exponent_for(row_max<LPR>(largest_finite<DT>(p)));
                    p.store_codes(to, scale_of(254 - e));
                    if (l == 0) a.pages.v_exp[at + (lo - p0) + r] = (uint8_t)e;
                } else {
                    p.store(to);
                }
            }
            __syncthreads();
            const int first = (int)(lo - p0), last = (int)(hi - p0);
            for (int i = tid; i < kTile / KG * D; i += kThreads) {
                const int g = i / D, d = i - g * D;                                  // piece: rows g KG .. of column d
                char* to = a.pages.v + ((at + g * KG) * D + (int64_t)d * KG) * PB;
                const char* from = lds + (g * KG * D + d) * PB;
                if (first <= g * KG && last >= (g + 1) * KG) {
                    alignas(16) char piece[16];
#pragma unroll
                    for (int j = 0; j < KG; ++j) __builtin_memcpy(piece + j * PB, from + j * (D * PB), PB);
                    *(i32x4*)to = *(const i32x4*)piece;
                } else {
                    for (int j = max(first - g * KG, 0); j < min(last - g * KG, KG); ++j) __builtin_memcpy(to + j * PB, from + j * (D * PB), PB);
                }
            }
            __syncthreads();
        }
        return;
    }

    // queries and keys: the positions' angles first
    float2* turns = (float2*)lds;
    for (int i = tid; i < n * a.half; i += kThreads) {
        const int t = i / a.half;
        turns[i] = turn(lo + t, a.inv_freq[i - t * a.half]);
    }
    P w;
    const void* weight = is_q ? a.q_weight : a.k_weight;
    if (weight) w.load((const char*)weight + l * 16);
    __syncthreads();
    const int chunk = is_q ? a.q_chunk : a.kv_chunk, heads = is_q ? a.Hq : a.Hkv;
    const int h0 = (is_q ? job : job - a.q_jobs) * chunk, nh = min(chunk, heads - h0);
    const Rows& in = is_q ? a.q : a.k;
    const Rows& out = is_q ? a.q_out : a.k_out;
    for (int r0 = 0; r0 < n * nh; r0 += RPB) {
        const int r = min(r0 + tid / LPR, n * nh - 1), t = r % n, h = h0 + r / n;     // (lanes of a row beyond the last take part in the sums)
        const int64_t row = lo - span.start + t;
        P p;
        p.load(in.data + (int64_t)b * in.seq + (int64_t)h * in.head + row * in.row + l * 16);
        norm_rotate<DT, D>(a, w, weight != nullptr, turns + t * a.half, l, p);
        if (r0 + tid / LPR >= n * nh) continue;
        if (!PAGED || is_q) {
            p.store(out.data + (int64_t)b * out.seq + (int64_t)h * out.head + row * out.row + l * 16);
        } else {
            const int64_t at = page_row + (int64_t)h * a.pages.rows + (lo - p0) + t;
            char* to = a.pages.k + (at * D + l * N) * PB;
            if constexpr (E4M3) {
                const int e = exponent_for(row_max<LPR>(largest_finite<DT>(p)));
                p.store_codes(to, scale_of(254 - e));
                if (l == 0) a.pages.k_exp[at] = (uint8_t)e;
            } else {
                p.store(to);
            }
        }
    }
}

// The way back: 16 positions of some heads of k or of v.
template <int DT, int D, bool E4M3>
__global__ __launch_bounds__(kThreads) void read_rows_kernel(const ReadArgs a)
{
    using P = Piece<DT>;
    constexpr int N = P::N, LPR = D / N, RPB = kThreads / LPR, PB = E4M3 ? 1 : P::EB, KG = 16 / PB;
    __shared__ alignas(16) char lds[kTile * D * PB];
    const int tid = threadIdx.x, b = blockIdx.z, l = tid % LPR;
    const Span span = row_span(a.start, a.count, b, a.n_rows);
    const int64_t p0 = (span.start / kTile + blockIdx.x) * kTile;
    const int64_t lo = span.lo > p0 ? span.lo : p0, hi = span.hi < p0 + kTile ? span.hi : p0 + kTile;
    if (lo >= hi) return;
    const int n = (int)(hi - lo), first = (int)(lo - p0);
    int pg = -1;
    if (p0 < (int64_t)a.pages.cols * a.pages.rows) pg = page_of(a.pages.table + (int64_t)b * a.pages.cols, p0, a.pages.rows_log2, a.pages.n_pages);
    const int64_t page_row = (int64_t)pg * a.pages.heads * a.pages.rows + (p0 & (a.pages.rows - 1));
    const bool is_v = (int)blockIdx.y >= a.k_jobs;
    const Rows& out = is_v ? a.v : a.k;
    const int h0 = (blockIdx.y - (is_v ? a.k_jobs : 0)) * a.chunk, h1 = min(h0 + a.chunk, a.pages.heads);
    for (int h = h0; h < h1; ++h) {
        const int64_t at = page_row + (int64_t)h * a.pages.rows;
        if (is_v && pg >= 0) {
            for (int i = tid; i < kTile / KG * D; i += kThreads) {
                const int g = i / D, d = i - g * D;
                alignas(16) char piece[16];
                *(i32x4*)piece = *(const i32x4*)(a.pages.v + ((at + g * KG) * D + (int64_t)d * KG) * PB);
#pragma unroll
                for (int j = 0; j < KG; ++j) __builtin_memcpy(lds + ((g * KG + j) * D + d) * PB, piece + j * PB, PB);
            }
            __syncthreads();
        }
        for (int r = tid / LPR; r < n; r += RPB) {
            P p;
            const char* from = is_v ? lds + ((first + r) * D + l * N) * PB : a.pages.k + ((at + first + r) * D + l * N) * PB;
            if (pg < 0) {
#pragma unroll
                for (int i = 0; i < N; ++i) p.x[i] = __builtin_nanf("");
            } else if constexpr (E4M3) {
                p.load_codes(from, scale_of((is_v ? a.pages.v_exp : a.pages.k_exp)[at + first + r]));
            } else {
                p.load(from);
            }
            p.store(out.data + (int64_t)b * out.seq + (int64_t)h * out.head + (lo - span.start + r) * out.row + l * 16);
        }
        if (is_v) __syncthreads();
    }
}

int ceil_div(int a, int b) { return (a + b - 1) / b; }

template <int DT, bool E4M3, bool PAGED> hipError_t launch(const RotateArgs& a, dim3 grid, hipStream_t st)
{
    switch (a.D) {
        case 64: hipLaunchKernelGGL((rotate_rows_kernel<DT, 64, E4M3, PAGED>), grid, dim3(kThreads), 0, st, a); break;
        case 128: hipLaunchKernelGGL((rotate_rows_kernel<DT, 128, E4M3, PAGED>), grid, dim3(kThreads), 0, st, a); break;
        case 256: hipLaunchKernelGGL((rotate_rows_kernel<DT, 256, E4M3, PAGED>), grid, dim3(kThreads), 0, st, a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

template <int DT, bool E4M3> hipError_t launch(const ReadArgs& a, dim3 grid, hipStream_t st)
{
    switch (a.pages.D) {
        case 64: hipLaunchKernelGGL((read_rows_kernel<DT, 64, E4M3>), grid, dim3(kThreads), 0, st, a); break;
        case 128: hipLaunchKernelGGL((read_rows_kernel<DT, 128, E4M3>), grid, dim3(kThreads), 0, st, a); break;
        case 256: hipLaunchKernelGGL((read_rows_kernel<DT, 256, E4M3>), grid, dim3(kThreads), 0, st, a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(int dtype, int page_dtype, const RotateArgs& args, int batch, hipStream_t st)
{
    RotateArgs a = args;
    const bool paged = a.pages.k != nullptr;
    a.q_chunk = 16;
    a.kv_chunk = 8;
    a.q_jobs = a.q.data ? ceil_div(a.Hq, a.q_chunk) : 0;
    a.k_jobs = a.k.data ? ceil_div(a.Hkv, a.kv_chunk) : 0;
    a.v_jobs = paged && a.v.data ? ceil_div(a.Hkv, a.kv_chunk) : 0;
    const dim3 grid((unsigned)tiles_of_rows(a.n_rows), a.q_jobs + a.k_jobs + a.v_jobs, batch);
    if (grid.x == 0 || grid.y == 0 || grid.z == 0) return hipSuccess;
    if (!paged) {
        switch (dtype) {
            case BUZZ_FP32: return launch<BUZZ_FP32, false, false>(a, grid, st);
            case BUZZ_FP16: return launch<BUZZ_FP16, false, false>(a, grid, st);
            case BUZZ_BF16: return launch<BUZZ_BF16, false, false>(a, grid, st);
        }
        return hipErrorInvalidValue;
    }
    const bool e4m3 = page_dtype == BUZZ_E4M3;
    switch (dtype) {
        case BUZZ_FP32: return launch<BUZZ_FP32, false, true>(a, grid, st);
        case BUZZ_FP16: return e4m3 ? launch<BUZZ_FP16, true, true>(a, grid, st) : launch<BUZZ_FP16, false, true>(a, grid, st);
        case BUZZ_BF16: return e4m3 ? launch<BUZZ_BF16, true, true>(a, grid, st) : launch<BUZZ_BF16, false, true>(a, grid, st);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_paged_read(int dtype, int page_dtype, const ReadArgs& args, int batch, hipStream_t st)
{
    ReadArgs a = args;
    a.chunk = 8;
    a.k_jobs = a.k.data ? ceil_div(a.pages.heads, a.chunk) : 0;
    a.v_jobs = a.v.data ? ceil_div(a.pages.heads, a.chunk) : 0;
    const dim3 grid((unsigned)tiles_of_rows(a.n_rows), a.k_jobs + a.v_jobs, batch);
    if (grid.x == 0 || grid.y == 0 || grid.z == 0) return hipSuccess;
    const bool e4m3 = page_dtype == BUZZ_E4M3;
    switch (dtype) {
        case BUZZ_FP32: return launch<BUZZ_FP32, false>(a, grid, st);
        case BUZZ_FP16: return e4m3 ? launch<BUZZ_FP16, true>(a, grid, st) : launch<BUZZ_FP16, false>(a, grid, st);
        case BUZZ_BF16: return e4m3 ? launch<BUZZ_BF16, true>(a, grid, st) : launch<BUZZ_BF16, false>(a, grid, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace buzz
