// Rows of queries, keys and values on their way: norm and position rotation, into and out of the pages of a paged cache.
//
// What bounds these kernels: every row is read once and written once, some ten operations per element in between:
// memory.  What they have to arrange is that the rest stays small beside that:
//   - a block works on 16 positions and some heads, a row on as many lanes as it has 16-byte pieces: mean and maximum are
//     sums over neighbouring lanes.  Of a row that is rotated a lane takes both elements of its pairs (8 bytes from either
//     half), and it stays with one position while it goes through the heads: sines and cosines are made once, in
//     registers, and nothing is exchanged between lanes;
//   - angles: 64 bits up to the reduction to one turn;
//   - values turn around on their way into a page ([row / g][dim][g]): a lane gathers the rows that share a dword there,
//     the dwords of 16 positions meet in LDS and leave as whole 16-byte pieces where all g rows of one are new, as single
//     elements where they are not.  Tiles are aligned to 16 positions of the sequence, so that a piece and a page belong
//     to one block, and its page is one number.
// Measured (a call in a captured graph): 32768 tokens of 32 + 8 bf16 heads of 128 turned 137 us, 4.9 TB/s read and written, of
// which a copy of these bytes takes 123; up to 8192 tokens of four sequences, the same heads into 8-bit pages, 107, and back 28;
// 131072 tokens of 8 heads out of 8-bit pages 150 us, 5.4 TB/s; one token of 8 sequences 4.0 us.
// 32 bits up to the rounding to 8: of 33 million codes some 38 are a neighbour of the exact value's.  In 64 bits it is 11, but
// a SIMD then holds two waves instead of four and the call takes 20% longer.
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
constexpr int kHeads = 4;                  // rows that a lane asks for at a time

template <int DT> struct Elem;
template <> struct Elem<BUZZ_FP32> { using vec = f32x4; using one = float; };
template <> struct Elem<BUZZ_FP16> { using vec = f16x8_t; using one = _Float16; };
template <> struct Elem<BUZZ_BF16> { using vec = bf16x8_t; using one = __bf16; };

// 16 bytes of a row as fp32: N elements, from one place or half from each of two; back rounded to nearest even.
template <int DT> struct Piece {
    static constexpr int EB = DT == BUZZ_FP32 ? 4 : 2, N = 16 / EB, HN = N / 2;
    float x[N];
    __device__ inline void from(i32x4 raw)
    {
        const auto v = __builtin_bit_cast(typename Elem<DT>::vec, raw);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (float)v[i];
    }
    __device__ inline i32x4 to() const
    {
        typename Elem<DT>::vec v;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = (typename Elem<DT>::one)x[i];
        return __builtin_bit_cast(i32x4, v);
    }
    // e4m3 codes of 4 elements from number i on
    __device__ inline int codes(int i, float by) const
    {
        const int w = __builtin_amdgcn_cvt_pk_fp8_f32(finite(x[i]) * by, finite(x[i + 1]) * by, 0, false);
        return __builtin_amdgcn_cvt_pk_fp8_f32(finite(x[i + 2]) * by, finite(x[i + 3]) * by, w, true);
    }
    __device__ inline void from_codes(int i, int w, float by)
    {
        x[i] = __builtin_amdgcn_cvt_f32_fp8(w, 0) * by;
        x[i + 1] = __builtin_amdgcn_cvt_f32_fp8(w, 1) * by;
        x[i + 2] = __builtin_amdgcn_cvt_f32_fp8(w, 2) * by;
        x[i + 3] = __builtin_amdgcn_cvt_f32_fp8(w, 3) * by;
    }
    // the type has no infinity: an infinite value becomes NaN
    __device__ static inline float finite(float v) { return fabsf(v) <= 3.4028234663852886e38f ? v : __builtin_nanf(""); }
};
__device__ inline i32x4 load16(const char* p) { return *(const i32x4*)p; }
// PAST: the caches of the dies would not hold what the call writes until it is read; past them it takes 3 to 27% less time
// (32768 tokens of 48 heads 138 -> 132 us, 16384 tokens of 8 heads out of 16-bit pages 28 -> 22).
template <bool PAST> __device__ inline void store16(char* p, i32x4 v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, (i32x4*)p);
    else *(i32x4*)p = v;
}
__device__ inline i32x2 load8(const char* p) { return *(const i32x2*)p; }
template <bool PAST> __device__ inline void store8(char* p, i32x2 v)
{
    if constexpr (PAST) __builtin_nontemporal_store(v, (i32x2*)p);
    else *(i32x2*)p = v;
}
__device__ inline i32x4 load8x2(const char* p, const char* q)
{
    const i32x2 x = load8(p), y = load8(q);
    return i32x4{x[0], x[1], y[0], y[1]};
}
template <bool PAST> __device__ inline void store8x2(char* p, char* q, i32x4 v)
{
    store8<PAST>(p, i32x2{v[0], v[1]});
    store8<PAST>(q, i32x2{v[2], v[3]});
}

// op over the LPR neighbouring lanes of a row, in all of them
template <int CTRL> __device__ inline float dpp(float v) { return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, false)); }
template <int LPR, class Op> __device__ inline float over_row(float v, Op op)
{
    v = op(v, dpp<0xB1>(v));               // quads: the lane 1 away, 2 away
    v = op(v, dpp<0x4E>(v));
    if constexpr (LPR >= 8) v = op(v, dpp<0x141>(v));      // the other quad of 8 lanes
    if constexpr (LPR >= 16) v = op(v, dpp<0x140>(v));     // the other half of 16
    if constexpr (LPR >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    if constexpr (LPR >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(r[0]), __uint_as_float(r[1]));
    }
    return v;
}
template <int LPR> __device__ inline float row_sum(float v) { return over_row<LPR>(v, [](float x, float y) { return x + y; }); }
template <int LPR> __device__ inline float row_max(float v) { return over_row<LPR>(v, [](float x, float y) { return fmaxf(x, y); }); }

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

// Sine and cosine of position * inv_freq, the latter given in turns.  The product and its reduction to an eighth of a turn take
// 64 bits: 2^28 radians are right to 2^-25.  What is left, at most pi / 4, goes into the first terms of the two power series: the
// next ones are 2e-9 and 5e-10 at most.
__device__ inline float2 turn(int64_t pos, double freq)
{
    const double t = (double)pos * freq, quarters = rint(t * 4.0);
    const float x = (float)(t - quarters * 0.25) * 6.2831853071795865f, y = x * x;
    const int k = (int)(quarters - rint(quarters * 0.25) * 4.0);       // -2 .. 2
    const float s = x * fmaf(y, fmaf(y, fmaf(y, fmaf(y, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
    const float c = fmaf(y, fmaf(y, fmaf(y, fmaf(y, fmaf(y, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
    const float u = k & 1 ? s : c, v = k & 1 ? c : s;                  // a quarter turn on, (cos, sin) is (-sin, cos)
    return make_float2((k + 1) & 2 ? -u : u, k & 2 ? -v : v);
}

// What of a block's 16 positions from p0 on a call handles, and the page they lie on.
struct TileSpan {
    int64_t p0, lo, hi, row;               // positions [lo, hi); row: of the caller's, of position p0
    __device__ inline TileSpan(const int32_t* start, const int32_t* count, int b, int64_t n_rows, int tile)
    {
        const Span span = row_span(start, count, b, n_rows);
        p0 = (span.start / kTile + tile) * kTile;
        lo = span.lo > p0 ? span.lo : p0;
        hi = span.hi < p0 + kTile ? span.hi : p0 + kTile;
        row = p0 - span.start;
    }
    __device__ inline int32_t page(const PageArgs& a, int b) const
    {
        return p0 < (int64_t)a.cols * a.rows ? page_of(a.table + (int64_t)b * a.cols, p0, a.rows_log2, a.n_pages) : -1;
    }
};

// The row of the pool that a tile's position p0 has in head 0 of page pg (-1: none, and the result is not to be used).
__device__ inline int64_t page_row(const PageArgs& a, const TileSpan& tile, int32_t pg)
{
    return (int64_t)pg * a.heads * a.rows + (tile.p0 & (a.rows - 1));
}

// How values share dwords in a page: T rows to one, so that a lane gathers T rows of its N columns.
template <int DT, int D, bool E4M3> struct ValueTile {
    using P = Piece<DT>;
    static constexpr int PB = E4M3 ? 1 : P::EB, T = 4 / PB, KG = 16 / PB;
    static constexpr int LPR = D / P::N, ROWS = kThreads / LPR;       // rows of dwords that the block's threads make at a time
    static constexpr int TG = kTile / T;                              // ... and a head has
    static constexpr int HEADS = ROWS > TG ? ROWS / TG : 1;           // heads at a time
    static constexpr int LDS = HEADS * TG * D * 4;
};

// Heads h0 .. h1 - 1 of v: 16 positions of each into page pg.
template <int DT, int D, bool E4M3, bool PAST>
__device__ inline void store_values(const RotateArgs& a, const TileSpan& tile, int b, int h0, int h1, int32_t pg, char* lds)
{
    using P = Piece<DT>;
    using V = ValueTile<DT, D, E4M3>;
    constexpr int N = P::N, T = V::T;
    const int tid = threadIdx.x, l = tid % V::LPR, first = (int)(tile.lo - tile.p0), last = (int)(tile.hi - tile.p0);
    const int64_t at0 = page_row(a.pages, tile, pg);
    for (int h = h0; h < h1; h += V::HEADS) {
        for (int r = tid / V::LPR; r < V::HEADS * V::TG; r += V::ROWS) {
            const int t = r % V::TG, hh = h + r / V::TG;
            if (hh >= h1 || t * T >= last || t * T + T <= first) continue;
            const char* src = a.v.data + (int64_t)b * a.v.seq + (int64_t)hh * a.v.head + l * 16;
            i32x4 raw[T];
#pragma unroll
            for (int j = 0; j < T; ++j) raw[j] = load16(src + (tile.row + min(max(t * T + j, first), last - 1)) * a.v.row);
            int w[N];
            if constexpr (E4M3) {
                int c[T][2];
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    P p;
                    p.from(raw[j]);
                    const int e = exponent_for(row_max<V::LPR>(largest_finite<DT>(p)));
                    c[j][0] = p.codes(0, scale_of(254 - e));
                    c[j][1] = p.codes(4, scale_of(254 - e));
                    const int row = t * T + j;
                    if (l == 0 && row >= first && row < last && pg >= 0) a.pages.v_exp[at0 + (int64_t)hh * a.pages.rows + row] = (uint8_t)e;
                }
                // byte i of dwords 0 .. 3 to bytes 0 .. 3 of dword i
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const unsigned x = __builtin_amdgcn_perm(c[1][k], c[0][k], 0x05010400), y = __builtin_amdgcn_perm(c[1][k], c[0][k], 0x07030602);
                    const unsigned u = __builtin_amdgcn_perm(c[3][k], c[2][k], 0x05010400), v = __builtin_amdgcn_perm(c[3][k], c[2][k], 0x07030602);
                    w[4 * k] = __builtin_amdgcn_perm(u, x, 0x05040100);
                    w[4 * k + 1] = __builtin_amdgcn_perm(u, x, 0x07060302);
                    w[4 * k + 2] = __builtin_amdgcn_perm(v, y, 0x05040100);
                    w[4 * k + 3] = __builtin_amdgcn_perm(v, y, 0x07060302);
                }
            } else if constexpr (T == 2) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[2 * i] = __builtin_amdgcn_perm(raw[1][i], raw[0][i], 0x05040100);
                    w[2 * i + 1] = __builtin_amdgcn_perm(raw[1][i], raw[0][i], 0x07060302);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = raw[0][i];
            }
            i32x4* to = (i32x4*)(lds + (r * D + l * N) * 4);
#pragma unroll
            for (int i = 0; i < N / 4; ++i) to[i] = i32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
        }
        __syncthreads();
        if (pg < 0) return;
        constexpr int G = kTile / V::KG;               // 16-byte pieces of a column
        for (int i = tid; i < V::HEADS * G * D; i += kThreads) {
            const int d = i % D, g = i / D % G, hd = i / (G * D), hh = h + hd;
            if (hh >= h1) break;
            const int* from = (const int*)lds + (hd * V::TG + g * 4) * D + d;
            const i32x4 piece = {from[0], from[D], from[2 * D], from[3 * D]};
            char* to = a.pages.v + ((at0 + (int64_t)hh * a.pages.rows + g * V::KG) * D + (int64_t)d * V::KG) * V::PB;
            if (first <= g * V::KG && last >= (g + 1) * V::KG) {
                store16<PAST>(to, piece);
            } else {
#pragma unroll
                for (int j = 0; j < V::KG; ++j) {
                    if (g * V::KG + j < first || g * V::KG + j >= last) continue;
                    const int w = piece[j * V::PB / 4] >> (j * V::PB % 4 * 8);
                    if constexpr (V::PB == 4) *(int*)(to + j * 4) = w;
                    else if constexpr (V::PB == 2) *(uint16_t*)(to + j * 2) = (uint16_t)w;
                    else *(uint8_t*)(to + j) = (uint8_t)w;
                }
            }
        }
        __syncthreads();
    }
}

// One block: the rows of 16 positions (those of them that are there) of some heads of q, of k or of v.
// E4M3: the pages hold 8 bits.  PAGED: keys and values go to pages.
template <int DT, int D, bool E4M3, bool PAGED, bool PAST>
__global__ __launch_bounds__(kThreads) void rotate_rows_kernel(const RotateArgs a)
{
    using P = Piece<DT>;
    constexpr int N = P::N, HN = P::HN, LPR = D / N, ROWS = kThreads / LPR, PB = E4M3 ? 1 : P::EB;
    __shared__ alignas(16) char lds[PAGED ? ValueTile<DT, D, E4M3>::LDS : 16];
    const int tid = threadIdx.x, b = blockIdx.z, l = tid % LPR, job = blockIdx.y;
    const TileSpan tile(a.start, a.count, b, a.n_rows, blockIdx.x);
    if (tile.lo >= tile.hi) return;
    const bool is_q = job < a.q_jobs;
    // The page, if there is one (rows without are dropped), is waited for only where something is stored.
    int32_t pg = -1;
    if constexpr (PAGED) {
        if (!is_q) pg = tile.page(a.pages, b);
        if (job >= a.q_jobs + a.k_jobs) {
            const int h0 = (job - a.q_jobs - a.k_jobs) * a.v_chunk;
            store_values<DT, D, E4M3, PAST>(a, tile, b, h0, min(h0 + a.v_chunk, a.Hkv), pg, lds);
            return;
        }
    }

    // A lane's elements: HN from o1 on and HN from o2 on, HN pairs; the pairs' turns are numbers p .. of the rotation's.
    const int p = l * HN, rot = 2 * a.half;
    const bool turns = p < a.half;
    int o1, o2;
    if (a.interleaved) { o1 = l * N; o2 = o1 + HN; }
    else if (turns) { o1 = p; o2 = p + a.half; }
    else { o1 = rot + (p - a.half); o2 = o1 + (D - rot) / 2; }
    const char* weight = (const char*)(is_q ? a.q_weight : a.k_weight);
    P w;
    if (weight) w.from(load8x2(weight + o1 * P::EB, weight + o2 * P::EB));
    double freq[HN];
#pragma unroll
    for (int i = 0; i < HN; ++i) freq[i] = turns ? a.inv_freq[p + i] * 0.15915494309189535 : 0.0;    // turns per position

    const int chunk = is_q ? a.q_chunk : a.kv_chunk, heads = is_q ? a.Hq : a.Hkv;
    const int h0 = (is_q ? job : job - a.q_jobs) * chunk, h1 = min(h0 + chunk, heads);
    const Rows& in = is_q ? a.q : a.k;
    const Rows& out = is_q ? a.q_out : a.k_out;
    const int n = (int)(tile.hi - tile.lo), slot = tid / LPR;
    const int step = ROWS >= n ? ROWS / n : 1;         // heads that the rows of threads take side by side
    for (int t = slot % n; t < n; t += ROWS) {         // (ROWS >= n: once)
        const int64_t pos = tile.lo + t, row = tile.row + (pos - tile.p0);
        if (ROWS >= n && slot >= step * n) break;
        int h = h0 + (ROWS >= n ? slot / n : 0);
        const char* x1 = in.data + (int64_t)b * in.seq + row * in.row + (int64_t)h * in.head + o1 * P::EB;
        const int64_t ahead = (int64_t)step * in.head, apart = (int64_t)(o2 - o1) * P::EB;
        i32x4 raw[kHeads] = {};            // of several heads at a time: one after the other, each would wait for memory
        auto request = [&]() {
#pragma unroll
            for (int u = 0; u < kHeads; ++u, x1 += ahead)
                if (h + u * step < h1) raw[u] = load8x2(x1, x1 + apart);
        };
        request();
        // What the pairs are multiplied with, weights included: (x1 a1 - x2 b1, x2 a2 + x1 b2).
        float a1[HN], a2[HN], b1[HN], b2[HN];
#pragma unroll
        for (int i = 0; i < HN; ++i) {
            const float2 cs = turns ? turn(pos, freq[i]) : make_float2(1.f, 0.f);
            const float w1 = weight ? (a.interleaved ? w.x[2 * i] : w.x[i]) : 1.f, w2 = weight ? (a.interleaved ? w.x[2 * i + 1] : w.x[HN + i]) : 1.f;
            a1[i] = w1 * cs.x; b1[i] = w2 * cs.y;
            a2[i] = w2 * cs.x; b2[i] = w1 * cs.y;
        }
        const bool to_page = PAGED && !is_q;
        const int64_t at = to_page ? page_row(a.pages, tile, pg) + (int64_t)h * a.pages.rows + (pos - tile.p0) : 0;
        char* y1 = to_page ? a.pages.k + at * (D * PB) + o1 * PB : out.data + (int64_t)b * out.seq + row * out.row + (int64_t)h * out.head + o1 * P::EB;
        const int64_t y_ahead = to_page ? (int64_t)step * a.pages.rows * (D * PB) : (int64_t)step * out.head;
        if (to_page && pg < 0) break;      // nowhere to store
        uint8_t* exps = E4M3 && to_page ? a.pages.k_exp + at : nullptr;
        for (; h < h1; h += kHeads * step, request()) {
#pragma unroll
            for (int u = 0; u < kHeads; ++u, y1 += y_ahead) {
                if (h + u * step >= h1) break;
                P x;
                x.from(raw[u]);
                float r = 1.f;
                if (weight) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < N; ++i) ss = fmaf(x.x[i], x.x[i], ss);
                    const float m = row_sum<LPR>(ss) * (1.0f / D) + a.eps;
                    r = rsqrtf(m);
                    const float off = fmaf(-m * r, r, 1.f);            // (its last bit is every element's: one step of Newton's)
                    if (off < 1.f) r = fmaf(0.5f * r, off, r);         // (m 0, tiny or infinite: as it is)
                }
#pragma unroll
                for (int i = 0; i < HN; ++i) {
                    float& u1 = a.interleaved ? x.x[2 * i] : x.x[i];
                    float& u2 = a.interleaved ? x.x[2 * i + 1] : x.x[HN + i];
                    const float v1 = u1, v2 = u2;
                    // (where nothing turns, the other element must not come in even with a weight of 0: it may be infinite)
                    u1 = (turns ? fmaf(v1, a1[i], -(v2 * b1[i])) : v1 * a1[i]) * r;
                    u2 = (turns ? fmaf(v2, a2[i], v1 * b2[i]) : v2 * a2[i]) * r;
                }
                if (E4M3 && to_page) {
                    const int e = exponent_for(row_max<LPR>(largest_finite<DT>(x)));
                    *(int*)y1 = x.codes(0, scale_of(254 - e));
                    *(int*)(y1 + (o2 - o1)) = x.codes(N == 8 ? 4 : 0, scale_of(254 - e));
                    if (l == 0) *exps = (uint8_t)e;
                    exps += step * a.pages.rows;
                } else {
                    store8x2<PAST>(y1, y1 + apart, x.to());
                }
            }
        }
    }
}

// The way back: 16 positions of some heads of k or of v.
template <int DT, int D, bool E4M3, bool PAST>
__global__ __launch_bounds__(kThreads) void read_rows_kernel(const ReadArgs a)
{
    using P = Piece<DT>;
    using V = ValueTile<DT, D, E4M3>;
    constexpr int N = P::N, LPR = D / N, ROWS = kThreads / LPR, PB = V::PB, T = V::T;
    __shared__ alignas(16) char lds[V::LDS];
    const int tid = threadIdx.x, b = blockIdx.z, l = tid % LPR, job = blockIdx.y;
    const TileSpan tile(a.start, a.count, b, a.n_rows, blockIdx.x);
    if (tile.lo >= tile.hi) return;
    const int first = (int)(tile.lo - tile.p0), last = (int)(tile.hi - tile.p0), n = last - first;
    const int32_t pg = tile.page(a.pages, b);
    const int64_t at0 = page_row(a.pages, tile, pg);
    const bool is_v = job >= a.k_jobs;
    const Rows& out = is_v ? a.v : a.k;
    const int h0 = (job - (is_v ? a.k_jobs : 0)) * a.chunk, h1 = min(h0 + a.chunk, a.pages.heads);
    char* const dst = out.data + (int64_t)b * out.seq + tile.row * out.row + l * 16;

    if (pg < 0) {                          // no page: NaN
        P p;
#pragma unroll
        for (int i = 0; i < N; ++i) p.x[i] = __builtin_nanf("");
        for (int r = tid / LPR; r < n * (h1 - h0); r += ROWS) store16<PAST>(dst + (int64_t)(h0 + r / n) * out.head + (first + r % n) * out.row, p.to());
        return;
    }
    if (!is_v) {
        const char* src = a.pages.k + at0 * (D * PB) + l * N * PB;
        for (int r0 = tid / LPR; r0 < n * (h1 - h0); r0 += kHeads * ROWS) {
            i32x4 raw[kHeads];
            uint8_t e[kHeads];
#pragma unroll
            for (int u = 0; u < kHeads; ++u) {
                const int r = min(r0 + u * ROWS, n * (h1 - h0) - 1);
                const int64_t at = (int64_t)(h0 + r / n) * a.pages.rows + first + r % n;
                if constexpr (E4M3) {
                    const i32x2 x = load8(src + at * D);
                    raw[u] = i32x4{x[0], x[1], 0, 0};
                    e[u] = a.pages.k_exp[at0 + at];
                } else {
                    raw[u] = load16(src + at * (D * PB));
                }
            }
#pragma unroll
            for (int u = 0; u < kHeads; ++u) {
                const int r = r0 + u * ROWS;
                if (r >= n * (h1 - h0)) break;
                char* to = dst + (int64_t)(h0 + r / n) * out.head + (first + r % n) * out.row;
                if constexpr (E4M3) {
                    P p;
                    p.from_codes(0, raw[u][0], scale_of(e[u]));
                    p.from_codes(4, raw[u][1], scale_of(e[u]));
                    store16<PAST>(to, p.to());
                } else {
                    store16<PAST>(to, raw[u]);
                }
            }
        }
        return;
    }
    constexpr int G = kTile / V::KG;
    for (int h = h0; h < h1; h += V::HEADS) {
        for (int i = tid; i < V::HEADS * G * D; i += kThreads) {
            const int d = i % D, g = i / D % G, hd = i / (G * D), hh = h + hd;
            if (hh >= h1) break;
            const i32x4 piece = load16(a.pages.v + ((at0 + (int64_t)hh * a.pages.rows + g * V::KG) * D + (int64_t)d * V::KG) * PB);
            int* to = (int*)lds + (hd * V::TG + g * 4) * D + d;
#pragma unroll
            for (int j = 0; j < 4; ++j) to[j * D] = piece[j];
        }
        __syncthreads();
        for (int r = tid / LPR; r < V::HEADS * V::TG; r += ROWS) {
            const int t = r % V::TG, hh = h + r / V::TG;
            if (hh >= h1) break;
            const i32x4* from = (const i32x4*)(lds + (r * D + l * N) * 4);
            int w[N];
#pragma unroll
            for (int i = 0; i < N / 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) w[4 * i + j] = from[i][j];
#pragma unroll
            for (int j = 0; j < T; ++j) {
                const int row = t * T + j;
                if (row < first || row >= last) continue;
                char* to = dst + (int64_t)hh * out.head + row * out.row;
                if constexpr (E4M3) {
                    P p;
                    const float by = scale_of(a.pages.v_exp[at0 + (int64_t)hh * a.pages.rows + row]);
#pragma unroll
                    for (int i = 0; i < N; ++i) p.x[i] = __builtin_amdgcn_cvt_f32_fp8((unsigned)w[i] >> (8 * j), 0) * by;
                    store16<PAST>(to, p.to());
                } else if constexpr (T == 2) {
                    const unsigned pick = j ? 0x07060302 : 0x05040100;
                    store16<PAST>(to, i32x4{(int)__builtin_amdgcn_perm(w[1], w[0], pick), (int)__builtin_amdgcn_perm(w[3], w[2], pick),
                                      (int)__builtin_amdgcn_perm(w[5], w[4], pick), (int)__builtin_amdgcn_perm(w[7], w[6], pick)});
                } else {
                    store16<PAST>(to, i32x4{w[0], w[1], w[2], w[3]});
                }
            }
        }
        __syncthreads();
    }
}

// Heads per block, of `heads` at `tiles` tiles: one tile's rows fill a block's threads `full` heads at a time; from there on as
// many more as leave so many blocks, up to 16 (the angles are made once for all of them).
constexpr int kMostHeads = 16;
int heads_per_block(int64_t tiles, int heads, int full, int blocks)
{
    int64_t chunk = tiles * heads / blocks;
    if (chunk > kMostHeads) chunk = kMostHeads;
    return (int)(chunk < full ? full : chunk);
}
// ... how many heads fill the threads with n_rows rows each
int heads_side_by_side(int dtype, int D, int64_t n_rows)
{
    const int rows = kThreads / (D / (dtype == BUZZ_FP32 ? 4 : 8)), n = n_rows < kTile ? (int)n_rows : kTile;
    return rows > n ? rows / n : 1;
}

// ... and how many heads of values (ValueTile::HEADS)
int values_side_by_side(int dtype, int page_dtype, int D)
{
    const int rows = kThreads / (D / (dtype == BUZZ_FP32 ? 4 : 8)), groups = page_dtype == BUZZ_E4M3 ? 4 : dtype == BUZZ_FP32 ? 16 : 8;
    return rows > groups ? rows / groups : 1;
}

// Whether a call writes more than the caches of the dies are good for (32 MB together, and others use them).
bool writes_past(int64_t rows, int batch, int heads, int row_bytes) { return (double)rows * batch * heads * row_bytes > 8.0e6; }

int ceil_div(int a, int b) { return (a + b - 1) / b; }

template <int DT, int D, bool E4M3, bool PAGED> hipError_t launch_d(const RotateArgs& a, dim3 grid, bool past, hipStream_t st)
{
    if (past) hipLaunchKernelGGL((rotate_rows_kernel<DT, D, E4M3, PAGED, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((rotate_rows_kernel<DT, D, E4M3, PAGED, false>), grid, dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

template <int DT, bool E4M3, bool PAGED> hipError_t launch(const RotateArgs& a, dim3 grid, bool past, hipStream_t st)
{
    switch (a.D) {
        case 64: return launch_d<DT, 64, E4M3, PAGED>(a, grid, past, st);
        case 128: return launch_d<DT, 128, E4M3, PAGED>(a, grid, past, st);
        case 256: return launch_d<DT, 256, E4M3, PAGED>(a, grid, past, st);
    }
    return hipErrorInvalidValue;
}

template <int DT, int D, bool E4M3> hipError_t launch_d(const ReadArgs& a, dim3 grid, bool past, hipStream_t st)
{
    if (past) hipLaunchKernelGGL((read_rows_kernel<DT, D, E4M3, true>), grid, dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((read_rows_kernel<DT, D, E4M3, false>), grid, dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

template <int DT, bool E4M3> hipError_t launch(const ReadArgs& a, dim3 grid, bool past, hipStream_t st)
{
    switch (a.pages.D) {
        case 64: return launch_d<DT, 64, E4M3>(a, grid, past, st);
        case 128: return launch_d<DT, 128, E4M3>(a, grid, past, st);
        case 256: return launch_d<DT, 256, E4M3>(a, grid, past, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_rotate(int dtype, int page_dtype, const RotateArgs& args, int batch, hipStream_t st)
{
    RotateArgs a = args;
    const bool paged = a.pages.k != nullptr;
    const int64_t tiles = tiles_of_rows(a.n_rows) * batch;
    const int full = heads_side_by_side(dtype, a.D, a.n_rows), all = (a.q.data ? a.Hq : 0) + (a.k.data ? a.Hkv : 0) + (paged ? a.Hkv : 0);
    a.q_chunk = a.kv_chunk = heads_per_block(tiles, all, full, 512);
    const bool past = writes_past(a.n_rows, batch, all, a.D * (dtype == BUZZ_FP32 ? 4 : 2));
    const int at_once = values_side_by_side(dtype, page_dtype, a.D);
    a.v_chunk = (heads_per_block(tiles, all, at_once, 512) + at_once - 1) / at_once * at_once;
    a.q_jobs = a.q.data ? ceil_div(a.Hq, a.q_chunk) : 0;
    a.k_jobs = a.k.data ? ceil_div(a.Hkv, a.kv_chunk) : 0;
    a.v_jobs = paged && a.v.data ? ceil_div(a.Hkv, a.v_chunk) : 0;
    // (the tiles of one job one after the other: what they write is contiguous. The other way round, a third more time for reads)
    const dim3 grid((unsigned)tiles_of_rows(a.n_rows), a.q_jobs + a.k_jobs + a.v_jobs, batch);
    if (grid.x == 0 || grid.y == 0 || grid.z == 0) return hipSuccess;
    if (!paged) {
        switch (dtype) {
            case BUZZ_FP32: return launch<BUZZ_FP32, false, false>(a, grid, past, st);
            case BUZZ_FP16: return launch<BUZZ_FP16, false, false>(a, grid, past, st);
            case BUZZ_BF16: return launch<BUZZ_BF16, false, false>(a, grid, past, st);
        }
        return hipErrorInvalidValue;
    }
    const bool e4m3 = page_dtype == BUZZ_E4M3;
    switch (dtype) {
        case BUZZ_FP32: return launch<BUZZ_FP32, false, true>(a, grid, past, st);
        case BUZZ_FP16: return e4m3 ? launch<BUZZ_FP16, true, true>(a, grid, past, st) : launch<BUZZ_FP16, false, true>(a, grid, past, st);
        case BUZZ_BF16: return e4m3 ? launch<BUZZ_BF16, true, true>(a, grid, past, st) : launch<BUZZ_BF16, false, true>(a, grid, past, st);
    }
    return hipErrorInvalidValue;
}

hipError_t launch_paged_read(int dtype, int page_dtype, const ReadArgs& args, int batch, hipStream_t st)
{
    ReadArgs a = args;
    a.chunk = heads_per_block(tiles_of_rows(a.n_rows) * batch, 2 * a.pages.heads, heads_side_by_side(dtype, a.pages.D, a.n_rows), 2048);
    const bool past = writes_past(a.n_rows, batch, 2 * a.pages.heads, a.pages.D * (dtype == BUZZ_FP32 ? 4 : 2));
    a.k_jobs = a.k.data ? ceil_div(a.pages.heads, a.chunk) : 0;
    a.v_jobs = a.v.data ? ceil_div(a.pages.heads, a.chunk) : 0;
    const dim3 grid((unsigned)tiles_of_rows(a.n_rows), a.k_jobs + a.v_jobs, batch);
    if (grid.x == 0 || grid.y == 0 || grid.z == 0) return hipSuccess;
    const bool e4m3 = page_dtype == BUZZ_E4M3;
    switch (dtype) {
        case BUZZ_FP32: return launch<BUZZ_FP32, false>(a, grid, past, st);
        case BUZZ_FP16: return e4m3 ? launch<BUZZ_FP16, true>(a, grid, past, st) : launch<BUZZ_FP16, false>(a, grid, past, st);
        case BUZZ_BF16: return e4m3 ? launch<BUZZ_BF16, true>(a, grid, past, st) : launch<BUZZ_BF16, false>(a, grid, past, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace buzz
