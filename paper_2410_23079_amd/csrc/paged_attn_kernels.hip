// Attention of one new token per sequence over a paged cache.
//
// Mathematics.  For every query head g of a kv head: s_j = scale q_g . k_j, p = softmax(s), out = sum_j p_j v_j, in one
// pass: a reference r is kept per head, and sum_j 2^(s_j - r) and sum_j 2^(s_j - r) v_j (logits in units of log 2) are
// rescaled when the reference moves.  Partial results (r, sum, sum v) of any two sets of keys add up after bringing
// them to the larger reference; that joins the waves of a block and the blocks of a sequence.
//
// What bounds it: every visible key and value row is read once, 2 head_dim elements for 4 head_dim * heads operations:
// memory.  The matrix instructions serve to make the arithmetic vanish beside that, and to need no shuffling:
//   - a wave takes 16 bytes per lane of keys as the first operand of a 16x16 product whose other side is the queries:
//     rows are keys, columns heads.  Which key stands in which row is free, and is chosen so that each lane ends up
//     with the logits of KG consecutive keys (KG = elements in 16 bytes) of one head;
//   - these, as weights, are one operand of the second product as they stand; its other operand is 16 bytes of one
//     column of V for the same KG keys, which is why the pages hold V that way.  No LDS, no transposition, no lane
//     crossing between the two products.
//   - Weights keep more than 16 bits: with 16-bit operands columns 0..7 carry the weights rounded to the operand's
//     type, columns 8..15 (the same heads again) what that rounding left over.  The unused half of the matrix
//     instruction does it for free; the sum of both halves has at least 16 bits.
//
// Layout of the work.  Sequences differ in length, and their lengths are known on the device only.  So the tiles of
// all (sequence, head) pairs, 4 KG keys each, are numbered through, and each block takes the same number of
// consecutive ones, whatever sequences they belong to: no block has more to do than another, and the grid does not
// depend on how long a sequence may get.  A block's tiles of one pair are joined in LDS; a pair that lies within one
// block is done, the others' partial results go through the workspace, and the block that finishes last for a pair
// adds them up in order, which is why the result does not depend on timing.
#include <math.h>

#include "paged_internal.h"

namespace buzz {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWaves = 4;                  // per block

// What a page holds and what the queries are.
enum { P_F32 = 0, P_F16, P_BF16, P_E4M3_F16, P_E4M3_BF16 };

template <int P> struct Form {
    static constexpr int EB = P == P_F32 ? 4 : P >= P_E4M3_F16 ? 1 : 2;   // bytes of an element of a page
    static constexpr int KG = 16 / EB;                                    // keys of a lane
    static constexpr int TILE = 4 * KG;                                   // keys of a wave's tile
    static constexpr bool E4M3 = P >= P_E4M3_F16;
    static constexpr bool F16Q = P == P_F16 || P == P_E4M3_F16;           // type of the first product
    static constexpr bool F16V = P == P_F16;                              // ... of the second: e4m3 values are weighted with
                                                                          // their row's power of two, which f16 cannot hold
    // f16 weights are taken 2^8 times as large, so that what is lost below the type's range is 2^-32 of the largest one
    static constexpr float BIAS = F16V ? 8.f : 0.f;
};
constexpr float kSlack = 7.f;              // the reference moves when a logit exceeds it by 2^7: seldom after the first tiles

__device__ inline float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float scale_of(unsigned e) { return __uint_as_float(e << 23); }        // 2^(e - 127), e 1 .. 254

template <bool F16> __device__ inline f32x4 mma(i32x4 a, i32x4 b, f32x4 c)
{
    if constexpr (F16) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// 8 e4m3 codes, two of the four dwords at `at`, in 16 bits each: exact in either type
template <bool F16> __device__ inline i32x4 widen(i32x4 x, int at)
{
    i32x4 r;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned w = (unsigned)x[2 * at + i];
        if constexpr (F16) {
            r[2 * i] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false));
            r[2 * i + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true));
        } else {
            r[2 * i] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
            r[2 * i + 1] = __builtin_bit_cast(int, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true));
        }
    }
    return r;
}

// Two weights as one dword of the second product's operand: rounded to its type, or (left = 1) what that left over.
template <bool F16> __device__ inline int pack(float x, float y, float left)
{
    if constexpr (F16) {
        const f16x2_t h = {(_Float16)x, (_Float16)y};
        const f16x2_t r = {(_Float16)fmaf(-left, (float)h[0], x), (_Float16)fmaf(-left, (float)h[1], y)};
        return __builtin_bit_cast(int, r);
    } else {
        const bf16x2_t h = {(__bf16)x, (__bf16)y};
        const bf16x2_t r = {(__bf16)fmaf(-left, (float)h[0], x), (__bf16)fmaf(-left, (float)h[1], y)};
        return __builtin_bit_cast(int, r);
    }
}

// the other lane of 8 in a row of 16
__device__ inline float across8(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, false));   // row_ror:8
}
// the maximum / sum over the four lanes of the same column
__device__ inline float column_max(float v) { v = fmaxf(v, __shfl_xor(v, 16)); return fmaxf(v, __shfl_xor(v, 32)); }
__device__ inline float column_sum(float v) { v += __shfl_xor(v, 16); return v + __shfl_xor(v, 32); }

// a value that all lanes agree on, in scalar registers
__device__ inline uint64_t uniform(uint64_t v)
{
    return (uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}

// Partial results pass between the blocks of one launch as in the decode step over the bounded cache (attn_kernels.hip
// gives the argument): device-scope stores, a wait for their acknowledgement, a block barrier, the ticket; and device-scope
// loads behind the ticket.
__device__ inline void publish(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline float acquire(const float* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The running results of one wave: lane (m, q) has column m of rows 4 q .. 4 q + 3 of each 16 output dimensions.
template <int D> struct WaveState {
    f32x4 o[D / 16];
    float sum, ref;
    bool bad;                              // a page number that is none was met
};

template <int P, int D> struct Attn {
    using F = Form<P>;
    static constexpr int NC = D * F::EB / 64;          // 16-byte pieces of a key row per lane
    static constexpr int NT = F::KG / 4;               // products of 16 keys per tile
    static constexpr int NQ = P == P_F32 ? D / 16 : D / 32;   // 16-byte pieces of queries per lane

    // One lane's pieces of the query rows: column m is head m % 8 (fp32: m), zeros where there is none.
    __device__ static inline void load_queries(const PagedAttnArgs& a, int b, int h, int lane, i32x4 (&q)[NQ])
    {
        const int g = lane & (P == P_F32 ? 15 : 7), part = lane >> 4;
        const char* row = a.q + (int64_t)b * a.q_seq + (int64_t)(h * a.G + g) * a.q_head;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            // piece i covers what the product of the keys' pieces i (e4m3: half of piece i / 2) multiplies
            const int at = F::E4M3 ? (i / 2) * 128 + part * 32 + (i & 1) * 16 : i * 64 + part * 16;
            q[i] = g < a.G ? *(const i32x4*)(row + at) : i32x4{0, 0, 0, 0};
        }
    }

    __device__ static inline void tile(const PagedAttnArgs& a, const int32_t* table_row, const Visible& vis, int h, int t0,
                                       int lane, const i32x4 (&q)[NQ], WaveState<D>& w)
    {
        const int m = lane & 15, part = lane >> 4;
        const int gk = t0 + F::KG * (m >> 2), gv = t0 + F::KG * part;    // first of the KG keys that the lane loads of K, of V
        // Pages.  Groups of keys of which none is visible are not looked up; their rows are page 0's, masked below.
        auto page = [&](int first) {
            const bool any = first < vis.length && (first + F::KG > vis.from || first < vis.sink_end);
            int pg = any ? page_of(table_row, first, a.pages.rows_log2, a.pages.n_pages) : 0;
            if (pg < 0) { w.bad = true; pg = 0; }
            return (int64_t)pg * a.pages.heads + h;
        };
        const int64_t pk = page(gk), pv = page(gv);
        const int R = a.pages.rows, in_k = gk & (R - 1), in_v = gv & (R - 1);
        const char* krow = a.pages.k + (pk * R + in_k + (m & 3)) * (D * F::EB) + part * 16;
        const char* vcol = a.pages.v + (pv * R + in_v) * (D * F::EB) + m * 16;
        i32x4 kk[NT][NC], vv[D / 16];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int c = 0; c < NC; ++c) kk[t][c] = *(const i32x4*)(krow + t * 4 * (D * F::EB) + c * 64);
        i32x4 ke{}, ve{};
        if constexpr (F::E4M3) {
            ke = *(const i32x4*)(a.pages.k_exp + pv * R + in_v);
            ve = *(const i32x4*)(a.pages.v_exp + pv * R + in_v);
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d) vv[d] = *(const i32x4*)(vcol + d * 256);

        f32x4 s[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                if constexpr (P == P_F32) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (int)kk[t][c][e]), __builtin_bit_cast(float, (int)q[c][e]), s[t], 0, 0, 0);
                } else if constexpr (F::E4M3) {
                    s[t] = mma<F::F16Q>(widen<F::F16Q>(kk[t][c], 0), q[2 * c], s[t]);
                    s[t] = mma<F::F16Q>(widen<F::F16Q>(kk[t][c], 1), q[2 * c + 1], s[t]);
                } else {
                    s[t] = mma<F::F16Q>(kk[t][c], q[c], s[t]);
                }
            }
        }
        const bool whole = t0 + F::TILE <= vis.length && (t0 >= vis.from || t0 + F::TILE <= vis.sink_end);
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = s[t][e] * a.scale_log2;
                if constexpr (F::E4M3) x *= scale_of(((unsigned)ke[t] >> (8 * e)) & 255u);
                if (!whole && !vis.sees(gv + 4 * t + e)) x = -INFINITY;
                s[t][e] = x;
                top = fmaxf(top, x);
            }
        if (__any(top > w.ref + (F::BIAS + kSlack))) {
            const float moved = fmaxf(w.ref, column_max(top) - F::BIAS), by = fast_exp2(w.ref - moved);
            w.sum *= by;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) w.o[d] *= by;
            w.ref = moved;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[t][e] = fast_exp2(s[t][e] - w.ref);
                w.sum += s[t][e];
            }
        // What a masked place of V holds must not matter: a weight of 0 does not cancel a NaN.
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned keep = 0;
#pragma unroll
                for (int e = 0; e < F::KG / 4; ++e)
                    if (vis.sees(gv + i * (F::KG / 4) + e)) keep |= (F::EB == 4 ? ~0u : F::EB == 2 ? 0xffffu << (16 * e) : 0xffu << (8 * e));
#pragma unroll
                for (int d = 0; d < D / 16; ++d) vv[d][i] &= (int)keep;
                if constexpr (F::E4M3) ve[i] &= (int)keep;
            }
        }
        if constexpr (P == P_F32) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w.o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (int)vv[d][e]), s[0][e], w.o[d], 0, 0, 0);
        } else {
            const float left = m < 8 ? 0.f : 1.f;
            if constexpr (F::E4M3) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][e] *= scale_of(((unsigned)ve[t] >> (8 * e)) & 255u);
            }
#pragma unroll
            for (int hf = 0; hf < NT / 2; ++hf) {
                const i32x4 p = {pack<F::F16V>(s[2 * hf][0], s[2 * hf][1], left), pack<F::F16V>(s[2 * hf][2], s[2 * hf][3], left),
                                 pack<F::F16V>(s[2 * hf + 1][0], s[2 * hf + 1][1], left), pack<F::F16V>(s[2 * hf + 1][2], s[2 * hf + 1][3], left)};
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
                    if constexpr (F::E4M3) w.o[d] = mma<false>(widen<false>(vv[d], hf), p, w.o[d]);
                    else w.o[d] = mma<F::F16V>(vv[d], p, w.o[d]);
                }
            }
        }
    }
};

template <int P, int D>
__global__ __launch_bounds__(kWaves * 64) void paged_attn_kernel(const PagedAttnArgs a)
{
    using F = Form<P>;
    using A = Attn<P, D>;
    __shared__ float acc[kWaves][8][D];
    __shared__ float2 stat[kWaves][8];     // (reference, sum)
    __shared__ int arrived;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), G = a.G, H = a.pages.heads;
    const int64_t most = (int64_t)a.pages.cols * a.pages.rows;
    // A pair without visible keys, or with a length that is none, counts as one tile: somebody has to write its output.
    auto tiles_in = [&](int b) {
        const int n = tiles_of(visible(a.length[b], a.sink, a.window, most), F::TILE).count;
        return (uint64_t)(n > 0 ? n : 1) * (unsigned)H;
    };
    // Every wave adds up the tiles of all sequences, `per` consecutive ones to a lane.
    const int per = (a.batch + 63) / 64;
    uint64_t mine = 0;
    for (int i = lane * per; i < min((lane + 1) * per, a.batch); ++i) mine += tiles_in(i);
    uint64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint64_t x = __shfl_up(upto, o);
        if (lane >= o) upto += x;
    }
    const uint64_t total = uniform(__shfl(upto, 63));
    const uint64_t share = tiles_per_block(total, gridDim.x);
    uint64_t cur = share * blockIdx.x;
    if (cur >= total) return;
    const uint64_t end = min(cur + share, total);
    const int owner = __ffsll((unsigned long long)__ballot(cur < upto)) - 1;
    uint64_t off = uniform(cur - __shfl(upto - mine, owner));   // tiles between the start of sequence b and the block's first
    int b = owner * per;
    for (uint64_t n; off >= (n = tiles_in(b)); ++b) off -= n;

    while (cur < end) {
        const Visible vis = visible(a.length[b], a.sink, a.window, most);
        const Tiles tiles = tiles_of(vis, F::TILE);
        const unsigned n = tiles.count > 0 ? tiles.count : 1;
        const int h = (int)(off / n);
        const unsigned first = (unsigned)(off - (uint64_t)h * n);
        const unsigned here = (unsigned)min((uint64_t)(n - first), end - cur);
        const int32_t* table_row = a.pages.table + (int64_t)b * a.pages.cols;

        WaveState<D> w;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) w.o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        w.sum = 0.f; w.ref = -3e38f; w.bad = vis.length < 0;
        if (tiles.count > 0) {
            i32x4 q[A::NQ];
            A::load_queries(a, b, h, lane, q);
            for (unsigned i = wave; i < here; i += kWaves)
                A::tile(a, table_row, vis, h, tiles.at(first + i) * F::TILE, lane, q, w);
        }
        const bool bad = __any(w.bad);
        w.sum = column_sum(w.sum);
        const int m = lane & 15, part = lane >> 4;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) {
            f32x4 x = w.o[d];
            if constexpr (P != P_F32) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] += across8(x[e]);
            }
            if (m < G) *(f32x4*)&acc[wave][m][d * 16 + part * 4] = x;
        }
        if (part == 0 && m < G) stat[wave][m] = make_float2(w.ref, bad ? __builtin_nanf("") : w.sum);
        __syncthreads();

        const bool alone = first == 0 && here == n;
        const int64_t unit = (int64_t)b * H + h;
        const int64_t slot = 2 * (int64_t)blockIdx.x + (first == 0 ? 1 : 0);
        for (int i = tid; i < G * D; i += kWaves * 64) {
            const int g = i / D, d = i - g * D;
            float ref = stat[0][g].x, sum = 0.f, o = 0.f;
#pragma unroll
            for (int x = 1; x < kWaves; ++x) ref = fmaxf(ref, stat[x][g].x);
#pragma unroll
            for (int x = 0; x < kWaves; ++x) {
                const float by = fast_exp2(stat[x][g].x - ref);
                sum = fmaf(by, stat[x][g].y, sum);
                o = fmaf(by, acc[x][g][d], o);
            }
            if (alone) {
                a.out[unit * G * D + i] = tiles.count > 0 ? o / sum : sum;       // nothing visible: 0, or NaN
                if (d == 0 && a.lse) a.lse[unit * G + g] = tiles.count > 0 ? (ref + log2f(sum)) * 0.6931471805599453f : sum - INFINITY;
            } else {
                publish(a.part_o + slot * G * D + i, o);
                if (d == 0) { publish(a.part_ml + (slot * G + g) * 2, ref); publish(a.part_ml + (slot * G + g) * 2 + 1, sum); }
            }
        }
        if (!alone) {
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
            __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt(0): this wave's partial results are acknowledged
            __syncthreads();
            const Parts all = parts_of(cur - first, n, share);
            if (tid == 0) arrived = __hip_atomic_fetch_add(a.ticket + unit, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __syncthreads();
            if (__builtin_amdgcn_readfirstlane(arrived) == all.parts - 1) {
                __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
                for (int i = tid; i < G * D; i += kWaves * 64) {
                    const int g = i / D, d = i - g * D;
                    float ref = -3e38f, sum = 0.f, o = 0.f;
                    for (int p = 0; p < all.parts; ++p) {
                        const int64_t s = all.slot(p);
                        const float r = acquire(a.part_ml + (s * G + g) * 2), l = acquire(a.part_ml + (s * G + g) * 2 + 1);
                        const float x = acquire(a.part_o + s * G * D + i);
                        const float moved = fmaxf(ref, r), old = fast_exp2(ref - moved), by = fast_exp2(r - moved);
                        sum = fmaf(sum, old, by * l);
                        o = fmaf(o, old, by * x);
                        ref = moved;
                    }
                    a.out[unit * G * D + i] = o / sum;
                    if (d == 0 && a.lse) a.lse[unit * G + g] = (ref + log2f(sum)) * 0.6931471805599453f;
                }
                if (tid == 0) __hip_atomic_store(a.ticket + unit, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next step
            }
        }
        __syncthreads();                               // the next pair's results go to the same LDS
        cur += here;
        off += here;
        if (off == (uint64_t)n * (unsigned)H) { off = 0; ++b; }
    }
}

template <int P> hipError_t launch(const PagedAttnArgs& a, int grid, hipStream_t st)
{
    switch (a.pages.D) {
        case 64: hipLaunchKernelGGL((paged_attn_kernel<P, 64>), dim3(grid), dim3(kWaves * 64), 0, st, a); break;
        case 128: hipLaunchKernelGGL((paged_attn_kernel<P, 128>), dim3(grid), dim3(kWaves * 64), 0, st, a); break;
        case 256: hipLaunchKernelGGL((paged_attn_kernel<P, 256>), dim3(grid), dim3(kWaves * 64), 0, st, a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_attn(int dtype, int page_dtype, const PagedAttnArgs& a, int compute_units, hipStream_t st)
{
    const bool e4m3 = page_dtype == BUZZ_E4M3;
    const int tile = e4m3 ? 64 : dtype == BUZZ_FP32 ? 16 : 32;
    int64_t grid = (int64_t)compute_units * 2;
    if (grid > kPagedMaxBlocks) grid = kPagedMaxBlocks;
    // no more blocks than could have tiles, four to a block
    const int64_t most = ((int64_t)a.pages.cols * a.pages.rows + tile - 1) / tile, tiles = (int64_t)a.batch * a.pages.heads * (most > 0 ? most : 1);
    if (grid > (tiles + kWaves - 1) / kWaves) grid = (tiles + kWaves - 1) / kWaves;
    if (dtype == BUZZ_FP32) return launch<P_F32>(a, (int)grid, st);
    if (dtype == BUZZ_FP16) return e4m3 ? launch<P_E4M3_F16>(a, (int)grid, st) : launch<P_F16>(a, (int)grid, st);
    return e4m3 ? launch<P_E4M3_BF16>(a, (int)grid, st) : launch<P_BF16>(a, (int)grid, st);
}

}  // namespace buzz
