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
//   - Weights keep 22 bits or more: with 16-bit operands columns 0..7 carry the weights rounded to the operand's type,
//     columns 8..15 (the same heads again) what that rounding left over, and in bf16 another product what is left then.
//     The unused half of the matrix instruction does most of it for free.
//
// Layout of the work.  Sequences differ in length, and their lengths are known on the device only.  So there is a block
// of eight waves to every compute unit, and each looks at all lengths and finds its share by itself:
//   - where pairs are short, or many and not long, a wave takes a whole pair and nothing is joined;
//   - otherwise the tiles of all (sequence, head) pairs, 4 KG keys each, are cut into units of four tiles or more (a whole
//     pair, where the longest is short; as much as gives every block one, where pairs are few), numbered through, and
//     each block takes the same number of consecutive ones, whatever sequences they belong to: no block has more to do
//     than another, and the grid does not depend on how long a sequence may get.  A block's tiles of one pair go to its
//     waves in turn and are joined in LDS; a pair that lies within one block is done, the others' partial results go
//     through the workspace, and the block that finishes last for a pair adds them up in order, which is why the result
//     does not depend on timing.  The next pair's first rows are under way meanwhile.
//
// Measured (a call in a captured graph): 16 sequences of 32 bf16 heads of 128, up to 16384 keys, 378 us, 6.34 TB/s of the
// 7.05 that a plain read reaches; 8 sequences of 32 fp16 heads, up to 4096, 57 us, 5.5 TB/s; 4 sequences of 8 pairs with 4
// heads, 32768 keys in 8 bits, 50 us, 5.4 TB/s; 8 pairs with 4 heads of 1517 bf16 keys 9.3 us, of 300 8.3, of one 3.9.  Of 9
// us: start 0.4 to 0.9 us, lengths 0.4, shares 0.6, page numbers 0.35, keys and
// values 1.3 to 1.7, LDS 0.7, publish and ticket 1.0, the parts back 1.0, output 0.7.
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

constexpr int NW = 8, kThreads = NW * 64;  // waves and threads of a block: one block to a compute unit, two waves to a SIMD

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
    // Tiles of a pair up to which one wave takes it: two, four where a tile costs little arithmetic.
    static constexpr int SOLO = EB == 2 ? 4 : 2;
};
constexpr float kSlack = 7.f;               // the reference moves when a logit exceeds it by 2^7: seldom after the first tiles

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

// Two weights as dwords of the second product's operands.  With f16, columns 0 .. 7 take them rounded (left 0), columns 8 .. 15
// what that rounding left over (left 1): 22 bits together.  bf16 has 8 bits, so what the second rounding leaves over goes into an
// operand of its own, columns 0 .. 7 (the others 0): 24 bits.
struct Packed { int both, rest; };
template <bool F16> __device__ inline Packed pack(float x, float y, float left)
{
    if constexpr (F16) {
        const f16x2_t h = {(_Float16)x, (_Float16)y};
        const f16x2_t r = {(_Float16)fmaf(-left, (float)h[0], x), (_Float16)fmaf(-left, (float)h[1], y)};
        return Packed{__builtin_bit_cast(int, r), 0};
    } else {
        const bf16x2_t h = {(__bf16)x, (__bf16)y};
        const float x1 = x - (float)h[0], y1 = y - (float)h[1];
        const bf16x2_t r = {(__bf16)x1, (__bf16)y1};
        const bf16x2_t e = {(__bf16)(x1 - (float)r[0]), (__bf16)(y1 - (float)r[1])};
        return Packed{__builtin_bit_cast(int, left == 0.f ? h : r), left == 0.f ? __builtin_bit_cast(int, e) : 0};
    }
}

// Lane moves within the wave that need no LDS: a row is 16 lanes.
template <int CTRL, int ROWS> __device__ inline int dpp(int v) { return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, CTRL < 0x120); }
__device__ inline float across8(float v) { return __builtin_bit_cast(float, dpp<0x128, 0xf>(__builtin_bit_cast(int, v))); }   // the lane 8 away in the row
// the maximum / sum over the four lanes of the same column (the same place in the four rows)
template <class Op> __device__ inline float column(float v, Op op)
{
    const unsigned x = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
    const unsigned y = __float_as_uint(op(__uint_as_float(r[0]), __uint_as_float(r[1])));
    const auto s = __builtin_amdgcn_permlane32_swap(y, y, false, false);
    return op(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ inline float column_max(float v) { return column(v, [](float x, float y) { return fmaxf(x, y); }); }
__device__ inline float column_sum(float v) { return column(v, [](float x, float y) { return x + y; }); }
// op over the lanes up to this one; 0 is op's neutral element
template <class Op> __device__ inline int scan(int v, Op op)
{
    v = op(v, dpp<0x111, 0xf>(v));         // row_shr 1, 2, 4, 8
    v = op(v, dpp<0x112, 0xf>(v));
    v = op(v, dpp<0x114, 0xf>(v));
    v = op(v, dpp<0x118, 0xf>(v));
    v = op(v, dpp<0x142, 0xa>(v));         // the last lane of row 0 to row 1, of row 2 to row 3
    return op(v, dpp<0x143, 0xc>(v));      // lane 31 to rows 2 and 3
}

// Partial results pass between the blocks of one launch as in the decode step over the bounded cache (attn_kernels.hip
// gives the argument): device-scope stores, a wait for their acknowledgement, a block barrier, the ticket; and device-scope
// loads behind the ticket.
__device__ inline void publish(float* p, float v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline float2 acquire2(const float* p)
{
    const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
// Partial results that a team of the merging block asks for at a time, and teams.  The code that joins them runs once per launch
// and is fetched while it runs, so more of either is slower: 8 pairs of 513 fp32 keys of 64 take 8.3 us with 16 and up to 16
// teams, 8.2 with 8 and 16, 7.3 with 8 and 2 or 4; 32 pairs of 32768 keys in 8 bits 49.9, 49.9 and 49.6.
constexpr int kParts = 8, kTeams = 2;

// A block barrier that orders LDS alone: loads and stores to memory stay under way.
__device__ inline void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ inline i32x4 fetch(const void* p) { return __builtin_nontemporal_load((const i32x4*)p); }

// A block's, or a wave's, share of one (sequence, head) pair: `count` of the pair's tiles from number `first` on.
struct Segment {
    int b, h;
    Visible vis;
    Tiles tiles;
    uint32_t first, count;
    __device__ inline int tile(uint32_t i) const { return tiles.at((int)(first + min(i, count - 1))); }   // number i of them, or the last
};

// One wave's way through its tiles of a segment.  The rows of the next tile are asked for as soon as the registers of the
// present one are read: keys after the first product, values after the second, page numbers a tile ahead of that; so a wave
// always has half a tile or more under way, in the registers of one.  (No branch lies between a load and the wait for it, or
// the compiler would wait for all that are under way: the last tile, which asks for nothing, has code of its own.)
// MASK: the cache has a window.
template <int P, int D, bool MASK> struct Attn {
    using F = Form<P>;
    static constexpr int NC = D * F::EB / 64;          // 16-byte pieces of a key row per lane
    static constexpr int NT = F::KG / 4;               // products of 16 keys per tile
    static constexpr int NQ = P == P_F32 ? D / 16 : D / 32;   // 16-byte pieces of queries per lane
    static constexpr int ROW = D * F::EB;
    // Heads of 256 leave no registers for the queries: they stay in LDS, and every tile reads them from there.
    static constexpr bool QLDS = D == 256;
    // ... and in 8 bits, whose elements are widened before each product, too few to have the next tile's keys under way behind
    // the values: both are asked for together (32 heads of 256, 4096 keys: 39.4 us with the keys first, 36.8 so).
    static constexpr bool LATE = D == 256 && F::E4M3;
    static constexpr uint32_t MANY = D == 64 ? 5 : 4;  // pairs to two blocks that are many (below)
    struct Tile { int t0; int32_t pk, pv; };           // first key; pages of the keys that the lane loads of K, of V

    const PagedAttnArgs& a;
    const int lane, m, part;               // the lane is column m, rows 4 part .. 4 part + 3 of a product
    i32x4* const ql;                       // [NQ][64 lanes]
    i32x4 q[QLDS ? 1 : NQ], kk[NT][NC], vv[D / 16], ke, ve;
    // The running results: column m of rows 4 part .. of each 16 output dimensions, relative to `ref`.
    f32x4 o[D / 16];
    float sum, ref;
    bool bad;                              // a page number that is none was met
    Tile t, next;                          // the tile that has been asked for, and the one after it

    __device__ inline Attn(const PagedAttnArgs& args, i32x4* lds) : a(args), lane(threadIdx.x & 63), m(lane & 15), part(lane >> 4), ql(lds) {}

    // Column m is head m % 8 (fp32: m), zeros where there is none.  Piece i covers what the product of the keys' pieces i
    // (e4m3: half of piece i / 2) multiplies.
    __device__ inline const char* query_row(const Segment& s) const
    {
        const int g = P == P_F32 ? m : m & 7;
        return a.q + (int64_t)s.b * a.q_seq + (int64_t)(s.h * a.G + min(g, a.G - 1)) * a.q_head + (F::E4M3 ? part * 32 : part * 16);
    }
    __device__ inline i32x4 query_piece(const char* row, int i) const
    {
        const i32x4 x = *(const i32x4*)(row + (F::E4M3 ? (i / 2) * 128 + (i & 1) * 16 : i * 64));
        return (P == P_F32 ? m : m & 7) < a.G ? x : i32x4{0, 0, 0, 0};
    }

    // First of the KG keys that the lane loads of K, of V.
    __device__ inline int key_group(int t0) const { return t0 + F::KG * (m >> 2); }
    __device__ inline int value_group(int t0) const { return t0 + F::KG * part; }
    // Their page: of a group of which no key is visible that of the sequence's last key, which always is.
    __device__ inline int32_t page_of_group(const Segment& s, int first) const
    {
        int j = min(first, s.vis.length - 1);
        if constexpr (MASK)
            if (first + F::KG <= s.vis.from && first >= s.vis.sink_end) j = s.vis.length - 1;
        return a.pages.table[(int64_t)s.b * a.pages.cols + (j >> a.pages.rows_log2)];
    }
    __device__ inline Tile look_up(const Segment& s, uint32_t i) const
    {
        const int t0 = s.tile(i) * F::TILE;
        return Tile{t0, page_of_group(s, key_group(t0)), page_of_group(s, value_group(t0))};
    }
    // A page's place and a row's within it; a page that is none stands for page 0, and is noted.
    __device__ inline uint64_t page_at(int32_t pg)
    {
        const bool none = (unsigned)pg >= (unsigned)a.pages.n_pages;
        bad |= none;
        return (uint64_t)(unsigned)(none ? 0 : pg) * a.page_bytes;
    }
    __device__ inline uint32_t row_in_page(const Segment& s, int first) const { return (uint32_t)s.h * a.pages.rows + (first & (a.pages.rows - 1)); }
    // (the keys' exponents come in the order of the logits: the lane's group of values)
    __device__ inline void request_keys(const Segment& s, const Tile& t)
    {
        const char* p = a.pages.k + page_at(t.pk) + (row_in_page(s, key_group(t.t0)) + (m & 3)) * ROW + part * 16;
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int c = 0; c < NC; ++c) kk[i][c] = fetch(p + i * 4 * ROW + c * 64);
        if constexpr (F::E4M3) ke = *(const i32x4*)(a.pages.k_exp + page_at(t.pv) / ROW + row_in_page(s, value_group(t.t0)));
    }
    __device__ inline void request_values(const Segment& s, const Tile& t)
    {
        const uint64_t page = page_at(t.pv);
        const uint32_t row = row_in_page(s, value_group(t.t0));
        if constexpr (F::E4M3) ve = *(const i32x4*)(a.pages.v_exp + page / ROW + row);
        const char* p = a.pages.v + page + row * ROW + m * 16;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) vv[d] = fetch(p + d * 256);
    }

    // logits of the tile's keys: s[t][e] is key value_group + 4 t + e of column m
    __device__ inline void logits(f32x4 (&s)[NT]) const
    {
        int z = lane;
        if constexpr (QLDS) asm volatile("" : "+v"(z));    // (or the compiler would take the reads out of the loop over the tiles)
        auto query = [&](int i) { return QLDS ? ql[z + i * 64] : q[QLDS ? 0 : i]; };
#pragma unroll
        for (int t = 0; t < NT; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            if constexpr (P == P_F32) {
                const i32x4 x = query(c);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (int)kk[0][c][e]), __builtin_bit_cast(float, (int)x[e]), s[0], 0, 0, 0);
            } else {
#pragma unroll
                for (int hf = 0; hf < (F::E4M3 ? 2 : 1); ++hf) {
                    const i32x4 x = query(F::E4M3 ? 2 * c + hf : c);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        if constexpr (F::E4M3) s[t] = mma<F::F16Q>(widen<F::F16Q>(kk[t][c], hf), x, s[t]);
                        else s[t] = mma<F::F16Q>(kk[t][c], x, s[t]);
                    }
                    if constexpr (QLDS) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }

    // weights of the tile's keys and their sum with the values
    __device__ inline void accumulate(const Visible& vis, int t0, f32x4 (&s)[NT], i32x4 exps)
    {
        const bool whole = t0 + F::TILE <= vis.length && (!MASK || t0 >= vis.from || t0 + F::TILE <= vis.sink_end);
        uint32_t seen = ~0u;
        if (!whole) seen = MASK ? vis.bits(value_group(t0), F::KG) : Visible::below(vis.length - value_group(t0), F::KG);
        float top = -INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = s[t][e] * a.scale_log2;
                if constexpr (F::E4M3) x *= scale_of(((unsigned)exps[t] >> (8 * e)) & 255u);
                if (!((seen >> (4 * t + e)) & 1)) x = -INFINITY;
                s[t][e] = x;
                top = fmaxf(top, x);
            }
        if (__any(top > ref + (F::BIAS + kSlack))) {
            const float moved = fmaxf(ref, column_max(top) - F::BIAS), by = fast_exp2(ref - moved);
            sum *= by;
#pragma unroll
            for (int d = 0; d < D / 16; ++d) o[d] *= by;
            ref = moved;
        }
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s[t][e] = fast_exp2(s[t][e] - ref);
                sum += s[t][e];
            }
        // What a masked place of V holds must not matter: a weight of 0 does not cancel a NaN.
        if (!whole) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                unsigned keep = 0;
#pragma unroll
                for (int e = 0; e < F::KG / 4; ++e)
                    if ((seen >> (i * (F::KG / 4) + e)) & 1) keep |= (F::EB == 4 ? ~0u : F::EB == 2 ? 0xffffu << (16 * e) : 0xffu << (8 * e));
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
                    o[d] = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (int)vv[d][e]), s[0][e], o[d], 0, 0, 0);
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
                i32x4 p, rest;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const Packed x = pack<F::F16V>(s[2 * hf + i / 2][i % 2 * 2], s[2 * hf + i / 2][i % 2 * 2 + 1], left);
                    p[i] = x.both;
                    rest[i] = x.rest;
                }
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
                    const i32x4 v = F::E4M3 ? widen<false>(vv[d], hf) : vv[d];
                    o[d] = mma<F::F16V>(v, p, o[d]);
                    if constexpr (!F::F16V) o[d] = mma<false>(v, rest, o[d]);
                    if constexpr (D == 256 && F::E4M3) if (d % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
    }

    // Asks for the queries and the first tile of a segment, of which the wave is to take tiles i, i + step, ..
    __device__ inline void begin(const Segment& s, uint32_t i, uint32_t step, int wave)
    {
        bad = s.vis.length < 0;
        if constexpr (QLDS) {
            if (s.count > 0) {
                const char* row = query_row(s);
                for (int x = wave; x < NQ; x += NW) ql[x * 64 + lane] = query_piece(row, x);
            }
            lds_barrier();
        }
        if constexpr (!QLDS) if (i < s.count) {
            const char* row = query_row(s);
#pragma unroll
            for (int x = 0; x < NQ; ++x) q[x] = query_piece(row, x);
            request_first(s, i, step);
        }
    }
    __device__ inline void request_first(const Segment& s, uint32_t i, uint32_t step)
    {
        t = look_up(s, i);
        next = look_up(s, i + step);
        request_keys(s, t);
        request_values(s, t);
    }

    // Takes them; afterwards columns 0 .. 7 hold the heads' results (fp32: all columns do).
    __device__ inline void run(const Segment& s, uint32_t i, uint32_t step)
    {
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
        sum = 0.f;
        ref = -3e38f;
        if (i < s.count) {
            if constexpr (QLDS) request_first(s, i, step);
            f32x4 x[NT];
            for (; i + step < s.count; i += step) {
                const i32x4 exps = ke;
                logits(x);
                const Tile after = look_up(s, i + 2 * step);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (!LATE) request_keys(s, next);
                __builtin_amdgcn_sched_barrier(0);
                accumulate(s.vis, t.t0, x, exps);
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (LATE) request_keys(s, next);
                request_values(s, next);
                __builtin_amdgcn_sched_barrier(0);
                t = next;
                next = after;
            }
            logits(x);
            accumulate(s.vis, t.t0, x, ke);
        }
        bad = __any(bad);
        sum = column_sum(sum);
        if (bad) sum = __builtin_nanf("");
        if constexpr (P != P_F32) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[d][e] += across8(o[d][e]);
        }
    }
};

// What is needed at the end only is fetched there: in scalar registers all along, it would crowd out what the loop needs.
typedef const __attribute__((address_space(4))) PagedAttnArgs* LateArgs;
__device__ inline LateArgs late_args()
{
    LateArgs p = (LateArgs)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return p;
}

// What this block has published before is there for whoever draws a later number from `counter`: true for the block that
// draws the last of `count`, which may then read what the others have published, and which resets the counter.
__device__ inline bool last_to_arrive(int32_t* counter, int count, int* shared)
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): this wave's partial results are acknowledged
    lds_barrier();
    if (threadIdx.x == 0) {
        const int before = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (before == count - 1) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next step
        *shared = before;
    }
    lds_barrier();
    const bool last = __builtin_amdgcn_readfirstlane(*shared) == count - 1;
    if (last) __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    return last;
}

struct Sum2 { float ref, sum; float2 o; };             // of two output elements

// A pair of which this block has only a part: publishes the part, and in the block that finishes last for the pair (for the
// part's group first, where there are many) adds up all of them in order.  A thread takes two output elements; the heads are
// laid over the threads once or twice, as teams that share the parts.  kParts parts are asked for at a time: one after
// the other, each would wait for memory.
template <int D> __device__ inline void join_parts(const Parts& all, int slot, int64_t unit, const float2 (&stat)[NW][8], float (&acc)[NW][8][D], int* arrived)
{
    constexpr int HT = D / 2, HL = HT < 64 ? HT : 64;  // threads of a head; lanes of a wave that work on one head
    constexpr int NH = kThreads / HT;                  // heads that the block has threads for
    LateArgs a = late_args();
    const int tid = threadIdx.x, lane = tid & 63, j = lane % HL, G = a->G, e = tid % HT * 2;
    float* const part_o = a->part_o;
    float* const part_ml = a->part_ml;
    const int padded = G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : 8, teams = padded < NH ? min(NH / padded, kTeams) : 1;
    const int group = group_of(all.parts);
    bool last = group == 1;
    int first = last ? 0 : ((int)blockIdx.x - all.from) / group * group, stride = 1, count = last ? all.parts : min(group, all.parts - first), to = all.slot(first);
    while (last_to_arrive(last ? a->ticket + unit : a->group_ticket + to, count, arrived)) {
        for (int g0 = 0; g0 < G; g0 += NH) {
            const int g = g0 + (tid / HT & (padded < NH ? padded - 1 : NH - 1)), team = tid / HT / padded;
            Sum2 s{-3e38f, 0.f, make_float2(0.f, 0.f)};
            if (g < G && team < teams) {
                for (int p0 = team; p0 < count; p0 += kParts * teams) {
                    // lane j of a head's lanes fetches the (reference, sum) of its team's part p0 + j
                    auto at = [&](int k) { return (all.slot(first + min(p0 + k * teams, count - 1) * stride) * G + g); };
                    const bool have = j < kParts && p0 + j * teams < count;
                    const float2 ml = acquire2(part_ml + at(j % kParts) * 2);
                    float2 x[kParts];
#pragma unroll
                    for (int k = 0; k < kParts; k += 4) {
                        if (p0 + k * teams >= count) break;
#pragma unroll
                        for (int i = k; i < k + 4; ++i) x[i] = acquire2(part_o + at(i) * D + e);
                    }
                    float ref = have ? ml.x : -3e38f;
#pragma unroll
                    for (int d = 1; d < kParts; d <<= 1) ref = fmaxf(ref, __shfl_xor(ref, d));
                    ref = fmaxf(s.ref, __shfl(ref, lane - j));
                    const float by = have ? fast_exp2(ml.x - ref) : 0.f, old = fast_exp2(s.ref - ref);
                    s.sum *= old; s.o.x *= old; s.o.y *= old; s.ref = ref;
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        if (p0 + k * teams >= count) break;
                        const float b = __shfl(by, lane - j + k);
                        s.sum = fmaf(b, __shfl(ml.y, lane - j + k), s.sum);
                        s.o.x = fmaf(b, x[k].x, s.o.x);
                        s.o.y = fmaf(b, x[k].y, s.o.y);
                    }
                }
            }
            Sum2* sums = (Sum2*)&acc[0][0][0];
            __syncthreads();                           // all have read what emitting a group's sum may overwrite
            if (teams > 1) {
                sums[tid] = s;
                lds_barrier();
                if (team == 0)
                    for (int t = 1; t < teams; ++t) {
                        const Sum2 x = sums[tid + t * padded * HT];
                        const float ref = fmaxf(s.ref, x.ref), u = fast_exp2(s.ref - ref), v = fast_exp2(x.ref - ref);
                        s = Sum2{ref, fmaf(s.sum, u, x.sum * v), make_float2(fmaf(s.o.x, u, x.o.x * v), fmaf(s.o.y, u, x.o.y * v))};
                    }
            }
            if (team == 0 && g < G) {
                if (last) {
                    *(float2*)(a->out + (unit * G + g) * D + e) = make_float2(s.o.x / s.sum, s.o.y / s.sum);
                    if (e == 0 && a->lse) a->lse[unit * G + g] = (s.ref + log2f(s.sum)) * 0.6931471805599453f;
                } else {
                    const int64_t row = (int64_t)to * G + g;
                    publish(part_o + row * D + e, s.o.x);
                    publish(part_o + row * D + e + 1, s.o.y);
                    if (e == 0) { publish(part_ml + row * 2, s.ref); publish(part_ml + row * 2 + 1, s.sum); }
                }
            }
        }
        if (last) break;
        last = true;
        first = 0; stride = group; count = (all.parts + group - 1) / group;
    }
}

template <int P, int D, bool MASK>
__global__ __launch_bounds__(kThreads) void paged_attn_kernel(const PagedAttnArgs a)
{
    using F = Form<P>;
    using A = Attn<P, D, MASK>;
    __shared__ float acc[NW][8][D];
    __shared__ float2 stat[NW][8];         // (reference, sum)
    __shared__ i32x4 queries[A::QLDS ? A::NQ * 64 : 1];
    __shared__ int arrived;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), H = a.pages.heads;
    const int32_t most = a.pages.cols << a.pages.rows_log2;
    auto visible_in = [&](int length) {
        if constexpr (MASK) return visible(length, a.sink, a.window, most);
        else return Visible{length > most ? -1 : length, 0, 0};
    };
    auto tiles_in = [&](const Visible& v) {
        if constexpr (MASK) return tiles_of(v, F::TILE);
        else return Tiles{0, 0, v.length > 0 ? (int)((uint32_t)(v.length - 1) / F::TILE) + 1 : 0};
    };
    // Every wave looks at the lengths of all sequences, `per` consecutive ones to a lane.
    const int per = (a.batch + 63) / 64;
    auto for_lengths = [&](auto f) {       // of the lane, eight asked for at a time
        const int to = min((lane + 1) * per, a.batch);
        for (int i = lane * per; i < to; i += 8) {
            int n[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) n[j] = a.length[min(i + j, to - 1)];
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i + j < to) f(n[j]);
        }
    };
    int one = 0, longest = 0;              // the lane's length and its tiles, where each has one; the most tiles of a pair
    if (per == 1) {
        one = a.length[min(lane, a.batch - 1)];
        longest = tiles_in(visible_in(one)).count;
    } else {
        for_lengths([&](int n) { longest = max(longest, tiles_in(visible_in(n)).count); });
    }
    const int own = longest;
    longest = __builtin_amdgcn_readlane(scan(longest, [](int x, int y) { return max(x, y); }), 63);
    auto segment = [&](int b, int h) {
        Segment s;
        s.b = b;
        s.h = h;
        s.vis = visible_in(per == 1 ? __builtin_amdgcn_readlane(one, b) : __builtin_amdgcn_readfirstlane(a.length[b]));
        s.tiles = tiles_in(s.vis);
        s.first = 0;
        s.count = s.tiles.count;
        return s;
    };
    A w(a, queries);

    // Pairs of a few tiles: a wave to each, which needs nobody else.  With two pairs and more to a block a few are three times as
    // many for each of them, as far as pairs would be left whole: short pairs do not wait for long ones, and nothing is joined.
    // (Heads of 64, whose tiles are half as much, from two and a half on: 16 sequences of 32 such heads with 600 8-bit keys take
    // 12.2 us by blocks, 15 by waves; 20 sequences 18.4, 16.1.  64 sequences of 32 heads of 128 with 900 bf16 keys: 162 us by blocks, 156 by
    // waves; of 90 to 900 keys 134 and 109; one of 900 and 63 of 90 118 and 37; 20 sequences of 500 35.4 and 33.0.)
    const uint32_t pairs = (uint32_t)a.batch * H, whole = whole_tiles(F::TILE * D * F::EB * 2, pairs, a.blocks);
    if (!A::QLDS && (uint32_t)longest <= (pairs < A::MANY * a.blocks / 2 ? (uint32_t)F::SOLO : min(whole, pairs / a.blocks * (3 * F::SOLO)))) {
        for (uint32_t pair = wave * a.blocks + blockIdx.x; pair < pairs; pair += a.blocks * NW) {   // over all compute units first
            const Segment s = segment(pair / H, pair % H);
            w.begin(s, 0, 1, wave);
            w.run(s, 0, 1);
            LateArgs l = late_args();
            const int G = l->G;
            if (w.m < G) {
                const int64_t row = (int64_t)pair * G + w.m;
                const bool any = s.count > 0;
                const float by = 1.f / w.sum;          // (a division for each output would be a fifth of the code that runs)
                float* out = l->out + row * D + w.part * 4;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) {
                    f32x4 x;
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = any ? w.o[d][e] * by : w.sum;   // nothing visible: 0, or NaN
                    *(f32x4*)(out + d * 16) = x;
                }
                if (w.part == 0 && l->lse) l->lse[row] = any ? (w.ref + log2f(w.sum)) * 0.6931471805599453f : w.sum - INFINITY;
            }
        }
        return;
    }

    // The unit, in tiles: a pair, where the longest is short; else what gives every block one unit, where the pairs are few (a
    // block with parts of two pairs pays for both), else the least.
    uint32_t unit = kUnitTiles, upto, total;
    auto add = [&](uint32_t n) { upto = scan(n, [](int x, int y) { return x + y; }); total = __builtin_amdgcn_readlane(upto, 63) * (uint32_t)H; return n; };
    auto units_in_lane = [&]() {
        if (per == 1) return lane < a.batch ? units_of(own, unit) : 0u;
        uint32_t sum = 0;
        for_lengths([&](int n) { sum += units_of(tiles_in(visible_in(n)).count, unit); });
        return sum;
    };
    if ((uint32_t)longest <= whole) unit = max(longest, 1);
    uint32_t mine = add(units_in_lane());
    if (per == 1 && 2 * pairs <= a.blocks && total > a.blocks) {
        unit *= units_per_block(total, a.blocks);
        unit = (unit + NW - 1) / NW * NW;              // (a round of a tile for each wave takes as long if some have none)
        for (const uint32_t more = max(unit / 64 * NW, (uint32_t)NW);; unit += more) {
            mine = add(units_in_lane());
            if (total <= a.blocks) break;
        }
    }
    const uint32_t share = units_per_block(total, a.blocks);
    uint32_t cur = share * blockIdx.x;
    if (cur >= total) return;
    const uint32_t end = min(cur + share, total);
    const int owner = __ffsll((unsigned long long)__ballot(cur < upto * H)) - 1;
    uint32_t off = cur - __builtin_amdgcn_readlane(upto - mine, owner) * H;   // units between the start of sequence b and the block's first
    int b = owner * per;
    auto units = [&](const Segment& s) { return units_of(s.tiles.count, unit); };
    if (per > 1)
        for (uint32_t n; off >= (n = units(segment(b, 0)) * H); ++b) off -= n;

    // the block's share of the pair that `off` lies in: `here` units from the pair's unit `first` of n on
    Segment s;
    uint32_t n, first, here;
    auto place = [&]() {
        s = segment(b, 0);
        n = units(s);
        s.h = off / n;
        first = off - s.h * n;
        here = min(n - first, end - cur);
        if (s.count > 0) {
            s.first = first * unit;
            s.count = min(here * unit, s.tiles.count - s.first);
        }
    };
    place();
    w.begin(s, wave, NW, wave);
    while (true) {
        w.run(s, wave, NW);
        const bool alone = here == n, any = s.tiles.count > 0;
        const uint32_t at = cur - first, of = n;       // the pair's units
        const int64_t pair = (int64_t)b * H + s.h;
        const int slot = 2 * (int)blockIdx.x + (first == 0 ? 1 : 0);
        cur += here;
        off += here;
        if (off == n * H) { off = 0; ++b; }
        const bool more = cur < end;
        if (more) {                                    // the next pair's first rows are under way while this one's results are joined
            place();
            if constexpr (!A::QLDS) w.begin(s, wave, NW, wave);
        }
        LateArgs l = late_args();
        const int G = l->G;
        if (w.m < G) {
#pragma unroll
            for (int d = 0; d < D / 16; ++d) *(f32x4*)&acc[wave][w.m][d * 16 + w.part * 4] = w.o[d];
            if (w.part == 0) stat[wave][w.m] = make_float2(w.ref, w.sum);
        }
        lds_barrier();

        for (int i = tid; i < G * D; i += kThreads) {
            const int g = i / D, d = i - g * D;
            float ref = stat[0][g].x, sum = 0.f, o = 0.f;
#pragma unroll
            for (int x = 1; x < NW; ++x) ref = fmaxf(ref, stat[x][g].x);
#pragma unroll
            for (int x = 0; x < NW; ++x) {
                const float by = fast_exp2(stat[x][g].x - ref);
                sum = fmaf(by, stat[x][g].y, sum);
                o = fmaf(by, acc[x][g][d], o);
            }
            if (alone) {
                l->out[pair * G * D + i] = any ? o / sum : sum;                  // nothing visible: 0, or NaN
                if (d == 0 && l->lse) l->lse[pair * G + g] = any ? (ref + log2f(sum)) * 0.6931471805599453f : sum - INFINITY;
            } else {
                publish(l->part_o + (int64_t)slot * G * D + i, o);
                if (d == 0) { publish(l->part_ml + ((int64_t)slot * G + g) * 2, ref); publish(l->part_ml + ((int64_t)slot * G + g) * 2 + 1, sum); }
            }
        }
        if (!alone) join_parts<D>(parts_of(at, of, share), slot, pair, stat, acc, &arrived);
        if (!more) break;
        lds_barrier();                                 // the next pair's results go to the same LDS
        if constexpr (A::QLDS) w.begin(s, wave, NW, wave);
    }
}

template <int P, int D> hipError_t launch(PagedAttnArgs a, int compute_units, hipStream_t st)
{
    int64_t grid = compute_units < kPagedMaxBlocks ? compute_units : kPagedMaxBlocks;
    // no more blocks than could have units
    constexpr int unit = Form<P>::TILE * kUnitTiles;
    const int64_t units = (int64_t)a.batch * a.pages.heads * (((int64_t)a.pages.cols * a.pages.rows + unit - 1) / unit);
    if (grid > units) grid = units;
    a.blocks = (uint32_t)grid;
    if (a.window > 0) hipLaunchKernelGGL((paged_attn_kernel<P, D, true>), dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    else hipLaunchKernelGGL((paged_attn_kernel<P, D, false>), dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    return hipGetLastError();
}

template <int P> hipError_t launch(const PagedAttnArgs& a, int compute_units, hipStream_t st)
{
    switch (a.pages.D) {
        case 64: return launch<P, 64>(a, compute_units, st);
        case 128: return launch<P, 128>(a, compute_units, st);
        case 256: return launch<P, 256>(a, compute_units, st);
    }
    return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_paged_attn(int dtype, int page_dtype, const PagedAttnArgs& a, int compute_units, hipStream_t st)
{
    const bool e4m3 = page_dtype == BUZZ_E4M3;
    if (dtype == BUZZ_FP32) return launch<P_F32>(a, compute_units, st);
    if (dtype == BUZZ_FP16) return e4m3 ? launch<P_E4M3_F16>(a, compute_units, st) : launch<P_F16>(a, compute_units, st);
    return e4m3 ? launch<P_E4M3_BF16>(a, compute_units, st) : launch<P_BF16>(a, compute_units, st);
}

}  // namespace buzz
