// Internal declarations of the paged cache and of the position rotation, shared by their host code and kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "buzz.h"

namespace buzz {

constexpr int kPagedMaxBlocks = 512;       // blocks of a decode step; the workspace holds two partial results for each
constexpr int kPagedTileTokens = 16;       // positions that one block of the row kernels works on: every page is whole tiles

struct Rows {                              // [sequence][head][row][head_dim], distances in bytes
    char* data;
    int64_t seq, head, row;
};

// The pages of one cache.  `rows` is a power of two, so are the elements in 16 bytes (g): page rows of a lane's
// 16-byte pieces never cross a page.
struct PageArgs {
    char* k; char* v;
    uint8_t* k_exp; uint8_t* v_exp;        // NULL unless the pages hold 8 bits
    const int32_t* table;                  // [batch][cols]
    int32_t n_pages, rows, rows_log2, cols;
    int32_t heads, D;
};

// The page of token j, or -1: a number that is none of the pool's is never followed.  The caller has made sure that
// 0 <= j < cols * rows.
__host__ __device__ inline int32_t page_of(const int32_t* table_row, int64_t j, int32_t rows_log2, int32_t n_pages)
{
    const int32_t p = table_row[j >> rows_log2];
    return p >= 0 && p < n_pages ? p : -1;
}

// Which rows of a sequence a call handles: positions [lo, hi) of rows lo - start ..; empty where nothing is there.
struct Span { int64_t start, lo, hi; };
__host__ __device__ inline Span row_span(const int32_t* start, const int32_t* count, int b, int64_t n_rows)
{
    const int64_t s = start ? start[b] : 0;
    int64_t n = count ? count[b] : n_rows;
    n = n < 0 ? 0 : n > n_rows ? n_rows : n;
    return s < 0 ? Span{0, 0, 0} : Span{s, s, s + n};
}

// Tiles of 16 positions that n rows can touch, wherever the first one stands.
__host__ __device__ inline int64_t tiles_of_rows(int64_t n) { return n <= 0 ? 0 : (n + 14) / kPagedTileTokens + 1; }
// Whether a grid has room for them: fewer than 2^32 threads, 256 for a tile and head at most.
inline bool rows_launchable(int64_t n, int64_t heads) { return heads <= 65535 && n <= 1 << 28 && tiles_of_rows(n) * heads <= UINT32_MAX / 256; }

// Keys that the new token of a sequence of `length` tokens attends to: [0, sink_end) and [from, length).
struct Visible {
    int32_t length, from, sink_end;        // length < 0: the caller's length is none
    __host__ __device__ inline bool sees(int32_t j) const { return j < length && (j >= from || j < sink_end); }
    // ... of the n <= 16 keys from j on, bit by bit
    __host__ __device__ inline uint32_t bits(int32_t j, int32_t n) const { return below(sink_end - j, n) | (below(length - j, n) & ~below(from - j, n)); }
    __host__ __device__ static inline uint32_t below(int32_t k, int32_t n) { return (1u << (k < 0 ? 0 : k > n ? n : k)) - 1u; }
};
__host__ __device__ inline Visible visible(int32_t length, int32_t sink, int32_t window, int64_t most)
{
    if (length < 0 || length > most) return Visible{-1, 0, 0};
    const int32_t from = window > 0 && length > window ? length - window : 0;
    return Visible{length, from, sink < from ? sink : from};
}

// The tiles of `tile` keys that hold them, in order: the first `low` ones, then those from `high` on; `count` in all.
struct Tiles {
    int32_t low, high, count;
    __host__ __device__ inline int32_t at(int32_t i) const { return i < low ? i : high + (i - low); }
};
__host__ __device__ inline Tiles tiles_of(const Visible& v, int32_t tile)
{
    if (v.length <= 0) return Tiles{0, 0, 0};
    const int32_t end = (v.length - 1) / tile + 1, high = v.from / tile;
    int32_t low = v.sink_end > 0 ? (v.sink_end - 1) / tile + 1 : 0;
    if (low > high) low = high;
    return Tiles{low, high, low + end - high};
}

// A decode step's work is cut into units of `unit` tiles of one (sequence, head) pair.  The units of all pairs are numbered
// through, `share` consecutive ones to a block.  A pair of n units from number `begin` on is worked on by `parts` blocks from
// `from` on; each but the one with the pair's first unit leaves its partial result in its slot 0, that one in slot 1, so a block
// that ends one pair and begins another needs two.
constexpr int kUnitTiles = 4;              // the least
__host__ __device__ inline uint32_t units_of(int32_t tiles, uint32_t unit) { return tiles > 0 ? ((uint32_t)tiles + unit - 1) / unit : 1; }   // somebody has to write an empty pair's output
__host__ __device__ inline uint32_t units_per_block(uint32_t total, uint32_t blocks) { return (total + blocks - 1) / blocks; }
// Up to how many tiles a pair is left whole.  Reading 128 KB takes a compute unit about as long as it takes to publish partial
// results and to add them up; with as many pairs as blocks four times that, because cutting pairs then leaves most blocks with
// parts of two (bf16, 4 heads of 128, tiles of 16 KB: 64 pairs of 13 tiles whole 10.1 us, cut 8.8; 256 of 10 to 19 tiles 13.6 / 17.5).
__host__ __device__ inline uint32_t whole_tiles(uint32_t tile_bytes, uint32_t pairs, uint32_t blocks)
{
    const uint32_t times = pairs >= blocks ? 4 : 4 * pairs / blocks;
    return 131072 / tile_bytes * (times < 1 ? 1 : times);
}
struct Parts {
    int from, parts;
    __host__ __device__ inline int slot(int i) const { return 2 * (from + i) + (i == 0 ? 1 : 0); }
};
__host__ __device__ inline Parts parts_of(uint32_t begin, uint32_t n, uint32_t share)
{
    const int from = (int)(begin / share);
    return Parts{from, (int)((begin + n - 1) / share) - from + 1};
}
// Partial results are added up sixteen or so at a time: those of a pair with more are added up by groups first.  Part i belongs
// to the group of part i / group * group, whose slot takes the group's sum and numbers the group's arrival counter.
__host__ __device__ inline int group_of(int parts) { return parts <= 16 ? 1 : parts <= 256 ? 16 : 32; }

// Most units that a cache's configuration can lead to, of the smallest tiles (16 keys): they have to be countable in 31 bits.
inline bool units_countable(int64_t batch, int64_t heads, int64_t cols, int64_t rows)
{
    return batch * heads <= INT32_MAX && (double)batch * (double)heads * (double)((cols * rows + 63) / 64) < 2147483648.0;
}

struct RotateArgs {
    Rows q, k, v, q_out, k_out;            // data NULL: not there; k_out of the dense form only
    const void* q_weight; const void* k_weight;
    const double* inv_freq;
    const int32_t* start; const int32_t* count;
    int64_t n_rows;
    float eps;
    int32_t half;                          // rot_dim / 2
    int32_t interleaved;
    int32_t Hq, Hkv, D;
    int32_t q_chunk, kv_chunk, v_chunk, q_jobs, k_jobs, v_jobs;   // heads per block; blocks per tile of positions (set by the launch)
    PageArgs pages;                        // k NULL: dense
};

struct ReadArgs {
    Rows k, v;
    const int32_t* start; const int32_t* count;
    int64_t n_rows;
    PageArgs pages;
    int32_t chunk, k_jobs, v_jobs;         // likewise
};

struct PagedAttnArgs {
    const char* q;
    int64_t q_seq, q_head;                 // bytes
    float* out; float* lse;
    const int32_t* length;
    PageArgs pages;
    float* part_o;                         // [blocks][2][G][D] unnormalised outputs
    float* part_ml;                        // [blocks][2][G][2] (reference, sum)
    int32_t* ticket;                       // [batch * heads], arrivals of a pair's parts or groups; zero between launches
    int32_t* group_ticket;                 // [2 * kPagedMaxBlocks], of a group's parts, by slot; likewise
    int32_t batch, G;
    int32_t sink, window;
    float scale_log2;
    uint32_t page_bytes;                   // of one page of K, or of V: under 4 GiB
    uint32_t blocks;                       // the grid (set by the launch)
};

hipError_t launch_rotate(int dtype, int page_dtype, const RotateArgs& a, int batch, hipStream_t st);
hipError_t launch_paged_read(int dtype, int page_dtype, const ReadArgs& a, int batch, hipStream_t st);
hipError_t launch_paged_attn(int dtype, int page_dtype, const PagedAttnArgs& a, int compute_units, hipStream_t st);
hipError_t launch_clear_f32(float* dst, int64_t n, hipStream_t st);

}  // namespace buzz
