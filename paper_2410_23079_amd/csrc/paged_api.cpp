// Host side of the paged cache and of the position rotation: C ABI, validation, workspace layout.  Lengths and pages are
// on the device; nothing is read back, and a call enqueues one kernel.
#include <math.h>
#include <new>

#include "paged_internal.h"

using namespace buzz;

namespace {

constexpr uint32_t kPagedMagic = 0xB0220CA6u;
constexpr int64_t kMaxTokens = (int64_t)1 << 28;       // tokens of a sequence in a cache

size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
bool is_power(int v) { return v > 0 && (v & (v - 1)) == 0; }
int elem_bytes(int dtype) { return dtype == BUZZ_FP32 ? 4 : 2; }
bool head_dim_ok(int d) { return d == 64 || d == 128 || d == 256; }
int hip_rc(hipError_t e) { return e == hipSuccess ? BUZZ_OK : BUZZ_EHIP; }

struct PagedLayout { size_t ticket, group_ticket, counters, part_ml, part_o, total; };

int make_layout(const buzz_paged_config_t* c, PagedLayout* L)
{
    if (!c || c->batch < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->n_pages < 1 || c->table_cols < 1) return BUZZ_EINVAL;
    if (c->n_q_heads % c->n_kv_heads || c->dtype < BUZZ_FP32 || c->dtype > BUZZ_BF16) return BUZZ_EINVAL;
    if (c->page_dtype != c->dtype && c->page_dtype != BUZZ_E4M3) return BUZZ_EINVAL;
    if (c->page_rows < 1 || c->sink < 0 || c->window < 0 || c->reserved != 0 || (c->flags & ~(uint32_t)BUZZ_FLAG_DRY_RUN)) return BUZZ_EINVAL;
    if (!(c->softmax_scale >= 0.f) || isinf(c->softmax_scale)) return BUZZ_EINVAL;
    const int G = c->n_q_heads / c->n_kv_heads;
    if (!head_dim_ok(c->head_dim) || G > 8 || (c->page_dtype == BUZZ_E4M3 && c->dtype == BUZZ_FP32)) return BUZZ_EUNSUPPORTED;
    if (!is_power(c->page_rows) || c->page_rows < kPagedTileTokens || c->page_rows > 256) return BUZZ_EUNSUPPORTED;
    if (c->batch > 65535 || c->n_kv_heads > 65535 || (int64_t)c->table_cols * c->page_rows > kMaxTokens) return BUZZ_EUNSUPPORTED;
    if ((double)c->n_kv_heads * c->page_rows * c->head_dim * elem_bytes(c->dtype) >= 4294967296.0) return BUZZ_EUNSUPPORTED;
    if (!units_countable(c->batch, c->n_kv_heads, c->table_cols, c->page_rows)) return BUZZ_EUNSUPPORTED;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += align_up(bytes); return at; };
    L->ticket = take((size_t)c->batch * c->n_kv_heads * sizeof(int32_t));
    L->group_ticket = take((size_t)2 * kPagedMaxBlocks * sizeof(int32_t));
    L->counters = off / sizeof(int32_t);               // all of them from the start of the workspace
    L->part_ml = take((size_t)2 * kPagedMaxBlocks * G * 2 * sizeof(float));
    L->part_o = take((size_t)2 * kPagedMaxBlocks * G * c->head_dim * sizeof(float));
    L->total = off;
    return BUZZ_OK;
}

// compute units of the current device (asked for once)
int compute_units()
{
    static int cus = 0;
    if (cus == 0) {
        int dev = 0, v = 0;
        cus = hipGetDevice(&dev) == hipSuccess && hipDeviceGetAttribute(&v, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && v > 0 ? v : 256;
    }
    return cus;
}

// Rows of the caller in bytes.  `rows`: the row distance counts; distances of a dimension of one do not.
int take_rows(const buzz_rows_t* r, int elem, int64_t batch, int64_t heads, int64_t rows, Rows* out)
{
    if (!r || !r->data) return BUZZ_EINVAL;
    *out = Rows{(char*)r->data, batch > 1 ? r->seq_stride * elem : 0, heads > 1 ? r->head_stride * elem : 0, rows > 1 ? r->row_stride * elem : 0};
    if (((uintptr_t)r->data | (uint64_t)out->seq | (uint64_t)out->head | (uint64_t)out->row) & 15) return BUZZ_EUNSUPPORTED;
    return BUZZ_OK;
}

// The rotary part of the kernel's arguments.
int take_rotary(const buzz_rotary_t* r, int D, RotateArgs* a)
{
    if (!r) return BUZZ_OK;
    if (r->reserved != 0 || r->rot_dim < 0 || r->rot_dim > D || (r->interleaved != 0 && r->interleaved != 1)) return BUZZ_EINVAL;
    if ((r->q_weight || r->k_weight) && !(r->eps >= 0.f)) return BUZZ_EINVAL;
    if (r->rot_dim > 0 && !r->inv_freq) return BUZZ_EINVAL;
    if (r->rot_dim % 16) return BUZZ_EUNSUPPORTED;
    if (((uintptr_t)r->q_weight | (uintptr_t)r->k_weight) & 15 || ((uintptr_t)r->inv_freq & 7)) return BUZZ_EUNSUPPORTED;
    a->q_weight = r->q_weight; a->k_weight = r->k_weight; a->inv_freq = r->inv_freq;
    a->eps = r->eps; a->half = r->rot_dim / 2; a->interleaved = r->interleaved;
    return BUZZ_OK;
}

}  // namespace

struct buzz_paged {
    uint32_t magic;
    buzz_paged_config_t cfg;
    PagedLayout L;
    buzz_pages_t pages;
    char* ws;
    float scale;
    bool dry;

    PageArgs args(const int32_t* table) const
    {
        PageArgs p{};
        p.k = (char*)pages.k; p.v = (char*)pages.v;
        p.k_exp = pages.k_exp; p.v_exp = pages.v_exp;
        p.table = table;
        p.n_pages = cfg.n_pages; p.rows = cfg.page_rows; p.rows_log2 = __builtin_ctz(cfg.page_rows); p.cols = cfg.table_cols;
        p.heads = cfg.n_kv_heads; p.D = cfg.head_dim;
        return p;
    }
};

namespace {

bool alive(const buzz_paged_t* c) { return c && c->magic == kPagedMagic; }

// What append and read ask of batch, rows and table.
int check_call(const buzz_paged_t* c, int32_t batch, int64_t n_rows, const int32_t* table)
{
    if (!alive(c) || batch < 0 || n_rows < 0) return BUZZ_EINVAL;
    if (!c->dry && batch > 0 && n_rows > 0 && !table) return BUZZ_EINVAL;
    if (batch > c->cfg.batch || n_rows > (int64_t)c->cfg.table_cols * c->cfg.page_rows) return BUZZ_ECAPACITY;
    return rows_launchable(n_rows, (int64_t)c->cfg.n_q_heads + 2 * (int64_t)c->cfg.n_kv_heads) ? BUZZ_OK : BUZZ_EUNSUPPORTED;
}

}  // namespace

extern "C" {

int buzz_qk_norm_rotate(int32_t dtype, int32_t head_dim, int32_t n_q_heads, int32_t n_kv_heads, const buzz_rotary_t* rotary,
                        const buzz_rows_t* q, const buzz_rows_t* k, const buzz_rows_t* q_out, const buzz_rows_t* k_out,
                        int32_t batch, int64_t n_rows, const int32_t* start, const int32_t* count, void* hip_stream)
{
    if (dtype < BUZZ_FP32 || dtype > BUZZ_BF16 || head_dim < 1 || batch < 0 || n_rows < 0 || !rotary) return BUZZ_EINVAL;
    if ((q != nullptr) != (q_out != nullptr) || (k != nullptr) != (k_out != nullptr)) return BUZZ_EINVAL;
    if ((q && n_q_heads < 1) || (k && n_kv_heads < 1)) return BUZZ_EINVAL;
    if (!head_dim_ok(head_dim) || batch > 65535 || !rows_launchable(n_rows, (q ? (int64_t)n_q_heads : 0) + (k ? (int64_t)n_kv_heads : 0))) return BUZZ_EUNSUPPORTED;
    RotateArgs a{};
    if (int rc = take_rotary(rotary, head_dim, &a)) return rc;
    if (batch == 0 || n_rows == 0) return BUZZ_OK;
    const int elem = elem_bytes(dtype);
    if (q) {
        if (int rc = take_rows(q, elem, batch, n_q_heads, n_rows, &a.q)) return rc;
        if (int rc = take_rows(q_out, elem, batch, n_q_heads, n_rows, &a.q_out)) return rc;
    }
    if (k) {
        if (int rc = take_rows(k, elem, batch, n_kv_heads, n_rows, &a.k)) return rc;
        if (int rc = take_rows(k_out, elem, batch, n_kv_heads, n_rows, &a.k_out)) return rc;
    }
    a.start = start; a.count = count; a.n_rows = n_rows;
    a.Hq = n_q_heads; a.Hkv = n_kv_heads; a.D = head_dim;
    return hip_rc(launch_rotate(dtype, dtype, a, batch, (hipStream_t)hip_stream));
}

int buzz_paged_workspace_bytes(const buzz_paged_config_t* cfg, size_t* bytes)
{
    if (!cfg || !bytes) return BUZZ_EINVAL;
    PagedLayout L;
    if (int rc = make_layout(cfg, &L)) return rc;
    *bytes = L.total;
    return BUZZ_OK;
}

int buzz_paged_create(const buzz_paged_config_t* cfg, const buzz_pages_t* pages, void* dev_workspace, size_t bytes,
                      void* hip_stream, buzz_paged_t** out)
{
    if (!cfg || !out) return BUZZ_EINVAL;
    PagedLayout L;
    if (int rc = make_layout(cfg, &L)) return rc;
    const bool dry = cfg->flags & BUZZ_FLAG_DRY_RUN, e4m3 = cfg->page_dtype == BUZZ_E4M3;
    if (!dry) {
        if (!pages || !pages->k || !pages->v || !dev_workspace || ((uintptr_t)dev_workspace & 255)) return BUZZ_EINVAL;
        if (e4m3 != (pages->k_exp != nullptr) || e4m3 != (pages->v_exp != nullptr)) return BUZZ_EINVAL;
        if (((uintptr_t)pages->k | (uintptr_t)pages->v | (uintptr_t)pages->k_exp | (uintptr_t)pages->v_exp) & 15) return BUZZ_EINVAL;
        if (bytes < L.total) return BUZZ_ECAPACITY;
    }
    buzz_paged_t* c = new (std::nothrow) buzz_paged_t();
    if (!c) return BUZZ_EINVAL;
    c->magic = kPagedMagic;
    c->cfg = *cfg;
    c->L = L;
    if (pages) c->pages = *pages;
    c->ws = (char*)dev_workspace;
    c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / sqrtf((float)cfg->head_dim);
    c->dry = dry;
    if (!dry) {
        if (hipError_t e = launch_clear_f32((float*)c->ws, (int64_t)L.counters, (hipStream_t)hip_stream)) {
            delete c;
            return hip_rc(e);
        }
    }
    *out = c;
    return BUZZ_OK;
}

int buzz_paged_destroy(buzz_paged_t* c)
{
    if (!c) return BUZZ_OK;
    if (!alive(c)) return BUZZ_EINVAL;
    c->magic = 0;
    delete c;
    return BUZZ_OK;
}

int buzz_paged_append(buzz_paged_t* c, const buzz_rotary_t* rotary, const buzz_rows_t* q, const buzz_rows_t* k,
                      const buzz_rows_t* v, const buzz_rows_t* q_out, int32_t batch, int64_t n_rows,
                      const int32_t* page_table, const int32_t* start, const int32_t* count, void* hip_stream)
{
    if (int rc = check_call(c, batch, n_rows, page_table)) return rc;
    const buzz_paged_config_t& cfg = c->cfg;
    if ((q != nullptr) != (q_out != nullptr)) return BUZZ_EINVAL;
    RotateArgs a{};
    if (int rc = take_rotary(rotary, cfg.head_dim, &a)) return rc;
    if (c->dry || batch == 0 || n_rows == 0) return BUZZ_OK;
    const int elem = elem_bytes(cfg.dtype);
    if (q) {
        if (int rc = take_rows(q, elem, batch, cfg.n_q_heads, n_rows, &a.q)) return rc;
        if (int rc = take_rows(q_out, elem, batch, cfg.n_q_heads, n_rows, &a.q_out)) return rc;
    }
    if (int rc = take_rows(k, elem, batch, cfg.n_kv_heads, n_rows, &a.k)) return rc;
    if (int rc = take_rows(v, elem, batch, cfg.n_kv_heads, n_rows, &a.v)) return rc;
    a.start = start; a.count = count; a.n_rows = n_rows;
    a.Hq = cfg.n_q_heads; a.Hkv = cfg.n_kv_heads; a.D = cfg.head_dim;
    a.pages = c->args(page_table);
    return hip_rc(launch_rotate(cfg.dtype, cfg.page_dtype, a, batch, (hipStream_t)hip_stream));
}

int buzz_paged_read(buzz_paged_t* c, const buzz_rows_t* k, const buzz_rows_t* v, int32_t batch, int64_t n_rows,
                    const int32_t* page_table, const int32_t* start, const int32_t* count, void* hip_stream)
{
    if (int rc = check_call(c, batch, n_rows, page_table)) return rc;
    if (c->dry || batch == 0 || n_rows == 0) return BUZZ_OK;
    ReadArgs a{};
    const int elem = elem_bytes(c->cfg.dtype);
    if (k)
        if (int rc = take_rows(k, elem, batch, c->cfg.n_kv_heads, n_rows, &a.k)) return rc;
    if (v)
        if (int rc = take_rows(v, elem, batch, c->cfg.n_kv_heads, n_rows, &a.v)) return rc;
    a.start = start; a.count = count; a.n_rows = n_rows;
    a.pages = c->args(page_table);
    return hip_rc(launch_paged_read(c->cfg.dtype, c->cfg.page_dtype, a, batch, (hipStream_t)hip_stream));
}

int buzz_paged_decode(buzz_paged_t* c, const buzz_rows_t* q, int32_t batch, const int32_t* page_table,
                      const int32_t* length, float* out, float* lse, void* hip_stream)
{
    if (!alive(c) || batch < 0) return BUZZ_EINVAL;
    if (batch > c->cfg.batch) return BUZZ_ECAPACITY;
    if (c->dry || batch == 0) return BUZZ_OK;
    if (!page_table || !length || !out) return BUZZ_EINVAL;
    const buzz_paged_config_t& cfg = c->cfg;
    Rows rows;
    if (int rc = take_rows(q, elem_bytes(cfg.dtype), batch, cfg.n_q_heads, 1, &rows)) return rc;
    if ((uintptr_t)out & 15) return BUZZ_EUNSUPPORTED;
    PagedAttnArgs a{};
    a.q = rows.data; a.q_seq = rows.seq; a.q_head = rows.head;
    a.out = out; a.lse = lse;
    a.length = length;
    a.pages = c->args(page_table);
    a.ticket = (int32_t*)(c->ws + c->L.ticket);
    a.group_ticket = (int32_t*)(c->ws + c->L.group_ticket);
    a.part_ml = (float*)(c->ws + c->L.part_ml);
    a.part_o = (float*)(c->ws + c->L.part_o);
    a.batch = batch; a.G = cfg.n_q_heads / cfg.n_kv_heads;
    a.sink = cfg.sink; a.window = cfg.window;
    a.scale_log2 = c->scale * 1.4426950408889634f;
    a.page_bytes = (uint32_t)cfg.n_kv_heads * cfg.page_rows * cfg.head_dim * (cfg.page_dtype == BUZZ_E4M3 ? 1 : elem_bytes(cfg.dtype));
    return hip_rc(launch_paged_attn(cfg.dtype, cfg.page_dtype, a, compute_units(), (hipStream_t)hip_stream));
}

}  // extern "C"
