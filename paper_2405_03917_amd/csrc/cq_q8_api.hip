// Host entry points of the 8-bit block cache (cq_*_q8): argument validation and sizes.  Every check runs before any HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cq_q8.hpp"

namespace cq {
namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// an array of a call (no bytes: one that is not there)
struct Span {
    const void* at;
    size_t bytes;
};
bool overlap(const Span& a, const Span& b)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return a.bytes && b.bytes && x < y + b.bytes && y < x + a.bytes;
}

cq_status check_format(const cq_q8_format* fmt)
{
    if (!fmt || fmt->head_dim <= 0 || fmt->n_kv_heads <= 0 || fmt->n_kv_heads > 65535) return CQ_ERR_INVALID_ARG;
    if (fmt->kind != CQ_Q8_INT8 && fmt->kind != CQ_Q8_E4M3) return CQ_ERR_INVALID_ARG;
    return fmt->head_dim == kQ8Head ? CQ_OK : CQ_ERR_UNSUPPORTED;
}

// What all calls share: the cache, where its tiles lie, the sequences' lengths.  `pages` or t_cap.
struct Call {
    Q8Cache cache;
    Span spans[5];                                          // code and scale arrays, block table
    cq_status check(const cq_q8_cache* c, const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, int32_t t_cap,
                    const cq_page_table* pages, bool paged, const int32_t* seq_lens)
    {
        const cq_status st = check_format(fmt);
        if (st != CQ_OK) return st;
        if (!c || !c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return CQ_ERR_INVALID_ARG;
        if (!aligned16(c->k_codes) || !aligned16(c->v_codes) || !aligned16(c->k_scales) || !aligned16(c->v_scales)) return CQ_ERR_INVALID_ARG;
        if (batch <= 0 || batch > 32767 || !aligned4(seq_lens)) return CQ_ERR_INVALID_ARG;
        size_t tiles;
        if (paged) {
            if (!pages || !pages->block_table || pages->n_pages <= 0 || pages->max_tiles <= 0 || pages->max_tiles > (1 << 24)) return CQ_ERR_INVALID_ARG;
            if (pages->row_stride < pages->max_tiles || !aligned4(pages->block_table)) return CQ_ERR_INVALID_ARG;
            cache.map = CacheMap{pages->block_table, pages->row_stride, pages->n_pages, 0, fmt->n_kv_heads};
            t_cap = pages->max_tiles * kTileTokens;
            tiles = (size_t)pages->n_pages * fmt->n_kv_heads;
            spans[4] = Span{pages->block_table, sizeof(int32_t) * ((size_t)(batch - 1) * pages->row_stride + pages->max_tiles)};
        } else {
            if (t_cap <= 0 || t_cap % kTileTokens != 0) return CQ_ERR_INVALID_ARG;
            cache.map = CacheMap{nullptr, 0, 0, t_cap / kTileTokens, fmt->n_kv_heads};
            tiles = (size_t)batch * fmt->n_kv_heads * (t_cap / kTileTokens);
            spans[4] = Span{nullptr, 0};
        }
        if (m <= 0 || t < m || t > t_cap) return CQ_ERR_INVALID_ARG;
        cache.codes[0] = static_cast<uint8_t*>(c->k_codes);
        cache.codes[1] = static_cast<uint8_t*>(c->v_codes);
        cache.scales[0] = c->k_scales;
        cache.scales[1] = c->v_scales;
        for (int i = 0; i < 2; ++i) {
            spans[i] = Span{cache.codes[i], tiles * kQ8TileBytes};
            spans[2 + i] = Span{cache.scales[i], tiles * sizeof(float)};
        }
        return CQ_OK;
    }
    bool touches(const Span& s) const
    {
        for (const Span& mine : spans)
            if (overlap(mine, s)) return true;
        return false;
    }
};

// fp16 [batch][m][width] by element strides (multiples of 8): checked, and the bytes from its first element to its last.
cq_status check_strided(const void* x, int64_t batch_stride, int64_t row_stride, int32_t batch, int32_t m, int64_t width, Span* span)
{
    if (!x || !aligned16(x)) return CQ_ERR_INVALID_ARG;
    if (row_stride < width || row_stride % 8 != 0 || row_stride > (int64_t{1} << 40)) return CQ_ERR_INVALID_ARG;
    if (batch > 1 && (batch_stride < (int64_t)m * row_stride || batch_stride % 8 != 0 || batch_stride > (int64_t{1} << 45))) return CQ_ERR_INVALID_ARG;
    *span = Span{x, sizeof(uint16_t) * (size_t)((batch > 1 ? (batch - 1) * batch_stride : 0) + (m - 1) * row_stride + width)};
    return CQ_OK;
}

// Whether two arrays of such rows, of the same strides, share an element: rows `apart` elements from one another, or that less
// whole batch strides and row strides.  All rows of a sequence lie within a batch stride, so two neighbouring multiples of it can do, and of
// row strides the two next to what is left.
bool rows_overlap(const void* x, const void* y, int64_t batch_stride, int64_t row_stride, int32_t batch, int32_t m, int64_t width)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(x), q = reinterpret_cast<uintptr_t>(y);
    const int64_t apart = (int64_t)((p < q ? q - p : p - q) / sizeof(uint16_t));
    const int64_t first = batch > 1 ? apart / batch_stride : 0;
    for (int64_t n = first; n <= first + 1 && n < batch; ++n) {
        const int64_t left = apart - (batch > 1 ? n * batch_stride : 0), within = left < 0 ? -left : left;
        for (int64_t j = within / row_stride; j <= within / row_stride + 1; ++j) {
            const int64_t rest = within - j * row_stride;
            if (j < m && rest < width && -rest < width) return true;
        }
    }
    return false;
}

void set_rows(Q8Rows* r, const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, const int32_t* seq_lens)
{
    r->batch = batch;
    r->m = m;
    r->t = t;
    r->n_kv_heads = fmt->n_kv_heads;
    r->seq_lens = seq_lens;
}

cq_status append_common(const void* x_k, const void* x_v, int64_t x_batch_stride, int64_t x_row_stride, const cq_q8_cache* cache,
                        const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, int32_t t_cap, const cq_page_table* pages, bool paged,
                        const int32_t* seq_lens, const void* rope_table, int32_t rope_positions,
                        const void* q, int64_t q_batch_stride, int64_t q_row_stride, int32_t n_q_heads, void* q_out, void* stream)
{
    Call call;
    cq_status st = call.check(cache, fmt, batch, m, t, t_cap, pages, paged, seq_lens);
    if (st != CQ_OK) return st;
    const int64_t width = (int64_t)fmt->n_kv_heads * kQ8Head;
    Span read[5] = {};
    if ((st = check_strided(x_k, x_batch_stride, x_row_stride, batch, m, width, &read[0])) != CQ_OK) return st;
    if ((st = check_strided(x_v, x_batch_stride, x_row_stride, batch, m, width, &read[1])) != CQ_OK) return st;
    read[2] = Span{seq_lens, seq_lens ? sizeof(int32_t) * batch : 0};
    if (rope_table) {
        if (!aligned16(rope_table) || rope_positions <= 0 || rope_positions % kTileTokens != 0 || rope_positions < t) return CQ_ERR_INVALID_ARG;
        read[3] = Span{rope_table, q8_rope_table_bytes(rope_positions)};
    } else if (rope_positions != 0) {
        return CQ_ERR_INVALID_ARG;
    }
    Span written{nullptr, 0};
    if (q || q_out) {
        if (!rope_table || !q_out || !aligned16(q_out) || n_q_heads <= 0 || n_q_heads % fmt->n_kv_heads != 0) return CQ_ERR_INVALID_ARG;
        const int64_t q_width = (int64_t)n_q_heads * kQ8Head;
        if ((st = check_strided(q, q_batch_stride, q_row_stride, batch, m, q_width, &read[4])) != CQ_OK) return st;
        written = Span{q_out, sizeof(uint16_t) * (size_t)((int64_t)batch * m * q_width)};
        if (q == q_out) {                                   // in place: every element where it was
            if ((m > 1 && q_row_stride != q_width) || (batch > 1 && q_batch_stride != m * q_width)) return CQ_ERR_INVALID_ARG;
            read[4].bytes = 0;
        }
        if (call.touches(written)) return CQ_ERR_INVALID_ARG;
    }
    for (int i = 0; i < 5; ++i) {
        if (overlap(written, read[i])) return CQ_ERR_INVALID_ARG;
        for (int k = 0; k < 4; ++k)
            if (overlap(call.spans[k], read[i]) || overlap(call.spans[k], call.spans[4])) return CQ_ERR_INVALID_ARG;
    }
    for (int i = 0; i < 4; ++i)
        for (int k = 0; k < i; ++k)
            if (overlap(call.spans[i], call.spans[k])) return CQ_ERR_INVALID_ARG;
    Q8AppendArgs a{};
    set_rows(&a, fmt, batch, m, t, seq_lens);
    a.x[0] = static_cast<const uint16_t*>(x_k);
    a.x[1] = static_cast<const uint16_t*>(x_v);
    a.x_batch_stride = x_batch_stride;
    a.x_row_stride = x_row_stride;
    a.cache = call.cache;
    if (rope_table) {
        a.tile_tab = static_cast<const double2*>(rope_table);
        a.lane_tab = a.tile_tab + (size_t)(rope_positions / kTileTokens) * kQ8Pairs;
    }
    a.q = static_cast<const uint16_t*>(q);
    a.q_batch_stride = q_batch_stride;
    a.q_row_stride = q_row_stride;
    a.n_q_heads = n_q_heads;
    a.q_out = static_cast<uint16_t*>(q_out);
    return launch_append_q8(a, fmt->kind, static_cast<hipStream_t>(stream));
}

cq_status dequantize_common(const cq_q8_cache* cache, const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, int32_t t_cap,
                            const cq_page_table* pages, bool paged, const int32_t* seq_lens,
                            void* k_out, void* v_out, int64_t out_batch_stride, int64_t out_row_stride, void* stream)
{
    Call call;
    cq_status st = call.check(cache, fmt, batch, m, t, t_cap, pages, paged, seq_lens);
    if (st != CQ_OK) return st;
    if (!k_out && !v_out) return CQ_ERR_INVALID_ARG;
    const int64_t width = (int64_t)fmt->n_kv_heads * kQ8Head;
    Span out[2] = {};
    void* const ptr[2] = {k_out, v_out};
    for (int i = 0; i < 2; ++i) {
        if (!ptr[i]) continue;
        if ((st = check_strided(ptr[i], out_batch_stride, out_row_stride, batch, m, width, &out[i])) != CQ_OK) return st;
        if (call.touches(out[i]) || overlap(out[i], Span{seq_lens, seq_lens ? sizeof(int32_t) * batch : 0})) return CQ_ERR_INVALID_ARG;
    }
    if (k_out && v_out && rows_overlap(k_out, v_out, out_batch_stride, out_row_stride, batch, m, width)) return CQ_ERR_INVALID_ARG;
    Q8DequantArgs a{};
    set_rows(&a, fmt, batch, m, t, seq_lens);
    a.cache = call.cache;
    a.out[0] = static_cast<uint16_t*>(k_out);
    a.out[1] = static_cast<uint16_t*>(v_out);
    a.out_batch_stride = out_batch_stride;
    a.out_row_stride = out_row_stride;
    return launch_dequantize_q8(a, fmt->kind, static_cast<hipStream_t>(stream));
}

bool good_attention(const cq_q8_format* fmt, int32_t batch, int32_t n_q_heads, int32_t m, int32_t t, int32_t tokens_per_split)
{
    return batch > 0 && batch <= 32767 && n_q_heads > 0 && n_q_heads % fmt->n_kv_heads == 0 && m > 0 && t >= m && tokens_per_split >= 0 &&
           tokens_per_split % kTileTokens == 0 && (int64_t)batch * m * n_q_heads <= 0x7fffffffLL;
}
size_t attention_workspace(int32_t batch, int32_t n_q_heads, int32_t m, const Q8Plan& plan)
{
    return plan.n_split == 1 ? 16 : sizeof(float) * (size_t)batch * m * n_q_heads * plan.n_split * kQ8Partial;
}

cq_status attention_common(const void* q, const cq_q8_cache* cache, float scale, const cq_q8_format* fmt, int32_t batch, int32_t n_q_heads,
                           int32_t m, int32_t t, int32_t t_cap, const cq_page_table* pages, bool paged, const int32_t* seq_lens,
                           int32_t tokens_per_split, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    Call call;
    cq_status st = call.check(cache, fmt, batch, m, t, t_cap, pages, paged, seq_lens);
    if (st != CQ_OK) return st;
    if (!good_attention(fmt, batch, n_q_heads, m, t, tokens_per_split) || !std::isfinite(scale)) return CQ_ERR_INVALID_ARG;
    if (!q || !out || !workspace || !aligned16(q) || !aligned16(out) || !aligned16(workspace)) return CQ_ERR_INVALID_ARG;
    const Q8Plan plan = q8_plan(batch, fmt->n_kv_heads, n_q_heads, m, t, tokens_per_split);
    const size_t need = attention_workspace(batch, n_q_heads, m, plan);
    if (workspace_bytes < need) return CQ_ERR_WORKSPACE_TOO_SMALL;
    const size_t bytes = sizeof(uint16_t) * (size_t)batch * m * n_q_heads * kQ8Head;
    const Span in{q, bytes}, lens{seq_lens, seq_lens ? sizeof(int32_t) * batch : 0}, to{out, bytes}, work{workspace, plan.n_split == 1 ? 0 : need};
    if (call.touches(to) || call.touches(work) || overlap(to, in) || overlap(to, lens) || overlap(to, work) || overlap(work, in) || overlap(work, lens))
        return CQ_ERR_INVALID_ARG;
    Q8AttentionArgs a{};
    set_rows(&a, fmt, batch, m, t, seq_lens);
    a.q = static_cast<const uint16_t*>(q);
    a.out = static_cast<uint16_t*>(out);
    a.cache = call.cache;
    a.scale_log2e = scale * 1.4426950408889634f;
    a.n_q_heads = n_q_heads;
    a.tiles_per_split = plan.tiles_per_split;
    a.n_split = plan.n_split;
    a.partials = static_cast<float*>(workspace);
    return launch_attention_q8(a, fmt->kind, plan, static_cast<hipStream_t>(stream));
}

}  // namespace
}  // namespace cq

using namespace cq;

extern "C" {

size_t cq_q8_cache_bytes(const cq_q8_format* fmt, int32_t batch, int32_t t_cap)
{
    if (check_format(fmt) != CQ_OK || batch <= 0 || t_cap <= 0 || t_cap % kTileTokens != 0) return 0;
    return (size_t)batch * fmt->n_kv_heads * (t_cap / kTileTokens) * kQ8TileBytes;
}

size_t cq_q8_paged_cache_bytes(const cq_q8_format* fmt, int32_t n_pages)
{
    if (check_format(fmt) != CQ_OK || n_pages <= 0) return 0;
    return (size_t)n_pages * fmt->n_kv_heads * kQ8TileBytes;
}

size_t cq_q8_rope_table_bytes(int32_t head_dim, int32_t positions)
{
    if (head_dim != kQ8Head || positions <= 0 || positions % kTileTokens != 0) return 0;
    return q8_rope_table_bytes(positions);
}

cq_status cq_q8_rope_table(double base, int32_t head_dim, int32_t positions, void* table, size_t table_bytes, void* stream)
{
    if (head_dim <= 0 || positions <= 0 || positions % kTileTokens != 0 || !(base > 0.0) || !std::isfinite(base)) return CQ_ERR_INVALID_ARG;
    if (head_dim != kQ8Head) return CQ_ERR_UNSUPPORTED;
    if (!table || !aligned16(table)) return CQ_ERR_INVALID_ARG;
    if (table_bytes < q8_rope_table_bytes(positions)) return CQ_ERR_WORKSPACE_TOO_SMALL;
    return launch_q8_rope_table(base, positions, table, static_cast<hipStream_t>(stream));
}

cq_status cq_append_q8(const void* x_k, const void* x_v, int64_t x_batch_stride, int64_t x_row_stride, const cq_q8_cache* cache,
                       const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, int32_t t_cap, const int32_t* seq_lens,
                       const void* rope_table, int32_t rope_positions,
                       const void* q, int64_t q_batch_stride, int64_t q_row_stride, int32_t n_q_heads, void* q_out, void* stream)
{
    return append_common(x_k, x_v, x_batch_stride, x_row_stride, cache, fmt, batch, m, t, t_cap, nullptr, false, seq_lens, rope_table,
                         rope_positions, q, q_batch_stride, q_row_stride, n_q_heads, q_out, stream);
}

cq_status cq_append_q8_paged(const void* x_k, const void* x_v, int64_t x_batch_stride, int64_t x_row_stride, const cq_q8_cache* cache,
                             const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, const cq_page_table* pages, const int32_t* seq_lens,
                             const void* rope_table, int32_t rope_positions,
                             const void* q, int64_t q_batch_stride, int64_t q_row_stride, int32_t n_q_heads, void* q_out, void* stream)
{
    return append_common(x_k, x_v, x_batch_stride, x_row_stride, cache, fmt, batch, m, t, 0, pages, true, seq_lens, rope_table,
                         rope_positions, q, q_batch_stride, q_row_stride, n_q_heads, q_out, stream);
}

cq_status cq_dequantize_q8(const cq_q8_cache* cache, const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t, int32_t t_cap,
                           const int32_t* seq_lens, void* k_out, void* v_out, int64_t out_batch_stride, int64_t out_row_stride, void* stream)
{
    return dequantize_common(cache, fmt, batch, m, t, t_cap, nullptr, false, seq_lens, k_out, v_out, out_batch_stride, out_row_stride, stream);
}

cq_status cq_dequantize_q8_paged(const cq_q8_cache* cache, const cq_q8_format* fmt, int32_t batch, int32_t m, int32_t t,
                                 const cq_page_table* pages, const int32_t* seq_lens,
                                 void* k_out, void* v_out, int64_t out_batch_stride, int64_t out_row_stride, void* stream)
{
    return dequantize_common(cache, fmt, batch, m, t, 0, pages, true, seq_lens, k_out, v_out, out_batch_stride, out_row_stride, stream);
}

int32_t cq_attention_q8_default_split(const cq_q8_format* fmt, int32_t batch, int32_t n_q_heads, int32_t m, int32_t t)
{
    if (check_format(fmt) != CQ_OK || !good_attention(fmt, batch, n_q_heads, m, t, 0)) return 0;
    return q8_plan(batch, fmt->n_kv_heads, n_q_heads, m, t, 0).tiles_per_split * kTileTokens;
}

size_t cq_attention_q8_workspace_bytes(const cq_q8_format* fmt, int32_t batch, int32_t n_q_heads, int32_t m, int32_t t,
                                       int32_t tokens_per_split)
{
    if (check_format(fmt) != CQ_OK || !good_attention(fmt, batch, n_q_heads, m, t, tokens_per_split)) return 0;
    return attention_workspace(batch, n_q_heads, m, q8_plan(batch, fmt->n_kv_heads, n_q_heads, m, t, tokens_per_split));
}

cq_status cq_decode_attention_q8(const void* q, const cq_q8_cache* cache, float scale, const cq_q8_format* fmt,
                                 int32_t batch, int32_t n_q_heads, int32_t t, int32_t t_cap, const int32_t* seq_lens, int32_t tokens_per_split,
                                 void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return attention_common(q, cache, scale, fmt, batch, n_q_heads, 1, t, t_cap, nullptr, false, seq_lens, tokens_per_split, out, workspace,
                            workspace_bytes, stream);
}

cq_status cq_decode_attention_q8_paged(const void* q, const cq_q8_cache* cache, float scale, const cq_q8_format* fmt,
                                       int32_t batch, int32_t n_q_heads, int32_t t, const cq_page_table* pages, const int32_t* seq_lens,
                                       int32_t tokens_per_split, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return attention_common(q, cache, scale, fmt, batch, n_q_heads, 1, t, 0, pages, true, seq_lens, tokens_per_split, out, workspace,
                            workspace_bytes, stream);
}

cq_status cq_chunk_attention_q8(const void* q, const cq_q8_cache* cache, float scale, const cq_q8_format* fmt,
                                int32_t batch, int32_t n_q_heads, int32_t m, int32_t t, int32_t t_cap, const int32_t* seq_lens,
                                int32_t tokens_per_split, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return attention_common(q, cache, scale, fmt, batch, n_q_heads, m, t, t_cap, nullptr, false, seq_lens, tokens_per_split, out, workspace,
                            workspace_bytes, stream);
}

cq_status cq_chunk_attention_q8_paged(const void* q, const cq_q8_cache* cache, float scale, const cq_q8_format* fmt,
                                      int32_t batch, int32_t n_q_heads, int32_t m, int32_t t, const cq_page_table* pages, const int32_t* seq_lens,
                                      int32_t tokens_per_split, void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    return attention_common(q, cache, scale, fmt, batch, n_q_heads, m, t, 0, pages, true, seq_lens, tokens_per_split, out, workspace,
                            workspace_bytes, stream);
}

}  // extern "C"
