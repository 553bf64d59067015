// C ABI of the operators around the paged key-value cache: argument validation and the views the kernels take.
// No arithmetic of the method lives here.
#include <cmath>

#include "internal.cuh"
#include "kv.cuh"

namespace bitlinear {
namespace {

bitlinear_status check_cache_shape(int64_t n_pages, int kv_heads, int head_dim, int page_size, int bits)
{
    if (bits != 16 && bits != 8) return BITLINEAR_ERR_ARG;
    if (kv_heads < 1 || kv_heads > kMaxKvHeads) return BITLINEAR_ERR_SHAPE;
    if (head_dim < 4 || head_dim > kMaxHeadDim || head_dim % 4 != 0) return BITLINEAR_ERR_SHAPE;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return BITLINEAR_ERR_SHAPE;
    if (n_pages < 1 || n_pages >= ((int64_t)1 << 31) / (kv_heads * page_size)) return BITLINEAR_ERR_SHAPE;
    return BITLINEAR_OK;
}

int log2_of(int x)
{
    int n = 0;
    while ((1 << n) < x) ++n;
    return n;
}

// Validates the cache and the sequences and fills the kernels' views.
bitlinear_status take_views(const bitlinear_kv_cache *c, const bitlinear_kv_batch *s, KvCache &kc, KvBatch &ks)
{
    if (!c || !s || !c->k || !c->v || !c->status) return BITLINEAR_ERR_ARG;
    const bitlinear_status st = check_cache_shape(c->n_pages, c->kv_heads, c->head_dim, c->page_size, c->bits);
    if (st != BITLINEAR_OK) return st;
    if ((c->bits == 8) != (c->k_scale != nullptr) || (c->bits == 8) != (c->v_scale != nullptr)) return BITLINEAR_ERR_ARG;
    if (s->n_seqs < 0 || s->n_seqs > (1 << 20)) return BITLINEAR_ERR_SHAPE;
    if (s->table_pages < 1 || s->table_pages > s->table_stride || s->table_pages > ((int64_t)1 << 30) / c->page_size) return BITLINEAR_ERR_SHAPE;
    if (s->table_stride > ((int64_t)1 << 40)) return BITLINEAR_ERR_SHAPE;
    if (s->n_seqs > 0 && (!s->page_table || !s->kv_lens)) return BITLINEAR_ERR_ARG;
    if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, 16) || !aligned(c->v_scale, 16) || !aligned(c->status, 4))
        return BITLINEAR_ERR_ALIGN;
    if (!aligned(s->page_table, 4) || !aligned(s->kv_lens, 4) || !aligned(s->cu_tokens, 4)) return BITLINEAR_ERR_ALIGN;
    kc.k = c->k;
    kc.v = c->v;
    kc.k_scale = c->k_scale;
    kc.v_scale = c->v_scale;
    kc.status = c->status;
    kc.n_pages = (int32_t)c->n_pages;
    kc.kv_heads = c->kv_heads;
    kc.head_dim = c->head_dim;
    kc.width = kv_row_width(c->head_dim);
    kc.page_shift = log2_of(c->page_size);
    ks.page_table = s->page_table;
    ks.kv_lens = s->kv_lens;
    ks.cu_tokens = s->cu_tokens;
    ks.n_seqs = (int32_t)s->n_seqs;
    ks.capacity = (int32_t)(s->table_pages << kc.page_shift);
    ks.table_stride = s->table_stride;
    return BITLINEAR_OK;
}

// Rows of `heads` heads: the stride covers them and keeps every row 16-byte aligned.
bitlinear_status check_rows(const void *p, int64_t stride, int heads, int head_dim)
{
    if (stride < (int64_t)heads * head_dim || stride % 8 != 0 || stride > ((int64_t)1 << 40)) return BITLINEAR_ERR_SHAPE;
    return aligned(p, 16) ? BITLINEAR_OK : BITLINEAR_ERR_ALIGN;
}

} // namespace
} // namespace bitlinear

using namespace bitlinear;

extern "C" {

size_t bitlinear_kv_cache_bytes(int64_t n_pages, int kv_heads, int head_dim, int page_size, int bits)
{
    if (check_cache_shape(n_pages, kv_heads, head_dim, page_size, bits) != BITLINEAR_OK) return 0;
    return (size_t)n_pages * kv_heads * page_size * kv_row_width(head_dim) * (bits / 8);
}

bitlinear_status bitlinear_rope_table(float *table, int64_t n_pos, int head_dim, double base, void *stream)
{
    if (!table || !(base > 0.0) || !std::isfinite(base)) return BITLINEAR_ERR_ARG;
    if (n_pos < 1 || n_pos > (1 << 24) || head_dim < 4 || head_dim > kMaxHeadDim || head_dim % 4 != 0) return BITLINEAR_ERR_SHAPE;
    if (!aligned(table, 16)) return BITLINEAR_ERR_ALIGN;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    return launch_rope_table(table, n_pos, head_dim, base, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

namespace {

// Checks what the two forms of appending have in common; `idle`: there is nothing to do.
bitlinear_status take_append(AppendArgs &a, bool &idle, const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *k,
                             int64_t k_stride, const void *v, int64_t v_stride, const void *q, int64_t q_stride, int64_t T, int heads,
                             const float *rope, int64_t rope_positions, int interleaved, void *q_out, int64_t q_out_stride)
{
    bitlinear_status st = take_views(cache, batch, a.cache, a.batch);
    if (st != BITLINEAR_OK) return st;
    if (T < 0 || T > (1 << 20) || (!batch->cu_tokens && T != batch->n_seqs)) return BITLINEAR_ERR_SHAPE;
    if (interleaved != 0 && interleaved != 1) return BITLINEAR_ERR_ARG;
    if (T > 0 && (!k || !v || (q && !q_out))) return BITLINEAR_ERR_ARG;
    if ((st = check_rows(k, k_stride, a.cache.kv_heads, a.cache.head_dim)) != BITLINEAR_OK) return st;
    if ((st = check_rows(v, v_stride, a.cache.kv_heads, a.cache.head_dim)) != BITLINEAR_OK) return st;
    if (q) {
        if (heads < 1 || heads > kMaxHeads) return BITLINEAR_ERR_SHAPE;
        if ((st = check_rows(q, q_stride, heads, a.cache.head_dim)) != BITLINEAR_OK) return st;
        if ((st = check_rows(q_out, q_out_stride, heads, a.cache.head_dim)) != BITLINEAR_OK) return st;
        if (q == q_out && q_stride != q_out_stride) return BITLINEAR_ERR_ARG;
    }
    if (rope) {
        if (rope_positions < 1 || rope_positions > (1 << 30)) return BITLINEAR_ERR_SHAPE;
        if (!aligned(rope, 16)) return BITLINEAR_ERR_ALIGN;
    }
    idle = T == 0 || batch->n_seqs == 0;
    a.k = reinterpret_cast<const __nv_bfloat16 *>(k);
    a.v = reinterpret_cast<const __nv_bfloat16 *>(v);
    a.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    a.q_out = reinterpret_cast<__nv_bfloat16 *>(q_out);
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.q_stride = q_stride;
    a.q_out_stride = q_out_stride;
    a.rope = reinterpret_cast<const float2 *>(rope);
    a.rope_positions = (int32_t)rope_positions;
    a.T = (int32_t)T;
    a.heads = q ? heads : 0;
    a.interleaved = interleaved;
    return BITLINEAR_OK;
}

bitlinear_status take_marks(const bitlinear_kv_marks *marks, KvMarks &m)
{
    if (!marks || !marks->mass || !marks->pos) return BITLINEAR_ERR_ARG;
    if (!aligned(marks->mass, 16) || !aligned(marks->pos, 16)) return BITLINEAR_ERR_ALIGN;
    m.mass = marks->mass;
    m.pos = marks->pos;
    return BITLINEAR_OK;
}

} // namespace

bitlinear_status bitlinear_kv_append(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *k,
                                     int64_t k_stride, const void *v, int64_t v_stride, const void *q, int64_t q_stride,
                                     int64_t T, int heads, const float *rope, int64_t rope_positions, int interleaved,
                                     void *q_out, int64_t q_out_stride, void *stream)
{
    AppendArgs a{};
    bool idle;
    const bitlinear_status st = take_append(a, idle, cache, batch, k, k_stride, v, v_stride, q, q_stride, T, heads, rope, rope_positions,
                                            interleaved, q_out, q_out_stride);
    if (st != BITLINEAR_OK) return st;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (idle) return BITLINEAR_OK;
    return launch_kv_append(a, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

bitlinear_status bitlinear_kv_append_rmsnorm(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *k,
                                             int64_t k_stride, const void *v, int64_t v_stride, const void *q, int64_t q_stride,
                                             int64_t T, int heads, const float *q_gain, const float *k_gain, float norm_eps,
                                             const float *rope, int64_t rope_positions, int interleaved, const int32_t *positions,
                                             const bitlinear_kv_marks *marks, void *q_out, int64_t q_out_stride, void *stream)
{
    AppendArgs a{};
    bool idle;
    bitlinear_status st = take_append(a, idle, cache, batch, k, k_stride, v, v_stride, q, q_stride, T, heads, rope, rope_positions,
                                      interleaved, q_out, q_out_stride);
    if (st != BITLINEAR_OK) return st;
    if (!(norm_eps >= 0.0f) || !std::isfinite(norm_eps)) return BITLINEAR_ERR_ARG;
    if (!aligned(q_gain, 16) || !aligned(k_gain, 16) || !aligned(positions, 4)) return BITLINEAR_ERR_ALIGN;
    if (marks && (st = take_marks(marks, a.marks)) != BITLINEAR_OK) return st;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (idle) return BITLINEAR_OK;
    a.q_gain = q ? q_gain : nullptr;
    a.k_gain = k_gain;
    a.norm_eps = norm_eps;
    a.positions = positions;
    return launch_kv_append_rmsnorm(a, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

namespace {

bool heads_ok(int heads, int kv_heads, int head_dim)
{
    return kv_heads >= 1 && kv_heads <= kMaxKvHeads && heads >= 1 && heads <= kMaxHeads && heads % kv_heads == 0 && head_dim >= 4 &&
           head_dim <= kMaxHeadDim && head_dim % 4 == 0;
}

size_t workspace_for(int heads, int kv_heads, int head_dim, bool prompt)
{
    return prompt ? attend_prompt_workspace_bytes(heads, kv_heads, head_dim) : attend_decode_workspace_bytes(heads, kv_heads, head_dim);
}

// Checks what the attentions have in common and fills their view.
bitlinear_status take_attend(AttendArgs &a, const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *q, int64_t q_stride,
                             int64_t T, int heads, float softmax_scale, void *out, int64_t out_stride, void *workspace, bool prompt)
{
    bitlinear_status st = take_views(cache, batch, a.cache, a.batch);
    if (st != BITLINEAR_OK) return st;
    if (T < 0 || T > (1 << 20) || !heads_ok(heads, a.cache.kv_heads, a.cache.head_dim)) return BITLINEAR_ERR_SHAPE;
    if (prompt && T * (heads / a.cache.kv_heads) > (1 << 30)) return BITLINEAR_ERR_SHAPE;
    if (prompt != (batch->cu_tokens != nullptr)) return BITLINEAR_ERR_ARG;
    if (!(softmax_scale > 0.0f) || !std::isfinite(softmax_scale) || !workspace || (T > 0 && (!q || !out || q == out))) return BITLINEAR_ERR_ARG;
    if ((st = check_rows(q, q_stride, heads, a.cache.head_dim)) != BITLINEAR_OK) return st;
    if ((st = check_rows(out, out_stride, heads, a.cache.head_dim)) != BITLINEAR_OK) return st;
    if (!aligned(workspace, 256)) return BITLINEAR_ERR_ALIGN;
    a.heads = heads;
    if (!prompt && !attend_decode_fits(a)) return BITLINEAR_ERR_SHAPE;
    a.scale = (float)((double)softmax_scale * 1.4426950408889634074); // log2 e
    if (!std::isfinite(a.scale)) return BITLINEAR_ERR_ARG;
    a.q = reinterpret_cast<const __nv_bfloat16 *>(q);
    a.out = reinterpret_cast<__nv_bfloat16 *>(out);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.T = (int32_t)T;
    a.workspace = workspace;
    a.parts = reinterpret_cast<float *>(reinterpret_cast<char *>(workspace) + decode_counter_bytes());
    return BITLINEAR_OK;
}

bitlinear_status attend(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *q, int64_t q_stride, int64_t T,
                        int heads, float softmax_scale, void *out, int64_t out_stride, void *workspace, size_t workspace_bytes,
                        void *stream, bool prompt)
{
    AttendArgs a{};
    const bitlinear_status st = take_attend(a, cache, batch, q, q_stride, T, heads, softmax_scale, out, out_stride, workspace, prompt);
    if (st != BITLINEAR_OK) return st;
    if (workspace_bytes < workspace_for(heads, a.cache.kv_heads, a.cache.head_dim, prompt)) return BITLINEAR_ERR_WORKSPACE;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (T == 0 || batch->n_seqs == 0) return BITLINEAR_OK;
    return (prompt ? launch_attend_prompt(a, (cudaStream_t)stream) : launch_attend_decode(a, (cudaStream_t)stream)) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

} // namespace

size_t bitlinear_attend_workspace_bytes(int heads, int kv_heads, int head_dim, int prompt)
{
    if (!heads_ok(heads, kv_heads, head_dim) || (prompt != 0 && prompt != 1)) return 0;
    return workspace_for(heads, kv_heads, head_dim, prompt != 0);
}

bitlinear_status bitlinear_attend_decode(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *q,
                                         int64_t q_stride, int heads, float softmax_scale, void *out, int64_t out_stride,
                                         void *workspace, size_t workspace_bytes, void *stream)
{
    return attend(cache, batch, q, q_stride, batch ? batch->n_seqs : 0, heads, softmax_scale, out, out_stride, workspace,
                  workspace_bytes, stream, false);
}

bitlinear_status bitlinear_attend_prompt(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const void *q,
                                         int64_t q_stride, int64_t T, int heads, float softmax_scale, void *out,
                                         int64_t out_stride, void *workspace, size_t workspace_bytes, void *stream)
{
    return attend(cache, batch, q, q_stride, T, heads, softmax_scale, out, out_stride, workspace, workspace_bytes, stream, true);
}

size_t bitlinear_attend_weigh_workspace_bytes(int heads, int kv_heads, int head_dim, int bits, int64_t n_seqs, int64_t max_keys)
{
    if (!heads_ok(heads, kv_heads, head_dim) || (bits != 16 && bits != 8) || n_seqs < 0 || n_seqs > (1 << 20) || max_keys < 0 ||
        max_keys > ((int64_t)1 << 40))
        return 0;
    return attend_weigh_workspace_bytes(heads, kv_heads, head_dim, bits == 8, n_seqs, max_keys);
}

bitlinear_status bitlinear_attend_decode_weigh(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch,
                                               const bitlinear_kv_marks *marks, const void *q, int64_t q_stride, int heads,
                                               float softmax_scale, void *out, int64_t out_stride, void *workspace,
                                               size_t workspace_bytes, void *stream)
{
    AttendArgs a{};
    KvMarks m{};
    const int64_t T = batch ? batch->n_seqs : 0;
    bitlinear_status st = take_attend(a, cache, batch, q, q_stride, T, heads, softmax_scale, out, out_stride, workspace, false);
    if (st != BITLINEAR_OK) return st;
    if ((st = take_marks(marks, m)) != BITLINEAR_OK) return st;
    if (workspace_bytes < attend_weigh_workspace_bytes(heads, a.cache.kv_heads, a.cache.head_dim, a.cache.k_scale != nullptr, T, 0))
        return BITLINEAR_ERR_WORKSPACE;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (T == 0) return BITLINEAR_OK;
    return launch_attend_decode_weigh(a, m, workspace_bytes, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

namespace {

// Workspace of the attention over shared beginnings: the prompt kernel's, whose counters are the decode kernel's (the shared form needs
// none), the decode kernel's partial results, then what the one hands to the other.
struct SharedLayout {
    size_t decode_parts, starts, where, ml, o, bytes;
    SharedLayout(int heads, int kv_heads, int head_dim, int64_t n_seqs)
    {
        decode_parts = attend_prompt_workspace_bytes(heads, kv_heads, head_dim);
        starts = decode_parts + attend_decode_workspace_bytes(heads, kv_heads, head_dim) - decode_counter_bytes();
        where = starts + align_up((size_t)n_seqs * sizeof(int32_t), 256);
        ml = where + align_up((size_t)n_seqs * heads * sizeof(int2), 256);
        o = ml + align_up((size_t)n_seqs * heads * sizeof(float2), 256);
        bytes = o + align_up((size_t)n_seqs * heads * kv_row_width(head_dim) * sizeof(float), 256);
    }
};

} // namespace

size_t bitlinear_attend_shared_workspace_bytes(int heads, int kv_heads, int head_dim, int64_t n_seqs)
{
    if (!heads_ok(heads, kv_heads, head_dim) || n_seqs < 0 || n_seqs > (1 << 20)) return 0;
    return SharedLayout(heads, kv_heads, head_dim, n_seqs).bytes;
}

bitlinear_status bitlinear_attend_decode_shared(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch,
                                                const bitlinear_kv_batch *groups, const void *q, int64_t q_stride, int heads,
                                                float softmax_scale, int64_t share_from, void *out, int64_t out_stride, void *workspace,
                                                size_t workspace_bytes, void *stream)
{
    AttendArgs a{}, p{};
    const int64_t T = batch ? batch->n_seqs : 0;
    bitlinear_status st = take_attend(a, cache, batch, q, q_stride, T, heads, softmax_scale, out, out_stride, workspace, false);
    if (st != BITLINEAR_OK) return st;
    p = a;
    if ((st = take_views(cache, groups, p.cache, p.batch)) != BITLINEAR_OK) return st;
    if (!groups->cu_tokens) return BITLINEAR_ERR_ARG;
    if (T * (heads / a.cache.kv_heads) > (1 << 30)) return BITLINEAR_ERR_SHAPE;
    const SharedLayout at(heads, a.cache.kv_heads, a.cache.head_dim, T);
    if (workspace_bytes < at.bytes) return BITLINEAR_ERR_WORKSPACE;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (T == 0) return BITLINEAR_OK;
    char *ws = reinterpret_cast<char *>(workspace);
    a.parts = reinterpret_cast<float *>(ws + at.decode_parts);
    SharedArgs shared;
    shared.starts = reinterpret_cast<int32_t *>(ws + at.starts);
    shared.where = reinterpret_cast<int2 *>(ws + at.where);
    shared.ml = reinterpret_cast<float2 *>(ws + at.ml);
    shared.parts = reinterpret_cast<float *>(ws + prompt_counter_bytes());
    shared.o = reinterpret_cast<float *>(ws + at.o);
    shared.seqs = a.batch;
    const int64_t row = (int64_t)a.cache.kv_heads * a.cache.head_dim, own_bound = a.cache.k_scale ? kShareFromCodes : kShareFrom,
                  least = share_from < 0 ? own_bound : share_from;
    shared.share_from = least / row + (least % row != 0);
    // (or where no lengths that the groups' page table has room for make it worth while)
    if (groups->n_seqs == 0 || T * p.batch.capacity < shared.share_from)
        return launch_attend_decode(a, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
    if (launch_attend_prefix(p, shared, (cudaStream_t)stream) != cudaSuccess) return BITLINEAR_ERR_CUDA;
    return launch_attend_decode_behind(a, shared, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

namespace {

bitlinear_status select_rows(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const bitlinear_kv_marks *marks, int64_t keep,
                             int64_t recent, bool any_order, int32_t *source, int32_t *new_lens, void *stream)
{
    SelectArgs a{};
    bitlinear_status st = take_views(cache, batch, a.cache, a.batch);
    if (st != BITLINEAR_OK) return st;
    if ((st = take_marks(marks, a.marks)) != BITLINEAR_OK) return st;
    if (keep < 1 || keep > ((int64_t)1 << 30) || recent < 0 || recent > keep) return BITLINEAR_ERR_SHAPE;
    if (a.batch.capacity > kSelectMaxRows || batch->n_seqs * a.cache.kv_heads > (1 << 27)) return BITLINEAR_ERR_SHAPE;
    if (batch->n_seqs > 0 && (!source || !new_lens)) return BITLINEAR_ERR_ARG;
    // (the lengths are read by every head's CTAs while one of them writes the new ones)
    const uintptr_t from = reinterpret_cast<uintptr_t>(batch->kv_lens), to = reinterpret_cast<uintptr_t>(new_lens), bytes = (uintptr_t)batch->n_seqs * 4;
    if (batch->n_seqs > 0 && from < to + bytes && to < from + bytes) return BITLINEAR_ERR_ARG;
    if (!aligned(source, 4) || !aligned(new_lens, 4)) return BITLINEAR_ERR_ALIGN;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (batch->n_seqs == 0) return BITLINEAR_OK;
    a.source = source;
    a.new_lens = new_lens;
    a.keep = (int32_t)keep;
    a.recent = (int32_t)recent;
    a.any_order = any_order;
    return launch_kv_select(a, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

} // namespace

bitlinear_status bitlinear_kv_select(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const bitlinear_kv_marks *marks,
                                     int64_t keep, int64_t recent, int32_t *source, int32_t *new_lens, void *stream)
{
    return select_rows(cache, batch, marks, keep, recent, false, source, new_lens, stream);
}

bitlinear_status bitlinear_kv_select_any_order(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const bitlinear_kv_marks *marks,
                                               int64_t keep, int64_t recent, int32_t *source, int32_t *new_lens, void *stream)
{
    return select_rows(cache, batch, marks, keep, recent, true, source, new_lens, stream);
}

bitlinear_status bitlinear_kv_compact(const bitlinear_kv_cache *cache, const bitlinear_kv_batch *batch, const int32_t *source,
                                      int64_t keep, const bitlinear_kv_marks *marks, void *stream)
{
    CompactArgs a{};
    bitlinear_status st = take_views(cache, batch, a.cache, a.batch);
    if (st != BITLINEAR_OK) return st;
    if (marks && (st = take_marks(marks, a.marks)) != BITLINEAR_OK) return st;
    if (keep < 1 || keep > ((int64_t)1 << 30)) return BITLINEAR_ERR_SHAPE;
    if (batch->n_seqs > 0 && !source) return BITLINEAR_ERR_ARG;
    if (!aligned(source, 4)) return BITLINEAR_ERR_ALIGN;
    if (!device_is_sm100()) return BITLINEAR_ERR_ARCH;
    if (batch->n_seqs == 0) return BITLINEAR_OK;
    a.source = source;
    a.keep = (int32_t)keep;
    return launch_kv_compact(a, (cudaStream_t)stream) == cudaSuccess ? BITLINEAR_OK : BITLINEAR_ERR_CUDA;
}

} // extern "C"
