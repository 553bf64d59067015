// What the kernels around the paged key-value cache share: the views of the cache and of a call's sequences, and the
// look-ups into them.  Nothing that comes from device memory (lengths, page numbers) is used as an index unchecked.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "internal.cuh"

namespace bitlinear {

constexpr int kMaxHeadDim = 128;
constexpr int kMaxKvHeads = 1024;
constexpr int kMaxHeads = 4096;

// Elements of a cache row: the head padded to 16 elements (a whole 32-byte sector in bf16, a 16-byte piece in int8).
__host__ __device__ inline int kv_row_width(int head_dim) { return (head_dim + 15) / 16 * 16; }

struct KvCache {
    void *k, *v;            // bf16 or int8 [n_pages][kv_heads][page_size][width]
    float *k_scale, *v_scale; // null for bf16
    int32_t *status;
    int32_t n_pages, kv_heads, head_dim, width, page_shift;
};

// What is kept about every row of a cache beside its key and value: [n_pages][kv_heads][page_size].
struct KvMarks {
    float *mass;  // the attention weight it has received
    int32_t *pos; // the position of its token
};

struct KvBatch {
    const int32_t *page_table, *kv_lens, *cu_tokens;
    int32_t n_seqs;
    int32_t capacity; // positions a row of the page table covers
    int64_t table_stride;
};

// Reports a bad page, length, position or token row.  An expired wait, which says more, stays where it is: its code is the larger
// one of the two as unsigned numbers, and both are larger than BITLINEAR_OK.
static_assert((uint32_t)BITLINEAR_ERR_TIMEOUT > (uint32_t)BITLINEAR_ERR_PAGE, "a timeout is not replaced");
__device__ __forceinline__ void kv_report(const KvCache &c) { atomicMax(reinterpret_cast<uint32_t *>(c.status), (uint32_t)BITLINEAR_ERR_PAGE); }

// The length of sequence b, cut to what its row of the page table covers; over_long: it was cut.
__host__ __device__ __forceinline__ int kv_length(const KvBatch &s, int b, bool &over_long)
{
    const int n = s.kv_lens[b];
    over_long = n > s.capacity;
    return n < 0 ? 0 : (over_long ? s.capacity : n);
}

// Page of a position inside the capacity; -1 if the table holds a number the cache does not have.
__host__ __device__ __forceinline__ int kv_page(const KvCache &c, const KvBatch &s, int b, int pos)
{
    const int page = s.page_table[(int64_t)b * s.table_stride + (pos >> c.page_shift)];
    return (uint32_t)page < (uint32_t)c.n_pages ? page : -1;
}

// Row of the cache, counted over all pages, heads and slots (less than 2^31 of them).
__host__ __device__ __forceinline__ int kv_row(const KvCache &c, int page, int head, int pos)
{
    return ((page * c.kv_heads + head) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

// Sequence of token row t, or -1 if it has none; `first` and `count`: its token rows.
__host__ __device__ __forceinline__ int kv_sequence_of(const KvBatch &s, int t, int &first, int &count)
{
    if (!s.cu_tokens) {
        first = t;
        count = 1;
        return t < s.n_seqs ? t : -1;
    }
    int lo = 0, hi = s.n_seqs; // the first b whose rows end behind t
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (s.cu_tokens[mid + 1] > t)
            hi = mid;
        else
            lo = mid + 1;
    }
    if (lo >= s.n_seqs) return -1;
    first = s.cu_tokens[lo];
    count = s.cu_tokens[lo + 1] - first;
    return first <= t ? lo : -1;
}

// Launches a kernel that may start while the launch before it on the stream is still running (its CTAs wait at griddep_wait,
// which returns when that launch is complete and its writes are visible).  Between small launches this hides the start.
template <typename... Args>
cudaError_t launch_dependent(void (*kernel)(Args...), unsigned blocks, unsigned threads, size_t smem, cudaStream_t stream,
                             const std::remove_const_t<Args> &...args)
{
    cudaLaunchAttribute attribute;
    attribute.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attribute.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(blocks);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = &attribute;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

// ---- launchers -----------------------------------------------------------------------------------------

cudaError_t launch_rope_table(float *table, int64_t n_pos, int head_dim, double base, cudaStream_t stream);

struct AppendArgs {
    KvCache cache;
    KvBatch batch;
    const __nv_bfloat16 *k, *v, *q;
    __nv_bfloat16 *q_out;
    int64_t k_stride, v_stride, q_stride, q_out_stride;
    const float2 *rope;
    int32_t rope_positions, T, heads, interleaved;
    // of the form that normalises (and takes positions and marks) alone
    const float *q_gain, *k_gain; // fp32 [head_dim], or null: not normalised
    const int32_t *positions;     // of the token rows, or null: the rows' places in their sequences
    KvMarks marks;                // null pointers: none
    float norm_eps;
};
cudaError_t launch_kv_append(const AppendArgs &a, cudaStream_t stream);
cudaError_t launch_kv_append_rmsnorm(const AppendArgs &a, cudaStream_t stream);

struct AttendArgs {
    KvCache cache;
    KvBatch batch;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    int64_t q_stride, out_stride;
    int32_t T, heads;
    float scale; // of the scores, times log2(e): the kernels work with powers of two
    void *workspace; // begins with the counters, of every kind of call and for any heads: they alone have to be zero between calls
    float *parts;    // in it: the decode kernel's partial results
};

// What the decode kernel that passes its weights on (to the marks) has besides.
struct WeighArgs {
    float *scores;     // of every unit of work with room for it: [kBlock keys][query heads of the chunk], scaled
    int64_t max_units; // units that there is room for
    float2 *sums;      // [n_seqs][heads]: reference and denominator of every softmax
    KvMarks marks;
};

// Groups of sequences that begin with the same rows, as a batch: pages, rows shared, and the bounds of each group's sequences.  With
// bounds that fall or lie outside the batch nothing is shared.  (Of one group: whether they do.)
__device__ __forceinline__ bool group_bounds_bad(const KvBatch &groups, int g, int n_seqs)
{
    return groups.cu_tokens[g] < 0 || groups.cu_tokens[g] > groups.cu_tokens[g + 1] || groups.cu_tokens[g + 1] > n_seqs;
}
// How many rows group g shares, a whole number of pages; none for a group of a single sequence (nothing is saved).
__device__ __forceinline__ int group_shares(const KvCache &c, const KvBatch &groups, int g, bool &over)
{
    const int n = max(0, groups.kv_lens[g]) >> c.page_shift << c.page_shift;
    over = n > groups.capacity;
    return groups.cu_tokens[g + 1] - groups.cu_tokens[g] < 2 ? 0 : min(n, groups.capacity);
}
// The rows of sequence b that are its group's; none for a sequence that is shorter than them.
__device__ __forceinline__ int shared_start(const KvCache &c, const KvBatch &groups, const KvBatch &s, int b)
{
    int first, count;
    bool over;
    const int g = kv_sequence_of(groups, b, first, count);
    const int n = g < 0 ? 0 : group_shares(c, groups, g, over);
    return kv_length(s, b, over) >= n ? n : 0;
}

// What the kernels that attend to shared beginnings hand to each other.
struct SharedArgs {
    int32_t *starts; // [n_seqs]: rows of the sequence that the shared part has dealt with
    int2 *where;     // [n_seqs][heads]: where its results stand: (first part, parts * 2^16 + row of the tile), or (-1, 0): in ml and o
    float2 *ml;      // [n_seqs][heads]: reference and sum of the shared part of every softmax
    float *o;        // [n_seqs][heads][width]: its weighted sum of the values
    float *parts;    // the partial results of tiles whose keys several CTAs share (see prompt_part_floats)
    KvBatch seqs;
    int64_t share_from; // rows that the groups' sequences read in all where nothing is shared: from here on it is
};
// Sharing costs a launch and 9 us of beginnings and ends; reading a shared row again for every sequence, mostly from the L2, goes at 7
// TB/s of keys and values.  Both meet near 40 M elements of keys (32/32 heads of 128, 4 sequences sharing 1000 rows: 22 us shared, 16
// apart; 2500 rows, 41 M: 29.6 and 29.2; 4000 rows: 32 and 42; 64/8 heads, 8 sequences sharing 2000: 21 and 17; 5000, 41 M: 28.7 and 28.8;
// 28/4 heads, 16 sharing 4000: 22 and 24; 24/8 heads of 64, 32 in two groups sharing 8000: 29 and 73).
constexpr int64_t kShareFrom = (int64_t)40 << 20;
// Codes are half as long to read apart, and have to become bf16 in the tiles: they meet near 64 M elements (64/8 heads, 8 sequences sharing
// 5000 rows, 41 M: 29.9 us shared, 24.4 apart; 8000, 65 M: 33.1 and 32.9; 10000: 35.8 and 38.5; 28/4 heads, 16 sharing 4000: 27 and 22; 8000,
// 65 M: 31.7 and 32.7; 24/8 heads of 64, 16 sharing 5000, 41 M: 26.3 and 24.9; 32 in two groups sharing 8000: 36 and 56).  Where few
// sequences share rows under many kv heads, later (32/32 heads, 4 sequences sharing 5000, 82 M: 45 and 39; 8000: 59 and 55).
constexpr int64_t kShareFromCodes = (int64_t)64 << 20;

// Workspace of the decode kernel: a counter per CTA, then the partial results (of the shared form elsewhere).  The grid has at most
// kDecodeMaxCtas CTAs.
constexpr int kDecodeMaxCtas = 512;
__host__ __device__ constexpr size_t decode_counter_bytes() { return kDecodeMaxCtas * sizeof(uint32_t); }
size_t attend_decode_workspace_bytes(int heads, int kv_heads, int head_dim);
bool attend_decode_fits(const AttendArgs &a); // the kernel counts its work in 31 bits
cudaError_t launch_attend_decode(const AttendArgs &a, cudaStream_t stream);
// The same, adding the weights to the marks: room for scores of max_keys keys in all, more in a workspace of more bytes.
size_t attend_weigh_workspace_bytes(int heads, int kv_heads, int head_dim, bool int8, int64_t n_seqs, int64_t max_keys);
cudaError_t launch_attend_decode_weigh(const AttendArgs &a, const KvMarks &marks, size_t workspace_bytes, cudaStream_t stream);
// The same for sequences whose first rows the call before it has dealt with.
cudaError_t launch_attend_decode_behind(const AttendArgs &a, const SharedArgs &shared, cudaStream_t stream);

// Workspace of the prompt kernel: two words per part (those of a tile's first part count its parts), then the partial results.  At
// most kPromptMaxParts CTAs share tiles of rows.
constexpr int kPromptMaxParts = 160;
__host__ __device__ constexpr size_t prompt_counter_bytes() { return 256 * 2 * sizeof(uint32_t); }
static_assert(kPromptMaxParts * 2 * sizeof(uint32_t) <= prompt_counter_bytes(), "a counter for every part");
static_assert(decode_counter_bytes() == prompt_counter_bytes(), "calls of both kinds may take turns in one workspace");
constexpr int kPromptRows = 256; // of a tile
// A part: (reference, sum) of its rows, then their outputs as [four elements][row], so that a row per thread writes and reads whole
// lines.
__host__ __device__ constexpr size_t prompt_part_floats(int width) { return (size_t)kPromptRows * (width + 2); }
size_t attend_prompt_workspace_bytes(int heads, int kv_heads, int head_dim);
cudaError_t launch_attend_prompt(const AttendArgs &a, cudaStream_t stream);
// The part of a decode step that groups of sequences share: a.batch holds the groups (their pages, how many rows they share, which
// sequences they are), a.T sequences in all.
cudaError_t launch_attend_prefix(const AttendArgs &a, const SharedArgs &shared, cudaStream_t stream);

struct SelectArgs {
    KvCache cache;
    KvBatch batch;
    KvMarks marks;
    int32_t *source, *new_lens;
    int32_t keep, recent;
    bool any_order; // the newest position is the largest of the rows', not the last row's
};
constexpr int64_t kSelectMaxRows = (int64_t)1 << 18; // of a sequence
cudaError_t launch_kv_select(const SelectArgs &a, cudaStream_t stream);

struct CompactArgs {
    KvCache cache;
    KvBatch batch;
    KvMarks marks; // null pointers: none
    const int32_t *source;
    int32_t keep;
};
cudaError_t launch_kv_compact(const CompactArgs &a, cudaStream_t stream);

} // namespace bitlinear
