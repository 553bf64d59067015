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
};
cudaError_t launch_kv_append(const AppendArgs &a, cudaStream_t stream);

struct AttendArgs {
    KvCache cache;
    KvBatch batch;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    int64_t q_stride, out_stride;
    int32_t T, heads;
    float scale; // of the scores, times log2(e): the kernels work with powers of two
    void *workspace;
};

// Workspace of the decode kernel: a counter per CTA, then the partial results.  The grid has at most kDecodeMaxCtas CTAs.
constexpr int kDecodeMaxCtas = 512;
__host__ __device__ constexpr size_t decode_counter_bytes() { return kDecodeMaxCtas * sizeof(uint32_t); }
size_t attend_decode_workspace_bytes(int heads, int kv_heads, int head_dim);
bool attend_decode_fits(const AttendArgs &a); // the kernel counts its work in 31 bits
cudaError_t launch_attend_decode(const AttendArgs &a, cudaStream_t stream);

// Workspace of the prompt kernel: two words per part (those of a tile's first part count its parts), then the partial results.  At
// most kPromptMaxParts CTAs share tiles of rows.
constexpr int kPromptMaxParts = 160;
__host__ __device__ constexpr size_t prompt_counter_bytes() { return 256 * 2 * sizeof(uint32_t); }
static_assert(kPromptMaxParts * 2 * sizeof(uint32_t) <= prompt_counter_bytes(), "a counter for every part");
size_t attend_prompt_workspace_bytes(int heads, int kv_heads, int head_dim);
cudaError_t launch_attend_prompt(const AttendArgs &a, cudaStream_t stream);

} // namespace bitlinear
