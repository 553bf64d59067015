// Which rows of a sequence stay in the cache, by the attention weight they have received, and moving them to the front.
//
// Selection, for every (sequence, kv head) of n rows of which `keep` stay.  A row's worth is a 32-bit number: the bits of its
// weight (not negative, so they order as the weights do), or the largest number for the rows of the `recent` newest positions.
// The keep-th largest worth is found digit by digit (11, 11 and 10 bits: a histogram of the rows that agree with the digits found so
// far, summed from above); rows above it stay, and of the rows equal to it the first ones.  Which rows stay is kept as a bit per
// row, with the number of bits in front of every word, so that the j-th hole (a row below `keep` that goes) finds the j-th row to be
// moved (at or behind `keep`) by a search in those numbers.  Nothing depends on the order in which threads run.
//
// A cluster of CTAs shares a (sequence, kv head), each of them a contiguous stretch of the rows.
#include <cooperative_groups.h>

#include <algorithm>

#include "internal.cuh"
#include "kv.cuh"
#include "ptx.cuh"

namespace bitlinear {
namespace {

namespace cg = cooperative_groups;

constexpr int kSelectThreads = 512, kSelectWarps = kSelectThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kDigits = 3, kBins = 2048;
__device__ __forceinline__ int digit_shift(int d) { return d == 0 ? 21 : (d == 1 ? 10 : 0); }

struct SelectShared {
    uint32_t bins[kDigits][kBins];
    int scan[kSelectWarps];
    int digit, above;        // found: the digit, and how many rows are above it
    int ties, holes, movers; // of this CTA's stretch
};

// Sum over the CTA of x of the threads in front of this one; total: of all of them.
__device__ __forceinline__ int scan_block(int x, int *scan, int &total)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    int upto = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += y;
    }
    __syncthreads(); // (scan may still be read from the call before)
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kSelectWarps; ++w) {
        if (w < warp) before += scan[w];
        total += scan[w];
    }
    return before + upto - x;
}

// Replaces counts[0 .. n) by the sums in front of each; returns the sum of all.
__device__ __forceinline__ int scan_words(int *counts, int n, int *scan)
{
    int sum = 0;
    for (int w0 = 0; w0 < n; w0 += kSelectThreads) {
        const int w = w0 + (int)threadIdx.x;
        int total;
        const int before = scan_block(w < n ? counts[w] : 0, scan, total);
        if (w < n) counts[w] = sum + before;
        sum += total;
    }
    __syncthreads();
    return sum;
}

// Words of 32 rows in a CTA's stretch of a sequence of so many rows.
int stretch_words(int64_t rows, int cluster) { return (int)(((rows + 31) / 32 + cluster - 1) / cluster); }

__global__ void __launch_bounds__(kSelectThreads) kv_select_kernel(const __grid_constant__ SelectArgs a, const int max_words)
{
    ptx::griddep_wait(); // everything below is read from memory that the launch before this one may have written
    ptx::griddep_launch_dependents();
    cg::cluster_group cluster = cg::this_cluster();
    const int C = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    extern __shared__ __align__(16) uint8_t smem[];
    SelectShared &sh = *reinterpret_cast<SelectShared *>(smem);
    uint32_t *stays = reinterpret_cast<uint32_t *>(smem + sizeof(SelectShared)); // a bit per row of the stretch
    int *before = reinterpret_cast<int *>(stays + max_words);                     // per word: what is in front of it in the stretch
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const int Hk = a.cache.kv_heads, keep = a.keep;
    const int pair = (int)blockIdx.x / C, b = pair / Hk, h = pair - b * Hk;
    bool over;
    const int n = kv_length(a.batch, b, over);
    if (tid == 0 && rank == 0 && h == 0) {
        if (over) kv_report(a.cache);
        a.new_lens[b] = min(n, keep);
    }
    int32_t *source = a.source + (int64_t)pair * keep;
    if (n <= keep) { // (the whole cluster)
        for (int i = rank * kSelectThreads + tid; i < keep; i += C * kSelectThreads) source[i] = i < n ? i : -1;
        return;
    }
    auto row_of = [&](int i) {
        const int page = kv_page(a.cache, a.batch, b, i);
        return page < 0 ? -1 : kv_row(a.cache, page, h, i);
    };
    const int last = row_of(n - 1);
    const int64_t oldest = last < 0 ? INT64_MAX : (int64_t)a.marks.pos[last] - a.recent; // what is newer stays
    auto worth = [&](int i, bool report) -> uint32_t {
        const int row = row_of(i);
        if (row < 0) {
            if (report) kv_report(a.cache);
            return 0u;
        }
        if ((int64_t)a.marks.pos[row] > oldest) return 0xFFFFFFFFu;
        const float w = a.marks.mass[row];
        return w > 0.0f ? __float_as_uint(w) : 0u; // (nothing, or not a number: 0)
    };
    const int all_words = (n + 31) / 32, each = (all_words + C - 1) / C;
    const int word0 = min(all_words, rank * each), words = min(all_words, word0 + each) - word0; // of this stretch

    // ---- the keep-th largest worth, and how many rows are above it -----------------------------------------
    for (int i = tid; i < kDigits * kBins; i += kSelectThreads) (&sh.bins[0][0])[i] = 0u;
    __syncthreads();
    uint32_t least = 0u; // its digits found so far
    int above = 0;
    for (int d = 0; d < kDigits; ++d) {
        const int shift = digit_shift(d);
        for (int w = warp; w < words; w += kSelectWarps) {
            const int i = (word0 + w) * 32 + lane;
            if (i >= n) continue;
            const uint32_t x = worth(i, d == 0);
            if (d == 0 || ((x ^ least) >> digit_shift(d - 1)) == 0u) atomicAdd(&sh.bins[d][(x >> shift) & (d == 2 ? 1023u : 2047u)], 1u);
        }
        cluster.sync();
        int mine[kBins / kSelectThreads], sum = 0; // from the largest digit down
#pragma unroll
        for (int u = 0; u < kBins / kSelectThreads; ++u) {
            const int bin = kBins - 1 - (tid * (kBins / kSelectThreads) + u);
            int x = 0;
            for (int r = 0; r < C; ++r) x += (int)*cluster.map_shared_rank(&sh.bins[d][bin], r);
            mine[u] = x;
            sum += x;
        }
        int total;
        int upto = above + scan_block(sum, sh.scan, total);
#pragma unroll
        for (int u = 0; u < kBins / kSelectThreads; ++u) {
            if (upto < keep && upto + mine[u] >= keep) { // (of exactly one thread)
                sh.digit = kBins - 1 - (tid * (kBins / kSelectThreads) + u);
                sh.above = upto;
            }
            upto += mine[u];
        }
        __syncthreads();
        least |= (uint32_t)sh.digit << shift;
        above = sh.above;
        __syncthreads();
    }

    // ---- which rows stay: those above, and the first of those equal to it --------------------------------------
    for (int w = warp; w < words; w += kSelectWarps) {
        const int i = (word0 + w) * 32 + lane;
        const uint32_t equal = __ballot_sync(0xFFFFFFFFu, i < n && worth(i, false) == least);
        if (lane == 0) before[w] = __popc(equal);
    }
    __syncthreads();
    const int ties = scan_words(before, words, sh.scan);
    if (tid == 0) sh.ties = ties;
    cluster.sync();
    int wanted = keep - above; // of the rows equal to it, from this stretch on
    for (int r = 0; r < rank; ++r) wanted -= *cluster.map_shared_rank(&sh.ties, r);
    for (int w = warp; w < words; w += kSelectWarps) {
        const int i = (word0 + w) * 32 + lane;
        const uint32_t x = i < n ? worth(i, false) : 0u;
        const bool is_equal = i < n && x == least;
        const uint32_t equal = __ballot_sync(0xFFFFFFFFu, is_equal);
        const bool in = (i < n && x > least) || (is_equal && before[w] + __popc(equal & ((1u << lane) - 1u)) < wanted);
        const uint32_t bits = __ballot_sync(0xFFFFFFFFu, in);
        const uint32_t below = __ballot_sync(0xFFFFFFFFu, i < keep); // (keep < n: all of them are rows)
        __syncwarp();
        if (lane == 0) {
            stays[w] = bits;
            before[w] = __popc(below & ~bits) + __popc(bits & ~below); // holes, and rows to be moved
        }
    }
    __syncthreads();

    // ---- the j-th row to be moved goes to the j-th hole.  All holes are in front of all rows to be moved ------------
    const int both = scan_words(before, words, sh.scan);
    // this stretch's holes: those in the words below keep, and the lower part of the word that keep lies in
    if (tid == 0) {
        const int w = keep / 32 - word0;
        int holes = w < 0 ? 0 : (w >= words ? both : before[w]);
        if (w >= 0 && w < words) holes += __popc(~stays[w] & ((1u << (keep % 32)) - 1u));
        sh.holes = holes;
        sh.movers = both - holes;
    }
    cluster.sync();
    int hole0 = 0, first_mover[kMaxCluster]; // holes in front of the stretch, rows to be moved in front of every stretch
#pragma unroll
    for (int r = 0, sum = 0; r < kMaxCluster; ++r) {
        first_mover[r] = sum;
        if (r < C) {
            if (r < rank) hole0 += *cluster.map_shared_rank(&sh.holes, r);
            sum += *cluster.map_shared_rank(&sh.movers, r);
        }
    }
    for (int w = warp; w < words; w += kSelectWarps) {
        const int i = (word0 + w) * 32 + lane;
        if (i >= keep) continue;
        const uint32_t bits = stays[w];
        int from = i;
        if (!((bits >> lane) & 1u)) {
            const int j = hole0 + before[w] + __popc(~bits & ((1u << lane) - 1u));
            int r = 0;
#pragma unroll
            for (int u = 1; u < kMaxCluster; ++u)
                if (u < C && first_mover[u] <= j) r = u;
            int at = j;
#pragma unroll
            for (int u = 1; u < kMaxCluster; ++u)
                if (u == r) at = j - first_mover[u];
            const uint32_t *its_stays = cluster.map_shared_rank(stays, r);
            const int *its_before = cluster.map_shared_rank(before, r);
            const int its_holes = *cluster.map_shared_rank(&sh.holes, r);
            // the last word with at most `at` rows to be moved in front of it
            int lo = 0, hi = min(all_words, r * each + each) - r * each;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (its_before[mid] - its_holes <= at)
                    lo = mid;
                else
                    hi = mid;
            }
            const int word = r * each + lo;
            uint32_t moved = its_stays[lo];
            if (word * 32 < keep) moved &= ~((1u << (keep - word * 32)) - 1u); // (keep lies in this word)
            for (int rest = at - max(0, its_before[lo] - its_holes); rest > 0; --rest) moved &= moved - 1u;
            from = word * 32 + __ffs(moved) - 1;
        }
        source[i] = from;
    }
    cluster.sync(); // (others may still look into this CTA's words)
}

// Moves row source[i] of every sequence and kv head to row i.  A warp takes 32 rows i at a time, looks at what moves with a
// lane each, and copies rows with all of its lanes: keys with one half, values with the other.  Rows that are copied from lie at or behind
// `keep`, rows that are copied to below it, so no row is both and all may be copied at once.
constexpr int kCompactThreads = 256;
constexpr int kRowsAtATime = 4;

__global__ void __launch_bounds__(kCompactThreads) kv_compact_kernel(const __grid_constant__ CompactArgs a, const int64_t items)
{
    ptx::griddep_wait(); // everything below is read from memory that the launch before this one may have written
    ptx::griddep_launch_dependents();
    const int lane = threadIdx.x % 32, Hk = a.cache.kv_heads, keep = a.keep;
    const int per_pair = (keep + 31) / 32;
    const bool int8 = a.cache.k_scale != nullptr;
    const int row_bytes = a.cache.width * (int8 ? 1 : 2), pieces = row_bytes / 16;
    const int64_t step = (int64_t)gridDim.x * (kCompactThreads / 32);
    char *pool = reinterpret_cast<char *>(lane < 16 ? a.cache.k : a.cache.v);
    for (int64_t item = (int64_t)blockIdx.x * (kCompactThreads / 32) + threadIdx.x / 32; item < items; item += step) {
        const int64_t pair = item / per_pair;
        const int i = (int)(item - pair * per_pair) * 32 + lane, b = (int)(pair / Hk), h = (int)(pair - (int64_t)b * Hk);
        int from = -1, to = -1;
        if (i < keep) {
            const int src = a.source[pair * keep + i];
            bool over;
            const int n = kv_length(a.batch, b, over);
            if (over && i == 0 && h == 0) kv_report(a.cache);
            if (src != i && src != -1) {
                bool good = src >= keep && src < n;
                if (good) {
                    const int src_page = kv_page(a.cache, a.batch, b, src), dst_page = kv_page(a.cache, a.batch, b, i);
                    good = src_page >= 0 && dst_page >= 0;
                    if (good) {
                        from = kv_row(a.cache, src_page, h, src);
                        to = kv_row(a.cache, dst_page, h, i);
                    }
                }
                if (!good) kv_report(a.cache);
            }
        }
        if (from >= 0) {
            if (int8) {
                a.cache.k_scale[to] = a.cache.k_scale[from];
                a.cache.v_scale[to] = a.cache.v_scale[from];
            }
            if (a.marks.mass) {
                a.marks.mass[to] = a.marks.mass[from];
                a.marks.pos[to] = a.marks.pos[from];
            }
        }
        uint32_t moves = __ballot_sync(0xFFFFFFFFu, from >= 0);
        while (moves) {
            uint4 x[kRowsAtATime];
            int64_t dst[kRowsAtATime];
#pragma unroll
            for (int u = 0; u < kRowsAtATime; ++u) {
                const int l = moves ? __ffs(moves) - 1 : -1;
                moves &= moves - 1u;
                const int src = __shfl_sync(0xFFFFFFFFu, from, max(l, 0));
                const int row = __shfl_sync(0xFFFFFFFFu, to, max(l, 0));
                dst[u] = l < 0 || lane % 16 >= pieces ? -1 : (int64_t)row * row_bytes + lane % 16 * 16;
                if (dst[u] >= 0) x[u] = *reinterpret_cast<const uint4 *>(pool + (int64_t)src * row_bytes + lane % 16 * 16);
            }
#pragma unroll
            for (int u = 0; u < kRowsAtATime; ++u)
                if (dst[u] >= 0) *reinterpret_cast<uint4 *>(pool + dst[u]) = x[u];
        }
    }
}

} // namespace

cudaError_t launch_kv_select(const SelectArgs &a, cudaStream_t stream)
{
    const int64_t pairs = (int64_t)a.batch.n_seqs * a.cache.kv_heads;
    // CTAs per (sequence, kv head): more while there are idle SMs and a stretch is long enough to be worth it, and as many as the
    // bits of the longest sequence need.
    constexpr size_t kMost = 200 * 1024;
    auto bytes_of = [&](int c) { return sizeof(SelectShared) + (size_t)stretch_words(a.batch.capacity, c) * 8; };
    int cluster = 1;
    while (cluster < kMaxCluster && (bytes_of(cluster) > kMost || (pairs * cluster * 2 <= 2 * sm_count() && a.batch.capacity / cluster > 4096))) cluster *= 2;
    const size_t smem = bytes_of(cluster);
    if (smem > kMost) return cudaErrorInvalidValue;
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(kv_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMost);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    cudaLaunchAttribute attributes[2];
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = (unsigned)cluster;
    attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3((unsigned)(pairs * cluster));
    config.blockDim = dim3(kSelectThreads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = attributes;
    config.numAttrs = 2;
    return cudaLaunchKernelEx(&config, kv_select_kernel, a, stretch_words(a.batch.capacity, cluster));
}

cudaError_t launch_kv_compact(const CompactArgs &a, cudaStream_t stream)
{
    const int64_t items = (int64_t)a.batch.n_seqs * a.cache.kv_heads * ((a.keep + 31) / 32);
    const int64_t blocks = std::min<int64_t>((items + kCompactThreads / 32 - 1) / (kCompactThreads / 32), 8 * sm_count());
    return launch_dependent(kv_compact_kernel, (unsigned)blocks, kCompactThreads, 0, stream, a, items);
}

} // namespace bitlinear
