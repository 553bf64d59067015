// Which rows of a sequence stay in the cache, by the attention weight they have received, and moving them to the front.
//
// Selection, for every (sequence, kv head) of n rows of which `keep` stay.  A row's worth is a 32-bit number: the bits of its
// weight (not negative, so they order as the weights do), or the largest number for the rows of the `recent` newest positions.
// The keep-th largest worth is found digit by digit (10, 11 and 11 bits: a histogram of the rows that agree with the digits found so
// far, summed from above, until the rows from there on are `keep` in all); rows above it stay, and of the rows equal to it the first
// ones.  Which rows stay is kept as a bit per row, with the number of holes (rows below `keep` that go) and of rows to be moved (at
// or behind `keep`) in front of every word; the j-th row to be moved takes its hole from a list of the holes in order.  Nothing
// depends on the order in which threads run.
//
// The newest position is the last row's, or, for rows in any order, the largest, found by a pass over the positions in front of the
// others (1 x 32 heads of 2064 rows: 0.1 us more; 16 sequences of 6000 to 65535 rows: 32 -> 37 us).
//
// A cluster of CTAs shares a (sequence, kv head), each of them a contiguous stretch of the rows, whose marks are read once and
// kept in shared memory.  Histograms are added up by atomics into every CTA's shared memory (of the few bins that hold anything: reading
// all bins of the others took 1000 cycles for each of them); a hole is written to the list of the CTA whose row is moved there (by way of
// the output array it took 4000 cycles longer).
//
// What bounds it: latency.  1 x 32 heads of 2064 rows: 8.4 us, 15000 cycles, of which 2300 load the marks and the rest are barriers and
// chains of a few dependent accesses in ten steps.  16 sequences of 6000 to 65535 rows, 8 heads: 32 us where the marks' 28 MB take
// 4.4: two waves of CTAs, the longest of 40000 cycles, 12000 of them (at 5.7 TB/s) loading.  Keys of 15 bits, with which 65536 rows fit into one
// CTA, and weights read again for those that agree in them: 30 us, and the short sequences 12 instead of 8.4.
#include <cooperative_groups.h>

#include <algorithm>

#include "internal.cuh"
#include "kv.cuh"
#include "ptx.cuh"

namespace bitlinear {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxCluster = 8;
constexpr size_t kSelectSmem = 220 * 1024;
constexpr int kSorted = 128; // sequences that are taken in the order of their lengths
constexpr int kDigits = 3;    // of 10, 11 and 11 bits
constexpr int kBins = 2048;
constexpr int kFirstBins = 1024, kCopies = 4; // the first digit's bins, exponents above all, are few, and so are kept four times
__device__ __forceinline__ int digit_shift(int d) { return d == 0 ? 22 : (d == 1 ? 11 : 0); }

struct alignas(16) SelectShared {
    union {
        uint32_t first[kFirstBins][kCopies];
        uint32_t sums[kDigits - 1][kBins]; // of the other digits' bins, over all CTAs
    };
    uint32_t first_sums[kFirstBins]; // of the first digit's bins, over the copies and all CTAs
    uint32_t bins[kDigits - 1][kBins];
    int scan[32];
    int4 found;           // the digit, how many rows are above it, and how many have it
    int ties[kMaxCluster]; // of every CTA's stretch
    int2 moves[kMaxCluster]; // the same: holes, and rows to be moved
    int newest[kMaxCluster]; // the same: the largest position
    int lens[kSorted];
    int4 taken;              // (the sequence of this CTA)
};

// Sum over the CTA of x of the threads in front of this one; total: of all of them.
template <int kThreads>
__device__ __forceinline__ int scan_block(int x, int *scan, int &total)
{
    constexpr int kWarps = kThreads / 32;
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
    const int own = lane < kWarps ? scan[lane] : 0;
    int sums = own;
#pragma unroll
    for (int d = 1; d < kWarps; d <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, sums, d);
        if (lane >= d) sums += y;
    }
    total = __shfl_sync(0xFFFFFFFFu, sums, kWarps - 1);
    return __shfl_sync(0xFFFFFFFFu, sums - own, warp) + upto - x;
}

// before[w] = the sum of count(0 .. w - 1); returns the sum of all n.
template <int kThreads, typename Count>
__device__ __forceinline__ int scan_words(int *before, int n, int *scan, Count &&count)
{
    int sum = 0;
    for (int w0 = 0; w0 < n; w0 += kThreads) {
        const int w = w0 + (int)threadIdx.x;
        int total;
        const int own = scan_block<kThreads>(w < n ? count(w) : 0, scan, total);
        if (w < n) before[w] = sum + own;
        sum += total;
    }
    return sum;
}

// Words of 32 rows in a CTA's stretch of a sequence of so many rows.
int stretch_words(int64_t rows, int cluster) { return (int)(((rows + 31) / 32 + cluster - 1) / cluster); }

// C: CTAs that share a (sequence, kv head).
template <int C, int kThreads>
__global__ void __launch_bounds__(kThreads) kv_select_kernel(const __grid_constant__ SelectArgs a, const int max_words, const bool sorted)
{
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = C > 1 ? (int)cluster.block_rank() : 0;
    auto sync_all = [&] {
        if (C > 1)
            cluster.sync();
        else
            __syncthreads();
    };
    auto for_all = [&](auto &&f) { // f(of): what `of` gives of a place in shared memory is that place of one CTA after the other
#pragma unroll
        for (int r = 0; r < C; ++r) f([&](auto *p) { return C > 1 ? cluster.map_shared_rank(p, r) : p; });
    };
    extern __shared__ __align__(16) uint8_t smem[];
    SelectShared &sh = *reinterpret_cast<SelectShared *>(smem);
    uint4 *cached = reinterpret_cast<uint4 *>(smem + sizeof(SelectShared)); // the worth of the stretch's rows
    int *list = reinterpret_cast<int *>(cached);                             // and later the holes that its rows are moved to
    uint32_t *stays = reinterpret_cast<uint32_t *>(cached + max_words * 8);  // a bit per row of the stretch
    int *before = reinterpret_cast<int *>(stays + max_words);                // per word: what is in front of it in the stretch
    const int tid = threadIdx.x;
    for (int i = tid; i < (kFirstBins * (kCopies + 1) + (kDigits - 1) * kBins) / 4; i += kThreads) reinterpret_cast<uint4 *>(&sh)[i] = make_uint4(0u, 0u, 0u, 0u);
    if (tid == 0) sh.found = make_int4(0, 0, 0, 0);
    __syncthreads();
    if (C > 1) cluster.barrier_arrive(); // (the others may add to these bins)
    ptx::griddep_wait(); // what follows is read from memory that the launch before this one may have written
    ptx::griddep_launch_dependents();
    const int Hk = a.cache.kv_heads, keep = a.keep;
    const int turn = (int)blockIdx.x / C / Hk, h = (int)blockIdx.x / C - turn * Hk;
    bool over;
    int b = turn;
    if (sorted) { // the longest sequences first
        const int seqs = a.batch.n_seqs;
        if (tid < seqs) sh.lens[tid] = kv_length(a.batch, tid, over);
        __syncthreads();
        if (tid < seqs) {
            const int mine = sh.lens[tid];
            int longer = 0;
            for (int i = 0; i < seqs; ++i) longer += sh.lens[i] > mine || (sh.lens[i] == mine && i < tid);
            if (longer == turn) sh.taken.x = tid;
        }
        __syncthreads();
        b = sh.taken.x;
    }
    const int n = kv_length(a.batch, b, over);
    if (tid == 0 && rank == 0 && h == 0) {
        if (over) kv_report(a.cache);
        a.new_lens[b] = min(n, keep);
    }
    int32_t *source = a.source + ((int64_t)b * Hk + h) * keep;
    if (n <= keep) { // (the whole cluster)
        for (int i = rank * kThreads + tid; i < keep; i += C * kThreads) source[i] = i < n ? i : -1;
        if (C > 1) cluster.barrier_wait();
        return;
    }
    auto row_of = [&](int i) {
        const int page = kv_page(a.cache, a.batch, b, i);
        return page < 0 ? -1 : kv_row(a.cache, page, h, i);
    };
    const int all_words = (n + 31) / 32, each = (all_words + C - 1) / C;
    const int word0 = min(all_words, rank * each), words = min(all_words, word0 + each) - word0; // of this stretch
    const int row0 = word0 * 32, rows = min(n, row0 + words * 32) - row0;
    int64_t after = INT64_MAX; // what is as new as this stays
    if (!a.any_order) {
        const int last = row_of(n - 1);
        if (last >= 0) after = (int64_t)a.marks.pos[last] - a.recent + 1;
    } else { // the largest position of the stretch, then of all stretches (no row of it on a page that exists: the smallest there is)
        int top = INT32_MIN;
        for (int i = tid * 4; i < rows; i += kThreads * 4) {
            const int row = row_of(row0 + i);
            if (row < 0) continue;
            const int4 p = *reinterpret_cast<const int4 *>(a.marks.pos + row);
            const int y[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < rows) top = max(top, y[e]);
        }
        top = __reduce_max_sync(0xFFFFFFFFu, top);
        if (tid % 32 == 0) sh.scan[tid / 32] = top;
        __syncthreads();
        top = __reduce_max_sync(0xFFFFFFFFu, tid % 32 < kThreads / 32 ? sh.scan[tid % 32] : INT32_MIN);
        if (C > 1) {
            cluster.barrier_wait(); // (all CTAs have begun)
            if (tid == 0) for_all([&](auto &&of) { *of(&sh.newest[rank]) = top; });
            cluster.sync();
            for (int r = 0; r < C; ++r) top = max(top, sh.newest[r]);
            cluster.barrier_arrive(); // (as in front of this)
        }
        after = (int64_t)top - a.recent + 1;
    }
    const bool some_new = after <= INT32_MAX;
    const int newest = (int)(after < INT32_MIN ? INT32_MIN : after);
    auto worth_of = [&](float mass, int pos) { // (nothing, or not a number: 0)
        return some_new && pos >= newest ? 0xFFFFFFFFu : (mass > 0.0f ? __float_as_uint(mass) : 0u);
    };
    // Rows are taken in pieces of four, which lie in one page and may reach behind the sequence's end.
    auto load_four = [&](int row) {
        if (row < 0) return make_uint4(0u, 0u, 0u, 0u);
        const float4 m = *reinterpret_cast<const float4 *>(a.marks.mass + row);
        const int4 p = *reinterpret_cast<const int4 *>(a.marks.pos + row);
        return make_uint4(worth_of(m.x, p.x), worth_of(m.y, p.y), worth_of(m.z, p.z), worth_of(m.w, p.w));
    };
    const int pieces = words * 8, lane = tid % 32;
    auto real_of = [&](int p) { return rows - p * 4 >= 4 ? 15u : (rows > p * 4 ? (1u << (rows - p * 4)) - 1u : 0u); }; // rows of a piece that exist
    auto bits_of = [&](int p, auto &&holds) { // the rows of a piece for which it holds
        const uint4 x = cached[p];
        return ((uint32_t)holds(x.x) | (uint32_t)holds(x.y) << 1 | (uint32_t)holds(x.z) << 2 | (uint32_t)holds(x.w) << 3) & real_of(p);
    };
    auto word_of = [&](uint32_t bits) { // the word whose pieces eight neighbouring lanes have
        bits <<= lane % 8 * 4;
        bits |= __shfl_xor_sync(0xFFFFFFFFu, bits, 1);
        bits |= __shfl_xor_sync(0xFFFFFFFFu, bits, 2);
        return bits | __shfl_xor_sync(0xFFFFFFFFu, bits, 4);
    };

    // ---- the keep-th largest worth, and how many rows are above it -----------------------------------------
    constexpr int kInFlight = 4; // pieces of a thread whose marks are being loaded
    for (int i0 = tid * 4; i0 < rows; i0 += kInFlight * kThreads * 4) {
        int row[kInFlight];
        uint4 x[kInFlight];
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int i = i0 + u * kThreads * 4;
            row[u] = i < rows ? row_of(row0 + i) : -1;
            if (i < rows && row[u] < 0) kv_report(a.cache);
        }
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) x[u] = load_four(row[u]);
#pragma unroll
        for (int u = 0; u < kInFlight; ++u) {
            const int i = i0 + u * kThreads * 4;
            if (i >= rows) break;
            cached[i / 4] = x[u];
            const uint32_t y[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < rows) atomicAdd(&sh.first[y[e] >> digit_shift(0)][lane % kCopies], 1u);
        }
    }
    uint32_t least = 0u; // its digits found so far, zeros behind them
    int above = 0;
    bool exact = false;  // the rows with a worth of `least` or more are `keep` in all
#pragma unroll
    for (int d = 0; d < kDigits; ++d) {
        if (exact) break;
        const int shift = digit_shift(d);
        if (d > 0) {
            const uint32_t span = 1u << digit_shift(d - 1); // (least begins with the digits found: those that agree are less than this above it)
            for (int p = tid; p < pieces; p += kThreads) {
                const uint32_t real = real_of(p);
                const uint4 x = cached[p];
                const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (y[e] - least < span && ((real >> e) & 1u)) atomicAdd(&sh.bins[d - 1][(y[e] - least) >> shift], 1u);
            }
        }
        // the bins of all CTAs are added up in each of them, by those that have something in them
        __syncthreads();
        if (d == 0) {
            if (C > 1) cluster.barrier_wait();
            for (int i = tid; i < kFirstBins; i += kThreads) {
                const uint4 y = *reinterpret_cast<const uint4 *>(sh.first[i]);
                const uint32_t x = y.x + y.y + y.z + y.w;
                *reinterpret_cast<uint4 *>(sh.first[i]) = make_uint4(0u, 0u, 0u, 0u); // (as the sums of the other digits)
                if (x != 0u) for_all([&](auto &&of) { atomicAdd(of(&sh.first_sums[i]), x); });
            }
        } else if (C > 1) {
            for (int i = tid; i < kBins; i += kThreads) {
                const uint32_t x = sh.bins[d - 1][i];
                if (x != 0u) for_all([&](auto &&of) { atomicAdd(of(&sh.sums[d - 1][i]), x); });
            }
        }
        if (C > 1 || d == 0) sync_all();
        const uint32_t *sums = d == 0 ? sh.first_sums : (C > 1 ? sh.sums[d - 1] : sh.bins[d - 1]);
        constexpr int kMine = kBins / kThreads;
        int mine[kMine], sum = 0; // from the largest digit down
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            const int bin = kBins - 1 - (tid * kMine + u);
            mine[u] = d > 0 || bin < kFirstBins ? (int)sums[bin] : 0;
            sum += mine[u];
        }
        int total;
        int upto = above + scan_block<kThreads>(sum, sh.scan, total);
#pragma unroll
        for (int u = 0; u < kMine; ++u) {
            if (upto < keep && upto + mine[u] >= keep) sh.found = make_int4(kBins - 1 - (tid * kMine + u), upto, mine[u], 0); // (one thread's)
            upto += mine[u];
        }
        __syncthreads();
        const int4 found = sh.found;
        least |= (uint32_t)found.x << shift;
        above = found.y;
        exact = above + found.z == keep; // (read again only behind the next round's barriers)
    }

    // ---- which rows stay: those above, and the first of those equal to it --------------------------------------
    int wanted = 0; // of the rows equal to it, from this stretch on
    if (!exact) {
        for (int p0 = tid - lane; p0 < pieces; p0 += kThreads) {
            const int p = p0 + lane;
            const uint32_t equal = word_of(p < pieces ? bits_of(p, [&](uint32_t x) { return x == least; }) : 0u);
            if (p < pieces && lane % 8 == 0) stays[p / 8] = equal;
        }
        __syncthreads();
        const int ties = scan_words<kThreads>(before, words, sh.scan, [&](int w) { return __popc(stays[w]); });
        if (tid == 0) for_all([&](auto &&of) { *of(&sh.ties[rank]) = ties; });
        sync_all();
        wanted = keep - above;
        for (int r = 0; r < rank; ++r) wanted -= sh.ties[r];
    }
    const uint32_t bound = exact ? least - 1u : least; // (with keep < n rows at or above it, an exact one is not 0)
    for (int p0 = tid - lane; p0 < pieces; p0 += kThreads) {
        const int p = p0 + lane;
        uint32_t bits = 0u;
        if (p < pieces) {
            bits = bits_of(p, [&](uint32_t x) { return x > bound; });
            if (!exact) {
                const uint32_t equal = stays[p / 8];
                uint32_t mine = (equal >> (p % 8 * 4)) & 15u;
                for (int some = wanted - before[p / 8] - __popc(equal & ((1u << (p % 8 * 4)) - 1u)); some > 0 && mine; --some, mine &= mine - 1u) bits |= mine & (0u - mine);
            }
        }
        bits = word_of(bits); // (and behind this all lanes have read the word of the equal rows)
        if (p < pieces && lane % 8 == 0) stays[p / 8] = bits;
    }
    __syncthreads();

    // ---- the j-th row to be moved goes to the j-th hole.  All holes are in front of all rows to be moved ------------
    const int keep_word = keep / 32 - word0; // the word that keep lies in (keep < n: the rows below it all exist)
    const uint32_t keep_mask = (1u << (keep % 32)) - 1u;
    auto below_of = [&](int w) { return w < keep_word ? ~0u : (w == keep_word ? keep_mask : 0u); };
    const int both = scan_words<kThreads>(before, words, sh.scan, [&](int w) { return __popc(stays[w] ^ below_of(w)); }); // holes, then rows to be moved
    __syncthreads();
    int my_holes = keep_word < 0 ? 0 : (keep_word >= words ? both : before[keep_word]);
    if (keep_word >= 0 && keep_word < words) my_holes += __popc(~stays[keep_word] & keep_mask);
    int hole0 = 0; // holes in front of this stretch
    if (C > 1) {
        if (tid == 0) for_all([&](auto &&of) { *of(&sh.moves[rank]) = make_int2(my_holes, both - my_holes); });
        cluster.sync(); // (and behind this no CTA looks at its rows' worth)
        for (int r = 0; r < rank; ++r) hole0 += sh.moves[r].x;
    }
    // The holes are listed where their rows' worth stood, each with the CTA whose row is moved there.
    for (int p = tid; p < min(pieces, max(0, (keep - row0 + 3) / 4)); p += kThreads) {
        const uint32_t bits = ~stays[p / 8];
        int j = hole0 + before[p / 8] + __popc(bits & ((1u << (p % 8 * 4)) - 1u));
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (!((bits >> (p % 8 * 4 + e)) & 1u) || row0 + p * 4 + e >= keep) continue;
            int k = j++, r = 0;
            if (C > 1)
                while (r < C && k >= sh.moves[r].y) k -= sh.moves[r++].y;
            if (r < C) *(C > 1 ? cluster.map_shared_rank(&list[k], r) : &list[k]) = row0 + p * 4 + e;
        }
    }
    sync_all();
    for (int i = tid; i < min(rows, keep - row0); i += kThreads)
        if ((stays[i / 32] >> (i % 32)) & 1u) source[row0 + i] = row0 + i;
    constexpr int kGroup = 4; // rows of a thread (the newest are neighbours and all of them moved: with a word each 1 to 3 us more)
    for (int g = max(0, keep_word) * (32 / kGroup) + tid; g < words * (32 / kGroup); g += kThreads) {
        const int w = g / (32 / kGroup), e = g % (32 / kGroup) * kGroup;
        const uint32_t all = stays[w] & ~below_of(w);
        int j = max(0, before[w] - my_holes) + __popc(all & ((1u << e) - 1u));
        for (uint32_t moved = all & (((1u << kGroup) - 1u) << e); moved; moved &= moved - 1u, ++j) {
            const int to = list[j];
            if ((uint32_t)to < (uint32_t)keep) source[to] = row0 + w * 32 + __ffs(moved) - 1; // (always, unless the marks change meanwhile)
        }
    }
}

// Moves row source[i] of every sequence and kv head to row i.  A warp takes 32 rows i at a time, looks at what moves with a
// lane each, and copies rows with all of its lanes: keys with one half, values with the other.  Rows that are copied from lie at or behind
// `keep`, rows that are copied to below it, so no row is both and all may be copied at once.
//
// What bounds it: memory, in pieces of a row (256 bytes of bf16).  64 sequences of 1500 to 8191 rows cut to 1024, 8 heads of 128: 66.6 us
// = 5.5 TB/s (0.84 of a copy's rate; two rows at a time 80 us, eight 67).  Pieces of 128 bytes, for which half of the lanes copy: the same
// rows in 8 bits 49 us (0.60), heads of 64 in bf16 44 (0.64).  32 heads, 16 rows of 2064 each: 2.7 us, the launch.
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

size_t select_smem(int64_t rows, int cluster) { return sizeof(SelectShared) + (size_t)stretch_words(rows, cluster) * (128 + 8); }
static_assert(sizeof(SelectShared) + kSelectMaxRows / 32 / kMaxCluster * (128 + 8) <= kSelectSmem, "the longest stretch");

template <int C, int kThreads>
cudaError_t launch_select(const SelectArgs &a, cudaStream_t stream)
{
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(kv_select_kernel<C, kThreads>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSelectSmem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    const int words = stretch_words(a.batch.capacity, C);
    cudaLaunchAttribute attributes[2];
    attributes[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attributes[0].val.programmaticStreamSerializationAllowed = 1;
    attributes[1].id = cudaLaunchAttributeClusterDimension;
    attributes[1].val.clusterDim.x = (unsigned)C;
    attributes[1].val.clusterDim.y = attributes[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t config = {};
    const int64_t ctas = (int64_t)a.batch.n_seqs * a.cache.kv_heads * C;
    config.gridDim = dim3((unsigned)ctas);
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = select_smem(a.batch.capacity, C);
    config.stream = stream;
    config.attrs = attributes;
    config.numAttrs = C > 1 ? 2 : 1;
    // With a few waves of CTAs a long sequence that comes last is waited for (16 sequences of 6000 to 65535 rows, 8 heads: 41 us in the
    // order of the batch, 32 sorted); with many waves it is not, and every CTA's sorting costs (2560 pairs: 28, 31).
    const bool sorted = a.batch.n_seqs > 1 && a.batch.n_seqs <= kSorted && ctas > sm_count() && ctas <= 4 * sm_count();
    return cudaLaunchKernelEx(&config, kv_select_kernel<C, kThreads>, a, words, sorted);
}

} // namespace

cudaError_t launch_kv_select(const SelectArgs &a, cudaStream_t stream)
{
    const int64_t pairs = (int64_t)a.batch.n_seqs * a.cache.kv_heads;
    // (The lengths are known on the device alone, so "rows" here are those that a row of the page table has room for: a table far wider than
    // the sequences costs time.  64 sequences of 100 to 900 rows, 8 heads, none of them to be cut: 2.5 us behind a table of 960 positions, 22
    // behind one of 131072; of 1100 to 2000 rows, cut to 1024: 10.7 and 129.)
    // CTAs per (sequence, kv head): as many as the rows of the longest sequence need shared memory of, and more where a stretch is long
    // enough to be worth the clusters' barriers (us with 1, 2, 4 and 8 CTAs: 32 pairs of 9000 rows 10.5, 12.3, 11.0; of 12000 11.3, 12.2; of
    // 20000 14.8, 13.8, 12.8; 8 pairs of 40000 17.9 with 2, 14.1, 13.3; of 131000 23.8 with 4, 19.5) and all clusters run at once, of which the
    // parts of the GPU that hold a cluster each have room for few (16 pairs of 131000: 8 CTAs 35.7, 4 25.4; 128 of 16000: 2 25, 1 13.3).
    int cluster = 1;
    auto all_run = [&](int ctas) { return pairs * ctas <= sm_count() * (ctas == 8 ? 3 : 4) / 4; };
    while (cluster < kMaxCluster && (select_smem(a.batch.capacity, cluster) > kSelectSmem || (a.batch.capacity > 12288 && a.batch.capacity / cluster > 8192 && all_run(2 * cluster))))
        cluster *= 2;
    // Many pairs take fewer threads, where several CTAs fit on an SM (2560 pairs of 200 to 500 rows: 28 us with 256 threads, 38 with 512, 61
    // with 1024; 512 pairs of 1500 to 8191: 18.3, 17.7, 21.3; 256 of 10000 to 20000, whose marks fill an SM's shared memory: 48, 31, 25).
    if (cluster == 1) {
        if (pairs <= sm_count() || select_smem(a.batch.capacity, 1) > kSelectSmem / 2) return launch_select<1, 1024>(a, stream);
        return a.batch.capacity <= 4096 ? launch_select<1, 256>(a, stream) : launch_select<1, 512>(a, stream);
    }
    if (cluster == 2) return launch_select<2, 1024>(a, stream);
    return cluster == 4 ? launch_select<4, 1024>(a, stream) : launch_select<8, 1024>(a, stream);
}

cudaError_t launch_kv_compact(const CompactArgs &a, cudaStream_t stream)
{
    const int64_t items = (int64_t)a.batch.n_seqs * a.cache.kv_heads * ((a.keep + 31) / 32);
    const int64_t blocks = std::min<int64_t>((items + kCompactThreads / 32 - 1) / (kCompactThreads / 32), 16 * sm_count());
    return launch_dependent(kv_compact_kernel, (unsigned)blocks, kCompactThreads, 0, stream, a, items);
}

} // namespace bitlinear
