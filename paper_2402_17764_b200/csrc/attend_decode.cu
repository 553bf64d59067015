// Attention of one new token per sequence over the paged cache.
//
//   out_h = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m),   s_j = scale log2(e) q_h . k_j,   m = max_j s_j
//
// in one pass over the cache: every warp keeps a running maximum, sum and output for its own keys, and partial results join by
//   m = max(m1, m2),  l = l1 2^(m1 - m) + l2 2^(m2 - m),  o = o1 2^(m1 - m) + o2 2^(m2 - m).
//
// What bounds it: reading the cache once (HBM).  So all query heads of a kv head are handled together (8 or 16 columns of
// a matrix instruction), and the work is cut by bytes, not by sequences: the blocks of all (sequence, kv head) pairs stand
// in one row of units, and every CTA takes an equal, contiguous share of it, wherever that begins and ends.  A pair ends with one
// unit that stands for what beginning and joining a pair costs, about the time of a block (without it CTAs whose share
// is many short sequences finished 30 us after the others: 32 sequences of 1 to 4096 tokens, 32 heads, 82 us).  A pair that
// several CTAs share is joined by whichever of them finishes last, in the order of the shares, so the result does not
// depend on which one it was.
//
// Inside a CTA each of the four warps streams keys of its own through a ring of its own (cp.async, 8 KB per stage, no
// barrier between warps before the end of a pair): the ring keeps loading the next pair's keys while this one's are
// finished.  Scores are K Q^T (keys are the 16 rows of the instruction, queries its 8 columns) and the output is
// V^T P^T (16 elements of the head, 8 queries), so that a group of 1 to 8 query heads wastes at most the columns it does not have;
// P^T changes from accumulator to operand by movmatrix.  The weights enter as two bf16 parts (value and remainder, 16 bits
// together): the tensor cores have time for it, and beside the rounding of the results to bf16 it does not show.
//
// int8 cache: a key's scale multiplies its score, a value's scale its weight.  Values become bf16 exactly (code_pair below, four
// instructions per two elements, which is what bounds the kernel then).  Keys stay codes: the queries are written as integers of
// 23 bits, relative to the power of two above their row's largest, in three signed bytes, and the scores are exact
// integer products of codes and bytes (three MMAs of twice the depth instead of 16 conversions per MMA).
//
// Measured: 128k tokens of one sequence, 64/8 heads: 94-95 us = 5.7 TB/s (0.86 of a copy's rate); 32 sequences of 1 to 4096 tokens,
// 32 heads: 46.5 us = 5.2 TB/s; int8, 128 sequences of 256 to 8192 tokens, 64/8 heads: 157-159 us = 4.5 TB/s (issue slots 57 %
// busy, so not at a limit; what they wait for is the chain from a stage's codes to its output); one sequence of 777 tokens, 32
// heads of 100: 9.5 us per call, a chain of dependent loads and the join of its parts.
//
// Two more forms.  The one that weighs keeps all scores (4 bytes for each query head and key, 6 % of the traffic with 8 heads per kv
// head) and every softmax's reference and sum, and a second launch adds up 2^(s - m) / l over a kv head's queries: the references are
// known at the end only, and reading the keys again would cost half as much once more.  128k tokens of one sequence, 64/8 heads:
// 117 us (93 without); int8, 24 sequences of 100 to 4096 tokens, 40/40 heads: 86 us (75); one sequence of 777, 32 heads of 100: 11.8 us
// (9.2) on the GPU, 12.4 per call.  What they add: the scores' way to the L2 and back, and a launch.  The form behind shared rows starts behind them and joins
// what attend_prompt.cu found for those (up to 32 parts of a row) when a pair is stored: 64 sequences of 1 to 801 keys, 64/8 heads, 26 us
// with nine parts to join each, 21 without any.
#include <algorithm>

#include "internal.cuh"
#include "kv.cuh"
#include "ptx.cuh"

namespace bitlinear {
namespace {

using namespace ptx;

constexpr int kWarps = 4;
constexpr int kStageBytes = 8192; // keys and values of a stage
constexpr int kLeastShare = 2;    // units: finer shares cost more in joining than they save (8 pairs of 2000 keys: 14.4 -> 12.4 us)
constexpr int kMaxSplits = 2;     // partial results of a CTA: of the pair it begins in the middle of, of the one it ends in the middle of

// WT: elements of a cache row in shared memory (the row's width rounded up to 64 or 128).  NT: 8-query tiles.
template <bool kInt8, int WT, int NT>
struct Shape {
    // int8 keys stay codes and need fewer registers, and the conversion of the values more warps to hide its latency: three
    // CTAs of two stages per warp instead of two CTAs of three (128 sequences, 64/8 heads: 167 -> 158 us)
    static constexpr int kCtas = kInt8 && NT == 1 ? 3 : 2; // per SM
    static constexpr int kRowBytes = WT * (kInt8 ? 1 : 2);
    static constexpr int kKeys = kStageBytes / 2 / kRowBytes; // of a stage: 16, 32 or 64
    static constexpr int kChunks = kRowBytes / 16;
    static constexpr int kScaleBytes = kInt8 ? kKeys * 8 : 0; // fp32 scales of the keys and the values
    static constexpr int kStage = kStageBytes + kScaleBytes;
    static constexpr int kStages = kCtas == 3 ? 2 : 3;
    static constexpr int kQ = 8 * NT;
    static constexpr int kMl = kWarps * kQ; // (maximum, sum) of the warps, and later of the parts
    static constexpr int kSmem = kWarps * kStages * kStage + kMl * 8;
    static_assert(kQ * WT * 4 <= kStageBytes, "a warp's output fits the stage that it has just used up");
    static constexpr int kPartFloats = kQ * (WT + 2); // a partial result in the workspace
};

__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src, bool real)
{
    const int n = real ? 16 : 0; // 0: the 16 bytes become zero and nothing is read
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// The same for what is to leave the L2 first.
__device__ __forceinline__ uint64_t leave_first()
{
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
__device__ __forceinline__ void cp_async_16(uint32_t dst, const void *src, bool real, uint64_t policy)
{
    const int n = real ? 16 : 0;
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2, %3;" ::"r"(dst), "l"(src), "r"(n), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x)
{
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_s8(int (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm volatile("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// Two signed bytes of w as two bf16 numbers, exactly.  0x43 in front of a byte makes the bf16 number 128 + its low seven bits
// when its top bit is 0; 128 or, with the top bit alone, 256 is then subtracted: b - 0 or b - 256.
template <uint32_t kSelect>
__device__ __forceinline__ uint32_t code_pair(uint32_t w)
{
    const uint32_t t = __byte_perm(w, 0x43434343u, kSelect);
    const uint32_t x = t & 0xFF7FFF7Fu, y = t & 0xFF80FF80u;
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&d);
}

__device__ __forceinline__ void add_scaled(float4 &x, float f, const float4 &y)
{
    x.x += f * y.x;
    x.y += f * y.y;
    x.z += f * y.z;
    x.w += f * y.w;
}

// Byte offset of 16-byte piece c of row r of a stage's keys or values: the eight rows that an ldmatrix reads at one
// c lie in eight different bank groups.
template <int kRowBytes>
__device__ __forceinline__ uint32_t piece(int r, int c)
{
    const int x = kRowBytes >= 128 ? (r & 7) : ((r >> 1) & 3);
    return (uint32_t)(r * kRowBytes + ((c ^ x) << 4));
}

// A block of keys: block `blk` of pair `pair` (kv head and chunk of its query heads) of sequence b, at `unit` in the row.
struct Place {
    int b, pair, blk, nblk, len, unit;
};
constexpr int kPairCost = 1; // units at the end of a pair

// Equal shares of the row: the first `rest` shares have one unit more.
struct Plan {
    int shares, each, rest;
    __device__ __forceinline__ Plan(int total, int most)
    {
        shares = min(total, most);
        each = shares > 0 ? total / shares : 0;
        rest = shares > 0 ? total - each * shares : 0;
    }
    __device__ __forceinline__ int begin_of(int i) const { return i * each + min(i, rest); }
    __device__ __forceinline__ int share_of(int unit) const
    {
        const int longer = rest * (each + 1);
        return unit < longer ? unit / (each + 1) : rest + (unit - longer) / each;
    }
};

// What the kernel does besides.
enum : int {
    kPlain = 0,
    kWeigh = 1,  // keeps the scores of its blocks and every softmax's maximum and sum for the kernel that adds up the weights
    kBehind = 2, // the sequences' first rows have been dealt with: begins behind them and joins their results to its own
};
template <int kMode>
struct More {};
template <>
struct More<kWeigh> : WeighArgs {};
template <>
struct More<kBehind> : SharedArgs {};

template <bool kInt8, int WT, int NT, int kMode>
__global__ void __launch_bounds__(kWarps * 32, Shape<kInt8, WT, NT>::kCtas)
attend_decode_kernel(const __grid_constant__ AttendArgs a, const int chunks, const int chunk_heads, const __grid_constant__ More<kMode> more)
{
    griddep_wait(); // everything below is read from memory that the launch before this one may have written
    griddep_launch_dependents();
    using S = Shape<kInt8, WT, NT>;
    constexpr int kKeys = S::kKeys, kBlock = kWarps * kKeys, kSteps = WT / 16, kRB = S::kRowBytes, kThreads = kWarps * 32;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ int scan[kWarps], found_b, found_rest, is_last;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, g = lane / 4, tq = lane % 4;
    const int group = a.heads / a.cache.kv_heads, D = a.cache.head_dim, W = a.cache.width;
    const int pairs = a.cache.kv_heads * chunks, n_seqs = a.batch.n_seqs;

    // ---- the row: its length (the host made sure that it fits 31 bits), and where this CTA's share begins --------------
    auto start_of = [&](int b) { // the first row that is this kernel's
        if constexpr (kMode == kBehind) return more.starts[b];
        return 0;
    };
    auto length = [&](int b) {
        bool over;
        const int n = kv_length(a.batch, b, over);
        return kMode == kBehind ? max(0, n - start_of(b)) : n;
    };
    auto blocks_of = [&](int len) { return (len + kBlock - 1) / kBlock; };
    auto units_of = [&](int len) { return len > 0 ? (blocks_of(len) + kPairCost) * pairs : 0; };
    const int per_thread = (n_seqs + kThreads - 1) / kThreads;
    const int b0 = min(n_seqs, tid * per_thread), b1 = min(n_seqs, b0 + per_thread);
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        bool over;
        const int n = kv_length(a.batch, b, over);
        if (over && blockIdx.x == 0) kv_report(a.cache);
        mine += units_of(kMode == kBehind ? max(0, n - start_of(b)) : n);
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) upto += scan[w];
        total += scan[w];
    }
    const Plan plan(total, min((int)gridDim.x, max(1, total / kLeastShare)));
    const bool works = (int)blockIdx.x < plan.shares;
    const int share_begin = plan.begin_of(blockIdx.x), share_end = plan.begin_of(blockIdx.x + 1);
    if (works && share_begin >= upto - mine && share_begin < upto) {
        int rest = share_begin - (upto - mine), b = b0;
        for (; b < b1 - 1; ++b) {
            const int units = units_of(length(b));
            if (rest < units) break;
            rest -= units;
        }
        found_b = b;
        found_rest = rest;
    }
    __syncthreads();

    // a place that is inside the share, or `unit` >= share_end
    auto settle = [&](Place &p) { // p.blk may be behind the pair's last block
        if (p.blk < p.nblk) return;
        p.unit += p.nblk + kPairCost - p.blk;
        p.blk = 0;
        if (p.unit >= share_end || ++p.pair < pairs) return;
        p.pair = 0;
        do p.len = length(++p.b);
        while (p.len == 0);
        p.nblk = blocks_of(p.len);
    };
    auto advance = [&](Place &p) {
        ++p.blk;
        ++p.unit;
        settle(p);
    };
    Place first;
    first.unit = share_end;
    if (works) {
        first.b = found_b;
        first.len = length(first.b);
        first.nblk = blocks_of(first.len);
        first.pair = found_rest / (first.nblk + kPairCost);
        first.blk = found_rest - first.pair * (first.nblk + kPairCost);
        first.unit = share_begin;
        settle(first);
    }

    // ---- the ring --------------------------------------------------------------------------------------
    uint8_t *ring = smem + warp * S::kStages * S::kStage;
    const uint32_t ring_addr = smem_u32(ring);
    float2 *join_ml = reinterpret_cast<float2 *>(smem + kWarps * S::kStages * S::kStage); // (m, l) of [warp][query]

    // page numbers of the 16-key groups of this warp's part of a block, one per lane
    auto pages_of = [&](const Place &p) {
        int page = -1;
        if (lane < kKeys / 16) {
            const int pos = p.blk * kBlock + warp * kKeys + lane * 16;
            if (pos < p.len) {
                page = kv_page(a.cache, a.batch, p.b, start_of(p.b) + pos);
                if (page < 0) kv_report(a.cache);
            }
        }
        return page;
    };
    // (kWeigh: the keys and values make room in the L2 for the scores, which the launch behind this one reads)
    const uint64_t policy = kMode == kWeigh ? leave_first() : 0;
    auto copy = [&](uint32_t dst, const void *src, bool real) {
        if (kMode == kWeigh)
            cp_async_16(dst, src, real, policy);
        else
            cp_async_16(dst, src, real);
    };
    auto fetch = [&](const Place &p, int pages, int stage) {
        const uint32_t at = ring_addr + stage * S::kStage;
        const int key0 = p.blk * kBlock + warp * kKeys;
        const int n = p.len - key0; // keys that exist
        if (n <= 0) return;
        const int head = p.pair / chunks;
        constexpr int kElement = kInt8 ? 1 : 2, kRowsAtOnce = 32 / S::kChunks;
        const int c = lane % S::kChunks, r0 = lane / S::kChunks;
        // all rows exist and are as long in the cache as in the ring: nothing to check per copy
        const bool plain = W == WT && n >= kKeys && !__any_sync(0xFFFFFFFFu, lane < kKeys / 16 && pages < 0);
        const bool real_c = c * 16 < W * kElement;
#pragma unroll
        for (int q = 0; q < kKeys / 16; ++q) {
            const int page = __shfl_sync(0xFFFFFFFFu, pages, q);
            const bool have = page >= 0;
            const int64_t row = have ? kv_row(a.cache, page, head, key0 + q * 16) : 0;
            const uint8_t *kp = reinterpret_cast<const uint8_t *>(a.cache.k), *vp = reinterpret_cast<const uint8_t *>(a.cache.v);
            if (plain) {
                const int64_t offset = row * kRB + lane * 16; // (the rows of a group follow each other)
                kp += offset;
                vp += offset;
#pragma unroll
                for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
                    const uint32_t dst = at + piece<kRB>(q * 16 + i * kRowsAtOnce + r0, c);
                    if (kMode == kWeigh) {
                        copy(dst, kp + i * 512, true);
                        copy(dst + kStageBytes / 2, vp + i * 512, true);
                    } else {
                        cp_async_16(dst, kp + i * 512);
                        cp_async_16(dst + kStageBytes / 2, vp + i * 512);
                    }
                }
            } else {
                const int64_t offset = row * W * kElement;
                kp += offset;
                vp += offset;
#pragma unroll
                for (int i = 0; i < 16 / kRowsAtOnce; ++i) {
                    const int r = i * kRowsAtOnce + r0;
                    const bool real = have && real_c && q * 16 + r < n;
                    const int skip = real ? r * W * kElement + c * 16 : 0; // (an address that exists in any case)
                    const uint32_t dst = at + piece<kRB>(q * 16 + r, c);
                    copy(dst, kp + skip, real);
                    copy(dst + kStageBytes / 2, vp + skip, real);
                }
            }
            if (kInt8 && lane < 8) { // 4 pieces of 4 scales for the keys, 4 for the values
                const float *src = lane < 4 ? a.cache.k_scale : a.cache.v_scale;
                cp_async_16(at + kStageBytes + (lane < 4 ? 0 : kKeys * 4) + q * 64 + (lane & 3) * 16, src + (have ? row + (lane & 3) * 4 : 0), have);
            }
        }
    };

    // ---- a pair's state ----------------------------------------------------------------------------------
    // (two tiles of queries as three bytes each would not fit the registers)
    constexpr bool kDigits = kInt8 && NT == 1;
    uint32_t qf[NT][kSteps][2];       // queries as the MMA's operand
    uint32_t qd[kDigits ? 3 : 1][kSteps]; // or their bytes, highest first
    float factor = 0.0f;              // kDigits: of the integer scores of query g
    float o[NT][kSteps][4], m[NT][2], l[NT][2];
    auto begin_pair = [&](const Place &p) {
        const int head = p.pair / chunks, chunk = p.pair % chunks;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int i = chunk * chunk_heads + t * 8 + g; // query head of the group that is this lane's column
            const bool have = t * 8 + g < chunk_heads && i < group;
            const __nv_bfloat16 *q = a.q + (int64_t)p.b * a.q_stride + (int64_t)(head * group + (have ? i : 0)) * D;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                // the instruction's k index runs over the head's elements in the order in which K's registers hold them
                const int e0 = s * 16 + (kInt8 ? 4 * tq : 2 * tq), e1 = e0 + (kInt8 ? 2 : 8);
                qf[t][s][0] = have && e0 < D ? *reinterpret_cast<const uint32_t *>(q + e0) : 0u;
                qf[t][s][1] = have && e1 < D ? *reinterpret_cast<const uint32_t *>(q + e1) : 0u;
                o[t][s][0] = o[t][s][1] = o[t][s][2] = o[t][s][3] = 0.0f;
            }
            m[t][0] = m[t][1] = -INFINITY;
            l[t][0] = l[t][1] = 0.0f;
        }
        if (kDigits) {
            // the largest magnitude of the row (as the bits of a non-negative bf16 number), over the four lanes that share it
            uint32_t top = 0;
#pragma unroll
            for (int s = 0; s < kSteps; ++s)
#pragma unroll
                for (int h = 0; h < 2; ++h) top = max(top, max(qf[0][s][h] & 0x7FFFu, (qf[0][s][h] >> 16) & 0x7FFFu));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            // 2^e with 2^21 <= largest 2^e < 2^22 (e is cut at 120: rows below 2^-99 keep fewer bits)
            const int e = min(120, 21 + 127 - (int)max(top >> 7, 1u));
            const float up = __int_as_float((127 + e) << 23);
            factor = (top >> 7) == 0xFFu ? __int_as_float(0x7FFFFFFF) : a.scale * __int_as_float((127 - e) << 23); // (not finite: NaN)
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint32_t d[3] = {0u, 0u, 0u};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t w = qf[0][s][i / 2];
                    const int v = __float2int_rn(__uint_as_float(i % 2 ? w & 0xFFFF0000u : w << 16) * up);
                    const int d2 = (int)(int8_t)v, v1 = (v - d2) >> 8, d1 = (int)(int8_t)v1, d0 = (v1 - d1) >> 8;
                    d[0] |= ((uint32_t)d0 & 0xFFu) << (8 * i);
                    d[1] |= ((uint32_t)d1 & 0xFFu) << (8 * i);
                    d[2] |= ((uint32_t)d2 & 0xFFu) << (8 * i);
                }
#pragma unroll
                for (int i = 0; i < (kDigits ? 3 : 1); ++i) qd[i][s] = d[i];
            }
        }
    };

    // one stage: the scores of its keys, the weights, and their share of the output
    auto consume = [&](const Place &p, int pages, int stage) {
        const int key0 = p.blk * kBlock + warp * kKeys;
        const int n = p.len - key0;
        if (n <= 0) return;
        const uint32_t at = ring_addr + stage * S::kStage;
        const float *scales = reinterpret_cast<const float *>(ring + stage * S::kStage + kStageBytes);
        constexpr int kGroups = kKeys / 16;
        float s[kGroups][NT][4];
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
#pragma unroll
            for (int t = 0; t < NT; ++t) s[q][t][0] = s[q][t][1] = s[q][t][2] = s[q][t][3] = 0.0f;
            const int r = q * 16 + (lane & 15);
            if (kDigits) {
                int sum[3][4] = {};
#pragma unroll
                for (int i = 0; i < kSteps; i += 2) {
                    uint32_t k[4];
                    ldmatrix_x4(at + piece<kRB>(r, i + (lane >> 4)), k);
#pragma unroll
                    for (int d = 0; d < (kDigits ? 3 : 1); ++d) mma_s8(sum[d], k, qd[d][i], qd[d][i + 1]);
                }
                // (the upper two sums together are below 2^31: 128 products of 2^7 and 2^14 + 2^7)
#pragma unroll
                for (int c = 0; c < 4; ++c) s[q][0][c] = (float)(sum[0][c] * 256 + sum[1][c]) * 256.0f + (float)sum[2][c];
            } else if (!kInt8) {
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    uint32_t k[4];
                    ldmatrix_x4(at + piece<kRB>(r, 2 * i + (lane >> 4)), k);
#pragma unroll
                    for (int t = 0; t < NT; ++t) mma_bf16(s[q][t], k, qf[t][i][0], qf[t][i][1]);
                }
            } else {
#pragma unroll
                for (int i = 0; i < kSteps; i += 2) {
                    uint32_t w[4];
                    ldmatrix_x4(at + piece<kRB>(r, i + (lane >> 4)), w);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t k[4] = {code_pair<0x4140>(w[2 * j]), code_pair<0x4140>(w[2 * j + 1]), code_pair<0x4342>(w[2 * j]),
                                               code_pair<0x4342>(w[2 * j + 1])};
#pragma unroll
                        for (int t = 0; t < NT; ++t) mma_bf16(s[q][t], k, qf[t][i + j][0], qf[t][i + j][1]);
                    }
                }
            }
        }
        // scale, mask, running maximum
        // (the factor of query 2 tq + j stands in the lanes of its column's operand)
        const float column_factor[2] = {kDigits ? __shfl_sync(0xFFFFFFFFu, factor, 8 * tq) : 0.0f, kDigits ? __shfl_sync(0xFFFFFFFFu, factor, 8 * tq + 4) : 0.0f};
        bool bad = false;
        if (lane < kGroups) bad = pages < 0;
        const uint32_t bad_groups = __ballot_sync(0xFFFFFFFFu, bad);
        const bool all = n >= kKeys && bad_groups == 0u;
        float top[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t) top[t][0] = m[t][0], top[t][1] = m[t][1];
#pragma unroll
        for (int q = 0; q < kGroups; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = q * 16 + h * 8 + g;
                const float f = kDigits ? scales[r] : (kInt8 ? a.scale * scales[r] : a.scale);
                const bool seen = all || (r < n && !((bad_groups >> q) & 1u));
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float &x = s[q][t][2 * h + j];
                        x = seen ? (kDigits ? __fmul_rn(x * f, column_factor[j]) : __fmul_rn(x, f)) : -INFINITY; // (rounded here: the largest minus itself is 0)
                        top[t][j] = fmaxf(top[t][j], x);
                    }
            }
        if constexpr (kMode == kWeigh) {
            if (p.unit < more.max_units) {
                float *to = more.scores + ((int64_t)p.unit * kBlock + warp * kKeys) * chunk_heads;
#pragma unroll
                for (int q = 0; q < kGroups; ++q)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int column = t * 8 + 2 * tq;
                            float *at = to + (q * 16 + h * 8 + g) * chunk_heads + column;
                            if (chunk_heads % 2 == 0) {
                                if (column < chunk_heads) *reinterpret_cast<float2 *>(at) = make_float2(s[q][t][2 * h], s[q][t][2 * h + 1]);
                            } else {
                                if (column < chunk_heads) at[0] = s[q][t][2 * h];
                                if (column + 1 < chunk_heads) at[1] = s[q][t][2 * h + 1];
                            }
                        }
            }
        }
        float base[NT][2];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) top[t][j] = fmaxf(top[t][j], __shfl_xor_sync(0xFFFFFFFFu, top[t][j], d));
                base[t][j] = top[t][j] == -INFINITY ? 0.0f : top[t][j];
                const float keep = exp2_approx(m[t][j] - base[t][j]);
                m[t][j] = top[t][j];
                l[t][j] *= keep;
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    o[t][i][j] *= keep;
                    o[t][i][2 + j] *= keep;
                }
            }
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = q * 16 + h * 8 + g;
                const bool seen = all || (r < n && !((bad_groups >> q) & 1u));
                const float vs = kInt8 ? (seen ? scales[kKeys + r] : 0.0f) : 1.0f;
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    float w[2], rest[2];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        w[j] = exp2_approx(s[q][t][2 * h + j] - base[t][j]);
                        l[t][j] += w[j];
                        if (kInt8) w[j] *= vs;
                    }
                    // bf16 values may be infinite: the first part is cut off, not rounded, and the second one positive where the weight
                    // is, or infinity times the two would be NaN (with a second part of 0 or below): at least 2^-24 of the weight, and a
                    // normal number
                    const uint32_t x = kInt8 ? pack_bf16(w[0], w[1]) : __byte_perm(__float_as_uint(w[0]), __float_as_uint(w[1]), 0x7632);
                    rest[0] = w[0] - __uint_as_float(x << 16);
                    rest[1] = w[1] - __uint_as_float(x & 0xFFFF0000u);
                    if (!kInt8)
                        for (int j = 0; j < 2; ++j) rest[j] = fmaxf(rest[j], fminf(w[j], fmaf(w[j], 0x1p-24f, 0x1p-126f)));
                    hi[t][h] = movmatrix(x);
                    lo[t][h] = movmatrix(pack_bf16(rest[0], rest[1]));
                }
            }
            if (!kInt8) {
                // matrices in the order (elements 0-7, keys 0-7), (8-15, 0-7), (0-7, 8-15), (8-15, 8-15)
                const int r = q * 16 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    uint32_t v[4];
                    ldmatrix_x4_trans(at + kStageBytes / 2 + piece<kRB>(r, 2 * i + ((lane >> 3) & 1)), v);
#pragma unroll
                    for (int t = 0; t < NT; ++t) {
                        mma_bf16(o[t][i], v, hi[t][0], hi[t][1]);
                        mma_bf16(o[t][i], v, lo[t][0], lo[t][1]);
                    }
                }
            } else {
                // a 16-bit element of the transposed matrices is two neighbours of the head: rows 0-7 of the instruction take
                // the even ones, rows 8-15 the odd ones
                const int r = q * 16 + (lane & 15);
#pragma unroll
                for (int i = 0; i < kSteps; i += 2) {
                    uint32_t w[4];
                    ldmatrix_x4_trans(at + kStageBytes / 2 + piece<kRB>(r, i + (lane >> 4)), w);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const uint32_t v[4] = {code_pair<0x4240>(w[2 * j]), code_pair<0x4341>(w[2 * j]), code_pair<0x4240>(w[2 * j + 1]),
                                               code_pair<0x4341>(w[2 * j + 1])};
#pragma unroll
                        for (int t = 0; t < NT; ++t) {
                            mma_bf16(o[t][i + j], v, hi[t][0], hi[t][1]);
                            mma_bf16(o[t][i + j], v, lo[t][0], lo[t][1]);
                        }
                    }
                }
            }
        }
    };

    // ---- the end of a pair, or of this CTA's part of it -----------------------------------------------------
    uint32_t *counters = reinterpret_cast<uint32_t *>(a.workspace);
    auto part_of = [&](int share, int which) { return a.parts + (int64_t)(share * kMaxSplits + which) * S::kPartFloats; };
    // Adds the shared rows' result for four elements of query head `at` (counted over all sequences) to (x, M, L).
    auto join_shared = [&](int64_t at, int e, float4 &x, float &M, float &L) {
        if constexpr (kMode == kBehind) {
            const int2 where = more.where[at];
            const bool direct = where.x < 0;
            const int n = direct ? 1 : where.y >> 16, row = where.y & 0xFFFF;
            const size_t part = direct ? 0 : prompt_part_floats(W);
            const float *from = more.parts + (direct ? 0 : (size_t)where.x * part);
            const float2 *ml = direct ? more.ml + at : reinterpret_cast<const float2 *>(from) + row;
            const float4 *o = direct ? reinterpret_cast<const float4 *>(more.o + at * W + e)
                                     : reinterpret_cast<const float4 *>(from + 2 * kPromptRows) + (size_t)(e / 4) * kPromptRows + row;
            constexpr int kAtATime = 4;
            for (int c = 0; c < n; c += kAtATime) {
                float2 y[kAtATime];
                float4 v[kAtATime];
#pragma unroll
                for (int u = 0; u < kAtATime; ++u) {
                    const int p = min(c + u, n - 1);
                    y[u] = ml[p * part / 2];
                    v[u] = o[p * part / 4];
                }
                float top = M;
#pragma unroll
                for (int u = 0; u < kAtATime; ++u) top = fmaxf(top, y[u].x);
                const float base = top == -INFINITY ? 0.0f : top, keep = exp2_approx(M - base);
                x = make_float4(x.x * keep, x.y * keep, x.z * keep, x.w * keep);
                L *= keep;
                M = top;
#pragma unroll
                for (int u = 0; u < kAtATime; ++u)
                    if (c + u < n) {
                        const float f = exp2_approx(y[u].x - base);
                        add_scaled(x, f, v[u]);
                        L += f * y[u].y;
                    }
            }
        }
    };
    auto store_out = [&](const Place &p, int q, int e, float4 x, float M, float L) { // four neighbours of a query head's output
        const int head = p.pair / chunks, i = (p.pair % chunks) * chunk_heads + q;
        if (i >= group || e >= D) return;
        if constexpr (kMode == kWeigh) {
            if (e == 0) more.sums[(int64_t)p.b * a.heads + head * group + i] = make_float2(M, L);
        }
        if constexpr (kMode == kBehind) {
            if (start_of(p.b) > 0) join_shared((int64_t)p.b * a.heads + head * group + i, e, x, M, L);
        }
        const float inv = L == 0.0f ? 0.0f : 1.0f / L;
        *reinterpret_cast<uint2 *>(a.out + (int64_t)p.b * a.out_stride + (int64_t)(head * group + i) * D + e) =
            make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
    };
    // The warps lay their outputs down as [query][element] in the stage they have just used up (the next fetch into it
    // comes after this); element e of query q stands at e ^ 8 (q / 2 % 4), so that the lanes of a store hit 32 banks.
    auto laid = [](int q, int e) { return q * WT + (e ^ (((q >> 1) & 3) << 3)); };
    auto end_pair = [&](const Place &p, int stage) { // p: the last block of the pair that this CTA has
        // A thread's item, four elements of a query: neighbouring threads take neighbouring elements, or, where the shared rows' parts
        // are joined, in which neighbouring rows lie side by side, neighbouring queries (64 sequences, nine parts each: 79 -> 76 us).
        const bool by_query = kMode == kBehind && start_of(p.b) > 0;
        auto item_query = [&](int i) { return by_query ? i % chunk_heads : i / (WT / 4); };
        auto item_element = [&](int i) { return by_query ? i / chunk_heads * 4 : i % (WT / 4) * 4; };
        __syncwarp();
        float *own = reinterpret_cast<float *>(ring + stage * S::kStage);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int q = t * 8 + 2 * tq + j;
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) l[t][j] += __shfl_xor_sync(0xFFFFFFFFu, l[t][j], d);
                if (q < chunk_heads) {
                    if (g == 0) join_ml[warp * S::kQ + q] = make_float2(m[t][j], l[t][j]);
#pragma unroll
                    for (int i = 0; i < kSteps; ++i) {
                        const int e = i * 16 + (kInt8 ? 2 * g : g);
                        own[laid(q, e)] = o[t][i][j];
                        own[laid(q, e + (kInt8 ? 1 : 8))] = o[t][i][2 + j];
                    }
                }
            }
        __syncthreads();
        const int pair_begin = p.unit - p.blk, pair_end = pair_begin + p.nblk; // its blocks
        const bool whole = pair_begin >= share_begin && pair_end <= share_end;
        const int items = chunk_heads * (WT / 4); // four elements of a query each
        // the four warps' results, in warp order
        float *part = whole ? nullptr : part_of(blockIdx.x, pair_begin < share_begin ? 0 : 1);
        for (int i = tid; i < items; i += kThreads) {
            const int q = item_query(i), e = item_element(i);
            float2 ml[kWarps];
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                ml[w] = join_ml[w * S::kQ + q];
                M = fmaxf(M, ml[w].x);
            }
            const float base = M == -INFINITY ? 0.0f : M;
            float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float L = 0.0f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float f = exp2_approx(ml[w].x - base);
                add_scaled(x, f, *reinterpret_cast<const float4 *>(smem + (w * S::kStages + stage) * S::kStage + 4 * laid(q, e)));
                L += f * ml[w].y;
            }
            if (whole) {
                store_out(p, q, e, x, M, L);
            } else {
                *reinterpret_cast<float4 *>(part + 2 * S::kQ + q * WT + e) = x;
                if (e == 0) *reinterpret_cast<float2 *>(part + 2 * q) = make_float2(M, L);
            }
        }
        if (!whole) {
            const int from = plan.share_of(pair_begin), to = plan.share_of(pair_end - 1);
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                // the counter of the CTA in which the pair begins: at most one shared pair begins in a share
                const uint32_t before = atomicAdd(counters + from, 1u);
                is_last = before == (uint32_t)(to - from);
                if (is_last) counters[from] = 0u; // as the next call expects it
            }
            __syncthreads();
            if (is_last) {
                __threadfence();
                // the parts in the order of the shares; with few items each one is summed by several threads, every one
                // over its own stretch of the parts, and their sums are added in order
                int lanes = 1;
                while (items * lanes * 2 <= kThreads) lanes *= 2;
                const int n = to - from + 1, stretch = (n + lanes - 1) / lanes;
                for (int i0 = 0; i0 < items; i0 += kThreads / lanes) {
                    const int i = i0 + tid / lanes, q = item_query(i), e = item_element(i);
                    const int c0 = from + min(n, tid % lanes * stretch), c1 = from + min(n, (tid % lanes + 1) * stretch);
                    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    float M = -INFINITY, L = 0.0f;
                    if (i < items) {
#pragma unroll 1
                        for (int c = c0; c < c1; c += 8) { // eight parts' loads at a time
                            float2 ml[8];
                            float4 v[8];
#pragma unroll
                            for (int u = 0; u < 8; ++u) {
                                const int cc = min(c + u, c1 - 1);
                                const float *src = part_of(cc, cc == from ? 1 : 0);
                                ml[u] = __ldcg(reinterpret_cast<const float2 *>(src + 2 * q));
                                v[u] = __ldcg(reinterpret_cast<const float4 *>(src + 2 * S::kQ + q * WT + e));
                            }
                            float top = M;
#pragma unroll
                            for (int u = 0; u < 8; ++u) top = fmaxf(top, ml[u].x);
                            const float base = top == -INFINITY ? 0.0f : top, keep = exp2_approx(M - base);
                            x = make_float4(x.x * keep, x.y * keep, x.z * keep, x.w * keep);
                            L *= keep;
                            M = top;
#pragma unroll
                            for (int u = 0; u < 8; ++u) {
                                const float f = c + u < c1 ? exp2_approx(ml[u].x - base) : 0.0f;
                                if (c + u < c1) add_scaled(x, f, v[u]);
                                L += c + u < c1 ? f * ml[u].y : 0.0f;
                            }
                        }
                    }
                    // (lanes of one item are neighbours: at most 32 / its lanes items per warp)
                    for (int d = 1; d < lanes; d <<= 1) {
                        const float M2 = __shfl_xor_sync(0xFFFFFFFFu, M, d), L2 = __shfl_xor_sync(0xFFFFFFFFu, L, d);
                        const float4 y = make_float4(__shfl_xor_sync(0xFFFFFFFFu, x.x, d), __shfl_xor_sync(0xFFFFFFFFu, x.y, d),
                                                     __shfl_xor_sync(0xFFFFFFFFu, x.z, d), __shfl_xor_sync(0xFFFFFFFFu, x.w, d));
                        const float top = fmaxf(M, M2), base = top == -INFINITY ? 0.0f : top;
                        const float f = exp2_approx(M - base), f2 = exp2_approx(M2 - base);
                        x = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
                        add_scaled(x, f2, y);
                        L = L * f + L2 * f2;
                        M = top;
                    }
                    if (i < items && tid % lanes == 0) store_out(p, q, e, x, M, L);
                }
            }
        }
        __syncthreads();
    };

    // ---- the share -----------------------------------------------------------------------------------------
    // Three places walk along the share: the block whose page numbers are being looked up, the one being fetched (one
    // block behind it) and the one being consumed (kStages - 1 behind that).
    constexpr int kAhead = S::kStages - 1;
    Place now = first, look = first;
    int pages_look = -1, pages_held[kAhead + 1];
    if (look.unit < share_end) pages_look = pages_of(look);
    auto fetch_next = [&](int stage) { // returns the page numbers of the block it fetched
        int pages = -1;
        if (look.unit < share_end) {
            const Place get = look;
            pages = pages_look;
            advance(look);
            if (look.unit < share_end) pages_look = pages_of(look);
            fetch(get, pages, stage);
        }
        cp_async_commit();
        return pages;
    };
    if (now.unit < share_end) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) pages_held[i] = fetch_next(i);
        begin_pair(now);
        int stage = 0;
        for (;;) {
            cp_async_wait<kAhead - 1>();
            __syncwarp();
            pages_held[kAhead] = fetch_next(stage == 0 ? kAhead : stage - 1);
            consume(now, pages_held[0], stage);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) pages_held[j] = pages_held[j + 1];
            const bool ends = now.blk + 1 == now.nblk;
            if (ends || now.unit + 1 >= share_end) end_pair(now, stage);
            stage = stage == kAhead ? 0 : stage + 1;
            advance(now);
            if (now.unit >= share_end) break;
            if (ends) begin_pair(now);
        }
        cp_async_wait<0>();
    }

    // empty slots of the batch get zeros
    for (int b = blockIdx.x; b < n_seqs; b += gridDim.x) {
        if (length(b) > 0) continue;
        if constexpr (kMode == kBehind) { // (or what the shared rows gave, for one that has no others)
            if (start_of(b) > 0) {
                for (int i = tid; i < a.heads * D / 4; i += kThreads) {
                    const int h = i / (D / 4), e = i % (D / 4) * 4;
                    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    float M = -INFINITY, L = 0.0f;
                    join_shared((int64_t)b * a.heads + h, e, x, M, L);
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
                    *reinterpret_cast<uint2 *>(a.out + (int64_t)b * a.out_stride + (int64_t)h * D + e) =
                        make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
                }
                continue;
            }
        }
        uint32_t *row = reinterpret_cast<uint32_t *>(a.out + (int64_t)b * a.out_stride);
        for (int i = tid; i < a.heads * D / 2; i += kThreads) row[i] = 0u;
    }
}

// The weights of all keys, from the scores that attend_decode_kernel kept: mass_j += sum over the kv head's queries of
// 2^(s_j - m) / l.  A warp takes an equal share of the blocks, a lane a key; the chunks of a kv head's queries are added up in their
// order, so every row gets one addition per call and sequence (atomic, as sequences may share a page).
constexpr int kWeighWarps = 4, kWeighCtas = 8; // of a CTA, per SM

template <int kBlock>
__global__ void __launch_bounds__(kWeighWarps * 32, kWeighCtas)
add_weights_kernel(const __grid_constant__ AttendArgs a, const int chunks, const int chunk_heads, const __grid_constant__ WeighArgs more)
{
    // (What is looked at before the wait, lengths and pages, the launch before this one has only read, and its CTAs let this one in
    // when what came before them was complete.)
    constexpr int kThreads = kWeighWarps * 32;
    __shared__ int upto_of[kThreads];
    __shared__ int scan[kWeighWarps];
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int Hk = a.cache.kv_heads, group = a.heads / Hk, n_seqs = a.batch.n_seqs;
    auto length = [&](int b) {
        bool over;
        return kv_length(a.batch, b, over);
    };
    auto blocks_of = [&](int len) { return (len + kBlock - 1) / kBlock; };
    // the units in front of a sequence (as attend_decode_kernel counts them), and its blocks
    const int per_thread = (n_seqs + kThreads - 1) / kThreads;
    const int b0 = min(n_seqs, tid * per_thread), b1 = min(n_seqs, b0 + per_thread);
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        const int blocks = blocks_of(length(b));
        mine += blocks > 0 ? (blocks + kPairCost) * Hk * chunks : 0;
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xFFFFFFFFu, upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    int total = 0;
#pragma unroll
    for (int w = 0; w < kWeighWarps; ++w) {
        if (w < warp) upto += scan[w];
        total += scan[w];
    }
    upto_of[tid] = upto;
    __syncthreads();
    const Plan plan(total, (int)gridDim.x * kWeighWarps);
    const int share = (int)blockIdx.x * kWeighWarps + warp;
    if (share >= plan.shares) {
        griddep_wait(); // (nor may this launch be over before the one in front of it)
        return;
    }
    int unit = plan.begin_of(share);
    const int end = plan.begin_of(share + 1);
    // the thread whose sequences the first unit lies in, then the sequence
    int before = 0;
#pragma unroll
    for (int i = 0; i < kWeighWarps; ++i) before += __popc(__ballot_sync(0xFFFFFFFFu, upto_of[i * 32 + lane] <= unit));
    int rest = unit - (before > 0 ? upto_of[before - 1] : 0), b = before * per_thread, len, nblk;
    for (;; ++b) {
        len = length(b);
        nblk = blocks_of(len);
        const int units = nblk > 0 ? (nblk + kPairCost) * Hk * chunks : 0;
        if (rest < units) break;
        rest -= units;
    }
    int pair = rest / (nblk + kPairCost), blk = rest - pair * (nblk + kPairCost);
    griddep_wait();
    griddep_launch_dependents();
    while (unit < end) {
        const int chunk = pair % chunks, head = pair / chunks;
        if (chunk != 0 || blk >= nblk) { // (the other chunks are added to the first one's keys; the end of a pair)
            const int step = min(end - unit, nblk + kPairCost - blk);
            unit += step;
            blk += step;
        } else {
            float sum[kBlock / 32] = {};
            int row[kBlock / 32]; // of the marks; -1: no key, or on a bad page
#pragma unroll
            for (int i = 0; i < kBlock / 32; ++i) {
                const int pos = blk * kBlock + i * 32 + lane, page = pos < len ? kv_page(a.cache, a.batch, b, pos) : -1;
                row[i] = page < 0 ? -1 : kv_row(a.cache, page, head, pos);
            }
            bool room = true;
            for (int c = 0; c < chunks; ++c) {
                const int u = unit + c * (nblk + kPairCost), heads_here = min(chunk_heads, group - c * chunk_heads);
                if (u >= more.max_units) {
                    room = false;
                    break;
                }
                float2 ml = make_float2(0.0f, 0.0f);
                if (lane < heads_here) ml = more.sums[(int64_t)b * a.heads + head * group + c * chunk_heads + lane];
                const float m = ml.x == -INFINITY ? 0.0f : ml.x, inv = ml.y == 0.0f ? 0.0f : 1.0f / ml.y;
                const float *from = more.scores + (int64_t)u * kBlock * chunk_heads;
                // (what stands behind the last key goes into sums that nobody stores)
                if (chunk_heads % 4 == 0 && heads_here == chunk_heads) {
                    for (int q = 0; q < heads_here; q += 4) {
                        float4 s[kBlock / 32];
#pragma unroll
                        for (int i = 0; i < kBlock / 32; ++i) s[i] = *reinterpret_cast<const float4 *>(from + (i * 32 + lane) * chunk_heads + q);
                        float mq[4], iq[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            mq[u] = __shfl_sync(0xFFFFFFFFu, m, q + u);
                            iq[u] = __shfl_sync(0xFFFFFFFFu, inv, q + u);
                        }
#pragma unroll
                        for (int i = 0; i < kBlock / 32; ++i) {
                            sum[i] += exp2_approx(s[i].x - mq[0]) * iq[0];
                            sum[i] += exp2_approx(s[i].y - mq[1]) * iq[1];
                            sum[i] += exp2_approx(s[i].z - mq[2]) * iq[2];
                            sum[i] += exp2_approx(s[i].w - mq[3]) * iq[3];
                        }
                    }
                } else {
                    for (int q = 0; q < heads_here; ++q) {
                        const float mq = __shfl_sync(0xFFFFFFFFu, m, q), iq = __shfl_sync(0xFFFFFFFFu, inv, q);
#pragma unroll
                        for (int i = 0; i < kBlock / 32; ++i) sum[i] += exp2_approx(from[(i * 32 + lane) * chunk_heads + q] - mq) * iq;
                    }
                }
            }
            if (!room && lane == 0) kv_report(a.cache);
#pragma unroll
            for (int i = 0; i < kBlock / 32; ++i)
                if (room && row[i] >= 0) atomicAdd(more.marks.mass + row[i], sum[i]);
            ++unit;
            ++blk;
        }
        if (blk >= nblk + kPairCost) {
            blk = 0;
            if (++pair == Hk * chunks && unit < end) {
                pair = 0;
                do len = length(++b);
                while (len == 0);
                nblk = blocks_of(len);
            }
        }
    }
}

template <bool kInt8, int WT, int NT, int kMode>
cudaError_t launch(const AttendArgs &a, int chunks, int chunk_heads, const More<kMode> &more, cudaStream_t stream)
{
    using S = Shape<kInt8, WT, NT>;
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(attend_decode_kernel<kInt8, WT, NT, kMode>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    e = launch_dependent(attend_decode_kernel<kInt8, WT, NT, kMode>, std::min(S::kCtas * sm_count(), kDecodeMaxCtas), kWarps * 32, S::kSmem, stream,
                         a, chunks, chunk_heads, more);
    if constexpr (kMode == kWeigh) {
        if (e == cudaSuccess)
            e = launch_dependent(add_weights_kernel<kWarps * S::kKeys>, kWeighCtas * sm_count(), kWeighWarps * 32, 0, stream, a, chunks, chunk_heads,
                                 static_cast<const WeighArgs &>(more));
    }
    return e;
}

// Query heads of a kv head are taken up to 16 at a time (two tiles of 8 columns; a single tile where at most 8 are left).
void decode_chunks(int group, int &chunks, int &chunk_heads)
{
    chunks = (group + 15) / 16;
    chunk_heads = (group + chunks - 1) / chunks;
}

template <int kMode>
cudaError_t launch_mode(const AttendArgs &a, const More<kMode> &more, cudaStream_t stream)
{
    int chunks, chunk_heads;
    decode_chunks(a.heads / a.cache.kv_heads, chunks, chunk_heads);
    const bool narrow = a.cache.width <= 64, one = chunk_heads <= 8;
    if (a.cache.k_scale) {
        if (narrow) return one ? launch<true, 64, 1, kMode>(a, chunks, chunk_heads, more, stream) : launch<true, 64, 2, kMode>(a, chunks, chunk_heads, more, stream);
        return one ? launch<true, 128, 1, kMode>(a, chunks, chunk_heads, more, stream) : launch<true, 128, 2, kMode>(a, chunks, chunk_heads, more, stream);
    }
    if (narrow) return one ? launch<false, 64, 1, kMode>(a, chunks, chunk_heads, more, stream) : launch<false, 64, 2, kMode>(a, chunks, chunk_heads, more, stream);
    return one ? launch<false, 128, 1, kMode>(a, chunks, chunk_heads, more, stream) : launch<false, 128, 2, kMode>(a, chunks, chunk_heads, more, stream);
}

// Keys of a block: a stage of each warp.
int block_keys(bool int8, int head_dim) { return kWarps * kStageBytes / 2 / ((kv_row_width(head_dim) <= 64 ? 64 : 128) * (int8 ? 1 : 2)); }

// Of the workspace of the weighing form: behind the decode kernel's own, the softmaxes' maxima and sums, then the scores.
size_t weigh_fixed_bytes(int heads, int kv_heads, int head_dim, int64_t n_seqs)
{
    return attend_decode_workspace_bytes(heads, kv_heads, head_dim) + align_up((size_t)n_seqs * heads * sizeof(float2), 256);
}

} // namespace

size_t attend_decode_workspace_bytes(int heads, int kv_heads, int head_dim)
{
    int chunks, chunk_heads;
    decode_chunks(heads / kv_heads, chunks, chunk_heads);
    const size_t q = chunk_heads <= 8 ? 8 : 16, width = kv_row_width(head_dim) <= 64 ? 64 : 128;
    return align_up(decode_counter_bytes() + (size_t)kDecodeMaxCtas * kMaxSplits * q * (width + 2) * 4, 256);
}

size_t attend_weigh_workspace_bytes(int heads, int kv_heads, int head_dim, bool int8, int64_t n_seqs, int64_t max_keys)
{
    int chunks, chunk_heads;
    decode_chunks(heads / kv_heads, chunks, chunk_heads);
    // every sequence has at most one block that is not full, and a unit behind its last one
    const int64_t keys = block_keys(int8, head_dim), units = (max_keys / keys + n_seqs * (1 + kPairCost)) * kv_heads * chunks;
    return align_up(weigh_fixed_bytes(heads, kv_heads, head_dim, n_seqs) + (size_t)units * keys * chunk_heads * 4, 256);
}

bool attend_decode_fits(const AttendArgs &a)
{
    int chunks, chunk_heads;
    decode_chunks(a.heads / a.cache.kv_heads, chunks, chunk_heads);
    const int64_t units = (a.batch.capacity + 63) / 64 + kPairCost; // (blocks are 64 keys or more)
    return units * a.cache.kv_heads * chunks <= 0x7FFFFFFF / std::max(a.batch.n_seqs, 1);
}

cudaError_t launch_attend_decode(const AttendArgs &a, cudaStream_t stream) { return launch_mode<kPlain>(a, More<kPlain>{}, stream); }

cudaError_t launch_attend_decode_weigh(const AttendArgs &a, const KvMarks &marks, size_t workspace_bytes, cudaStream_t stream)
{
    int chunks, chunk_heads;
    decode_chunks(a.heads / a.cache.kv_heads, chunks, chunk_heads);
    const bool int8 = a.cache.k_scale != nullptr;
    const size_t own = attend_decode_workspace_bytes(a.heads, a.cache.kv_heads, a.cache.head_dim);
    const size_t fixed = weigh_fixed_bytes(a.heads, a.cache.kv_heads, a.cache.head_dim, a.batch.n_seqs);
    char *ws = reinterpret_cast<char *>(a.workspace);
    More<kWeigh> more;
    more.sums = reinterpret_cast<float2 *>(ws + own);
    more.scores = reinterpret_cast<float *>(ws + fixed);
    more.max_units = (int64_t)((workspace_bytes - fixed) / ((size_t)block_keys(int8, a.cache.head_dim) * chunk_heads * 4));
    more.marks = marks;
    return launch_mode<kWeigh>(a, more, stream);
}

cudaError_t launch_attend_decode_behind(const AttendArgs &a, const SharedArgs &shared, cudaStream_t stream)
{
    More<kBehind> more;
    static_cast<SharedArgs &>(more) = shared;
    return launch_mode<kBehind>(a, more, stream);
}

} // namespace bitlinear
