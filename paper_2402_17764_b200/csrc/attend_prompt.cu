// Causal attention of the new tokens of prompts and prompt chunks over the paged cache, on the tcgen05 tensor cores.
//
//   out = P V / sum P,  P_ij = 2^(s_ij - m_i),  S = scale log2(e) Q K^T,  in one pass over the keys with a running reference m_i
//
// Rows.  The query heads that share a kv head are taken together: row R of a (sequence, kv head) is token R / group, head
// R % group of the group, so one tile of keys serves them all and a chunk of few tokens still fills a tile.  A CTA owns
// 256 rows as two tiles of 128 (the MMA's M), and walks the keys they see in blocks of 128.
//
// Roles (16 warps):
//   warps 0-3, 4-7 : the softmax of tile 0 and of tile 1, one row per thread: scores from tensor memory, maximum, 2^x, the
//                    weights as bf16 back into tensor memory, over the scores they came from;
//   warps 8, 9     : issue the MMAs of tile 0 and tile 1: S = Q K^T (both operands in shared memory) and O += P V (P in
//                    tensor memory, V as it lies in the cache: keys are its rows, so it is the MN-major operand);
//   warps 10-13    : bf16 producers: TMA of one page's rows and 64 elements of the head per copy (128-byte swizzle); an
//                    issued copy costs its thread 100 to 150 cycles, hence four issuing warps;
//   int8 cache     : warps 10 and 11 copy the codes and scales of keys and of values into a ring of their own, warps 12-15
//                    turn them into bf16 (exactly) in the layout of the MMA.
// Tensor memory: 2 x 128 columns of scores, 2 x 128 of output.  The softmax works in steps of 64 keys, and a tile's two halves
// of the score columns take the steps in turn: while step k is worked on, P V of step k - 1 and the scores of step k + 1 run in
// the other half, so the softmax does not wait for the tensor cores between steps.  The MMAs that one thread issues execute in
// order, so the scores of step k + 2 may overwrite the weights that the P V of step k in front of them reads.  (With steps
// of 128 keys the scores of the next step could only start after P V of this one: softmax and MMAs of a tile took turns,
// 3900 cycles per block of 128 keys.)
//
// Rescaling.  The output stands in tensor memory, and moving it for every new maximum would cost as much as the softmax.  The
// reference m_i is therefore raised only when a score exceeds it by more than 8 (a factor 256, which fp32 sums and bf16 weights
// carry without loss); the result does not depend on the reference.  (A known refinement of the softmax in one pass, whose running
// maximum and sum are Milakov and Gimelshein's, "Online normalizer calculation for softmax", 2018.)
//
// Rounding of the reference.  m is a rounded product (score times scale), and one fma takes x scale - m from the exact one: all weights
// of a row carry the factor 2^(what m's rounding cut off), which cancels out as long as it stays inside fp32's range.  From |m| = 2^31
// on it need not (half a unit of m is 128), so beyond 2^24 a row's products are rounded first, as m was, and the largest becomes
// exactly m.  int8: in place, in front of the exponentials.  bf16: the tile is done again row by row; the branch that the int8
// form has costs this one 8 % (8192 tokens, 32 heads: 589 -> 642 us), and no score of a trained model comes near.
//
// What bounds it (heads of 128).  64 keys for 256 rows cost 16384 exponentials at 16 per cycle and SM, 1024 cycles, and 1280 cycles of
// the tensor pipe: P V 512, and Q K^T 768 instead of 512, because an MMA of 64 columns reads 4 KB of queries and 2 KB of keys from
// shared memory, at 128 bytes per cycle, for 32 cycles of arithmetic.  They take about 2040: neither unit is busy all the time
// (tensor pipe 67 %, exponentials 53 %), since a softmax warp loads its scores, finds their maximum and only then begins its
// exponentials.  8192 tokens, 32 heads: 586-594 us = 0.93 PFLOP/s, where the board's power limit holds the clock near 1.55 GHz
// (the same launch takes about 930 000 cycles at any clock).  int8: the converters' shared-memory traffic and arithmetic come on
// top, 57 % of the issue slots (chunks of 86 to 512 tokens behind 3300 to 12000, 64/8 heads: 393-405 us = 0.73 PFLOP/s).
// Prompts of few hundred tokens: half the time is each tile's beginning and end (pages, queries, first scores; results).
// Registers: the bf16 form spills 4 bytes (12 loaded; for shared rows 12, 28 loaded), the int8 form none.
//
// The form for rows that sequences share (single tokens of many sequences over the same keys) has the queries of a group's sequences
// as rows, no masks, and leaves its parts, in fp32, to be joined by the decode kernel behind it, a sequence's rows at a time: joined by
// the last CTA of a tile, as above, nine parts of 133 KB took 10 us.  Its weights enter as two bf16 parts (value and remainder, 16 bits
// together), as the decode kernel's do, so that a result is as exact with rows shared as without; the second parts stand behind the first
// ones, in the other half of the scores' columns, and meet the same values (64 sequences over 16384 shared rows, 64/8 heads: 77 us with
// one part and an error of 0.0023 against 64 bits, 82-83 with two and 0.0017, that of results rounded to bf16).  Of these 82 about 54
// are the tiles, 28 steps of some 2300 cycles and 18000 for the beginning (search, queries, first scores) and the end (parts).
#include <cuda.h>

#include <algorithm>
#include <type_traits>

#include "internal.cuh"
#include "kv.cuh"
#include "ptx.cuh"
#include "tma_host.cuh"

namespace bitlinear {
namespace {

using namespace ptx;

constexpr int kTile = 128;               // rows of a query tile, keys of a block
constexpr int kStep = 64;                // keys of a softmax step
constexpr int kRows = 2 * kTile;         // rows of a CTA
static_assert(kRows == kPromptRows, "the parts' layout");
constexpr int kHalfBytes = kTile * 128;  // 128 rows of 64 bf16 elements, 128-byte swizzle
constexpr int kTileBytes16 = 2 * kHalfBytes;
constexpr int kMaxStages = 5;
constexpr int kInfo = 8;                 // ring of per-block notes (at most three blocks are in flight)
constexpr int kMmaWarp = 8;        // and the next one
constexpr int kFirstProducer = 10, kProducers = 4;
constexpr int kFirstConverter = 12, kConverters = 4; // int8
constexpr int kThreads = 16 * 32;
constexpr uint32_t kTmemColumns = 512;
constexpr float kRaise = 8.0f;
constexpr float kFar = 16777216.0f; // 2^24: references up to here are rounded by at most half a unit (see the header on rounding)
constexpr int kMaxParts = 16; // of a tile's keys
constexpr int kMaxSharedParts = 32;
// kv heads whose tiles follow each other: the keys and values of eight heads stay in the L2 while their tiles are worked on
// (8192 tokens, 32 heads: 134 MB in all, 590 us with all heads at a time, 576 with eight; at 128k tokens eight heads are
// 0.5 GB and do not stay there either, and of short prompts all heads would)
constexpr int kHeadGroup = 8;
template <bool kInt8>
struct Shared {
    static constexpr int kStages = kInt8 ? 3 : 5; // blocks of keys or values in shared memory
    static constexpr int kRaw = kInt8 ? 3 : 0;    // blocks of int8 keys or values in front of their conversion
    static constexpr int kRawBytes = kTile * 128 + kTile * 4; // codes, then scales
    static constexpr int kScaled = 4;             // blocks whose scales are kept
    float scales[kInt8 ? kScaled : 1][2][kInt8 ? kTile : 4]; // of the keys and of the values of a block
    uint64_t q_full[2], kv_full[kMaxStages], kv_empty[kMaxStages], s_full[2][2], p_ready[2][2], o_done[2], o_last[2], raw_full[3], raw_empty[3];
    uint32_t tmem_base;
    int abort_flag;
    int poisoned[2];
    int is_last;
    int found_b;
    int64_t found_local, scan[kThreads / 32];
    uint32_t bad_groups[kInfo]; // 16-key groups of a block whose page does not exist
    static constexpr int bytes();
};
template <bool kInt8>
constexpr int Shared<kInt8>::bytes()
{
    return 1024 + (2 + kStages) * kTileBytes16 + kRaw * kRawBytes + (int)sizeof(Shared<kInt8>);
}
static_assert(Shared<false>::bytes() <= 232448 && Shared<true>::bytes() <= 232448, "shared memory of an SM");

// Registers: 512 threads are launched with 128 each; the softmax warps (a row of 128 scores each) take 184, the others keep 72.
constexpr int kLaunchRegs = 128, kSoftmaxRegs = 184, kOtherRegs = 72;
static_assert(kSoftmaxRegs * 256 + kOtherRegs * 256 <= kLaunchRegs * kThreads, "setmaxnreg hands on what the launch was given");
template <int N>
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

struct PromptArgs {
    CUtensorMap k_map, v_map;
    AttendArgs a;
    int splits;       // CTAs that may share the keys of a tile of rows
    int slots;        // > 0: CTAs among which the tiles are to be split, once their number is known
    WaitHooks hooks;
};

// The shared form: the "sequences" of a.batch are groups of sequences, a group's new tokens are one token of each of its
// sequences (token row = sequence), and all of them see all rows that the group shares (what comes out for a sequence that is
// shorter is not used).  References, sums and outputs stay fp32 and are handed on.
template <bool kShared>
struct PromptMore {};
template <>
struct PromptMore<true> : SharedArgs {};

__device__ __forceinline__ float exp2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// The largest of three, or NaN if one of them is.
__device__ __forceinline__ float max3(float x, float y, float z)
{
    float m;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
    return m;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
// Copies kBytes to shared memory, or fills them with zeros (nothing is read then).
template <int kBytes>
__device__ __forceinline__ void cp_async(uint32_t dst, const void *src, bool real)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(kBytes), "r"(real ? kBytes : 0) : "memory");
}
__device__ __forceinline__ void named_barrier(int id, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }

// Two signed bytes of w as two bf16 numbers, exactly (attend_decode.cu has the same step on its operands).
template <uint32_t kSelect>
__device__ __forceinline__ uint32_t code_pair(uint32_t w)
{
    const uint32_t t = __byte_perm(w, 0x43434343u, kSelect);
    const uint32_t x = t & 0xFF7FFF7Fu, y = t & 0xFF80FF80u;
    const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&d);
}

// A CTA's rows: 256 of the rows of (sequence b, kv head), and the blocks of keys it walks.
struct Work {
    int b, head;          // sequence and kv head
    int first_token;      // token row of the sequence's first new token
    int row0, rows;       // first row of the tile; rows of the sequence in all
    int len;              // keys of the sequence
    int offset;           // position of the first new token (may be negative)
    int group;
    // keys that row r of the sequence sees
    __device__ __forceinline__ int sees(int r) const
    {
        const int n = offset + r / group + 1;
        return n < 0 ? 0 : (n > len ? len : n);
    }
};

// (Not inlined: the registers of the main loop are allotted without it, 584 -> 576 us for 8192 tokens, 32 heads.)
// One row by plain arithmetic, one warp: for tiles in which a non-finite value stands behind keys that some of the rows do not
// see (0 x NaN would reach them through the MMA), or in which a reference lies beyond kFar.
// to: the shared form's place for the result, in fp32.
struct RowResult {
    float2 *ml;
    float *o;
    int step; // between four elements and the next
};
template <bool kShared>
__device__ __noinline__ void attend_row(const AttendArgs &a, const Work &w, int r, int lane, int begin, int end, const RowResult &to)
{
    const int D = a.cache.head_dim, t = w.first_token + r / w.group, h = w.head * w.group + r % w.group;
    const bool mine = 4 * lane < D;
    auto load = [&](const __nv_bfloat16 *p) {
        if (!mine) return make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        const uint2 u = *reinterpret_cast<const uint2 *>(p + 4 * lane);
        return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xFFFF0000u), __uint_as_float(u.y << 16),
                           __uint_as_float(u.y & 0xFFFF0000u));
    };
    const float4 q = load(a.q + (int64_t)t * a.q_stride + h * D);
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    constexpr int kAtATime = 4; // keys (a page holds 16 or more)
    for (int j = begin; j < end; j += kAtATime) {
        const int page = kv_page(a.cache, a.batch, w.b, j);
        if (page < 0) continue;
        const int64_t row = (int64_t)kv_row(a.cache, page, w.head, j) * a.cache.width;
        const __nv_bfloat16 *kp = reinterpret_cast<const __nv_bfloat16 *>(a.cache.k) + row, *vp = reinterpret_cast<const __nv_bfloat16 *>(a.cache.v) + row;
        float4 k[kAtATime], v[kAtATime];
        float s[kAtATime];
#pragma unroll
        for (int i = 0; i < kAtATime; ++i) {
            const int at = j + i < end ? i * a.cache.width : 0;
            k[i] = load(kp + at);
            v[i] = load(vp + at);
        }
#pragma unroll
        for (int i = 0; i < kAtATime; ++i) {
            s[i] = q.x * k[i].x + q.y * k[i].y + q.z * k[i].z + q.w * k[i].w;
#pragma unroll
            for (int d = 16; d; d >>= 1) s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], d);
            s[i] = j + i < end ? __fmul_rn(s[i], a.scale) : -INFINITY;
        }
        float mn = m;
#pragma unroll
        for (int i = 0; i < kAtATime; ++i) mn = fmaxf(mn, s[i]);
        const float base = mn == -INFINITY ? 0.0f : mn, keep = exp2_approx(m - base);
        l *= keep;
        o = make_float4(o.x * keep, o.y * keep, o.z * keep, o.w * keep);
#pragma unroll
        for (int i = 0; i < kAtATime; ++i) {
            const float p = exp2_approx(s[i] - base);
            l += p;
            if (j + i < end) o = make_float4(o.x + p * v[i].x, o.y + p * v[i].y, o.z + p * v[i].z, o.w + p * v[i].w);
        }
        m = mn;
    }
    if constexpr (kShared) {
        if (lane == 0) *to.ml = make_float2(m, l);
        if (4 * lane < a.cache.width) *reinterpret_cast<float4 *>(to.o + lane * to.step) = o;
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (mine)
        *reinterpret_cast<uint2 *>(a.out + (int64_t)t * a.out_stride + h * D + 4 * lane) =
            make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

template <bool kInt8, bool kShared>
__global__ void __launch_bounds__(kThreads, 1) attend_prompt_kernel(const __grid_constant__ PromptArgs args, const __grid_constant__ PromptMore<kShared> more)
{
    if (kShared && !kInt8 && threadIdx.x == 0) {
        prefetch_tensormap(&args.k_map);
        prefetch_tensormap(&args.v_map);
    }
    griddep_wait(); // everything below is read from memory that the launch before this one may have written
    const AttendArgs &a = args.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    constexpr int kStages = Shared<kInt8>::kStages, kScaled = Shared<kInt8>::kScaled;
    constexpr int kRaw = Shared<kInt8>::kRaw, kRawBytes = Shared<kInt8>::kRawBytes;
    uint8_t *raw_ring = smem + (2 + kStages) * kTileBytes16;
    Shared<kInt8> &sh = *reinterpret_cast<Shared<kInt8> *>(raw_ring + kRaw * kRawBytes);
    volatile int *abort_flag = &sh.abort_flag;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int D = a.cache.head_dim, W = a.cache.width, group = a.heads / a.cache.kv_heads, n_seqs = a.batch.n_seqs;
    const uint32_t limit = args.hooks.limit_us;

    auto set_up = [&] {
        if (tid == 0) {
            for (int t = 0; t < 2; ++t) {
                mbar_init(smem_u32(&sh.q_full[t]), 4);
                for (int h = 0; h < 2; ++h) {
                    mbar_init(smem_u32(&sh.s_full[t][h]), 1);
                    mbar_init(smem_u32(&sh.p_ready[t][h]), 4);
                }
                mbar_init(smem_u32(&sh.o_done[t]), 1);
                mbar_init(smem_u32(&sh.o_last[t]), 1);
                sh.poisoned[t] = 0;
            }
            for (int s = 0; s < kStages; ++s) {
                mbar_init(smem_u32(&sh.kv_full[s]), kInt8 ? kConverters : 1);
                mbar_init(smem_u32(&sh.kv_empty[s]), 2);
            }
            for (int s = 0; s < kRaw; ++s) {
                mbar_init(smem_u32(&sh.raw_full[s]), 1);
                mbar_init(smem_u32(&sh.raw_empty[s]), kConverters);
            }
            sh.abort_flag = 0;
            fence_mbar_init();
        }
        if (warp == kMmaWarp) {
            tmem_alloc(smem_u32(&sh.tmem_base), kTmemColumns);
            tmem_relinquish();
        }
    };
    // The shared form: what is set up does not wait for the search for the rows, and a CTA that finds none gives it back.
    auto leave = [&] {
        tc_fence_before_sync();
        __syncthreads();
        tc_fence_after_sync();
        if (warp == kMmaWarp) tmem_dealloc(sh.tmem_base, kTmemColumns);
    };
    bool none = false; // (nothing is shared)
    auto write_starts = [&] {
        if constexpr (kShared)
            for (int b = blockIdx.x * kThreads + tid; b < a.T; b += gridDim.x * kThreads) more.starts[b] = none ? 0 : shared_start(a.cache, a.batch, more.seqs, b);
    };
    if (kShared) set_up();

    // ---- which rows: tiles are counted sequence by sequence, the longest first, and within a sequence, for every group of kv
    // heads, the last rows (which see most) first, so that the CTAs that start last have the least to do (four chunks of 86
    // to 512 tokens behind 3300 to 12000: 459 -> 383 us) ----
    int splits = args.splits;
    {
        auto tiles_of = [&](int b) -> int64_t {
            const int64_t n = (int64_t)a.batch.cu_tokens[b + 1] - a.batch.cu_tokens[b];
            if constexpr (kShared) {
                bool over;
                if (group_shares(a.cache, a.batch, b, over) == 0) return 0;
            }
            return n <= 0 || n > a.T ? 0 : (n * group + kRows - 1) / kRows * a.cache.kv_heads;
        };

        // (rows that the caller did not hand over: the sequence has none then, here or where its first row is looked at below)
        auto rows_missing = [&](int b) { return a.batch.cu_tokens[b] < 0 || a.batch.cu_tokens[b] > a.batch.cu_tokens[b + 1] || a.batch.cu_tokens[b + 1] > a.T; };
        const int per_thread = (n_seqs + kThreads - 1) / kThreads;
        const int b0 = min(n_seqs, tid * per_thread), b1 = min(n_seqs, b0 + per_thread);
        int64_t mine = 0;
        if constexpr (kShared) { // with bounds that fall, or lie outside the batch, nothing is shared at all
            bool bad = false;
            int64_t rows_again = 0; // what the groups' sequences would read where nothing is shared
            for (int b = b0; b < b1; ++b) {
                bool over;
                bad = bad || group_bounds_bad(a.batch, b, a.T);
                mine += tiles_of(b);
                rows_again += (int64_t)(a.batch.cu_tokens[b + 1] - a.batch.cu_tokens[b]) * group_shares(a.cache, a.batch, b, over);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) rows_again += __shfl_xor_sync(0xFFFFFFFFu, rows_again, d);
            if (lane == 0) sh.scan[warp] = rows_again;
            bad = __syncthreads_or(bad);
            rows_again = 0;
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) rows_again += sh.scan[w];
            __syncthreads(); // (the sums are written to below)
            none = bad || rows_again < more.share_from;
            if (none) {
                if (bad && blockIdx.x == 0 && tid == 0) kv_report(a.cache);
                write_starts();
                leave();
                return;
            }
        } else {
            for (int b = b0; b < b1; ++b) {
                mine += tiles_of(b);
                if (blockIdx.x == 0 && rows_missing(b)) kv_report(a.cache);
            }
        }
        int first_b = b0;
        if (!kShared && per_thread == 1) { // (longer lists of sequences are taken as they are)
            int64_t *tiles_by_rank = reinterpret_cast<int64_t *>(smem);
            int *lens = reinterpret_cast<int *>(tiles_by_rank + kThreads), *b_by_rank = lens + kThreads;
            const int len = mine > 0 ? a.batch.kv_lens[b0] : 0;
            lens[tid] = len;
            __syncthreads();
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n_seqs; ++j) rank += lens[j] > len || (lens[j] == len && j < tid);
            if (tid < n_seqs) {
                tiles_by_rank[rank] = mine;
                b_by_rank[rank] = tid;
            }
            __syncthreads();
            if (tid < n_seqs) {
                mine = tiles_by_rank[tid];
                first_b = b_by_rank[tid];
            }
            fence_proxy_async_smem(); // (the same bytes are copied to by the async proxy later)
        }
        int64_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t y = __shfl_up_sync(0xFFFFFFFFu, upto, d);
            if (lane >= d) upto += y;
        }
        if (lane == 31) sh.scan[warp] = upto;
        if (tid == 0) sh.found_b = -1;
        __syncthreads();
        for (int w = 0; w < warp; ++w) upto += sh.scan[w];
        if (args.slots > 0) {
            int tiles = 0; // (at most one per sequence and kv head, and what the host counted)
#pragma unroll
            for (int w = 0; w < kThreads / 32; ++w) tiles += (int)sh.scan[w];
            splits = min(kShared ? kMaxSharedParts : kMaxParts, max(1, args.slots / max(tiles, 1)));
        }
        const int64_t x = (int)blockIdx.x / splits;
        if (x >= upto - mine && x < upto) {
            int64_t rest = x - (upto - mine);
            int b = first_b;
            for (int i = 1; i < per_thread; ++i) {
                const int64_t n = tiles_of(b);
                if (rest < n) break;
                rest -= n;
                ++b;
            }
            sh.found_b = b;
            sh.found_local = rest;
        }
        __syncthreads();
    }
    if (sh.found_b < 0) {
        if (kShared) {
            write_starts();
            leave();
        }
        return;
    }
    const int split = blockIdx.x % splits;
    Work w;
    w.b = sh.found_b;
    w.group = group;
    w.first_token = a.batch.cu_tokens[w.b];
    const int n_tokens = a.batch.cu_tokens[w.b + 1] - w.first_token;
    if (!kShared && (w.first_token < 0 || (int64_t)w.first_token + n_tokens > a.T)) return; // (reported above)
    w.rows = n_tokens * group;
    {
        const int tiles = (w.rows + kRows - 1) / kRows;
        const int per_group = min(kHeadGroup, a.cache.kv_heads), in_group = tiles * per_group;
        const int which = (int)(sh.found_local / in_group), rest = (int)(sh.found_local - (int64_t)which * in_group);
        const int heads_here = min(per_group, a.cache.kv_heads - which * per_group);
        w.head = which * per_group + rest % heads_here;
        w.row0 = (tiles - 1 - rest / heads_here) * kRows;
    }
    bool over;
    w.len = kShared ? group_shares(a.cache, a.batch, w.b, over) : kv_length(a.batch, w.b, over);
    if (over && tid == 0) kv_report(a.cache);
    w.offset = kShared ? w.len : a.batch.kv_lens[w.b] - n_tokens; // (shared form: every row sees all keys)

    // blocks of keys of the two tiles, and this CTA's part of them (a part is at least four blocks, so that joining the parts
    // does not cost more than they save)
    const int most = (w.sees(min(w.row0 + kRows, w.rows) - 1) + kTile - 1) / kTile;
    // (The parts of the shared form are joined by the kernel behind it, a sequence's rows at a time: two blocks are enough.)
    const int parts = max(1, min(splits, most / (kShared ? 2 : 4)));
    if (split >= parts) {
        if (kShared) {
            write_starts();
            leave();
        }
        return;
    }
    using Product = std::conditional_t<kShared, int, int64_t>; // (blocks are below 2^23, the shared form's parts at most 32)
    const int from = (int)((Product)most * split / parts), to_block = (int)((Product)most * (split + 1) / parts);
    int n_steps[2];
    for (int t = 0; t < 2; ++t) {
        const int first = w.row0 + t * kTile, last = min(first + kTile, w.rows) - 1;
        n_steps[t] = first < w.rows ? max(0, min((w.sees(last) + kStep - 1) / kStep, 2 * to_block) - 2 * from) : 0;
    }
    const int total = (max(n_steps[0], n_steps[1]) + 1) / 2; // blocks

    if (!kShared) set_up();
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    const uint32_t q_addr = base, ring = base + 2 * kTileBytes16;

    if (warp >= kMmaWarp) {
        give_registers<kOtherRegs>();
        if (kInt8 && warp >= kFirstConverter) {
            // ---- int8: codes to bf16, blocks in the order K 0, V 0, K 1, V 1, ...; each warp a quarter of the rows ------------
            const int pieces = W / 16, c = lane % 8, r0 = lane / 8; // this lane: piece c (16 codes) of every fourth row
            for (int i = 0; i < 2 * total; ++i) {
                const int s = i % kStages, round = i / kStages, rs = kInt8 ? i % 3 : 0, j = from + i / 2;
                if (round > 0 && !mbar_wait_bounded(smem_u32(&sh.kv_empty[s]), (round - 1) & 1, abort_flag, limit, 0)) break;
                if (!mbar_wait_bounded(smem_u32(&sh.raw_full[rs]), (i / 3) & 1, abort_flag, limit, 0)) break;
                const uint8_t *codes = raw_ring + rs * kRawBytes;
                uint8_t *out = smem + (2 + s) * kTileBytes16 + (c / 4) * kHalfBytes;
                const int p = (c % 4) * 2;
                {
                    const int r = (warp - kFirstConverter) * 32 + lane; // (scales of keys that do not exist may be anything)
                    const float f = reinterpret_cast<const float *>(codes + kTile * 128)[r];
                    sh.scales[(i / 2) % kScaled][i & 1][r] = j * kTile + r < w.len ? f : 0.0f;
                }
                if (c < pieces) {
#pragma unroll 4
                    for (int u = 0; u < 8; ++u) {
                        const int r = (warp - kFirstConverter) * 32 + u * 4 + r0;
                        const uint4 x = *reinterpret_cast<const uint4 *>(codes + r * W + c * 16);
                        *reinterpret_cast<uint4 *>(out + r * 128 + ((p ^ (r & 7)) << 4)) =
                            make_uint4(code_pair<0x4140>(x.x), code_pair<0x4342>(x.x), code_pair<0x4140>(x.y), code_pair<0x4342>(x.y));
                        *reinterpret_cast<uint4 *>(out + r * 128 + (((p + 1) ^ (r & 7)) << 4)) =
                            make_uint4(code_pair<0x4140>(x.z), code_pair<0x4342>(x.z), code_pair<0x4140>(x.w), code_pair<0x4342>(x.w));
                    }
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(smem_u32(&sh.kv_full[s]));
                    mbar_arrive(smem_u32(&sh.raw_empty[rs]));
                }
            }
        } else if (warp >= kFirstProducer) {
            // ---- producers: bf16: every fourth block of K 0, V 0, K 1, V 1, ... each; int8: one the keys, one the values --------
            constexpr int kWarps = kInt8 ? 2 : kProducers, kRing = kInt8 ? 3 : kStages;
            const int halves = W > 64 ? 2 : 1;
            if (warp - kFirstProducer < kWarps)
                for (int i = warp - kFirstProducer; i < 2 * total; i += kWarps) {
                    const int s = i % kRing, round = i / kRing, j = from + i / 2;
                    const bool values = i & 1;
                    uint64_t *const full_bar = kInt8 ? &sh.raw_full[s % 3] : &sh.kv_full[s], *const empty_bar = kInt8 ? &sh.raw_empty[s % 3] : &sh.kv_empty[s];
                    // the rows of the block's eight 16-key groups, one per lane
                    int row = -1;
                    bool bad = false;
                    if (lane < 8) {
                        const int pos = j * kTile + lane * 16;
                        if (pos < w.len) {
                            const int page = kv_page(a.cache, a.batch, w.b, pos);
                            bad = page < 0;
                            if (!bad) row = kv_row(a.cache, page, w.head, pos);
                        }
                    }
                    const uint32_t bad_groups = __ballot_sync(0xFFFFFFFFu, bad);
                    if (bad_groups != 0u && lane == 0) kv_report(a.cache);
                    if (round > 0 && !mbar_wait_bounded(smem_u32(empty_bar), (round - 1) & 1, abort_flag, limit)) break;
                    if (!values && lane == 0) sh.bad_groups[(i / 2) % kInfo] = bad_groups;
                    const uint32_t full = smem_u32(full_bar);
                    const int per_copy = min(kTile, 1 << a.cache.page_shift); // rows of a copy
                    // (test device: the first CTA leaves out its first arrival and the copies that it announces)
                    const bool skip = args.hooks.skip_arrive && blockIdx.x == 0 && i == 0;
                    const uint32_t have = __ballot_sync(0xFFFFFFFFu, row >= 0);
                    uint32_t bytes = (uint32_t)(halves * kHalfBytes);
                    if (kInt8) {
                        bytes = 0;
                        for (int g = 0; g < kTile / 16; g += per_copy / 16)
                            if ((have >> g) & 1u) bytes += (uint32_t)(per_copy * (W + 4));
                    }
                    if (lane == 0 && !skip) mbar_arrive_expect_tx(full, bytes);
                    __syncwarp();
                    for (int g = 0; g < kTile / 16; g += per_copy / 16) {
                        const int r = __shfl_sync(0xFFFFFFFFu, row, g);
                        if (lane != 0 || skip) continue;
                        if (!kInt8) {
                            const int absent = (a.cache.n_pages * a.cache.kv_heads) << a.cache.page_shift; // a row behind the cache: reads zeros
                            for (int h = 0; h < halves; ++h)
                                tma_load_2d(ring + s * kTileBytes16 + h * kHalfBytes + g * 16 * 128, values ? &args.v_map : &args.k_map, h * 64,
                                            r < 0 ? absent : r, full);
                        } else if (r >= 0) {
                            const uint32_t dst = smem_u32(raw_ring) + s * kRawBytes;
                            bulk_copy_g2s(dst + g * 16 * W, reinterpret_cast<const int8_t *>(values ? a.cache.v : a.cache.k) + (int64_t)r * W,
                                          (uint32_t)(per_copy * W), full);
                            bulk_copy_g2s(dst + kTile * 128 + g * 64, (values ? a.cache.v_scale : a.cache.k_scale) + r, (uint32_t)(per_copy * 4), full);
                        }
                    }
                }
        } else {
            // ---- MMAs of tile t ----------------------------------------------------------------------------------
            const int t = warp - kMmaWarp, n = n_steps[t], k_steps = W / 16;
            const uint32_t idesc_s = idesc_bf16(kTile, kStep, 0), idesc_o = idesc_bf16(kTile, W, 1);
            const uint32_t s_tmem = tmem + t * kTile, o_tmem = tmem + kRows + t * kTile;
            const uint64_t q_desc = smem_desc_k_sw128(q_addr + t * kTileBytes16);
            auto wait = [&](uint64_t *bar, int phase) { return mbar_spin_bounded(smem_u32(bar), phase & 1, abort_flag, limit); };
            auto full = [&](int i) { return wait(&sh.kv_full[i % kStages], i / kStages); }; // K of block j: i = 2 j, V: i = 2 j + 1
            // S = Q K^T of step k, into half k % 2 of the tile's score columns
            auto scores = [&](int k) {
                const int stage = (k & ~1) % kStages;
                const uint64_t k_desc = smem_desc_k_sw128(ring + stage * kTileBytes16 + (k & 1) * kStep * 128);
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (i < k_steps) {
                            const uint64_t at = ((i / 4) * kHalfBytes + (i % 4) * 32) >> 4;
                            mma_f16_ss(s_tmem + (k & 1) * kStep, q_desc + at, k_desc + at, idesc_s, i > 0);
                        }
                    mma_commit(smem_u32(&sh.s_full[t][k & 1]));
                    if ((k & 1) || k + 1 == n) mma_commit(smem_u32(&sh.kv_empty[stage]));
                }
                __syncwarp();
            };
            bool ok = true;
            if (n > 0) {
                ok = full(0) && wait(&sh.q_full[t], 0);
                tc_fence_after_sync();
                if (ok) scores(0);
                if (ok && n > 1) scores(1);
            }
            for (int k = 0; k < n && ok; ++k) {
                const int v = k | 1, stage = v % kStages; // block k / 2: values are tile 2 (k / 2) + 1
                if (!(ok = full(v) && wait(&sh.p_ready[t][k & 1], k >> 1))) break;
                tc_fence_after_sync();
                const uint64_t v_desc = smem_desc_mn_sw128(ring + stage * kTileBytes16 + (k & 1) * kStep * 128, kHalfBytes);
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) // O += P V, 16 keys each
                        mma_f16_ts(o_tmem, s_tmem + (k & 1) * kStep + i * 8, v_desc + ((i * 16 * 128) >> 4), idesc_o, k > 0 || i > 0);
                    if (kShared) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) // (the weights' second parts)
                            mma_f16_ts(o_tmem, s_tmem + (k & 1) * kStep + kStep / 2 + i * 8, v_desc + ((i * 16 * 128) >> 4), idesc_o, true);
                    }
                    mma_commit(smem_u32(&sh.o_done[t]));
                    if (k + 1 == n) mma_commit(smem_u32(&sh.o_last[t]));
                    if ((k & 1) || k + 1 == n) mma_commit(smem_u32(&sh.kv_empty[stage]));
                }
                __syncwarp();
                if (k + 2 < n) {
                    if (!(ok = full((k + 2) & ~1))) break;
                    tc_fence_after_sync();
                    scores(k + 2);
                }
            }
            // blocks that only the other tile needs
            for (int i = (n + 1) / 2 * 2; i < 2 * total && ok; ++i) {
                ok = full(i);
                if (ok && lane == 0) mbar_arrive(smem_u32(&sh.kv_empty[i % kStages]));
            }
        }
    } else {
        take_registers<kSoftmaxRegs>();
        // ---- softmax: one row per thread ------------------------------------------------------------------------
        const int t = warp / 4, r = tid % kTile, row = w.row0 + t * kTile + r;
        const bool exists = row < w.rows;
        const uint32_t lane_base = tmem + ((uint32_t)(32 * (warp % 4)) << 16), s_col = lane_base + t * kTile, o_col = lane_base + kRows + t * kTile;
        uint8_t *q_tile = smem + t * kTileBytes16;
        if (n_steps[t] > 0) {
            // the tile's queries, in the layout of the MMA: this warp's 32 rows, two at a time, 16 bytes per lane (heads of 100
            // elements are only 8-byte aligned: two halves)
            const int64_t mine = exists ? (int64_t)(w.first_token + row / group) * a.q_stride + (w.head * group + row % group) * D : -1;
            const int c = lane % 16, left = D - c * 8; // elements of the head from this lane's piece on
            const uint32_t dst = smem_u32(q_tile) + (c / 8) * kHalfBytes;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int64_t at = __shfl_sync(0xFFFFFFFFu, mine, 2 * i + lane / 16);
                const int qr = warp % 4 * 32 + 2 * i + lane / 16;
                const uint32_t to = dst + qr * 128 + (((c % 8) ^ (qr & 7)) << 4);
                const __nv_bfloat16 *src = a.q + (at < 0 || left <= 0 ? 0 : at + c * 8);
                if (D % 8 == 0) {
                    cp_async<16>(to, src, at >= 0 && left > 0);
                } else {
                    cp_async<8>(to, src, at >= 0 && left > 0);
                    cp_async<8>(to + 8, left > 4 ? src + 4 : src, at >= 0 && left > 4);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.q_full[t]));
        }
        const int sees = exists ? w.sees(row) : 0x7FFFFFFF; // (rows that do not exist: nothing to hide from them)
        const int least = w.sees(w.row0 + t * kTile);       // of the tile's rows
        float m = -INFINITY, l = 0.0f;                      // reference and sum of this row
        bool far = false;                                   // a reference beyond kFar (int8: of any row of the warp, at present)
        bool ok = true;
        for (int k = 0; k < n_steps[t]; ++k) {
            if (!mbar_spin_bounded(smem_u32(&sh.s_full[t][k & 1]), (k >> 1) & 1, abort_flag, limit)) {
                ok = false;
                break;
            }
            tc_fence_after_sync();
            const int j = k >> 1, key0 = (from + j) * kTile + (k & 1) * kStep;
            const uint32_t s_half = s_col + (k & 1) * kStep;
            uint32_t u[2][32];
            tmem_ld_32x32(s_half, u[0]);
            tmem_ld_32x32(s_half + 32, u[1]);
            // (the producer's notes on a block of keys were written before its arrival, which Q K^T waited for; `kv_full` of
            // the keys itself cannot be asked any more, it may be a phase further)
            const uint32_t bad_groups = sh.bad_groups[j % kInfo] >> (4 * (k & 1)) & 0xFu;
            const bool masked = key0 + kStep > least || bad_groups != 0u;
            const int kv = 2 * j + 1, v_stage = kv % kStages;
            if ((masked || kInt8) && !mbar_spin_bounded(smem_u32(&sh.kv_full[v_stage]), (kv / kStages) & 1, abort_flag, limit)) {
                ok = false; // (the values, or their scales, are looked at below)
                break;
            }
            if (masked && !kInt8) {
                // Values behind the sequence's end are whatever an earlier owner of the page left: they become zero.
                // Values inside that are not finite would reach rows that do not see them (0 x NaN): such a tile is done
                // again, row by row.  Two threads per key, 64 elements each.
                const int key = (k & 1) * kStep + r % kStep;
                uint8_t *v = smem + (2 + v_stage) * kTileBytes16 + (r / kStep) * kHalfBytes + key * 128;
                if (r < kStep || W > 64) {
                    const bool behind = (from + j) * kTile + key >= w.len;
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        uint4 *p = reinterpret_cast<uint4 *>(v + (((i + r) & 7) << 4));
                        if (behind) {
                            *p = make_uint4(0, 0, 0, 0);
                        } else {
                            const uint4 x = *p;
                            const uint32_t y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) odd = odd || (y[e] & 0x7F800000u) == 0x7F800000u || (y[e] & 0x7F80u) == 0x7F80u;
                        }
                    }
                    if (odd) sh.poisoned[t] = 1;
                    fence_proxy_async_smem();
                }
            }
            tmem_ld_wait_for(u[0]);
            tmem_ld_wait_for(u[1]);
            if (kInt8) {
                const float4 *ks = reinterpret_cast<const float4 *>(sh.scales[j % kScaled][0] + (k & 1) * kStep);
#pragma unroll
                for (int c = 0; c < kStep / 4; ++c) {
                    const float4 f = ks[c];
                    uint32_t *x = &u[c / 8][c % 8 * 4];
                    const float2 y = mul2(make_float2(__uint_as_float(x[0]), __uint_as_float(x[1])), make_float2(f.x, f.y));
                    const float2 z = mul2(make_float2(__uint_as_float(x[2]), __uint_as_float(x[3])), make_float2(f.z, f.w));
                    x[0] = __float_as_uint(y.x);
                    x[1] = __float_as_uint(y.y);
                    x[2] = __float_as_uint(z.x);
                    x[3] = __float_as_uint(z.y);
                }
            }
            if (masked) {
                const int n = sees - key0;
#pragma unroll
                for (int c = 0; c < kStep; ++c)
                    if (c >= n || ((bad_groups >> (c / 16)) & 1u)) u[c / 32][c % 32] = 0xFF800000u; // -infinity
            }
            float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int c = 0; c < kStep; c += 2) top[c / 2 % 4] = max3(top[c / 2 % 4], __uint_as_float(u[c / 32][c % 32]), __uint_as_float(u[c / 32][c % 32 + 1]));
            // (a NaN among the scores, or an infinite one, makes the row NaN as it does by the formula; NaN is kept by max3)
            float peak = max3(max3(top[0], top[1], top[2]), top[3], top[3]) * a.scale;
            if (peak == INFINITY) peak = __int_as_float(0x7FFFFFFF);
            auto is_far = [&] { return fabsf(m) > kFar && m != -INFINITY; };
            if (k == 0) {
                m = peak;
                if (kInt8) far = __any_sync(0xFFFFFFFFu, is_far());
            } else if (__any_sync(0xFFFFFFFFu, !(peak <= m + kRaise))) {
                const float raised = peak <= m ? m : peak;
                const float keep = raised == -INFINITY ? 1.0f : exp2_approx(m - raised);
                if (!kInt8) far = far || is_far();
                m = raised;
                if (kInt8) far = __any_sync(0xFFFFFFFFu, is_far());
                l *= keep;
                // the P V in front of this step has to be at rest (the next one waits for this step's weights; the one before
                // it is done, as the scores of this step were issued behind it, so the phase asked for is the current one or
                // the one just completed)
                if (!mbar_spin_bounded(smem_u32(&sh.o_done[t]), (k - 1) & 1, abort_flag, limit)) {
                    ok = false;
                    break;
                }
                tc_fence_after_sync();
#pragma unroll 1
                for (int c = 0; c < W; c += 16) {
                    uint32_t o[16];
                    tmem_ld_32x16(o_col + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                    tmem_st_32x16(o_col + c, o);
                }
            }
            float nb = m == -INFINITY ? 0.0f : -m;
            if (kInt8 && far) {
                const float per_unit = 1.0f / a.scale;
#pragma unroll
                for (int c = 0; c < kStep; ++c) // (no fma: the product has to be rounded as m was)
                    u[c / 32][c % 32] = __float_as_uint((__fmul_rn(__uint_as_float(u[c / 32][c % 32]), a.scale) + nb) * per_unit);
                nb = 0.0f;
            }
            const float2 scale2 = make_float2(a.scale, a.scale), nb2 = make_float2(nb, nb);
            float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
            const float4 *vs = reinterpret_cast<const float4 *>(sh.scales[j % kScaled][1] + (k & 1) * kStep);
            auto weights = [&](auto hidden) { // hidden: some of the scores are
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t p[16];
                    [[maybe_unused]] uint32_t rest[kShared ? 16 : 1];
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float4 f = make_float4(1.0f, 1.0f, 1.0f, 1.0f);
                        if (kInt8) f = vs[c * 8 + e / 4];
                        const float2 fs[2] = {make_float2(f.x, f.y), make_float2(f.z, f.w)};
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t u0 = u[c][e + 2 * h], u1 = u[c][e + 2 * h + 1];
                            float2 y = fma2(make_float2(__uint_as_float(u0), __uint_as_float(u1)), scale2, nb2);
                            y = make_float2(exp2_approx(y.x), exp2_approx(y.y));
                            sum[h] = add2(sum[h], y);
                            if (kInt8) {
                                y = mul2(y, fs[h]);
                                // (0 times the scale of a row that is not finite)
                                if (decltype(hidden)::value) y = make_float2(u0 == 0xFF800000u ? 0.0f : y.x, u1 == 0xFF800000u ? 0.0f : y.y);
                            }
                            if constexpr (kShared) {
                                // (as in attend_decode.cu: bf16 values may be infinite, so the first part is cut off and the second one positive; here
                                // of a weight of 0 too, which may count as 2^-126: keys that do not exist have values of 0)
                                const uint32_t x = kInt8 ? pack_bf16(y.x, y.y) : __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x7632);
                                float2 z = fma2(make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xFFFF0000u)), make_float2(-1.0f, -1.0f), y);
                                if (!kInt8) {
                                    const float2 least = fma2(y, make_float2(0x1p-24f, 0x1p-24f), make_float2(0x1p-126f, 0x1p-126f));
                                    z = make_float2(fmaxf(z.x, least.x), fmaxf(z.y, least.y));
                                }
                                p[e / 2 + h] = x;
                                rest[e / 2 + h] = pack_bf16(z.x, z.y);
                            } else {
                                p[e / 2 + h] = pack_bf16(y.x, y.y);
                            }
                        }
                    }
                    tmem_st_32x16(s_half + c * 16, p); // (the scores have been read)
                    if constexpr (kShared) tmem_st_32x16(s_half + kStep / 2 + c * 16, rest);
                }
            };
            if (kInt8 && masked)
                weights(std::true_type{});
            else
                weights(std::false_type{});
            const float2 both = add2(sum[0], sum[1]);
            l += both.x + both.y;
            tmem_st_wait();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.p_ready[t][k & 1]));
        }
        if (n_steps[t] > 0) ok = ok && mbar_spin_bounded(smem_u32(&sh.o_last[t]), 0, abort_flag, limit);
        tc_fence_after_sync();
        // The next launch may start when all tiles are at their ends, not before: what it lets in early in its turn may be a matmul,
        // whose bounded waits would run while a long tile is worked on.  (bf16: below, when no row has to be done again.)
        if (kInt8 && tid == 0) griddep_launch_dependents();
        if (!kInt8 && exists && (far || (fabsf(m) > kFar && m != -INFINITY))) sh.poisoned[t] = 1; // (to be done again, like a poisoned tile)

        // ---- the result, or this CTA's part of it --------------------------------------------------------------
        float *ws_parts = reinterpret_cast<float *>(reinterpret_cast<char *>(a.workspace) + prompt_counter_bytes());
        if constexpr (kShared) {
            ws_parts = more.parts;
            if (exists && split == 0)
                more.where[(int64_t)(w.first_token + row / group) * a.heads + w.head * group + row % group] =
                    parts > 1 ? make_int2(blockIdx.x, parts << 16 | (t * kTile + r)) : make_int2(-1, 0);
        }
        const int first_part = blockIdx.x - split; // of this tile
        auto part_of = [&](int p) { return ws_parts + (size_t)(first_part + p) * prompt_part_floats(W); };
        if (ok) {
            const float inv = kShared || parts > 1 ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);
            __nv_bfloat16 *dst = a.out + (int64_t)(w.first_token + row / group) * a.out_stride + (w.head * group + row % group) * D;
            const int pr = t * kTile + r;
            const bool some = n_steps[t] > 0 && l != 0.0f;
            uint32_t o[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (c * 32 < W) tmem_ld_32x32(o_col + c * 32, o[c]);
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_wait_for(o[c]);
            auto at = [&](int e) { return some ? __uint_as_float(o[e / 32][e % 32]) * inv : 0.0f; };
            if (parts > 1) {
                if (exists) {
                    float4 *part = reinterpret_cast<float4 *>(part_of(split) + 2 * kRows) + pr;
                    *reinterpret_cast<float2 *>(part_of(split) + 2 * pr) = make_float2(n_steps[t] > 0 ? m : -INFINITY, l);
#pragma unroll
                    for (int e = 0; e < kTile; e += 4)
                        if (e < W) part[e / 4 * kRows] = make_float4(at(e), at(e + 1), at(e + 2), at(e + 3));
                }
            } else if constexpr (kShared) {
                if (exists) {
                    const int64_t to = (int64_t)(w.first_token + row / group) * a.heads + w.head * group + row % group;
                    more.ml[to] = make_float2(n_steps[t] > 0 ? m : -INFINITY, l);
                    float4 *out = reinterpret_cast<float4 *>(more.o + to * W);
#pragma unroll
                    for (int e = 0; e < kTile; e += 4)
                        if (e < W) out[e / 4] = make_float4(at(e), at(e + 1), at(e + 2), at(e + 3));
                }
            } else {
                // by way of the tile's queries, which are not needed any more, so that a warp stores whole rows
                uint8_t *own = q_tile + (warp % 4) * 32 * 256;
#pragma unroll
                for (int e = 0; e < kTile; e += 8)
                    *reinterpret_cast<uint4 *>(own + lane * 256 + (((e / 8) ^ (lane & 7)) << 4)) =
                        make_uint4(pack_bf16(at(e), at(e + 1)), pack_bf16(at(e + 2), at(e + 3)), pack_bf16(at(e + 4), at(e + 5)),
                                   pack_bf16(at(e + 6), at(e + 7)));
                __syncwarp();
                const int64_t mine = exists ? dst - a.out : -1;
                const int c = lane % 16, left = D - c * 8;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int sr = 2 * i + lane / 16;
                    const int64_t to = __shfl_sync(0xFFFFFFFFu, mine, sr);
                    const uint4 y = *reinterpret_cast<const uint4 *>(own + sr * 256 + ((c ^ (sr & 7)) << 4));
                    if (to < 0 || left <= 0) continue;
                    if (D % 8 == 0) {
                        *reinterpret_cast<uint4 *>(a.out + to + c * 8) = y;
                    } else {
                        *reinterpret_cast<uint2 *>(a.out + to + c * 8) = make_uint2(y.x, y.y);
                        if (left > 4) *reinterpret_cast<uint2 *>(a.out + to + c * 8 + 4) = make_uint2(y.z, y.w);
                    }
                }
            }
        }
        if (!kShared && parts > 1) {
            // the CTA that finishes last joins the parts in their order and leaves the counter at zero
            uint32_t *counter = reinterpret_cast<uint32_t *>(a.workspace) + 2 * first_part;
            __threadfence();
            named_barrier(1, kRows);
            if (tid == 0) {
                if (sh.poisoned[0] || sh.poisoned[1]) atomicOr(counter + 1, 1u);
                __threadfence();
                const uint32_t before = atomicAdd(counter, 1u);
                sh.is_last = before == (uint32_t)(parts - 1);
                if (sh.is_last) {
                    __threadfence();
                    const uint32_t odd = atomicExch(counter + 1, 0u);
                    sh.poisoned[0] = sh.poisoned[1] = (int)odd;
                    counter[0] = 0u;
                }
            }
            named_barrier(1, kRows);
            if (sh.is_last) {
                __threadfence();
                const int pr = tid, rr = w.row0 + pr; // a row per thread
                if (rr < w.rows) {
                    float M = -INFINITY, L = 0.0f;
#pragma unroll 4
                    for (int p = 0; p < parts; ++p) M = fmaxf(M, __ldcg(part_of(p) + 2 * pr));
                    const float ref = M == -INFINITY ? 0.0f : M;
                    float *factor = reinterpret_cast<float *>(smem) + tid; // (where the queries were)
#pragma unroll 4
                    for (int p = 0; p < parts; ++p) {
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(part_of(p) + 2 * pr));
                        const float f = exp2_approx(ml.x - ref);
                        factor[p * kRows] = f;
                        L += f * ml.y;
                    }
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
                    __nv_bfloat16 *dst = a.out + (int64_t)(w.first_token + rr / group) * a.out_stride + (w.head * group + rr % group) * D;
                    for (int e0 = 0; e0 < D; e0 += 16) { // (W is a multiple of 16)
                        float4 x[4];
#pragma unroll
                        for (int u = 0; u < 4; ++u) x[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
                        for (int p = 0; p < parts; ++p) {
                            const float4 *src = reinterpret_cast<const float4 *>(part_of(p) + 2 * kRows) + (size_t)(e0 / 4) * kRows + pr;
                            const float f = factor[p * kRows];
#pragma unroll
                            for (int u = 0; u < 4; ++u) {
                                const float4 v = __ldcg(src + u * kRows);
                                x[u] = make_float4(x[u].x + f * v.x, x[u].y + f * v.y, x[u].z + f * v.z, x[u].w + f * v.w);
                            }
                        }
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if (e0 + 4 * u < D)
                                *reinterpret_cast<uint2 *>(dst + e0 + 4 * u) =
                                    make_uint2(pack_bf16(x[u].x * inv, x[u].y * inv), pack_bf16(x[u].z * inv, x[u].w * inv));
                    }
                }
            }
        }
        if (!kInt8) {
            named_barrier(1, kRows);
            // The next launch may start, unless rows have to be done again: that takes long when they see many keys, and the
            // waits of a matmul that were resident meanwhile would run out.
            const bool again = kShared || parts == 1 || sh.is_last; // (the shared form's parts are each done again by their own CTA)
            if (tid == 0 && !(again && (sh.poisoned[0] || sh.poisoned[1]))) griddep_launch_dependents();
            if (again) {
                if (sh.poisoned[t])
                    for (int i = warp % 4; i < kTile; i += 4)
                        if (const int rr = w.row0 + t * kTile + i; rr < w.rows) {
                            RowResult to = {};
                            int begin = 0, end = w.sees(rr);
                            if constexpr (kShared) {
                                const int64_t at = (int64_t)(w.first_token + rr / group) * a.heads + w.head * group + rr % group;
                                begin = from * kTile;
                                end = min(end, to_block * kTile);
                                if (parts > 1)
                                    to = {reinterpret_cast<float2 *>(part_of(split)) + t * kTile + i, part_of(split) + 2 * kRows + 4 * (t * kTile + i), 4 * kRows};
                                else
                                    to = {more.ml + at, more.o + at * W, 4};
                            }
                            attend_row<kShared>(a, w, rr, lane, begin, end, to);
                        }
            }
        }
    }

    write_starts();

    // every thread arrives here, also after an expired wait
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) atomicMax(reinterpret_cast<uint32_t *>(a.cache.status), (uint32_t)BITLINEAR_ERR_TIMEOUT); // (see kv_report)
        // give copies and MMAs that may still be in flight time to land before shared and tensor memory go away
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
        __syncthreads();
    }
    if (warp == kMmaWarp) {
        tc_fence_after_sync();
        tmem_dealloc(tmem, kTmemColumns);
    }
}

// The cache as rows of `width` bf16 elements; a copy takes 64 of them from the rows of one page (at most 128).
bool encode_cache_map(CUtensorMap *map, void *pool, const KvCache &c)
{
    EncodeTiledFn encode = encode_tiled_fn();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)c.width, (cuuint64_t)c.n_pages * (cuuint64_t)c.kv_heads << c.page_shift};
    const cuuint64_t strides[1] = {(cuuint64_t)c.width * 2};
    const cuuint32_t box[2] = {64u, (cuuint32_t)std::min(kTile, 1 << c.page_shift)};
    const cuuint32_t step[2] = {1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, pool, dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool kInt8, bool kShared>
cudaError_t launch(const PromptArgs &p, const PromptMore<kShared> &more, int ctas, cudaStream_t stream)
{
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        cudaFuncAttributes have;
        e = cudaFuncGetAttributes(&have, attend_prompt_kernel<kInt8, kShared>);
        if (e != cudaSuccess) return e;
        if (have.numRegs != kLaunchRegs) return cudaErrorInvalidConfiguration; // (the split of the registers would not add up)
        e = cudaFuncSetAttribute(attend_prompt_kernel<kInt8, kShared>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shared<kInt8>::bytes());
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    return launch_dependent(attend_prompt_kernel<kInt8, kShared>, (unsigned)ctas, kThreads, Shared<kInt8>::bytes(), stream, p, more);
}

template <bool kShared>
cudaError_t launch_tiles(const AttendArgs &a, const PromptMore<kShared> &more, cudaStream_t stream)
{
    PromptArgs p{};
    p.a = a;
    p.hooks = take_wait_hooks();
    if (!a.cache.k_scale && (!encode_cache_map(&p.k_map, a.cache.k, a.cache) || !encode_cache_map(&p.v_map, a.cache.v, a.cache)))
        return cudaErrorInvalidValue;
    // No more tiles of rows than this can exist: every sequence has at most one that is not full.  (Of one sequence whose rows fill
    // their tiles exactly this is one per kv head too many: some CTAs find no tile, and the keys of the others are split less.)
    const int64_t group = a.heads / a.cache.kv_heads;
    const int64_t tiles = ((int64_t)a.T * group / kRows + std::min<int64_t>(a.batch.n_seqs, a.T)) * a.cache.kv_heads;
    // With fewer tiles than SMs the keys of a tile are split among several CTAs, no more than run at the same time (2 tokens behind
    // 10994, 32 heads of 100: with five CTAs for each of the 32 tiles twelve had to wait for an SM, 87 us; with four 57).  Of
    // several sequences only the device knows how many tiles they have (5 sequences of 50 tokens behind 4000, 24/8 heads
    // of 64: 48 -> 42 us against the bound above); it is asked where the bound is below the number of SMs, so a batch with many
    // empty slots is not split.
    const int slots = std::min(sm_count(), kPromptMaxParts);
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(kMaxParts, slots / tiles));
    p.slots = (kShared || a.batch.n_seqs > 1) && tiles < slots ? slots : 0;
    const int ctas = p.slots > 0 ? slots : (int)tiles * p.splits;
    return a.cache.k_scale ? launch<true, kShared>(p, more, ctas, stream) : launch<false, kShared>(p, more, ctas, stream);
}

} // namespace

size_t attend_prompt_workspace_bytes(int heads, int kv_heads, int head_dim)
{
    (void)heads;
    (void)kv_heads;
    return align_up(prompt_counter_bytes() + kPromptMaxParts * prompt_part_floats(kv_row_width(head_dim)) * 4, 256);
}

cudaError_t launch_attend_prompt(const AttendArgs &a, cudaStream_t stream) { return launch_tiles<false>(a, PromptMore<false>{}, stream); }

cudaError_t launch_attend_prefix(const AttendArgs &a, const SharedArgs &shared, cudaStream_t stream)
{
    PromptMore<true> more;
    static_cast<SharedArgs &>(more) = shared;
    return launch_tiles<true>(a, more, stream);
}

} // namespace bitlinear
