// Causal attention of the new tokens of prompts and prompt chunks over the paged cache, on the tcgen05 tensor cores.
//
//   out = P V / sum P,  P_ij = 2^(s_ij - m_i),  S = scale log2(e) Q K^T,  in one pass over the keys with a running reference m_i
//
// Rows.  The query heads that share a kv head are taken together: row R of a (sequence, kv head) is token R / group, head
// R % group of the group, so one tile of keys serves them all and a chunk of few tokens still fills a tile.  A CTA owns
// 256 rows as two tiles of 128 (the MMA's M), and walks the keys they see in blocks of 128.
//
// Roles (12 warps):
//   warps 0-3, 4-7 : the softmax of tile 0 and of tile 1, one row per thread: scores from tensor memory, maximum, 2^x, the
//                    weights as bf16 back into tensor memory, over the scores they came from; while one tile's weights are
//                    computed, the tensor cores work for the other tile;
//   warp 8         : issues the MMAs: S = Q K^T (both operands in shared memory) and O += P V (P in tensor memory, V as it
//                    lies in the cache: keys are its rows, so it is the MN-major operand);
//   warps 9-11     : producers.  bf16: TMA of one page's rows and 64 elements of the head per copy (128-byte swizzle); an
//                    issued copy costs its thread 100 to 150 cycles, hence three issuing warps.  int8: the
//                    three warps load the codes, turn them into bf16 (exactly) and store them in the same layout.
// Tensor memory: 2 x 128 columns of scores, 2 x 128 of output.  The tensor pipe executes the MMAs of one thread in order, so
// the commit behind Q K^T of a block also says that the P V before it is done, and the scores of the next block may overwrite
// the weights that the P V in front of them reads.
//
// Rescaling.  The output stands in tensor memory, and moving it for every new maximum would cost as much as the softmax.  The
// reference m_i is therefore raised only when a score exceeds it by more than 8 (a factor 256, which fp32 sums and bf16 weights
// carry without loss); the result does not depend on the reference.
//
// What bounds it: 128 x 128 scores need 16384 exponentials, 16 per cycle and SM = 1024 cycles, while their two MMAs take 512
// cycles at a head of 128.
#include <cuda.h>

#include <algorithm>

#include "internal.cuh"
#include "kv.cuh"
#include "ptx.cuh"
#include "tma_host.cuh"

namespace bitlinear {
namespace {

using namespace ptx;

constexpr int kTile = 128;               // rows of a query tile, keys of a block
constexpr int kRows = 2 * kTile;         // rows of a CTA
constexpr int kHalfBytes = kTile * 128;  // 128 rows of 64 bf16 elements, 128-byte swizzle
constexpr int kTileBytes16 = 2 * kHalfBytes;
constexpr int kMaxStages = 5;
constexpr int kInfo = 8;                 // ring of per-block notes (at most three blocks are in flight)
constexpr int kMmaWarp = 8, kFirstProducer = 9, kProducers = 3;
constexpr int kThreads = 12 * 32;
constexpr uint32_t kTmemColumns = 512;
constexpr float kRaise = 8.0f;

template <bool kInt8>
struct Shared {
    static constexpr int kStages = kInt8 ? 4 : 5; // blocks of keys or values in shared memory
    static constexpr int kScaled = 4;             // blocks whose scales are kept
    float scales[kInt8 ? kScaled : 1][2][kInt8 ? kTile : 4]; // of the keys and of the values of a block
    uint64_t q_full[2], kv_full[kMaxStages], kv_empty[kMaxStages], s_full[2], p_ready[2], o_done[2];
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
    return 1024 + (2 + kStages) * kTileBytes16 + (int)sizeof(Shared<kInt8>);
}
static_assert(Shared<false>::bytes() <= 232448 && Shared<true>::bytes() <= 232448, "shared memory of an SM");

struct PromptArgs {
    CUtensorMap k_map, v_map;
    AttendArgs a;
    int splits;       // CTAs that may share the keys of a tile of rows
    WaitHooks hooks;
};

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
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
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

// One row by plain arithmetic, one warp: for tiles in which a non-finite value stands behind keys that some of the rows do not
// see (0 x NaN would reach them through the MMA).
__device__ void attend_row(const AttendArgs &a, const Work &w, int r, int lane)
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
    const int end = w.sees(r);
    for (int j = 0; j < end; ++j) {
        const int page = kv_page(a.cache, a.batch, w.b, j);
        if (page < 0) continue;
        const int64_t row = (int64_t)kv_row(a.cache, page, w.head, j) * a.cache.width;
        const float4 k = load(reinterpret_cast<const __nv_bfloat16 *>(a.cache.k) + row);
        const float4 v = load(reinterpret_cast<const __nv_bfloat16 *>(a.cache.v) + row);
        float s = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        s *= a.scale;
        const float mn = fmaxf(m, s);
        const float base = mn == -INFINITY ? 0.0f : mn;
        const float keep = exp2_approx(m - base), p = exp2_approx(s - base);
        l = l * keep + p;
        o = make_float4(o.x * keep + p * v.x, o.y * keep + p * v.y, o.z * keep + p * v.z, o.w * keep + p * v.w);
        m = mn;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (mine)
        *reinterpret_cast<uint2 *>(a.out + (int64_t)t * a.out_stride + h * D + 4 * lane) =
            make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

// Partial results of the CTAs that share a tile of rows: (reference, sum) of 256 rows, then their outputs.
__host__ __device__ constexpr size_t part_floats(int width) { return (size_t)kRows * (width + 2); }

template <bool kInt8>
__global__ void __launch_bounds__(kThreads, 1) attend_prompt_kernel(const __grid_constant__ PromptArgs args)
{
    const AttendArgs &a = args.a;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t *smem = smem_raw + (base - raw);
    constexpr int kStages = Shared<kInt8>::kStages, kScaled = Shared<kInt8>::kScaled;
    Shared<kInt8> &sh = *reinterpret_cast<Shared<kInt8> *>(smem + (2 + kStages) * kTileBytes16);
    volatile int *abort_flag = &sh.abort_flag;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;
    const int D = a.cache.head_dim, W = a.cache.width, group = a.heads / a.cache.kv_heads, n_seqs = a.batch.n_seqs;
    const uint32_t limit = args.hooks.limit_us;

    // ---- which rows: tiles are counted sequence by sequence, kv head by kv head, the last rows (which see most) first ----
    const int split = blockIdx.x % args.splits;
    {
        const int64_t x = blockIdx.x / args.splits;
        auto tiles_of = [&](int b) -> int64_t {
            const int64_t n = (int64_t)a.batch.cu_tokens[b + 1] - a.batch.cu_tokens[b];
            return n <= 0 || n > a.T ? 0 : (n * group + kRows - 1) / kRows * a.cache.kv_heads;
        };
        const int per_thread = (n_seqs + kThreads - 1) / kThreads;
        const int b0 = min(n_seqs, tid * per_thread), b1 = min(n_seqs, b0 + per_thread);
        int64_t mine = 0;
        for (int b = b0; b < b1; ++b) mine += tiles_of(b);
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
        if (x >= upto - mine && x < upto) {
            int64_t rest = x - (upto - mine);
            int b = b0;
            for (; b < b1 - 1; ++b) {
                const int64_t n = tiles_of(b);
                if (rest < n) break;
                rest -= n;
            }
            sh.found_b = b;
            sh.found_local = rest;
        }
        __syncthreads();
    }
    if (sh.found_b < 0) return;
    Work w;
    w.b = sh.found_b;
    w.group = group;
    w.first_token = a.batch.cu_tokens[w.b];
    const int n_tokens = a.batch.cu_tokens[w.b + 1] - w.first_token;
    if (w.first_token < 0 || (int64_t)w.first_token + n_tokens > a.T) return; // (rows that the caller did not hand over)
    w.rows = n_tokens * group;
    {
        const int tiles = (w.rows + kRows - 1) / kRows;
        w.head = (int)(sh.found_local / tiles);
        w.row0 = (tiles - 1 - (int)(sh.found_local % tiles)) * kRows;
    }
    bool over;
    w.len = kv_length(a.batch, w.b, over);
    if (over && tid == 0) kv_report(a.cache);
    w.offset = a.batch.kv_lens[w.b] - n_tokens;

    // blocks of keys of the two tiles, and this CTA's part of them (a part is at least four blocks, so that joining the parts
    // does not cost more than they save)
    const int most = (w.sees(min(w.row0 + kRows, w.rows) - 1) + kTile - 1) / kTile;
    const int parts = max(1, min(args.splits, most / 4));
    if (split >= parts) return;
    const int from = (int)((int64_t)most * split / parts), to = (int)((int64_t)most * (split + 1) / parts);
    int blocks[2];
    for (int t = 0; t < 2; ++t) {
        const int first = w.row0 + t * kTile, last = min(first + kTile, w.rows) - 1;
        blocks[t] = first < w.rows ? max(0, min((w.sees(last) + kTile - 1) / kTile, to) - from) : 0;
    }
    const int total = max(blocks[0], blocks[1]);

    if (tid == 0) {
        for (int t = 0; t < 2; ++t) {
            mbar_init(smem_u32(&sh.q_full[t]), 4);
            mbar_init(smem_u32(&sh.s_full[t]), 1);
            mbar_init(smem_u32(&sh.p_ready[t]), 4);
            mbar_init(smem_u32(&sh.o_done[t]), 1);
            sh.poisoned[t] = 0;
        }
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_u32(&sh.kv_full[s]), 1);
            mbar_init(smem_u32(&sh.kv_empty[s]), 1);
        }
        sh.abort_flag = 0;
        fence_mbar_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(smem_u32(&sh.tmem_base), kTmemColumns);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem = sh.tmem_base;
    const uint32_t q_addr = base, ring = base + 2 * kTileBytes16;

    if (warp >= kFirstProducer) {
        // ---- producers: blocks in the order K 0, V 0, K 1, V 1, ..., each warp every third of them ----------------
        const int halves = W > 64 ? 2 : 1;
        for (int i = warp - kFirstProducer; i < 2 * total; i += kProducers) {
            const int s = i % kStages, round = i / kStages, j = from + i / 2;
            const bool values = i & 1;
            if (round > 0 && !mbar_wait_bounded(smem_u32(&sh.kv_empty[s]), (round - 1) & 1, abort_flag, limit)) break;
            const uint32_t full = smem_u32(&sh.kv_full[s]), dst = ring + s * kTileBytes16;
            // the pages of the block's eight 16-key groups, one per lane
            int row = -1;
            bool bad = false;
            if (lane < 8) {
                const int pos = j * kTile + lane * 16;
                if (pos < w.len) {
                    const int page = kv_page(a.cache, a.batch, w.b, pos);
                    bad = page < 0;
                    if (bad)
                        kv_report(a.cache);
                    else
                        row = kv_row(a.cache, page, w.head, pos);
                }
            }
            const uint32_t bad_groups = __ballot_sync(0xFFFFFFFFu, bad);
            if (!values && lane == 0) sh.bad_groups[(i / 2) % kInfo] = bad_groups;
            if (!kInt8) {
                const int per_copy = min(kTile, 1 << a.cache.page_shift); // rows of a copy
                const int absent = (a.cache.n_pages * a.cache.kv_heads) << a.cache.page_shift; // a row behind the cache: reads zeros
                const CUtensorMap *map = values ? &args.v_map : &args.k_map;
                const bool skip = args.hooks.skip_arrive && blockIdx.x == 0 && i == 0;
                if (lane == 0 && !skip) mbar_arrive_expect_tx(full, (uint32_t)(halves * kHalfBytes));
                __syncwarp();
                for (int g = 0; g < kTile / 16; g += per_copy / 16) {
                    const int r = __shfl_sync(0xFFFFFFFFu, row, g);
                    if (lane == 0 && !skip) {
                        for (int h = 0; h < halves; ++h)
                            tma_load_2d(dst + h * kHalfBytes + g * 16 * 128, map, h * 64, r < 0 ? absent : r, full);
                    }
                }
            } else {
                const int8_t *pool = reinterpret_cast<const int8_t *>(values ? a.cache.v : a.cache.k);
                const float *scale = values ? a.cache.v_scale : a.cache.k_scale;
                uint8_t *out = smem + (2 + s) * kTileBytes16;
                const int pieces = W / 16; // 16 codes each
                // lane: piece c of row r; rows 4 (or more) at a time
                const int c = lane % 8, r0 = lane / 8;
#pragma unroll 2
                for (int g = 0; g < 8; ++g) {
                    const int first = __shfl_sync(0xFFFFFFFFu, row, g);
                    uint4 x[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int r = g * 16 + u * 4 + r0;
                        const bool real = first >= 0 && c < pieces && j * kTile + r < w.len;
                        x[u] = real ? *reinterpret_cast<const uint4 *>(pool + (int64_t)(first + u * 4 + r0) * W + c * 16) : make_uint4(0, 0, 0, 0);
                    }
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int r = g * 16 + u * 4 + r0;
                        uint8_t *half = out + (c / 4) * kHalfBytes + r * 128;
                        const int p = (c % 4) * 2;
                        *reinterpret_cast<uint4 *>(half + ((p ^ (r & 7)) << 4)) =
                            make_uint4(code_pair<0x4140>(x[u].x), code_pair<0x4342>(x[u].x), code_pair<0x4140>(x[u].y), code_pair<0x4342>(x[u].y));
                        *reinterpret_cast<uint4 *>(half + (((p + 1) ^ (r & 7)) << 4)) =
                            make_uint4(code_pair<0x4140>(x[u].z), code_pair<0x4342>(x[u].z), code_pair<0x4140>(x[u].w), code_pair<0x4342>(x[u].w));
                    }
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int r = u * 32 + lane, first = __shfl_sync(0xFFFFFFFFu, row, r / 16);
                    sh.scales[(i / 2) % kScaled][values][r] = first >= 0 && j * kTile + r < w.len ? scale[first + r % 16] : 0.0f;
                }
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0 && !(args.hooks.skip_arrive && blockIdx.x == 0 && i == 0)) mbar_arrive(full);
            }
        }
    } else if (warp == kMmaWarp) {
        // ---- MMAs -------------------------------------------------------------------------------------------
        const int steps = W / 16;
        const uint32_t idesc_s = idesc_bf16(kTile, kTile, 0), idesc_o = idesc_bf16(kTile, W, 1);
        bool ok = true;
        auto wait = [&](uint64_t *bar, int phase) { ok = ok && mbar_wait_bounded(smem_u32(bar), phase & 1, abort_flag, limit); };
        auto scores = [&](int t, int j) { // S_t = Q_t K_j^T
            const uint32_t k = ring + (uint32_t)((2 * j) % kStages) * kTileBytes16, q = q_addr + t * kTileBytes16;
            if (elect_one()) {
#pragma unroll
                for (int s = 0; s < 8; ++s)
                    if (s < steps) {
                        const uint32_t at = (s / 4) * kHalfBytes + (s % 4) * 32;
                        mma_f16_ss(tmem + t * kTile, smem_desc_k_sw128(q + at), smem_desc_k_sw128(k + at), idesc_s, s > 0);
                    }
                mma_commit(smem_u32(&sh.s_full[t]));
            }
            __syncwarp();
        };
        if (total > 0) wait(&sh.kv_full[0], 0);
        for (int t = 0; t < 2 && ok; ++t) {
            if (blocks[t] == 0) continue;
            wait(&sh.q_full[t], 0);
            tc_fence_after_sync();
            if (ok) scores(t, 0);
        }
        if (ok && total > 0 && elect_one()) mma_commit(smem_u32(&sh.kv_empty[0]));
        __syncwarp();
        for (int j = 0; j < total && ok; ++j) {
            const int kv = 2 * j + 1, s_v = kv % kStages, k_next = 2 * j + 2, s_k = k_next % kStages;
            wait(&sh.kv_full[s_v], kv / kStages);
            if (j + 1 < total) wait(&sh.kv_full[s_k], k_next / kStages);
            for (int t = 0; t < 2 && ok; ++t) {
                if (j >= blocks[t]) continue;
                wait(&sh.p_ready[t], j);
                if (!ok) break;
                tc_fence_after_sync();
                const uint32_t v = ring + s_v * kTileBytes16;
                if (elect_one()) {
#pragma unroll
                    for (int s = 0; s < 8; ++s)
                        mma_f16_ts(tmem + kRows + t * kTile, tmem + t * kTile + s * 8, smem_desc_mn_sw128(v + s * 16 * 128, kHalfBytes),
                                   idesc_o, j > 0 || s > 0);
                    if (j + 1 == blocks[t]) mma_commit(smem_u32(&sh.o_done[t]));
                }
                __syncwarp();
                if (j + 1 < blocks[t]) scores(t, j + 1);
            }
            if (ok && elect_one()) {
                mma_commit(smem_u32(&sh.kv_empty[s_v]));
                if (j + 1 < total) mma_commit(smem_u32(&sh.kv_empty[s_k]));
            }
            __syncwarp();
        }
    } else {
        // ---- softmax: one row per thread ------------------------------------------------------------------------
        const int t = warp / 4, r = tid % kTile, row = w.row0 + t * kTile + r;
        const bool exists = row < w.rows;
        const uint32_t lane_base = tmem + ((uint32_t)(32 * (warp % 4)) << 16), s_col = lane_base + t * kTile, o_col = lane_base + kRows + t * kTile;
        uint8_t *q_tile = smem + t * kTileBytes16;
        if (blocks[t] > 0) {
            // the tile's queries, in the layout of the MMA (8-byte loads: heads of 100 elements are not 16-byte aligned)
#pragma unroll 4
            for (int i = r; i < kTile * 16; i += kTile) {
                const int qr = i / 16, c = i % 16, rr = w.row0 + t * kTile + qr;
                uint2 x = make_uint2(0, 0), y = make_uint2(0, 0);
                if (rr < w.rows) {
                    const __nv_bfloat16 *src = a.q + (int64_t)(w.first_token + rr / group) * a.q_stride + (w.head * group + rr % group) * D + c * 8;
                    if (c * 8 < D) x = *reinterpret_cast<const uint2 *>(src);
                    if (c * 8 + 4 < D) y = *reinterpret_cast<const uint2 *>(src + 4);
                }
                *reinterpret_cast<uint4 *>(q_tile + (c / 8) * kHalfBytes + qr * 128 + (((c % 8) ^ (qr & 7)) << 4)) = make_uint4(x.x, x.y, y.x, y.y);
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.q_full[t]));
        }
        const int sees = exists ? w.sees(row) : 0x7FFFFFFF; // (rows that do not exist: nothing to hide from them)
        const int least = w.sees(w.row0 + t * kTile);       // of the tile's rows
        float m = -INFINITY, l = 0.0f;                      // reference and sum of this row
        bool ok = true;
        for (int j = 0; j < blocks[t]; ++j) {
            if (!mbar_wait_bounded(smem_u32(&sh.s_full[t]), j & 1, abort_flag, limit)) {
                ok = false;
                break;
            }
            tc_fence_after_sync();
            const int key0 = (from + j) * kTile;
            // (the producer's notes on a block of keys were written before its arrival, which Q K^T waited for; `kv_full` of
            // the keys itself cannot be asked any more, it may be a phase further)
            const uint32_t bad_groups = sh.bad_groups[j % kInfo];
            const bool masked = key0 + kTile > least || bad_groups != 0u;
            const int n_seen = sees - key0;
            // 32 scores of this row, scaled by their keys and masked.  They are read twice, for the maximum and for the weights,
            // rather than held in 128 registers.
            auto load = [&](int c, uint32_t (&u)[32]) { tmem_ld_32x32(s_col + c * 32, u); };
            auto settle = [&](int c, const uint32_t (&u)[32], float (&x)[32]) {
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = __uint_as_float(u[e]);
                if (kInt8) {
                    const float4 *ks = reinterpret_cast<const float4 *>(sh.scales[j % kScaled][0]) + c * 8;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float4 f = ks[e];
                        x[4 * e] *= f.x;
                        x[4 * e + 1] *= f.y;
                        x[4 * e + 2] *= f.z;
                        x[4 * e + 3] *= f.w;
                    }
                }
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c * 32 + e >= n_seen || ((bad_groups >> (2 * c + e / 16)) & 1u)) x[e] = -INFINITY;
                }
            };
            if (masked) {
                if (!kInt8) {
                    // Values behind the sequence's end are whatever an earlier owner of the page left: they become zero.
                    // Values inside that are not finite would reach rows that do not see them (0 x NaN): such a tile
                    // is done again, row by row.
                    const int kv = 2 * j + 1, st = kv % kStages;
                    if (!mbar_wait_bounded(smem_u32(&sh.kv_full[st]), (kv / kStages) & 1, abort_flag, limit)) {
                        ok = false;
                        break;
                    }
                    uint8_t *v = smem + (2 + st) * kTileBytes16 + r * 128;
                    const bool behind = key0 + r >= w.len;
                    bool odd = false;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        if (i >= 8 && W <= 64) break;
                        uint4 *p = reinterpret_cast<uint4 *>(v + (i / 8) * kHalfBytes + (((i + r) & 7) << 4));
                        if (behind) {
                            *p = make_uint4(0, 0, 0, 0);
                        } else {
                            const uint4 x = *p;
                            const uint32_t u[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
                            for (int e = 0; e < 4; ++e) odd = odd || (u[e] & 0x7F800000u) == 0x7F800000u || (u[e] & 0x7F80u) == 0x7F80u;
                        }
                    }
                    if (odd) sh.poisoned[t] = 1;
                    fence_proxy_async_smem();
                }
            }
            uint32_t u[2][32];
            float x[32], top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            load(0, u[0]);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                tmem_ld_wait_for(u[c & 1]);
                if (c < 3) load(c + 1, u[(c + 1) & 1]);
                settle(c, u[c & 1], x);
#pragma unroll
                for (int e = 0; e < 32; ++e) top[e & 3] = fmaxf(top[e & 3], x[e]);
            }
            load(0, u[0]); // (for the second reading)
            const float peak = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * a.scale;
            if (j == 0) {
                m = peak;
            } else if (__any_sync(0xFFFFFFFFu, peak > m + kRaise)) {
                const float raised = fmaxf(m, peak);
                const float keep = raised == -INFINITY ? 1.0f : exp2_approx(m - raised);
                m = raised;
                l *= keep;
                // (the commit behind this block's scores covers the P V before it: the output is at rest)
#pragma unroll 1
                for (int c = 0; c < W; c += 16) {
                    uint32_t o[16];
                    tmem_ld_32x16(o_col + c, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                    tmem_st_32x16(o_col + c, o);
                }
                tmem_st_wait();
            }
            const float nb = m == -INFINITY ? 0.0f : -m;
            const float2 scale2 = make_float2(a.scale, a.scale), nb2 = make_float2(nb, nb);
            float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
            const float2 *vs = reinterpret_cast<const float2 *>(sh.scales[j % kScaled][1]);
            if (kInt8) {
                const int kv = 2 * j + 1;
                if (!mbar_wait_bounded(smem_u32(&sh.kv_full[kv % kStages]), (kv / kStages) & 1, abort_flag, limit)) {
                    ok = false;
                    break;
                }
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                tmem_ld_wait_for(u[c & 1]);
                if (c < 3) load(c + 1, u[(c + 1) & 1]);
                settle(c, u[c & 1], x);
                uint32_t p[16];
#pragma unroll
                for (int e = 0; e < 32; e += 2) {
                    float2 y = fma2(make_float2(x[e], x[e + 1]), scale2, nb2);
                    y = make_float2(exp2_approx(y.x), exp2_approx(y.y));
                    sum[(e / 2) & 1] = add2(sum[(e / 2) & 1], y);
                    if (kInt8) {
                        const float2 f = vs[c * 16 + e / 2];
                        y.x = masked && x[e] == -INFINITY ? 0.0f : y.x * f.x;
                        y.y = masked && x[e + 1] == -INFINITY ? 0.0f : y.y * f.y;
                    }
                    p[e / 2] = pack_bf16(y.x, y.y);
                }
                tmem_st_32x16(s_col + c * 16, p); // (columns of scores that have been read twice)
            }
            const float2 both = add2(sum[0], sum[1]);
            l += both.x + both.y;
            tmem_st_wait();
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.p_ready[t]));
        }
        if (blocks[t] > 0) ok = ok && mbar_wait_bounded(smem_u32(&sh.o_done[t]), 0, abort_flag, limit);
        tc_fence_after_sync();

        // ---- the result, or this CTA's part of it --------------------------------------------------------------
        float *ws_parts = reinterpret_cast<float *>(reinterpret_cast<char *>(a.workspace) + prompt_counter_bytes());
        const int tile_x = blockIdx.x / args.splits;
        auto part_of = [&](int p) { return ws_parts + (size_t)(tile_x * args.splits + p) * part_floats(W); };
        if (ok) {
            const float inv = parts > 1 ? 1.0f : (l == 0.0f ? 0.0f : 1.0f / l);
            __nv_bfloat16 *dst = a.out + (int64_t)(w.first_token + row / group) * a.out_stride + (w.head * group + row % group) * D;
            float *part = part_of(split) + 2 * kRows + (size_t)(t * kTile + r) * W;
            if (parts > 1) *reinterpret_cast<float2 *>(part_of(split) + 2 * (t * kTile + r)) = make_float2(blocks[t] > 0 ? m : -INFINITY, l);
#pragma unroll 1
            for (int c = 0; c < W; c += 16) {
                uint32_t o[16];
                tmem_ld_32x16(o_col + c, o);
                tmem_ld_wait();
                float x[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = blocks[t] > 0 && l != 0.0f ? __uint_as_float(o[e]) * inv : 0.0f;
                if (parts > 1) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) *reinterpret_cast<float4 *>(part + c + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
                } else if (exists) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4)
                        if (c + e < D) *reinterpret_cast<uint2 *>(dst + c + e) = make_uint2(pack_bf16(x[e], x[e + 1]), pack_bf16(x[e + 2], x[e + 3]));
                }
            }
        }
        if (parts > 1) {
            // the CTA that finishes last joins the parts in their order and leaves the counter at zero
            uint32_t *counter = reinterpret_cast<uint32_t *>(a.workspace) + 2 * tile_x;
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
                for (int i = tid; i < kRows * (W / 4); i += kRows) {
                    const int pr = i / (W / 4), e = i % (W / 4) * 4, rr = w.row0 + pr;
                    if (rr >= w.rows || e >= D) continue;
                    float M = -INFINITY;
                    for (int p = 0; p < parts; ++p) M = fmaxf(M, __ldcg(part_of(p) + 2 * pr));
                    const float ref = M == -INFINITY ? 0.0f : M;
                    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    float L = 0.0f;
                    for (int p = 0; p < parts; ++p) {
                        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(part_of(p) + 2 * pr));
                        const float4 v = __ldcg(reinterpret_cast<const float4 *>(part_of(p) + 2 * kRows + (size_t)pr * W + e));
                        const float f = exp2_approx(ml.x - ref);
                        x.x += f * v.x;
                        x.y += f * v.y;
                        x.z += f * v.z;
                        x.w += f * v.w;
                        L += f * ml.y;
                    }
                    const float inv = L == 0.0f ? 0.0f : 1.0f / L;
                    __nv_bfloat16 *dst = a.out + (int64_t)(w.first_token + rr / group) * a.out_stride + (w.head * group + rr % group) * D + e;
                    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(x.x * inv, x.y * inv), pack_bf16(x.z * inv, x.w * inv));
                }
            }
        }
        if (!kInt8) {
            named_barrier(1, kRows);
            if (parts == 1 || sh.is_last) {
                if (sh.poisoned[t])
                    for (int i = warp % 4; i < kTile; i += 4)
                        if (w.row0 + t * kTile + i < w.rows) attend_row(a, w, w.row0 + t * kTile + i, lane);
            }
        }
    }

    // every thread arrives here, also after an expired wait
    tc_fence_before_sync();
    __syncthreads();
    if (*abort_flag) {
        if (tid == 0) atomicExch(a.cache.status, (int32_t)BITLINEAR_ERR_TIMEOUT);
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

template <bool kInt8>
cudaError_t launch(const PromptArgs &p, int ctas, cudaStream_t stream)
{
    static bool ready[64] = {false};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        e = cudaFuncSetAttribute(attend_prompt_kernel<kInt8>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shared<kInt8>::bytes());
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    attend_prompt_kernel<kInt8><<<(unsigned)ctas, kThreads, Shared<kInt8>::bytes(), stream>>>(p);
    return cudaGetLastError();
}

} // namespace

size_t attend_prompt_workspace_bytes(int heads, int kv_heads, int head_dim)
{
    (void)heads;
    (void)kv_heads;
    return align_up(prompt_counter_bytes() + kPromptMaxParts * part_floats(kv_row_width(head_dim)) * 4, 256);
}

cudaError_t launch_attend_prompt(const AttendArgs &a, cudaStream_t stream)
{
    PromptArgs p{};
    p.a = a;
    p.hooks = take_wait_hooks();
    if (!a.cache.k_scale && (!encode_cache_map(&p.k_map, a.cache.k, a.cache) || !encode_cache_map(&p.v_map, a.cache.v, a.cache)))
        return cudaErrorInvalidValue;
    // No more tiles of rows than this can exist: every sequence has at most one that is not full.
    const int64_t group = a.heads / a.cache.kv_heads;
    const int64_t tiles = ((int64_t)a.T * group / kRows + std::min<int64_t>(a.batch.n_seqs, a.T)) * a.cache.kv_heads;
    // With fewer tiles than SMs the keys of a tile are split among several CTAs.
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(16, kPromptMaxParts / std::max<int64_t>(tiles, 1)));
    if (tiles >= sm_count()) p.splits = 1;
    return a.cache.k_scale ? launch<true>(p, (int)(tiles * p.splits), stream) : launch<false>(p, (int)(tiles * p.splits), stream);
}

} // namespace bitlinear
