// Appending to the paged key-value cache with the rotary embedding applied on the way (one launch for q, k and v), and the
// table of angles it reads.
//
// A pair (a, b) of a head becomes (a c - b s, b c + a s) with (c, s) of its position and its place i in the head.  Every
// (token, head) is one group of lanes: 8 lanes with 16-byte pieces where the head is a multiple of 16 elements, a warp with
// 4-byte pieces otherwise (the 100-wide heads of the 3B shape are only 8-byte aligned).  A lane holds both halves of
// its pairs, so nothing but the 8-bit cache's row maximum crosses lanes.  A warp serves one token: its sequence, position, page
// and angles are looked up once, and its groups walk the token's heads; with few tokens several warps share a token.  The warps
// of a CTA may serve different tokens.
//
// 8 bits: code = round(127 x / beta) has to come out as in exact arithmetic, also for values half way between two codes.  All is
// done in fp32 first; the few elements that fp32 cannot settle (candidates for the row's maximum, quotients near the
// middle between two codes) are computed again in double from memory.  Codes are rounded by adding 1.5 2^23, which leaves them in the
// low bytes of the sums (conversions go through a unit a quarter as wide: 2436 tokens, 40/40 heads: 52 -> 46 us with it).
//
// What bounds it: memory (every byte read and written once) for prompts, the launch and one chain of dependent loads
// (length, page number, row) for a decode step.  Measured (without the norm): 4096 tokens, 64/8 heads of 128: 32.2 us = 5.3 TB/s (0.80 of a copy's
// rate); heads of 100, 32/32 of them: 57 us = 2.8 TB/s, held by the 4-byte accesses; single tokens 8.4 us per call, the time the
// host needs for one; int8, 2436 tokens, 40/40 heads: 46 us = 2.8 TB/s: issue slots 66 % busy (row maxima, quotients and the test
// that settles each code), not at a limit.  Registers: nothing is spilled but 4 bytes in the rotating int8 form of 4-byte pieces.
//
// The form that normalises: y = x g r, r = 1 / sqrt(max(mean x^2 + eps, 2^-126)), the squares summed in fp32 over a group's lanes (four
// heads of a warp at a time where a head takes all lanes: one root for each, and half the shuffles).  4096 tokens, 64/8 heads of 128:
// 36.7 us = 4.6 TB/s (0.71 of a copy's rate), 27 million instructions where the form without has 17; heads of 100, 32/32 of them: 87
// us (56 without), 76 million instructions where 50 are without, issue slots 78 % busy; int8, 2436 tokens, 40/40 heads: 65 us (48),
// 41 million for 31, issue slots 66 % busy with three CTAs; a single token, 32/32 heads of 100: 5.0 us on the GPU (3.7), 10.7 per call (8.4).
#include <math.h>

#include <algorithm>

#include "internal.cuh"
#include "kv.cuh"
#include "ptx.cuh"

namespace bitlinear {
namespace {

__global__ void __launch_bounds__(256) rope_table_kernel(float2 *table, int64_t n, int half, double base)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    const int64_t pos = i / half;
    const int e = (int)(i - pos * half);
    const double angle = (double)pos * pow(base, -(double)e / (double)half);
    double s, c;
    sincos(angle, &s, &c);
    table[i] = make_float2((float)c, (float)s);
}

template <int VEC>
struct Piece; // VEC bf16 elements as one access
template <>
struct Piece<8> {
    uint4 w;
};
template <>
struct Piece<2> {
    uint32_t w;
};

template <int VEC>
__device__ __forceinline__ void unpack(const Piece<VEC> &w, float (&x)[VEC])
{
    const uint32_t *u = reinterpret_cast<const uint32_t *>(&w);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
}

template <int VEC>
__device__ __forceinline__ void store_piece(__nv_bfloat16 *p, const float (&x)[VEC])
{
    Piece<VEC> w;
    uint32_t *u = reinterpret_cast<uint32_t *>(&w);
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    *reinterpret_cast<Piece<VEC> *>(p) = w;
}

// Two products, or two products and sums, at a time.
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
        "fma.rn.f32x2 x, x, y, z;\n\tmov.b64 {%0, %1}, x;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

// The largest magnitude of three, or NaN if one of them is.
__device__ __forceinline__ float largest(float x, float y, float z)
{
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
    return m;
}

// Heads that a group of lanes takes at a time.  With 4-byte pieces four heads' loads have to be in flight to hide the
// memory's latency (4096 tokens, 32/32 heads of 100: one at a time 74 us, two or four 57, eight 66); with 16-byte pieces the
// registers are worth more as warps (64/8 heads of 128: one 32 us, two 38).  An 8-bit row works on more values: one.
template <int VEC, bool kInt8>
constexpr int kHeadsAtATime = VEC == 2 && !kInt8 ? 4 : 1;

// Three CTAs per SM for the 8-bit rows of 16-byte pieces: their values need 80 registers (four CTAs, with spills: 4 us more).
// kRotate: 0 none, 1 pairs half a head apart, 2 adjacent pairs.  kNorm: query and key heads may be normalised first, the
// positions of the angles may be the caller's, and rows may be marked.
template <int VEC, bool kInt8, int kRotate, bool kNorm>
__global__ void __launch_bounds__(256, kInt8 && VEC == 8 ? 3 : 4) kv_append_kernel(const __grid_constant__ AppendArgs a, const int shares) // warps per token
{
    ptx::griddep_wait(); // everything below is read from memory that the launch before this one may have written
    ptx::griddep_launch_dependents();
    constexpr int kLanes = VEC == 8 ? 8 : 32, kGroups = 32 / kLanes; // of a warp
    constexpr int kBatch = kHeadsAtATime<VEC, kInt8>;
    const int D = a.cache.head_dim, half = D / 2, Hk = a.cache.kv_heads;
    const int tasks = a.heads + 2 * Hk; // query heads, key heads, value heads
    const int warp = blockIdx.x * 8 + threadIdx.x / 32, t = warp / shares, share = warp - t * shares;
    const int lane = threadIdx.x % kLanes, group = threadIdx.x % 32 / kLanes;
    if (t >= a.T) return;

    // rows that the caller did not hand over (those of the same sequence that exist are stored)
    if (a.batch.cu_tokens && ((t == 0 && a.batch.cu_tokens[0] < 0) || (t == a.T - 1 && a.batch.cu_tokens[a.batch.n_seqs] > a.T))) kv_report(a.cache);
    int first, count;
    const int b = kv_sequence_of(a.batch, t, first, count);
    if (b < 0) return;
    const int pos = a.batch.kv_lens[b] - count + (t - first);
    if (pos < 0) return;
    const int angle_pos = kNorm && a.positions ? a.positions[t] : pos;
    if (pos >= a.batch.capacity || (kRotate != 0 && (angle_pos >= a.rope_positions || (kNorm && angle_pos < 0)))) {
        kv_report(a.cache);
        return;
    }
    const int page = kv_page(a.cache, a.batch, b, pos);
    if (page < 0) kv_report(a.cache);

    const bool mine = lane * 2 * VEC < D;
    const int o0 = kRotate == 2 ? lane * 2 * VEC : lane * VEC;
    const int o1 = kRotate == 2 ? o0 + VEC : half + lane * VEC;
    float2 cs[VEC] = {};
    // Whether gains and angles are multiplied with each other once: for the few elements of a lane with 4-byte pieces (4096 tokens, 32/32
    // heads of 100: 109 -> 87 us).  16-byte pieces would hold twice the registers for it, or load the factors as often (64/8 heads of
    // 128: 36.7 us with gains loaded for every head and four CTAs, 43 with products held and three).
    constexpr bool kFold = kNorm && VEC == 2 && !kInt8;
    if (!kFold && kRotate != 0 && mine) {
        const float4 *p = reinterpret_cast<const float4 *>(a.rope + (int64_t)angle_pos * half + lane * VEC);
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const float4 w = p[i];
            cs[2 * i] = make_float2(w.x, w.y);
            cs[2 * i + 1] = make_float2(w.z, w.w);
        }
    }
    // every lane of a warp goes through the same rounds (the 8-bit row maximum is a shuffle)
    auto source = [&](int task) {
        const int h = task < a.heads ? task : (task < a.heads + Hk ? task - a.heads : task - a.heads - Hk);
        return (task < a.heads ? a.q + (int64_t)t * a.q_stride
                               : (task < a.heads + Hk ? a.k + (int64_t)t * a.k_stride : a.v + (int64_t)t * a.v_stride)) + h * D;
    };
    auto works = [&](int task) { return task < tasks && mine && (task < a.heads || page >= 0); };
    Piece<VEC> next0[kBatch] = {}, next1[kBatch] = {};
    auto prefetch = [&](int first_task) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int task = first_task + u * kGroups;
            if (!works(task)) continue;
            const __nv_bfloat16 *src = source(task);
            next0[u] = *reinterpret_cast<const Piece<VEC> *>(src + o0);
            next1[u] = *reinterpret_cast<const Piece<VEC> *>(src + o1);
        }
    };
    // Normalised forms: an element becomes own_factor times itself and other_factor times its partner in the rotation, which are
    // products of the gain and the angle's cosine and sine, as pairs of neighbours.  They are those of queries or of keys.
    int held = 0;
    float2 own_factor[kFold ? VEC : 1], other_factor[kFold && kRotate != 0 ? VEC : 1];
    auto make_factors = [&](const float *gain) {
        if constexpr (kFold) {
            auto gain_at = [&](int e) { return gain ? *reinterpret_cast<const float2 *>(gain + e) : make_float2(1.0f, 1.0f); };
            const float2 *angles = a.rope + (int64_t)angle_pos * half;
#pragma unroll
            for (int p = 0; p < VEC; ++p) {
                const int e = p < VEC / 2 ? o0 + 2 * p : o1 + 2 * p - VEC; // and its neighbour
                const float2 g = gain_at(e);
                if constexpr (kRotate == 0) {
                    own_factor[p] = g;
                } else if constexpr (kRotate == 1) {
                    const int i = lane * VEC + (p < VEC / 2 ? 2 * p : 2 * p - VEC);
                    const float4 w = *reinterpret_cast<const float4 *>(angles + i); // (c, s) of the two
                    const float2 of = gain_at(p < VEC / 2 ? o1 + 2 * p : o0 + 2 * p - VEC);
                    own_factor[p] = make_float2(g.x * w.x, g.y * w.z);
                    other_factor[p] = p < VEC / 2 ? make_float2(-of.x * w.y, -of.y * w.w) : make_float2(of.x * w.y, of.y * w.w);
                } else {
                    const float2 w = angles[e / 2];
                    own_factor[p] = make_float2(g.x * w.x, g.y * w.x);
                    other_factor[p] = make_float2(-g.y * w.y, g.x * w.y);
                }
            }
        }
    };
    // 1 / rms of the heads that the warp has at hand.
    auto over_rms_of = [&](const Piece<VEC> (&now0)[kBatch], const Piece<VEC> (&now1)[kBatch], float (&r)[kBatch]) {
        auto squares_of = [&](float unit) { // of one of the heads per lane: kLanes / kBatch neighbours have the same
            float s[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                float x0[VEC], x1[VEC];
                unpack<VEC>(now0[u], x0);
                unpack<VEC>(now1[u], x1);
                float2 sum[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
                const float2 unit2 = make_float2(unit, unit);
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    float2 y = make_float2(x0[i], x0[i + 1]), z = make_float2(x1[i], x1[i + 1]);
                    if (unit != 1.0f) y = mul2(y, unit2), z = mul2(z, unit2);
                    sum[0] = fma2(y, y, sum[0]);
                    sum[1] = fma2(z, z, sum[1]);
                }
                s[u] = mine ? (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y) : 0.0f;
            }
            if constexpr (kBatch == 4) { // each half, then each quarter of the warp keeps the heads that become its own
                const bool upper = lane & 16, odd = lane & 8;
                const float y = (upper ? s[2] : s[0]) + __shfl_xor_sync(0xFFFFFFFFu, upper ? s[0] : s[2], 16);
                const float z = (upper ? s[3] : s[1]) + __shfl_xor_sync(0xFFFFFFFFu, upper ? s[1] : s[3], 16);
                s[0] = (odd ? z : y) + __shfl_xor_sync(0xFFFFFFFFu, odd ? y : z, 8);
            }
#pragma unroll
            for (int d = kLanes / kBatch / 2; d > 0; d >>= 1) s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], d);
            return s[0];
        };
        // (Squares below fp32's range do not matter beside the least mean, 2^-126.  Squares above it: again, in a smaller unit.)
        float squares = squares_of(1.0f), unit = 1.0f;
        if (__any_sync(0xFFFFFFFFu, !(squares <= 3e38f))) {
            const float small = squares_of(0x1p-80f);
            if (!(squares <= 3e38f)) {
                squares = small;
                unit = 0x1p-80f;
            }
        }
        const float mean = squares / (float)D + a.norm_eps * unit * unit;
        const float own = rsqrtf(mean < 0x1p-126f ? 0x1p-126f : mean) * unit; // (a NaN stays one)
#pragma unroll
        for (int u = 0; u < kBatch; ++u) r[u] = kBatch > 1 ? __shfl_sync(0xFFFFFFFFu, own, u * (32 / kBatch)) : own;
    };
    auto serve = [&](const int task, const Piece<VEC> &now0, const Piece<VEC> &now1, const float over_rms) {
        const bool is_q = task < a.heads, is_k = !is_q && task < a.heads + Hk;
        const int h = is_q ? task : (is_k ? task - a.heads : task - a.heads - Hk);
        const bool work = works(task);
        const __nv_bfloat16 *src = source(task);
        float x0[VEC] = {}, x1[VEC] = {};
        if (work) {
            unpack<VEC>(now0, x0);
            unpack<VEC>(now1, x1);
        }
        // the j-th pair of this lane: (x0[j], x1[j]), or two neighbours
        auto first_of = [&](int j) -> float & { return kRotate == 2 ? (j < VEC / 2 ? x0[2 * j] : x1[2 * j - VEC]) : x0[j]; };
        auto second_of = [&](int j) -> float & { return kRotate == 2 ? (j < VEC / 2 ? x0[2 * j + 1] : x1[2 * j + 1 - VEC]) : x1[j]; };
        const float *gain = !kNorm ? nullptr : (is_q ? a.q_gain : (is_k ? a.k_gain : nullptr));
        const bool rotate = kRotate != 0 && (is_q || is_k);
        if (kFold) {
            if (work && (is_q || is_k)) {
                const int kind = is_q ? 1 : 2;
                if (kind != held) {
                    held = kind;
                    make_factors(gain);
                }
                const float r = gain ? over_rms : 1.0f;
                float2 x[VEC];
#pragma unroll
                for (int p = 0; p < VEC; ++p)
                    x[p] = mul2(p < VEC / 2 ? make_float2(x0[2 * p], x0[2 * p + 1]) : make_float2(x1[2 * p - VEC], x1[2 * p + 1 - VEC]), make_float2(r, r));
#pragma unroll
                for (int p = 0; p < VEC; ++p) {
                    // (the partner's product is rounded first, as the form without a norm does it)
                    const float2 y = kRotate == 0 ? mul2(x[p], own_factor[p])
                                                  : fma2(x[p], own_factor[p],
                                                         mul2(kRotate == 1 ? x[p < VEC / 2 ? p + VEC / 2 : p - VEC / 2] : make_float2(x[p].y, x[p].x), other_factor[p]));
                    (p < VEC / 2 ? x0[2 * p] : x1[2 * p - VEC]) = y.x;
                    (p < VEC / 2 ? x0[2 * p + 1] : x1[2 * p + 1 - VEC]) = y.y;
                }
            }
        } else {
            if (kNorm && gain && work) {
                // (An 8-bit row's factor 1 / rms cancels out of its codes: it enters the scale alone.)
                const float f = kInt8 && !is_q ? 1.0f : over_rms;
#pragma unroll
                for (int i = 0; i < VEC; i += 2) {
                    const float2 g0 = *reinterpret_cast<const float2 *>(gain + o0 + i), g1 = *reinterpret_cast<const float2 *>(gain + o1 + i);
                    const float2 y = mul2(mul2(make_float2(x0[i], x0[i + 1]), make_float2(f, f)), g0);
                    const float2 z = mul2(mul2(make_float2(x1[i], x1[i + 1]), make_float2(f, f)), g1);
                    x0[i] = y.x, x0[i + 1] = y.y;
                    x1[i] = z.x, x1[i + 1] = z.y;
                }
            }
            if (kNorm && kRotate == 1 && rotate) {
#pragma unroll
                for (int j = 0; j < VEC; j += 2) {
                    const float2 y = make_float2(x0[j], x0[j + 1]), z = make_float2(x1[j], x1[j + 1]);
                    const float2 c = make_float2(cs[j].x, cs[j + 1].x), n = make_float2(cs[j].y, cs[j + 1].y);
                    const float2 u = mul2(z, n), lo = fma2(y, c, make_float2(-u.x, -u.y)), hi = fma2(z, c, mul2(y, n));
                    x0[j] = lo.x, x0[j + 1] = lo.y;
                    x1[j] = hi.x, x1[j + 1] = hi.y;
                }
            } else if (rotate) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    const float p = first_of(j), r = second_of(j);
                    first_of(j) = p * cs[j].x - r * cs[j].y;
                    second_of(j) = r * cs[j].x + p * cs[j].y;
                }
            }
        }
        const int64_t row = is_q || page < 0 ? 0 : kv_row(a.cache, page, h, pos);
        if (kNorm && a.marks.mass && is_k && page >= 0 && lane == 0) {
            a.marks.mass[row] = 0.0f;
            a.marks.pos[row] = angle_pos;
        }
        if (!kInt8 || is_q) {
            if (work) {
                __nv_bfloat16 *dst = is_q ? a.q_out + (int64_t)t * a.q_out_stride + h * D
                                          : reinterpret_cast<__nv_bfloat16 *>(is_k ? a.cache.k : a.cache.v) + row * a.cache.width;
                store_piece<VEC>(dst + o0, x0);
                store_piece<VEC>(dst + o1, x1);
            }
            if (VEC == 2 && !kInt8 && !is_q && task < tasks && page >= 0 && lane < a.cache.width - D) // (the row's padding)
                reinterpret_cast<__nv_bfloat16 *>(is_k ? a.cache.k : a.cache.v)[row * a.cache.width + D + lane] = __float2bfloat16(0.0f);
        }
        if (kInt8 && task - group + kGroups > a.heads) { // (not for a warp that has queries alone)
            // element i of x0, then of x1, exactly (up to 2^-53; with a gain, whose product with an element is exact, 2^-51)
            auto element = [&](int e) -> double {
                const double x = __bfloat162float(src[e]);
                return kNorm && gain ? x * gain[e] : x;
            };
            auto exact = [&](int i) -> double {
                const int e = i < VEC ? o0 + i : o1 + i - VEC;
                const double x = element(e);
                if (!rotate) return x;
                const int pair = kRotate == 2 ? e >> 1 : (e < half ? e : e - half);
                const bool second = kRotate == 2 ? (e & 1) != 0 : e >= half;
                const float2 w = a.rope[(int64_t)angle_pos * half + pair];
                const double y = element(kRotate == 2 ? e ^ 1 : (second ? e - half : e + half));
                return second ? x * (double)w.x + y * (double)w.y : x * (double)w.x - y * (double)w.y;
            };
            float top = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) top = largest(top, x0[i], x1[i]);
#pragma unroll
            for (int d = 1; d < kLanes; d <<= 1) top = largest(top, __shfl_xor_sync(0xFFFFFFFFu, top, d), 0.0f);
            // The rotated fp32 values are within 2^-22 of the row's maximum of the exact ones (three roundings of a c and b s,
            // |a c| + |b s| <= 2 max; with a gain, two more, 5 2^-24 in all): only those within 2^-20 of the largest can be the exact
            // maximum.  (Near the end of
            // fp32's range, where a rotation may overflow, nothing is settled in fp32.)
            const bool huge = !(top <= 8e37f);
            bool finite = true; // a row that is not finite stays so when it is rotated: such rows are among the huge ones
            if (__any_sync(0xFFFFFFFFu, huge)) {
                bool all = true;
                if (work)
                    for (int i = 0; i < VEC; ++i) {
                        all = all && isfinite(__bfloat162float(src[o0 + i])) && isfinite(__bfloat162float(src[o1 + i]));
                        if (kNorm && gain) all = all && isfinite(gain[o0 + i]) && isfinite(gain[o1 + i]);
                    }
#pragma unroll
                for (int d = 1; d < kLanes; d <<= 1) all = __shfl_xor_sync(0xFFFFFFFFu, (int)all, d) && all;
                finite = all;
            }
            constexpr uint32_t kAll = 2 * VEC == 32 ? ~0u : (1u << (2 * VEC)) - 1u;
            double beta = top;
            // (asked of the whole warp, whose rows may be keys and values: the values of a row that is neither rotated nor
            // multiplied are exact, and so is what comes out here)
            if (__any_sync(0xFFFFFFFFu, rotate || (kNorm && gain != nullptr))) {
                beta = 0.0;
                uint32_t candidates = 0;
#pragma unroll
                for (int i = 0; i < 2 * VEC; ++i) candidates |= (uint32_t)(fabsf(i < VEC ? x0[i] : x1[i - VEC]) >= top * 0.99999905f) << i;
                if (huge) candidates = kAll;
                if (!work || is_q || !finite) candidates = 0;
                const uint32_t holders = __ballot_sync(0xFFFFFFFFu, candidates != 0u) & (kLanes == 32 ? ~0u : 0xFFu << (8 * group)); // lanes of this row
                for (; candidates; candidates &= candidates - 1) beta = fmax(beta, fabs(exact(__ffs(candidates) - 1)));
                if (__any_sync(0xFFFFFFFFu, __popc(holders) > 1)) {
#pragma unroll
                    for (int d = 1; d < kLanes; d <<= 1) beta = fmax(beta, __shfl_xor_sync(0xFFFFFFFFu, beta, d));
                } else {
                    beta = __shfl_sync(0xFFFFFFFFu, beta, holders ? __ffs(holders) - 1 : 0);
                }
            }
            if (is_q || task >= tasks || page < 0) return;
            if (kNorm && gain) {
                if (!((float)beta * over_rms > 1.01e-5f)) beta = fmax(beta, 1e-5 / (double)over_rms);
            } else {
                beta = fmax(beta, 1e-5);
            }
            int8_t *dst = reinterpret_cast<int8_t *>(is_k ? a.cache.k : a.cache.v) + row * a.cache.width;
            if (mine) {
                const float inv = __fdividef(127.0f, (float)beta); // (within 2 ulp up to 2^126 > 8e37)
                // t = 1.5 2^23 + round(x inv): its low byte is the code, and x inv - code is exact but for its last bit.
                // The estimate of 127 x / beta is off by 127 (2^-22 + 2^-22 + 2^-24) < 7e-5 at most (with a gain by 8e-5).
                constexpr float kShift = 12582912.0f, kSettled = 0.4999f;
                auto value = [&](int i) { return i < VEC ? x0[i] : x1[i - VEC]; };
                auto beside = [&](float x, float t) { return fmaf(x, inv, kShift - t); };
                uint32_t t[2 * VEC];
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < 2 * VEC; i += 2) {
                    const float y = fmaf(value(i), inv, kShift), z = fmaf(value(i + 1), inv, kShift);
                    most = largest(most, beside(value(i), y), beside(value(i + 1), z));
                    t[i] = __float_as_uint(y);
                    t[i + 1] = __float_as_uint(z);
                }
                uint32_t unsettled = 0;
                if (huge) {
                    unsettled = finite ? kAll : 0u;
                } else if (most > kSettled) {
#pragma unroll
                    for (int i = 0; i < 2 * VEC; ++i) unsettled |= (uint32_t)(fabsf(beside(value(i), __uint_as_float(t[i]))) > kSettled) << i;
                }
                auto four = [&](int i) { // (a row that is not finite: 0)
                    const uint32_t w = __byte_perm(__byte_perm(t[i], t[i + 1], 0x0040), __byte_perm(t[i + 2], t[i + 3], 0x0040), 0x5410);
                    return finite ? w : 0u;
                };
                if constexpr (VEC == 8) {
                    *reinterpret_cast<uint2 *>(dst + o0) = make_uint2(four(0), four(4));
                    *reinterpret_cast<uint2 *>(dst + o1) = make_uint2(four(8), four(12));
                } else {
                    const uint32_t w = four(0);
                    *reinterpret_cast<uint16_t *>(dst + o0) = (uint16_t)w;
                    *reinterpret_cast<uint16_t *>(dst + o1) = (uint16_t)(w >> 16);
                }
                for (; unsettled; unsettled &= unsettled - 1) {
                    const int i = __ffs(unsettled) - 1;
                    dst[i < VEC ? o0 + i : o1 + i - VEC] = (int8_t)(int)rint(exact(i) * 127.0 / beta);
                }
            }
            if (VEC == 2 && lane < a.cache.width - D) dst[D + lane] = 0;
            if (lane == 0) {
                // beta / 127 is within 2^-52 of this product, so it rounds to the same fp32 number unless that lies within a few
                // units of the middle between two
                double scale = beta * (1.0 / 127.0);
                if (kNorm && gain) scale *= (double)over_rms;
                const int below = (int)(__double_as_longlong(scale) & 0x1FFFFFFF) - 0x10000000;
                if (below >= -8 && below <= 8 && !(kNorm && gain)) scale = beta / 127.0;
                (is_k ? a.cache.k_scale : a.cache.v_scale)[row] = finite ? (float)scale : __int_as_float(0x7FFFFFFF);
            }
        }
    };

    const int step = shares * kGroups * kBatch;
    prefetch(share * kGroups * kBatch + group);
    for (int round = share * kGroups * kBatch; round < tasks; round += step) {
        Piece<VEC> now0[kBatch], now1[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            now0[u] = next0[u];
            now1[u] = next1[u];
        }
        prefetch(round + step + group);
        float factor[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) factor[u] = 1.0f;
        if (kNorm && (a.q_gain || a.k_gain)) over_rms_of(now0, now1, factor);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) serve(round + u * kGroups + group, now0[u], now1[u], factor[u]);
    }
}

template <int VEC, bool kInt8, bool kNorm>
cudaError_t launch_append(const AppendArgs &a, cudaStream_t stream)
{
    // Warps per token: one round of heads per warp while that does not make more warps than the GPU holds.
    const int groups = (VEC == 8 ? 4 : 1) * kHeadsAtATime<VEC, kInt8>, rounds = (a.heads + 2 * a.cache.kv_heads + groups - 1) / groups;
    const int shares = std::max(1, std::min(rounds, 64 * sm_count() / a.T));
    const unsigned blocks = (unsigned)(((int64_t)a.T * shares + 7) / 8);
    return launch_dependent(!a.rope ? kv_append_kernel<VEC, kInt8, 0, kNorm>
                                    : (!a.interleaved ? kv_append_kernel<VEC, kInt8, 1, kNorm> : kv_append_kernel<VEC, kInt8, 2, kNorm>),
                            blocks, 256, 0, stream, a, shares);
}

template <bool kNorm>
cudaError_t launch_append(const AppendArgs &a, cudaStream_t stream)
{
    // 16-byte pieces need halves of a head that are multiples of 8 elements
    const bool wide = a.cache.head_dim % 16 == 0;
    if (a.cache.k_scale) return wide ? launch_append<8, true, kNorm>(a, stream) : launch_append<2, true, kNorm>(a, stream);
    return wide ? launch_append<8, false, kNorm>(a, stream) : launch_append<2, false, kNorm>(a, stream);
}

} // namespace

cudaError_t launch_rope_table(float *table, int64_t n_pos, int head_dim, double base, cudaStream_t stream)
{
    const int64_t n = n_pos * (head_dim / 2);
    rope_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(reinterpret_cast<float2 *>(table), n, head_dim / 2, base);
    return cudaGetLastError();
}

cudaError_t launch_kv_append(const AppendArgs &a, cudaStream_t stream) { return launch_append<false>(a, stream); }
cudaError_t launch_kv_append_rmsnorm(const AppendArgs &a, cudaStream_t stream) { return launch_append<true>(a, stream); }

} // namespace bitlinear
