// Appending to the paged key-value cache with the rotary embedding applied on the way (one launch for q, k and v), and the
// table of angles it reads.
//
// A pair (a, b) of a head becomes (a c - b s, b c + a s) with (c, s) of its position and its place i in the head.  Every
// (token, head) is one group of lanes: 8 lanes with 16-byte pieces where the head is a multiple of 16 elements, a warp with
// 4-byte pieces otherwise (the 100-wide heads of the 3B shape are only 8-byte aligned).  A lane holds both halves of
// its pairs, so nothing but the 8-bit cache's row maximum crosses lanes.
//
// What bounds it: memory (every byte read and written once) for prompts, the launch and one chain of dependent loads
// (length, page number, row) for a decode step.
#include <math.h>

#include "internal.cuh"
#include "kv.cuh"

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
__device__ __forceinline__ void load_piece(const __nv_bfloat16 *p, float (&x)[VEC])
{
    const Piece<VEC> w = *reinterpret_cast<const Piece<VEC> *>(p);
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

// round(127 x / beta), half to even.  y32 is 127 x / beta up to 1e-4 (its few fp32 roundings at magnitude 127), which
// settles all values except those near the middle between two codes; those are divided in double.
__device__ __forceinline__ int code_of(float y32, double x, double beta)
{
    const float c = rintf(y32);
    if (fabsf(fabsf(y32 - c) - 0.5f) > 4e-4f) return (int)c;
    return (int)rint(x * 127.0 / beta);
}

// kRotate: 0 none, 1 pairs half a head apart, 2 adjacent pairs.
template <int VEC, bool kInt8, int kRotate>
__global__ void __launch_bounds__(256) kv_append_kernel(const __grid_constant__ AppendArgs a)
{
    constexpr int kLanes = VEC == 8 ? 8 : 32;
    const int D = a.cache.head_dim, half = D / 2, Hk = a.cache.kv_heads;
    const int tasks = a.heads + 2 * Hk;
    const int64_t group = (int64_t)blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes;
    const int lane = threadIdx.x % kLanes;
    const int64_t t64 = group / tasks;
    const int task = (int)(group - t64 * tasks);
    const int t = (int)t64;
    bool active = t64 < a.T;
    int b = -1, first = 0, count = 0, pos = -1;
    if (active) b = kv_sequence_of(a.batch, t, first, count);
    if (b >= 0) pos = a.batch.kv_lens[b] - count + (t - first);
    active = active && b >= 0 && pos >= 0;
    if (active && (pos >= a.batch.capacity || (kRotate != 0 && pos >= a.rope_positions))) {
        kv_report(a.cache);
        active = false;
    }
    const bool is_q = task < a.heads;
    const bool is_k = !is_q && task < a.heads + Hk;
    const int h = is_q ? task : (task - a.heads) % Hk;
    int row = -1;
    if (active && !is_q) {
        const int page = kv_page(a.cache, a.batch, b, pos);
        if (page < 0)
            kv_report(a.cache);
        else
            row = kv_row(a.cache, page, h, pos);
    }
    const bool mine = lane * 2 * VEC < D;
    const int o0 = kRotate == 2 ? lane * 2 * VEC : lane * VEC;
    const int o1 = kRotate == 2 ? o0 + VEC : half + lane * VEC;
    const __nv_bfloat16 *src = is_q ? a.q + t64 * a.q_stride : (is_k ? a.k + t64 * a.k_stride : a.v + t64 * a.v_stride);
    const bool work = active && mine && (is_q || row >= 0);
    float x0[VEC] = {}, x1[VEC] = {};
    float2 cs[VEC] = {};
    const bool rotate = kRotate != 0 && !(task >= a.heads + Hk);
    if (work) {
        load_piece<VEC>(src + h * D + o0, x0);
        load_piece<VEC>(src + h * D + o1, x1);
        if (rotate) {
            const float4 *p = reinterpret_cast<const float4 *>(a.rope + (int64_t)pos * half + lane * VEC);
#pragma unroll
            for (int i = 0; i < VEC / 2; ++i) {
                const float4 w = p[i];
                cs[2 * i] = make_float2(w.x, w.y);
                cs[2 * i + 1] = make_float2(w.z, w.w);
            }
        }
    }
    // the j-th pair of this lane: (x0[j], x1[j]), or two neighbours
    auto first_of = [&](int j) -> float & { return kRotate == 2 ? (j < VEC / 2 ? x0[2 * j] : x1[2 * j - VEC]) : x0[j]; };
    auto second_of = [&](int j) -> float & { return kRotate == 2 ? (j < VEC / 2 ? x0[2 * j + 1] : x1[2 * j + 1 - VEC]) : x1[j]; };

    if (!kInt8 || is_q) {
        if (rotate) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float p = first_of(j), r = second_of(j);
                first_of(j) = p * cs[j].x - r * cs[j].y;
                second_of(j) = r * cs[j].x + p * cs[j].y;
            }
        }
        if (work) {
            __nv_bfloat16 *dst = is_q ? a.q_out + t64 * a.q_out_stride + h * D
                                      : reinterpret_cast<__nv_bfloat16 *>(is_k ? a.cache.k : a.cache.v) + (int64_t)row * a.cache.width;
            store_piece<VEC>(dst + o0, x0);
            store_piece<VEC>(dst + o1, x1);
        }
        if (!kInt8 && row >= 0 && lane < a.cache.width - D)
            reinterpret_cast<__nv_bfloat16 *>(is_k ? a.cache.k : a.cache.v)[(int64_t)row * a.cache.width + D + lane] = __float2bfloat16(0.0f);
    }
    if (kInt8) {
        // every lane of the warp takes part in the shuffles, whatever its group does
        double z0[VEC], z1[VEC], top = 0.0;
        bool finite = true;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            double p = first_of(j), r = second_of(j);
            if (rotate) {
                const double c = cs[j].x, s = cs[j].y, u = p * c - r * s;
                r = r * c + p * s;
                p = u;
            }
            z0[j] = p;
            z1[j] = r;
            finite = finite && fabs(p) <= 1e300 && fabs(r) <= 1e300;
            top = fmax(top, fmax(fabs(p), fabs(r)));
        }
#pragma unroll
        for (int d = 1; d < kLanes; d <<= 1) {
            top = fmax(top, __shfl_xor_sync(0xFFFFFFFFu, top, d));
            finite = __shfl_xor_sync(0xFFFFFFFFu, (int)finite, d) && finite;
        }
        if (!is_q && row >= 0) {
            const double beta = fmax(top, 1e-5);
            const float inv = 127.0f / (float)beta;
            int8_t c0[VEC], c1[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const int p = finite ? code_of((float)z0[j] * inv, z0[j], beta) : 0;
                const int r = finite ? code_of((float)z1[j] * inv, z1[j], beta) : 0;
                if (kRotate == 2) {
                    if (j < VEC / 2) {
                        c0[2 * j] = (int8_t)p;
                        c0[2 * j + 1] = (int8_t)r;
                    } else {
                        c1[2 * j - VEC] = (int8_t)p;
                        c1[2 * j + 1 - VEC] = (int8_t)r;
                    }
                } else {
                    c0[j] = (int8_t)p;
                    c1[j] = (int8_t)r;
                }
            }
            int8_t *dst = reinterpret_cast<int8_t *>(is_k ? a.cache.k : a.cache.v) + (int64_t)row * a.cache.width;
            if (mine) {
                if (VEC == 8) {
                    uint2 w0, w1;
                    memcpy(&w0, c0, 8);
                    memcpy(&w1, c1, 8);
                    *reinterpret_cast<uint2 *>(dst + o0) = w0;
                    *reinterpret_cast<uint2 *>(dst + o1) = w1;
                } else {
                    *reinterpret_cast<char2 *>(dst + o0) = make_char2(c0[0], c0[1]);
                    *reinterpret_cast<char2 *>(dst + o1) = make_char2(c1[0], c1[1]);
                }
            }
            if (lane < a.cache.width - D) dst[D + lane] = 0;
            if (lane == 0) (is_k ? a.cache.k_scale : a.cache.v_scale)[row] = finite ? (float)(beta / 127.0) : __int_as_float(0x7FFFFFFF);
        }
    }
}

template <int VEC, bool kInt8>
cudaError_t launch_append(const AppendArgs &a, cudaStream_t stream)
{
    const int64_t groups = (int64_t)a.T * (a.heads + 2 * a.cache.kv_heads);
    const int per_block = 256 / (VEC == 8 ? 8 : 32);
    const unsigned blocks = (unsigned)((groups + per_block - 1) / per_block);
    if (!a.rope)
        kv_append_kernel<VEC, kInt8, 0><<<blocks, 256, 0, stream>>>(a);
    else if (!a.interleaved)
        kv_append_kernel<VEC, kInt8, 1><<<blocks, 256, 0, stream>>>(a);
    else
        kv_append_kernel<VEC, kInt8, 2><<<blocks, 256, 0, stream>>>(a);
    return cudaGetLastError();
}

} // namespace

cudaError_t launch_rope_table(float *table, int64_t n_pos, int head_dim, double base, cudaStream_t stream)
{
    const int64_t n = n_pos * (head_dim / 2);
    rope_table_kernel<<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(reinterpret_cast<float2 *>(table), n, head_dim / 2, base);
    return cudaGetLastError();
}

cudaError_t launch_kv_append(const AppendArgs &a, cudaStream_t stream)
{
    // 16-byte pieces need halves of a head that are multiples of 8 elements
    const bool wide = a.cache.head_dim % 16 == 0;
    if (a.cache.k_scale) return wide ? launch_append<8, true>(a, stream) : launch_append<2, true>(a, stream);
    return wide ? launch_append<8, false>(a, stream) : launch_append<2, false>(a, stream);
}

} // namespace bitlinear
