// Softmax attention over the paged key-value cache: out = sum_j p_j v_j, p = softmax_j(scale q . k_j), one pass over the
// keys with the running maximum m and sum l of the softmax:
//   m' = max(m, s_j),  l' = l 2^(m - m') + 2^(s_j - m'),  o' = o 2^(m - m') + 2^(s_j - m') v_j,
// with scores in units of log2 (the scale carries log2 e).
//
// The simplest form that is right for every case: one warp per (token, head), four elements of the head per lane.
#include "internal.cuh"
#include "kv.cuh"

namespace bitlinear {
namespace {

template <bool kInt8>
__device__ __forceinline__ float4 load_row(const void *pool, const float *scale, int64_t row, int width, int lane, bool mine)
{
    float4 x = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (!mine) return x;
    if (kInt8) {
        const char4 c = *reinterpret_cast<const char4 *>(reinterpret_cast<const int8_t *>(pool) + row * width + 4 * lane);
        const float s = scale[row];
        x = make_float4(c.x * s, c.y * s, c.z * s, c.w * s);
    } else {
        const uint2 w = *reinterpret_cast<const uint2 *>(reinterpret_cast<const __nv_bfloat16 *>(pool) + row * width + 4 * lane);
        x = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                        __uint_as_float(w.y & 0xFFFF0000u));
    }
    return x;
}

template <bool kInt8>
__global__ void __launch_bounds__(128) attend_rows_kernel(const __grid_constant__ AttendArgs a)
{
    const int64_t unit = (int64_t)blockIdx.x * 4 + threadIdx.x / 32;
    const int lane = threadIdx.x % 32;
    const int64_t t = unit / a.heads;
    const int h = (int)(unit - t * a.heads);
    if (t >= a.T) return;
    int first, count;
    const int b = kv_sequence_of(a.batch, (int)t, first, count);
    if (b < 0) return;
    bool over;
    const int len = kv_length(a.batch, b, over);
    if (over && lane == 0) kv_report(a.cache);
    int end = a.batch.kv_lens[b] - count + ((int)t - first) + 1;
    end = end > len ? len : end;
    const int D = a.cache.head_dim, kvh = h / (a.heads / a.cache.kv_heads);
    const bool mine = 4 * lane < D;
    float4 q = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (mine) {
        const uint2 w = *reinterpret_cast<const uint2 *>(a.q + t * a.q_stride + h * D + 4 * lane);
        q = make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16),
                        __uint_as_float(w.y & 0xFFFF0000u));
    }
    float m = -INFINITY, l = 0.0f;
    float4 o = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    for (int j = 0; j < end; ++j) {
        const int page = kv_page(a.cache, a.batch, b, j);
        if (page < 0) {
            if (lane == 0) kv_report(a.cache);
            continue;
        }
        const int64_t row = kv_row(a.cache, page, kvh, j);
        const float4 k = load_row<kInt8>(a.cache.k, a.cache.k_scale, row, a.cache.width, lane, mine);
        const float4 v = load_row<kInt8>(a.cache.v, a.cache.v_scale, row, a.cache.width, lane, mine);
        float s = q.x * k.x + q.y * k.y + q.z * k.z + q.w * k.w;
#pragma unroll
        for (int d = 16; d; d >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, d);
        s *= a.scale;
        const float mn = fmaxf(m, s);
        if (mn == -INFINITY) continue;
        const float keep = exp2f(m - mn), p = exp2f(s - mn);
        l = l * keep + p;
        o = make_float4(o.x * keep + p * v.x, o.y * keep + p * v.y, o.z * keep + p * v.z, o.w * keep + p * v.w);
        m = mn;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (mine) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(o.x * inv, o.y * inv), y = __floats2bfloat162_rn(o.z * inv, o.w * inv);
        uint2 w;
        w.x = *reinterpret_cast<const uint32_t *>(&x);
        w.y = *reinterpret_cast<const uint32_t *>(&y);
        *reinterpret_cast<uint2 *>(a.out + t * a.out_stride + h * D + 4 * lane) = w;
    }
}

} // namespace

size_t attend_prompt_workspace_bytes(int heads, int kv_heads, int head_dim)
{
    (void)heads;
    (void)kv_heads;
    (void)head_dim;
    return 256;
}

cudaError_t launch_attend_prompt(const AttendArgs &a, cudaStream_t stream)
{
    const int64_t units = (int64_t)a.T * a.heads;
    const unsigned blocks = (unsigned)((units + 3) / 4);
    if (a.cache.k_scale)
        attend_rows_kernel<true><<<blocks, 128, 0, stream>>>(a);
    else
        attend_rows_kernel<false><<<blocks, 128, 0, stream>>>(a);
    return cudaGetLastError();
}

} // namespace bitlinear
