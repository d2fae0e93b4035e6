// The residual's addition, RMSNorm and the result in blocks of 32 e4m3 elements (mx.cuh), one pass over the row:
//   h = x + delta (rounded to x's type),  n = h / sqrt(mean(h^2) + eps) * gamma,  q, s = blocks of n.
// A row is one CTA, eight elements a thread, kept in registers between the sum of squares and the quantisation, so HBM sees every byte
// once; the sum is held in f32 (eight terms a thread, then a tree).
#include "mx.cuh"

namespace cs {

namespace {

template <typename T> __device__ __forceinline__ void load_row8(const T *p, float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        uint4 u;
        asm volatile("ld.global.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "l"(p));
        Chunk<__nv_bfloat16>::widen(u, v);
    } else {
        const float4 a = ld_dep4(p), b = ld_dep4(p + 4);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}
template <typename T> __device__ __forceinline__ void store_row8(T *p, const float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        __nv_bfloat162 o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
        *reinterpret_cast<uint4 *>(p) = *reinterpret_cast<const uint4 *>(o);
    } else {
        reinterpret_cast<float4 *>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
        reinterpret_cast<float4 *>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// x_out may be x.  d / 8 threads, rounded up to whole warps.  CTAs behind the last row clear the scales of the rows that its tile of 128 has left over.
template <typename TX, typename TD> __global__ void __launch_bounds__(1024)
mx_norm_kernel(const TX *x, const TD *delta, const float *__restrict__ gamma, int B, int d, float eps, TX *x_out, float *n_out, uint8_t *q, uint8_t *s) {
    __shared__ float part[32];
    const int kblocks = d >> 7;
    if ((int)blockIdx.x >= B) {
        pdl_launch_dependents();
        pdl_wait();
        const int quarter = blockIdx.x - B, tile = (B - 1) >> 7;      // 32 rows of the last tile
        for (int i = threadIdx.x; i < 32 * kblocks; i += blockDim.x) {
            const int r = i & 31;
            if (tile * 128 + quarter * 32 + r >= B)
                reinterpret_cast<uint32_t *>(s + ((size_t)tile * kblocks + (i >> 5)) * kMxTileBytes)[r * 4 + quarter] = 0;
        }
        return;
    }
    const int t = threadIdx.x, row = blockIdx.x;
    const bool in = t * 8 < d;
    const size_t at = (size_t)row * d + t * 8;
    float g[8], h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) { g[j] = 1.f; h[j] = 0.f; }
    if (in && gamma != nullptr) {
        const float4 a = __ldg(reinterpret_cast<const float4 *>(gamma) + 2 * t), b = __ldg(reinterpret_cast<const float4 *>(gamma) + 2 * t + 1);
        g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
    }
    pdl_launch_dependents();
    pdl_wait();
    float sum = 0.f;
    if (in) {
        load_row8(x + at, h);
        if (delta != nullptr) {
            float a[8];
            load_row8(delta + at, a);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                h[j] += a[j];
                if (sizeof(TX) == 2) h[j] = __bfloat162float(__float2bfloat16_rn(h[j]));   // the norm is that of the stored residual
            }
        }
        if (x_out != nullptr) store_row8(x_out + at, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(h[j], h[j], sum);
    }
    sum = warp_sum(sum);
    const int warps = blockDim.x >> 5;
    if ((t & 31) == 0) part[t >> 5] = sum;
    __syncthreads();
    sum = warp_sum((t & 31) < warps ? part[t & 31] : 0.f);
    const float rstd = 1.f / sqrtf(sum / (float)d + eps);
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) { h[j] = h[j] * rstd * g[j]; m = max(m, abs_bits(h[j])); }
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t byte = mx_scale_byte<true>(m);
    const float inv = mx_inverse(byte);
    // the four scales of 128 columns are one word of the tile
    uint32_t word = byte << (8 * ((t >> 2) & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    if (!in) return;
    if (n_out != nullptr) store_row8(n_out + at, h);
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = byte == 255 ? 0.f : h[j] * inv;
    *reinterpret_cast<uint2 *>(q + at) = make_uint2(pack_e4m3(h[0], h[1], h[2], h[3]), pack_e4m3(h[4], h[5], h[6], h[7]));
    if ((t & 15) == 0)
        reinterpret_cast<uint32_t *>(s + ((size_t)(row >> 7) * kblocks + (t >> 4)) * kMxTileBytes)[(row & 31) * 4 + ((row & 127) >> 5)] = word;
}

}  // namespace

cs_status launch_mx_norm(cs_plan *plan, const void *x, int x_dtype, const void *delta, int delta_dtype, const float *gamma, int B,
                         void *x_out, float *n_out, uint8_t *q, uint8_t *s, cudaStream_t st) {
    const int d = plan->cfg.d;
    const dim3 grid(B + (B % 128 != 0 ? 4 : 0)), block((d / 8 + 31) / 32 * 32);
    cudaError_t e;
    auto go = [&](auto tx, auto td) {
        using TX = decltype(tx);
        using TD = decltype(td);
        e = launch_pdl(true, mx_norm_kernel<TX, TD>, grid, block, 0, st, static_cast<const TX *>(x), static_cast<const TD *>(delta), gamma, B, d,
                       plan->cfg.rms_eps, static_cast<TX *>(x_out), n_out, q, s);
    };
    if (x_dtype == CS_F32) {
        if (delta_dtype == CS_F32) go(0.f, 0.f); else go(0.f, __nv_bfloat16());
    } else {
        if (delta_dtype == CS_F32) go(__nv_bfloat16(), 0.f); else go(__nv_bfloat16(), __nv_bfloat16());
    }
    if (e != cudaSuccess) return record_cuda(plan, e, "mx_norm_kernel");
    plan->launches += 1;
    return CS_OK;
}

}  // namespace cs
