// The residual's addition, RMSNorm and the result in blocks of 32 e4m3 elements (mx.cuh), one pass over the row:
//   h = x + delta (rounded to x's type),  n = h / sqrt(mean(h^2) + eps) * gamma,  q, s = blocks of n.
// A row is one pass of one CTA, eight elements a thread, kept in registers between the sum of squares and the quantisation, so HBM sees every byte
// once.  mx_norm_kernel is a CTA per row: one round of latencies, for as many rows as are
// resident at once.  More rows take mx_norm_rows_kernel, whose CTAs stay and have the next rows' bulk copies in flight while they work on one: with a CTA
// per row the loads wait for the row before (2048 rows of 5120 bf16 took 21.5 us; now 18.8 with inputs beyond L2, 3.9 TB/s; f32 26.3).  What bounds it is a
// row's chain of latencies - load, sum, two reductions, a barrier, the scale, the store - with 18 warps to an SM: 31 instructions an element, issued at 2.1 a
// cycle of the 4 that an SM can.
#include "mx_core.cuh"

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

// 1 / sqrt(mean square + eps) as a sum of two floats: the approximate reciprocal root (2^-22) and one Newton step in f64 (2^-43).
struct RowScale { float hi, lo; };
__device__ __forceinline__ RowScale row_scale(double sum, double per, float eps) {      // per: 1 / d
    const double m = sum * per + (double)eps;
    double r = (double)rsqrtf((float)m);
    if (r > 0. && r < 1e30) r = r * (1.5 - 0.5 * m * r * r);      // not where m left the range of f32
    RowScale s;
    s.hi = (float)r;
    s.lo = isfinite(s.hi) ? (float)(r - (double)s.hi) : 0.f;
    return s;
}

// n = h r g with the products' rounding errors carried along, as the odd one of the two floats around the true value (or the value, where it is a float): what
// rounds to fewer bits as the true value does, unless that is within 2^-42 of itself of a middle.
__device__ __forceinline__ float exact_n(float h, float g, RowScale r) {
    const float t = h * r.hi, tl = fmaf(h, r.lo, fmaf(h, r.hi, -t));
    const float u = t * g, ul = fmaf(tl, g, fmaf(t, g, -u));
    const float n = u + ul, left = ul - (n - u);
    const uint32_t bits = __float_as_uint(n);
    if (left == 0.f || (bits & 1) != 0 || n == 0.f || left != left) return n;
    return __uint_as_float((bits ^ __float_as_uint(left)) >> 31 ? bits - 1 : bits + 1);
}

// Eight elements of gamma, chunk c.  An input like x, which the launch ahead may have written: so these are ordinary loads through a pointer that may alias, which
// stay behind the wait.
__device__ __forceinline__ void load_gamma(const float *gamma, int c, bool in, float (&g)[8]) {
    if (gamma != nullptr && in) {
        const float4 a = reinterpret_cast<const float4 *>(gamma)[2 * c], b = reinterpret_cast<const float4 *>(gamma)[2 * c + 1];
        g[0] = a.x; g[1] = a.y; g[2] = a.z; g[3] = a.w; g[4] = b.x; g[5] = b.y; g[6] = b.z; g[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.f;
    }
}

// Eight elements of a row, chunk c, once the row's scale is known; `in`: there are any.  Sixteen neighbouring lanes hold sixteen neighbouring chunks.
// n by single products is within 4 units in the last place.  That decides the 8-bit rounding unless it stands so near a value whose low 19 bits are zero: all middles
// between two e4m3 values under a power of two are such values, and so is the border of the next scale.  There (one element in 60000) the chunk takes
// exact_n.  Without, one element in 300000 went the other way; with exact_n throughout, 2048 rows of 5120 took 23.3 us, with it where it
// counts 21.4.
// `g` holds gamma of this chunk and then of chunk `next`, unless that is negative: loaded as soon as its registers are free, and ahead of the stores, which an ordinary
// load cannot pass (2048 x 5120 bf16, back to back in a graph, 16.3 us; loaded at the start of its own chunk 16.8, with two chunks' registers 19.0).
__device__ __forceinline__ void finish_chunk(float (&h)[8], float (&g)[8], const float *gamma, int next, RowScale r, int d, int row, int c, bool in, float *n_out,
                                             uint8_t *q, uint8_t *s) {
    float n[8];
    bool near = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        n[j] = h[j] * r.hi * g[j];
        near |= ((__float_as_uint(n[j]) + 4) & 0x7ffff) <= 8 && n[j] != 0.f;      // (zeros are exact, and sums of bf16 are often zero)
    }
    const size_t at = (size_t)row * d + c * 8;
    if (next >= 0) load_gamma(gamma, next, in, g);
    if (n_out != nullptr && in) store_row8(n_out + at, n);
    if (near) {
        asm volatile("" ::: "memory");      // a branch, not eight selections
        float again[8];
        load_gamma(gamma, c, in, again);
#pragma unroll
        for (int j = 0; j < 8; ++j) n[j] = exact_n(h[j], again[j], r);
    }
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max_abs(top, n[j]);
    uint32_t m = __float_as_uint(top);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    const uint32_t byte = mx_scale_byte<true>(m);
    const float inv = mx_inverse(byte);
    // the four scales of 128 columns are one word of the tile
    uint32_t word = byte << (8 * ((c >> 2) & 3));
    word |= __shfl_xor_sync(0xffffffffu, word, 4);
    word |= __shfl_xor_sync(0xffffffffu, word, 8);
    if (!in) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) n[j] *= inv;
    uint2 v = make_uint2(pack_e4m3(n[0], n[1], n[2], n[3]), pack_e4m3(n[4], n[5], n[6], n[7]));
    if (byte == 255) v = make_uint2(0, 0);
    *reinterpret_cast<uint2 *>(q + at) = v;
    if ((c & 15) == 0)
        reinterpret_cast<uint32_t *>(s + ((size_t)(row >> 7) * (d >> 7) + (c >> 4)) * kMxTileBytes)[(row & 31) * 4 + ((row & 127) >> 5)] = word;
}
// h += delta, rounded to the residual's type: the norm is that of the stored residual.
template <typename TX> __device__ __forceinline__ void add_delta(float (&h)[8], const float (&a)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        h[j] += a[j];
        if (sizeof(TX) == 2) h[j] = __bfloat162float(__float2bfloat16_rn(h[j]));
    }
}
__device__ __forceinline__ uint32_t add_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// In f64 from the first product on: where a few channels hold most of the sum, their f32 squares alone move the row's scale by 2^-23, and with it the roundings
// next to a middle.  (2048 x 5120 bf16 back to back 17.0 us; f32 within a thread 16.4, f32 with the lost parts carried along 18.2.)
__device__ __forceinline__ double squares(const float (&h)[8]) {
    double a = 0., b = 0.;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        a = fma((double)h[j], (double)h[j], a);
        b = fma((double)h[j + 1], (double)h[j + 1], b);
    }
    return a + b;
}
__device__ __forceinline__ double warp_sum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// A quarter (32 rows) of the last tile of scales: zeros in the rows from B on.
__device__ __forceinline__ void clear_scales(uint8_t *s, int B, int kblocks, int quarter) {
    const int tile = (B - 1) >> 7;
    for (int i = threadIdx.x; i < 32 * kblocks; i += blockDim.x) {
        const int r = i & 31;
        if (tile * 128 + quarter * 32 + r >= B)
            reinterpret_cast<uint32_t *>(s + ((size_t)tile * kblocks + (i >> 5)) * kMxTileBytes)[r * 4 + quarter] = 0;
    }
}

// x_out may be x.  d / 8 threads, rounded up to whole warps.  Four CTAs behind the last row clear the scales of rows that its tile of 128 has left over.
template <typename TX, typename TD> __global__ void __launch_bounds__(1024)
mx_norm_kernel(const TX *x, const TD *delta, const float *gamma, int B, int d, double per, float eps, TX *x_out, float *n_out, uint8_t *q, uint8_t *s) {
    __shared__ double part[32];
    const int t = threadIdx.x, row = blockIdx.x;
    if (row >= B) {
        pdl_launch_dependents();
        pdl_wait();
        clear_scales(s, B, d >> 7, row - B);
        return;
    }
    const bool in = t * 8 < d;
    const size_t at = (size_t)row * d + t * 8;
    float g[8], h[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = 0.f;
    pdl_launch_dependents();
    pdl_wait();
    load_gamma(gamma, t, in, g);
    if (in) {
        float a[8];
        load_row8(x + at, h);
        if (delta != nullptr) { load_row8(delta + at, a); add_delta<TX>(h, a); }
        if (x_out != nullptr) store_row8(x_out + at, h);
    }
    double sum = warp_sum(squares(h));
    if ((t & 31) == 0) part[t >> 5] = sum;
    __syncthreads();
    sum = warp_sum((t & 31) < (int)(blockDim.x >> 5) ? part[t & 31] : 0.);
    finish_chunk(h, g, gamma, -1, row_scale(sum, per, eps), d, row, t, in, n_out, q, s);
}

constexpr int kNormStages = 8;
struct NormBars {
    uint64_t full[kNormStages];
    uint32_t aborted;
    double part[2][32];
};
template <typename T> __device__ __forceinline__ void read_row8(const uint8_t *p, float (&v)[8]) {
    if constexpr (sizeof(T) == 2) {
        Chunk<__nv_bfloat16>::widen(*reinterpret_cast<const uint4 *>(p), v);
    } else {
        const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
}

// Persistent CTAs: CTA c takes rows c, c + gridDim.x, ...; `stages` rows of x (and delta) are in flight or at work in shared memory.  The barrier of a row's
// sum comes after every thread has read the row, so it also frees the row's place.  E chunks of eight elements a thread, d / (8 E) apart: with four, what a
// thread does once a row (two reductions, the row's scale) is spread over 32 elements (two chunks 21.4 us, four 19.3).
template <typename TX, typename TD, int E> __global__ void __launch_bounds__(1024 / E, E == 4 ? 3 : E)
mx_norm_rows_kernel(const TX *x, const TD *delta, const float *gamma, int B, int d, double per, float eps, TX *x_out, float *n_out, uint8_t *q, uint8_t *s,
                    int stages, DeviceStatus *status) {
    extern __shared__ __align__(128) uint8_t ring_rows[];
    __shared__ NormBars bars;
    const int t = threadIdx.x, step = gridDim.x, apart = d / (8 * E);
    const bool in = t < apart;
    const uint32_t xb = d * sizeof(TX), db = delta != nullptr ? d * sizeof(TD) : 0, bytes = xb + db;
    if (t == 0) {
        for (int i = 0; i < stages; ++i) mbar_init(&bars.full[i], 1);
        bars.aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();
    auto fetch = [&](int row, int stage) {
        uint8_t *to = ring_rows + stage * bytes;
        mbar_expect_tx(&bars.full[stage], bytes);
        bulk_load(to, x + (size_t)row * d, xb, &bars.full[stage]);
        if (db != 0) bulk_load(to + xb, delta + (size_t)row * d, db, &bars.full[stage]);
    };
    if (t == 0)
        for (int i = 0, row = blockIdx.x; i < stages && row < B; ++i, row += step) fetch(row, i);
    if (B % 128 != 0 && (int)blockIdx.x < 4) clear_scales(s, B, d >> 7, blockIdx.x);
    MxRing ring;
    int turn = 0;
    for (int row = blockIdx.x; row < B; row += step, turn ^= 1) {
        const bool ok = mx_wait(&bars.full[ring.stage], ring.phase, &bars.aborted, status);
        const uint8_t *from = ring_rows + ring.stage * bytes;
        float h[E][8];
        double sum = 0.;
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
            for (int j = 0; j < 8; ++j) h[e][j] = 0.f;
            if (ok && in) {
                const int c = t + e * apart;
                if constexpr (sizeof(TX) == 2 && sizeof(TD) == 2) {      // one addition and one rounding, two at a time
                    uint4 u = *reinterpret_cast<const uint4 *>(from + c * 16);
                    if (db != 0) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(from + xb + c * 16);
                        u = make_uint4(add_bf16x2(u.x, v.x), add_bf16x2(u.y, v.y), add_bf16x2(u.z, v.z), add_bf16x2(u.w, v.w));
                    }
                    if (x_out != nullptr) *reinterpret_cast<uint4 *>(x_out + (size_t)row * d + c * 8) = u;
                    Chunk<__nv_bfloat16>::widen(u, h[e]);
                } else {
                    float a[8];
                    read_row8<TX>(from + c * 8 * sizeof(TX), h[e]);
                    if (db != 0) { read_row8<TD>(from + xb + c * 8 * sizeof(TD), a); add_delta<TX>(h[e], a); }
                    if (x_out != nullptr) store_row8(x_out + (size_t)row * d + c * 8, h[e]);
                }
            }
            sum += squares(h[e]);
        }
        sum = warp_sum(sum);
        if ((t & 31) == 0) bars.part[turn][t >> 5] = sum;
        if (!__syncthreads_and(ok)) {      // a wait gave up: the status word says so
            mx_settle(&bars.aborted);
            return;
        }
        if (t == 0 && row + stages * step < B) fetch(row + stages * step, ring.stage);
        float g[8];
        load_gamma(gamma, t, in, g);
        sum = warp_sum((t & 31) < (int)(blockDim.x >> 5) ? bars.part[turn][t & 31] : 0.);
        const RowScale rstd = row_scale(sum, per, eps);
#pragma unroll
        for (int e = 0; e < E; ++e) finish_chunk(h[e], g, gamma, e + 1 < E ? t + (e + 1) * apart : -1, rstd, d, row, t + e * apart, in, n_out, q, s);
        ring.next(stages);
    }
}

constexpr int kNormRings = 208 * 1024;      // an SM's, over its CTAs

template <typename TX, typename TD> cs_status prepare_rows() {
    for (auto *k : {mx_norm_rows_kernel<TX, TD, 1>, mx_norm_rows_kernel<TX, TD, 2>, mx_norm_rows_kernel<TX, TD, 4>})
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kNormRings) != cudaSuccess || prefer_shared(k) != cudaSuccess)
            return CS_ERR_CUDA;
    return CS_OK;
}

}  // namespace

cs_status prepare_mx_norm() {
    for (cs_status s : {prepare_rows<float, float>(), prepare_rows<float, __nv_bfloat16>(), prepare_rows<__nv_bfloat16, float>(),
                        prepare_rows<__nv_bfloat16, __nv_bfloat16>()})
        if (s != CS_OK) return s;
    return CS_OK;
}

cs_status launch_mx_norm(cs_plan *plan, const void *x, int x_dtype, const void *delta, int delta_dtype, const float *gamma, int B,
                         void *x_out, float *n_out, uint8_t *q, uint8_t *s, cudaStream_t st) {
    const int d = plan->cfg.d;
    const dim3 block((d / 8 + 31) / 32 * 32);
    // One CTA per row while all of them are resident at once.  Beyond, CTAs that stay: as many to an SM as leave each two rows of ring.
    const bool stay = B > plan->sm_count * (2048 / (int)block.x);
    const int row_bytes = d * ((x_dtype == CS_F32 ? 4 : 2) + (delta == nullptr ? 0 : delta_dtype == CS_F32 ? 4 : 2));
    const int each = d % 512 == 0 ? 4 : d % 256 == 0 ? 2 : 1, threads = (d / (8 * each) + 31) / 32 * 32;
    // (four small CTAs: with five 2048 rows of 5120 bf16 took 21.8 us against 19.3)
    const int ctas = max(1, min(min(each == 4 ? 4 : 3, (each == 4 ? 768 : 1024) / threads), kNormRings / (2 * row_bytes)));
    const int stages = min(kNormStages, kNormRings / ctas / row_bytes);
    cudaError_t e;
    auto go = [&](auto tx, auto td) {
        using TX = decltype(tx);
        using TD = decltype(td);
        if (stay)
            e = launch_pdl(true, each == 4 ? mx_norm_rows_kernel<TX, TD, 4> : each == 2 ? mx_norm_rows_kernel<TX, TD, 2> : mx_norm_rows_kernel<TX, TD, 1>,
                           dim3(ctas * plan->sm_count), dim3(threads), (size_t)stages * row_bytes, st, static_cast<const TX *>(x),
                           static_cast<const TD *>(delta), gamma, B, d, 1. / d, plan->cfg.rms_eps, static_cast<TX *>(x_out), n_out, q, s, stages,
                           plan->status);
        else
            e = launch_pdl(true, mx_norm_kernel<TX, TD>, dim3(B + (B % 128 != 0 ? 4 : 0)), block, 0, st, static_cast<const TX *>(x),
                           static_cast<const TD *>(delta), gamma, B, d, 1. / d, plan->cfg.rms_eps, static_cast<TX *>(x_out), n_out, q, s);
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
