// Weights to blocks of four-bit elements and back, and the order in which the FFN kernels read them.  See mx.cuh for the block format.
//
// All of it is bound by HBM: an element is read once (2 or 4 bytes) and written once (17/32 byte), or the reverse.
#include <type_traits>

#include "mx.cuh"

namespace cs {

namespace {

// A const __restrict__ pointer whose plain loads stay behind the wait: the launch ahead may have written what it points at, and through the parameter itself
// they could be taken for loads of constant data and moved ahead of it (see ld_dep).
template <typename T> __device__ __forceinline__ T *behind_wait(T *p) {
    asm volatile("" : "+l"(p)::"memory");
    return p;
}

constexpr int kQThreads = 256;
constexpr int kQUnroll = 4;     // 16- or 32-byte chunks a thread has in flight

template <typename T> __device__ __forceinline__ T narrow(float v);
template <> __device__ __forceinline__ float narrow<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight consecutive elements as they are stored, and what a block needs of them.
template <typename T> struct Eight;
template <> struct Eight<float> {
    float v[8];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 0.f;
    }
    __device__ __forceinline__ void load(const float *p) {
        const float4 a = __ldcs(reinterpret_cast<const float4 *>(p)), b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
    __device__ __forceinline__ void load(const float *p, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < n ? p[i] : 0.f;
    }
    __device__ __forceinline__ uint32_t largest() const {     // magnitude bits; a NaN's or an infinity's are above all others
        uint32_t m = abs_bits(v[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = max(m, abs_bits(v[i]));
        return m;
    }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i];
    }
};
template <> struct Eight<__nv_bfloat16> {
    uint32_t v[4];      // pairs
    __device__ __forceinline__ void zero() { v[0] = v[1] = v[2] = v[3] = 0; }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) {
        const uint4 a = __ldcs(reinterpret_cast<const uint4 *>(p));
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    }
    __device__ __forceinline__ void load(const __nv_bfloat16 *p, int n) {
        const uint16_t *u = reinterpret_cast<const uint16_t *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (2 * i < n ? u[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)u[2 * i + 1] << 16 : 0u);
    }
    __device__ __forceinline__ uint32_t largest() const {
        const uint32_t m = __vmaxu2(__vmaxu2(v[0] & 0x7fff7fffu, v[1] & 0x7fff7fffu), __vmaxu2(v[2] & 0x7fff7fffu, v[3] & 0x7fff7fffu));
        return max(m << 16, m & 0xffff0000u);
    }
    __device__ __forceinline__ void floats(float (&f)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_lo(v[i]); f[2 * i + 1] = bf16_hi(v[i]); }
    }
};

// Eight elements' codes under a scale byte; a block of NaN has zeros.
__device__ __forceinline__ uint32_t codes_of(float (&f)[8], uint32_t byte) {
    const float inv = mx_inverse(byte);
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] *= inv;
    const uint32_t q = pack_e2m1(f);
    return byte == 255 ? 0u : q;
}

// Four threads per block of 32 elements along the rows.  VEC: whole chunks of eight elements, 16-byte aligned.
template <typename T, bool VEC> __global__ void __launch_bounds__(kQThreads)
quantize_rows_kernel(const T *__restrict__ w, int rows, int cols, int64_t ld, uint32_t nb, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    pdl_launch_dependents();
    pdl_wait();
    w = behind_wait(w);
    const uint32_t parts = (uint32_t)rows * nb * 4;      // the host bounds it by 2^31
    const uint32_t base = blockIdx.x * (kQThreads * kQUnroll) + threadIdx.x;
    Eight<T> v[kQUnroll];
#pragma unroll
    for (int u = 0; u < kQUnroll; ++u) {
        const uint32_t i = base + u * kQThreads;
        const uint32_t row = i / (4 * nb), part = i - row * (4 * nb);
        const T *p = w + (int64_t)row * ld + part * 8;
        const int n = i < parts ? cols - (int)part * 8 : 0;
        if (n <= 0) v[u].zero();
        else if (VEC) v[u].load(p);
        else v[u].load(p, n);
    }
#pragma unroll
    for (int u = 0; u < kQUnroll; ++u) {
        const uint32_t i = base + u * kQThreads;
        uint32_t m = v[u].largest();
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
        const uint32_t byte = mx_scale_byte<false>(m);
        float f[8];
        v[u].floats(f);
        if (i < parts) {
            reinterpret_cast<uint32_t *>(codes)[i] = codes_of(f, byte);
            if ((i & 3) == 0) scales[i >> 2] = (uint8_t)byte;
        }
    }
}

// Blocks down the columns, written as rows of the transpose.  A thread takes two columns of 32 rows (no exchange between threads); eight warps stand
// below one another, so that a column's codes leave as 128 contiguous bytes through shared memory.  bf16 pairs stay packed until their scale
// is known: with 32 registers of data instead of 64 twice as many loads are in flight (11008 x 4096 bf16: 21.0 us of 17.4 that its bytes
// take, 56 with floats; f32, whose loads are twice as wide, 34.8 of 31.2; an odd number of bf16 columns, element by element, 85).
constexpr int kTCols = 64, kTBlocks = 8;
template <typename T, bool VEC> __global__ void __launch_bounds__(32 * kTBlocks)
quantize_cols_kernel(const T *__restrict__ w, int rows, int cols, int64_t ld, int nb, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    constexpr bool kPairs = sizeof(T) == 2;
    using Cell = typename std::conditional<kPairs, uint32_t, float2>::type;
    __shared__ uint4 tile[kTCols][kTBlocks + 1];     // the odd pitch spreads a column of 16-byte cells over the banks
    __shared__ uint8_t st[kTCols][kTBlocks];
    pdl_launch_dependents();
    pdl_wait();
    w = behind_wait(w);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * kTCols + 2 * lane, b = blockIdx.y * kTBlocks + warp, r0 = b * kMxBlock;
    Cell v[kMxBlock];
    const T *p = w + (int64_t)r0 * ld + c;
#pragma unroll
    for (int r = 0; r < kMxBlock; ++r, p += ld) {
        v[r] = Cell();
        if (r0 + r < rows && c < cols) {
            if constexpr (VEC) {
                v[r] = __ldcs(reinterpret_cast<const Cell *>(p));
            } else if constexpr (kPairs) {
                const uint16_t *u = reinterpret_cast<const uint16_t *>(p);
                v[r] = u[0] | (c + 1 < cols ? (uint32_t)u[1] << 16 : 0u);
            } else {
                v[r] = make_float2(p[0], c + 1 < cols ? p[1] : 0.f);
            }
        }
    }
    uint32_t m0 = 0, m1 = 0;
    if constexpr (kPairs) {
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < kMxBlock; ++r) m = __vmaxu2(m, v[r] & 0x7fff7fffu);
        m0 = m << 16; m1 = m & 0xffff0000u;
    } else {
#pragma unroll
        for (int r = 0; r < kMxBlock; ++r) { m0 = max(m0, abs_bits(v[r].x)); m1 = max(m1, abs_bits(v[r].y)); }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t byte = mx_scale_byte<false>(h ? m1 : m0);
        uint32_t q[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            float f[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if constexpr (kPairs) f[j] = h ? bf16_hi(v[8 * g + j]) : bf16_lo(v[8 * g + j]);
                else f[j] = h ? v[8 * g + j].y : v[8 * g + j].x;
            }
            q[g] = codes_of(f, byte);
        }
        tile[2 * lane + h][warp] = make_uint4(q[0], q[1], q[2], q[3]);
        st[2 * lane + h][warp] = (uint8_t)byte;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTCols * kTBlocks; i += 32 * kTBlocks) {
        const int col = blockIdx.x * kTCols + i / kTBlocks, blk = blockIdx.y * kTBlocks + i % kTBlocks;
        if (col < cols && blk < nb) {
            reinterpret_cast<uint4 *>(codes)[(int64_t)col * nb + blk] = tile[i / kTBlocks][i % kTBlocks];
            scales[(int64_t)col * nb + blk] = st[i / kTBlocks][i % kTBlocks];
        }
    }
}

// Eight codes to floats: two e2m1 become a pair of f16 (exactly), times the scale.
__device__ __forceinline__ void unpack_e2m1(uint32_t q, float s, float (&v)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t h;
        asm("{\n.reg .b8 a, b, c, d;\nmov.b32 {a, b, c, d}, %1;\ncvt.rn.f16x2.e2m1x2 %0, a;\n}" : "=r"(h) : "r"(q >> (8 * i)));
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h));
        v[2 * i] = f.x * s; v[2 * i + 1] = f.y * s;
    }
}

// Does not trigger the launch behind it: what it writes are weights, which this library's other calls may read ahead of their wait (parameters, cs.h).
template <typename T, bool VEC> __global__ void __launch_bounds__(kQThreads)
dequantize_kernel(const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales, int rows, int cols, uint32_t nb, T *__restrict__ w, int64_t ld) {
    pdl_wait();
    const uint32_t parts = (uint32_t)rows * nb * 4;
    const uint32_t base = blockIdx.x * (kQThreads * kQUnroll) + threadIdx.x;
    uint32_t q[kQUnroll]; uint32_t s[kQUnroll];
#pragma unroll
    for (int u = 0; u < kQUnroll; ++u) {
        const uint32_t i = base + u * kQThreads;
        q[u] = 0; s[u] = 0;
        if (i < parts) { q[u] = __ldcs(reinterpret_cast<const uint32_t *>(codes) + i); s[u] = __ldcs(scales + (i >> 2)); }
    }
#pragma unroll
    for (int u = 0; u < kQUnroll; ++u) {
        const uint32_t i = base + u * kQThreads;
        if (i >= parts) break;
        const uint32_t row = i / (4 * nb), part = i - row * (4 * nb);
        T *p = w + (int64_t)row * ld + part * 8;
        const int n = cols - (int)part * 8;
        float v[8];
        unpack_e2m1(q[u], mx_scale(s[u]), v);
        if (VEC) {
            if (n > 0) {
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
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) p[j] = narrow<T>(v[j]);
        }
    }
}

// Row-major codes and scales to the FFN's tiles of 128 rows x 128 columns (8 KB of codes, row by row, and 512 scales in tile order).
// GATE_UP: tile (group, k block, half): rows 0..63 are 64 channels of W_gate, rows 64..127 the same channels of W_up; `inner` k blocks.
// Otherwise tile (group, row tile): 128 rows of W_down, the group's 128 columns; `inner` row tiles.
template <bool GATE_UP> __global__ void __launch_bounds__(256)
pack_tiles_kernel(const uint8_t *__restrict__ c0, const uint8_t *__restrict__ s0, const uint8_t *__restrict__ c1, const uint8_t *__restrict__ s1,
                  int inner, int groups, uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    pdl_launch_dependents();
    pdl_wait();
    c0 = behind_wait(c0); s0 = behind_wait(s0);
    if (GATE_UP) { c1 = behind_wait(c1); s1 = behind_wait(s1); }
    const int64_t tile = blockIdx.x;
    const int half = GATE_UP ? (int)(tile & 1) : 0;
    const int64_t q = GATE_UP ? tile >> 1 : tile, g = q / inner;
    const int at = (int)(q - g * inner);
    auto source = [&](int r) {      // of row r: in blocks of 128 columns
        return GATE_UP ? (g * 128 + half * 64 + (r & 63)) * inner + at : ((int64_t)at * 128 + r) * groups + g;
    };
    for (int i = threadIdx.x; i < 512; i += 256) {    // 128 rows x 4 chunks of 16 bytes
        const int r = i >> 2;
        const uint8_t *src = (GATE_UP && r >= 64 ? c1 : c0) + source(r) * 64;
        reinterpret_cast<uint4 *>(codes + tile * 8192)[i] = reinterpret_cast<const uint4 *>(src)[i & 3];
    }
    if (threadIdx.x < 128) {
        const int r = threadIdx.x;
        const uint32_t v = reinterpret_cast<const uint32_t *>(GATE_UP && r >= 64 ? s1 : s0)[source(r)];
        reinterpret_cast<uint32_t *>(scales + tile * kMxTileBytes)[(r & 31) * 4 + (r >> 5)] = v;
    }
}

int64_t blocks_of(int64_t cols) { return (cols + 31) / 32; }      // 64 bits: cols may be the largest int32
bool fits(int64_t rows, int64_t cols) { return rows > 0 && cols > 0 && rows * blocks_of(cols) * 4 < (int64_t)1 << 31; }
bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
cs_status status_of(cudaError_t e) { return e == cudaSuccess ? CS_OK : CS_ERR_CUDA; }

template <typename T> cs_status quantize(const T *w, int rows, int cols, int64_t ld, bool transpose, uint8_t *codes, uint8_t *scales, cudaStream_t st) {
    if (transpose) {
        const int nb = (int)blocks_of(rows);
        const dim3 grid((cols + kTCols - 1) / kTCols, (nb + kTBlocks - 1) / kTBlocks);
        if (grid.y > 65535) return CS_ERR_SHAPE;
        const bool vec = cols % 2 == 0 && ld % 2 == 0 && aligned(w, 2 * sizeof(T));
        return status_of(launch_pdl(true, vec ? quantize_cols_kernel<T, true> : quantize_cols_kernel<T, false>, grid, dim3(32 * kTBlocks), 0, st, w, rows,
                                    cols, ld, nb, codes, scales));
    }
    const uint32_t nb = (uint32_t)blocks_of(cols);
    const int64_t parts = (int64_t)rows * nb * 4;
    const dim3 grid((unsigned)((parts + kQThreads * kQUnroll - 1) / (kQThreads * kQUnroll)));
    const bool vec = cols % 8 == 0 && (ld * sizeof(T)) % 16 == 0 && aligned(w, 16);
    return status_of(launch_pdl(true, vec ? quantize_rows_kernel<T, true> : quantize_rows_kernel<T, false>, grid, dim3(kQThreads), 0, st, w, rows, cols, ld,
                                nb, codes, scales));
}

template <typename T> cs_status dequantize(const uint8_t *codes, const uint8_t *scales, int rows, int cols, T *w, int64_t ld, cudaStream_t st) {
    const uint32_t nb = (uint32_t)blocks_of(cols);
    const int64_t parts = (int64_t)rows * nb * 4;
    const dim3 grid((unsigned)((parts + kQThreads * kQUnroll - 1) / (kQThreads * kQUnroll)));
    const bool vec = cols % 8 == 0 && (ld * sizeof(T)) % 16 == 0 && aligned(w, 16);
    return status_of(launch_pdl(true, vec ? dequantize_kernel<T, true> : dequantize_kernel<T, false>, grid, dim3(kQThreads), 0, st, codes, scales, rows,
                                cols, nb, w, ld));
}

}  // namespace

}  // namespace cs

using namespace cs;

extern "C" {

cs_status cs_mx_quantize(const void *w, int32_t dtype, int32_t rows, int32_t cols, int64_t ld, int32_t transpose, uint8_t *codes,
                         uint8_t *scales, void *stream) {
    if (w == nullptr || codes == nullptr || scales == nullptr) return CS_ERR_NULL;
    if (dtype != CS_F32 && dtype != CS_BF16) return CS_ERR_UNSUPPORTED;
    if (ld < cols || !fits(transpose ? cols : rows, transpose ? rows : cols)) return CS_ERR_SHAPE;
    if (!aligned(codes, 16) || !aligned(w, dtype == CS_F32 ? 4 : 2)) return CS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == CS_F32 ? quantize(static_cast<const float *>(w), rows, cols, ld, transpose != 0, codes, scales, st)
                           : quantize(static_cast<const __nv_bfloat16 *>(w), rows, cols, ld, transpose != 0, codes, scales, st);
}

cs_status cs_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int32_t rows, int32_t cols, int32_t dtype, void *w, int64_t ld,
                           void *stream) {
    if (w == nullptr || codes == nullptr || scales == nullptr) return CS_ERR_NULL;
    if (dtype != CS_F32 && dtype != CS_BF16) return CS_ERR_UNSUPPORTED;
    if (ld < cols || !fits(rows, cols)) return CS_ERR_SHAPE;
    if (!aligned(codes, 16) || !aligned(w, dtype == CS_F32 ? 4 : 2)) return CS_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == CS_F32 ? dequantize(codes, scales, rows, cols, static_cast<float *>(w), ld, st)
                           : dequantize(codes, scales, rows, cols, static_cast<__nv_bfloat16 *>(w), ld, st);
}

cs_status cs_mx_pack(const cs_plan *plan, const cs_mx_matrix *gate, const cs_mx_matrix *up, const cs_mx_matrix *down, uint8_t *gate_up_codes,
                     uint8_t *gate_up_scales, uint8_t *down_codes, uint8_t *down_scales, void *stream) {
    if (plan == nullptr || gate == nullptr || up == nullptr || down == nullptr || gate_up_codes == nullptr || gate_up_scales == nullptr ||
        down_codes == nullptr || down_scales == nullptr)
        return CS_ERR_NULL;
    if (plan->cfg.w_dtype != CS_MX4) return CS_ERR_UNSUPPORTED;
    for (const cs_mx_matrix *m : {gate, up, down}) {
        if (m->codes == nullptr || m->scales == nullptr) return CS_ERR_NULL;
        if (!aligned(m->codes, 16) || !aligned(m->scales, 4)) return CS_ERR_UNSUPPORTED;
    }
    if (!aligned(gate_up_codes, 32) || !aligned(gate_up_scales, 16) || !aligned(down_codes, 32) || !aligned(down_scales, 16))
        return CS_ERR_UNSUPPORTED;
    const int dk = plan->cfg.d / 128, G = plan->G;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e = launch_pdl(true, pack_tiles_kernel<true>, dim3(2 * G * dk), dim3(256), 0, st, gate->codes, gate->scales, up->codes, up->scales, dk, G,
                               gate_up_codes, gate_up_scales);
    if (e == cudaSuccess)
        e = launch_pdl(true, pack_tiles_kernel<false>, dim3(dk * G), dim3(256), 0, st, down->codes, down->scales, nullptr, nullptr, dk, G, down_codes,
                       down_scales);
    return status_of(e);
}

}  // extern "C"
