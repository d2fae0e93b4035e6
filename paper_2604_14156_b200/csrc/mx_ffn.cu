// Actuator on microscaled operands: the SwiGLU FFN over the groups of the supports, weights in blocks of e2m1, activations in blocks of e4m3.
//
//   mx_list_kernel     the union of the supports, and each token's membership bits
//   mx_gateup_kernel   a[t, c] = silu(Wg_c . n_t) (Wu_c . n_t), rounded to blocks of 32 channels in e4m3; blocks of groups outside the
//                      token's support are zero
//   mx_down_kernel     out[t, :] = sum_c a[t, c] Wd[:, c] over the union's channels, rounded to bf16
//
// Both products are tcgen05.mma kind::mxf8f6f4 with block scales: the tensor core multiplies the two block scales into every partial product of 32
// and adds in f32, so neither operand is ever widened.  Weights are the M side: a tile is 128 rows x 128 columns, 8 KB in memory and 16 KB in
// shared memory (TMA spreads 16 codes over 16 bytes, the form the instruction wants).  Tokens are the N side, 16 to 256 columns.  In
// gate/up 64 channels of W_gate and the same 64 of W_up share a tile: one accumulator holds both, and 172 tiles for 86 groups spread better over
// 148 SMs than 86.  The scales go from shared memory to tensor memory with tcgen05.cp, in a place of their own per stage of the ring.
//
// Work is split over a cluster where there are fewer tiles than SMs can hold: each CTA of a cluster takes a part of the k blocks, and the
// accumulators are added over distributed shared memory in a fixed order.
#include <stdio.h>

#include "mma_core.cuh"
#include "mx.cuh"

namespace cs {

namespace {

constexpr int kMxEpiWarps = 8;
constexpr int kMxThreads = 64 + 32 * kMxEpiWarps;    // TMA warp, MMA warp, epilogue
constexpr int kMxMaxTile = 256;                      // tokens of a tile
constexpr int kMxMaxStages = 8;
constexpr int kMxWBytes = 128 * 128;                 // a weight tile in shared memory
constexpr int kMxWLoad = 128 * 64;                   // ... and in memory, which is what the barrier counts
constexpr int kMxMaxCluster = 8;

// What a launch needs to know beside its tensor maps.
struct MxArgs {
    const uint8_t *w_scales, *x_scales;
    const int32_t *list, *count;    // groups of the union, ascending
    const uint32_t *mask;           // [B, 4] membership bits, or NULL: every token uses every listed group
    uint8_t *a, *a_scales;          // gate/up's result
    __nv_bfloat16 *out;             // down's
    DeviceStatus *status;
    int B, d, G;
    int cap;                        // groups the list can hold: pitch of a and its scales
    int tile, stages;               // tokens of a tile, ring stages
    int w_once;                     // weights are read by one token tile only
};

struct MxBars {
    uint64_t full[kMxMaxStages], empty[kMxMaxStages], acc;
    uint32_t tmem, aborted;
};

__host__ __device__ inline int mx_chunks(int tile) { return (tile + 127) / 128; }
__host__ __device__ inline int mx_stage_bytes(int tile) {     // weights, tokens, scales of both: a multiple of 1024
    return (kMxWBytes + tile * 128 + kMxTileBytes * (1 + mx_chunks(tile)) + 1023) / 1024 * 1024;
}
__host__ __device__ inline int mx_tmem_cols(int tile, int stages) {
    const int need = tile + 4 * stages * (1 + mx_chunks(tile));
    int c = 32;
    while (c < need) c *= 2;
    return c;
}

__device__ __forceinline__ bool mx_wait(uint64_t *bar, uint32_t parity, MxBars *b, DeviceStatus *status) {
    const uint32_t addr = smem_u32(bar);
    for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(addr), "r"(parity) : "memory");
        if (done) return true;
        if (*reinterpret_cast<volatile uint32_t *>(&b->aborted)) return false;
    }
    b->aborted = 1;
    atomicCAS(&status->code, 0, (int)CS_ERR_TIMEOUT);
    return false;
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// 512 bytes of scales to four tensor-memory columns, repeated in the four lane quarters.
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint32_t saddr) {
    const uint64_t desc = (uint64_t)((saddr & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
// e2m1 x e4m3 with block scales, M = 128, n columns; kk: which of the four blocks of 32 the scales' words hold.
__device__ __forceinline__ uint32_t mx_idesc(int n, int kk) {
    return ((uint32_t)kk << 4) | (5u << 7) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (1u << 27) | ((uint32_t)kk << 29);
}
__device__ __forceinline__ void tc_mma_mx(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::1.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
}
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kMxEpiWarps) : "memory"); }
__device__ __forceinline__ float ld_cluster(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}

// One CTA: the union of all rows of `support`, the rows' membership bits (when mask != NULL), validation.  A thread per entry, so that all loads
// of up to kMxListRows rows are in flight together.
constexpr int kMxListRows = 512;
__global__ void __launch_bounds__(1024)
mx_list_kernel(const int32_t *support, int rows, int k, int G, uint32_t *mask, int32_t *list, int32_t *count, DeviceStatus *status) {
    __shared__ uint32_t bits[kMxListRows][4];
    __shared__ uint32_t all[4];
    if (threadIdx.x < 4) all[threadIdx.x] = 0;
    pdl_launch_dependents();
    pdl_wait();
    bool bad = false;
    for (int t0 = 0; t0 < rows; t0 += kMxListRows) {
        const int nt = min(kMxListRows, rows - t0), n = nt * k;
        for (int i = threadIdx.x; i < nt * 4; i += blockDim.x) bits[i >> 2][i & 3] = 0;
        __syncthreads();
        const int32_t *rowsup = support + (size_t)t0 * k;
        for (int i0 = threadIdx.x; i0 < n; i0 += 4 * blockDim.x) {
            int g[4], last[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * (int)blockDim.x;
                g[u] = i < n ? ld_dep(rowsup + i) : 0;
                last[u] = i < n && i % k != 0 ? ld_dep(rowsup + i - 1) : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * (int)blockDim.x;
                if (i >= n) break;
                bad |= g[u] <= last[u] || g[u] >= G;
                if (g[u] >= 0 && g[u] < G) atomicOr(&bits[i / k][g[u] >> 5], 1u << (g[u] & 31));
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < nt * 4; i += blockDim.x) {
            const uint32_t m = bits[i >> 2][i & 3];
            if (mask != nullptr) mask[4 * (size_t)t0 + i] = m;
            if (m & ~*reinterpret_cast<volatile uint32_t *>(&all[i & 3])) atomicOr(&all[i & 3], m);
        }
        __syncthreads();
    }
    if (bad) atomicCAS(&status->code, 0, (int)CS_ERR_SUPPORT);
    if (threadIdx.x < 128) {
        const int g = threadIdx.x, w = g >> 5;
        int before = 0, n = 0;
        for (int i = 0; i < 4; ++i) {
            if (i < w) before += __popc(all[i]);
            n += __popc(all[i]);
        }
        before += __popc(all[w] & ((1u << (g & 31)) - 1));
        if (all[w] >> (g & 31) & 1) list[before] = g;
        if (g == 0) *count = n;
    }
}

// The part both products share: accumulators of this CTA's k blocks [first, first + n) of weight tile row `wrow` (in tiles: the first k
// block's index in the packed matrix; listed: k block j is list[j]) against token tile `z`.  Leaves the accumulators in the shared tile
// [columns][128], zeros where there was no k block.
struct MxRange { int first, n; };

template <bool DOWN>
__device__ __forceinline__ void mx_mainloop(const CUtensorMap *wmap, const CUtensorMap *xmap, const MxArgs &p, uint8_t *smem, MxBars *bars, int64_t wtile,
                                            MxRange r, int z, int columns) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int stage_bytes = mx_stage_bytes(p.tile), chunks = mx_chunks(p.tile);
    const int kpitch = DOWN ? p.cap : p.d >> 7;          // k blocks of the token operand
    if (warp == 0) {
        if (lane == 0) {
            const uint64_t policy = policy_evict_first();
            const uint32_t bytes = kMxWLoad + p.tile * 128 + kMxTileBytes * (1 + chunks);
            const int last_chunk = (p.B - 1) >> 7;
            for (int i = 0; i < r.n; ++i) {
                const int s = i % p.stages, j = r.first + i;
                if (i >= p.stages && !mx_wait(&bars->empty[s], (i / p.stages - 1) & 1, bars, p.status)) break;
                uint8_t *w = smem + (size_t)s * stage_bytes, *x = w + kMxWBytes, *sc = x + p.tile * 128;
                const int64_t tile = wtile + (DOWN ? ld_dep(p.list + j) : j);
                mbar_expect_tx(&bars->full[s], bytes);
                if (p.w_once) tma_load_2d(w, wmap, 0, (int)(tile * 128), &bars->full[s], policy);
                else tma_load_2d(w, wmap, 0, (int)(tile * 128), &bars->full[s]);
                tma_load_2d(x, xmap, j * 128, z * p.tile, &bars->full[s]);
                bulk_load(sc, p.w_scales + tile * kMxTileBytes, kMxTileBytes, &bars->full[s]);
                for (int c = 0; c < chunks; ++c)      // behind the last row: any tile that exists
                    bulk_load(sc + kMxTileBytes * (1 + c), p.x_scales + ((size_t)min(z * p.tile / 128 + c, last_chunk) * kpitch + j) * kMxTileBytes,
                              kMxTileBytes, &bars->full[s]);
            }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t scales = bars->tmem + p.tile;
            for (int i = 0; i < r.n; ++i) {
                const int s = i % p.stages;
                if (!mx_wait(&bars->full[s], (i / p.stages) & 1, bars, p.status)) break;
                tc_fence_after();
                const uint32_t w = smem_u32(smem + (size_t)s * stage_bytes), x = w + kMxWBytes, sc = x + p.tile * 128;
                const uint32_t sa = scales + s * 4 * (1 + chunks), sb = sa + 4;
                tc_copy_scales(sa, sc);
                for (int c = 0; c < chunks; ++c) tc_copy_scales(sb + 4 * c, sc + kMxTileBytes * (1 + c));
                const uint64_t ad = desc_sw128(w, 0), bd = desc_sw128(x, 0);
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) tc_mma_mx(bars->tmem, ad + 2 * kk, bd + 2 * kk, mx_idesc(columns, kk), sa, sb, (i | kk) != 0);
                tc_commit(&bars->empty[s]);
            }
            if (r.n > 0) tc_commit(&bars->acc);
        }
        __syncwarp();
    } else {
        const int e = warp - 2, quarter = warp & 3, half = e >> 2;
        float *tile = reinterpret_cast<float *>(smem);
        const bool ok = r.n > 0 && mx_wait(&bars->acc, 0, bars, p.status);
        tc_fence_after();
        // the ring is drained: the tile takes its place
        for (int c = 16 * half; c < columns; c += 32) {
            uint32_t v[16];
            if (ok) { tc_ld16(bars->tmem + ((uint32_t)quarter << 21) + c, v); tc_wait_ld(); }
#pragma unroll
            for (int j = 0; j < 16; ++j) tile[(c + j) * 128 + quarter * 32 + lane] = ok ? __uint_as_float(v[j]) : 0.f;
        }
    }
}

__device__ __forceinline__ uint8_t *mx_setup(MxBars *bars, int stages, int cols) {
    extern __shared__ uint8_t raw[];
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(&bars->full[s], 1); mbar_init(&bars->empty[s], 1); }
        mbar_init(&bars->acc, 1);
        bars->aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x >> 5 == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars->tmem)), "r"(cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    return reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
}
__device__ __forceinline__ void mx_teardown(MxBars *bars, int cols) {
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x >> 5 == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(bars->tmem), "r"(cols) : "memory");
    }
}

// Grid (cluster, 2 cap, token tiles): tile y is one half (64 channels) of list entry y / 2; the CTAs of a cluster split d.
__global__ void __launch_bounds__(kMxThreads)
mx_gateup_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const MxArgs p) {
    __shared__ MxBars bars;
    const int cs = gridDim.x, rank = blockIdx.x, entry = blockIdx.y >> 1, half = blockIdx.y & 1, z = blockIdx.z;
    const int kb = p.d >> 7, cols = mx_tmem_cols(p.tile, p.stages);
    uint8_t *smem = mx_setup(&bars, p.stages, cols);
    pdl_wait();
    pdl_launch_dependents();
    if (entry < ld_dep(p.count)) {      // the same in every CTA of a cluster
        const int g = ld_dep(p.list + entry);
        const int columns = min(p.tile, (p.B - z * p.tile + 15) & ~15);
        const MxRange r = {kb * rank / cs, kb * (rank + 1) / cs - kb * rank / cs};
        mx_mainloop<false>(&wmap, &xmap, p, smem, &bars, (int64_t)(2 * g + half) * kb, r, z, columns);
        if (cs > 1) cluster_sync_all();
        const int e = (int)(threadIdx.x >> 5) - 2, lane = threadIdx.x & 31;
        if (e >= 0) {
            if (cs == 1) epilogue_sync();
            // (column, block of 32 channels) pairs, a warp each: a lane is a channel
            const uint32_t base = smem_u32(smem);
            for (int i = e; (i >> 1) * cs < columns; i += kMxEpiWarps) {
                const int c = (i >> 1) * cs + rank, b = i & 1, t = z * p.tile + c;
                if (c >= columns || t >= p.B) continue;
                float gate = 0.f, up = 0.f;
                const uint32_t at = base + (uint32_t)(c * 128 + b * 32 + lane) * 4;
                if (cs == 1) {
                    const float *tile = reinterpret_cast<const float *>(smem) + c * 128 + b * 32 + lane;
                    gate = tile[0]; up = tile[64];
                } else {
                    for (int q = 0; q < cs; ++q) {
                        const uint32_t peer = map_to_cta(at, q);
                        gate += ld_cluster(peer); up += ld_cluster(peer + 256);
                    }
                }
                const bool member = p.mask == nullptr || (p.mask[4 * (size_t)t + (g >> 5)] >> (g & 31) & 1);
                const float a = member ? silu_f(gate) * up : 0.f;
                const uint32_t byte = mx_scale_byte<true>(__reduce_max_sync(0xffffffffu, abs_bits(a)));
                const uint8_t v = to_e4m3(byte == 255 ? 0.f : a * mx_inverse(byte));
                p.a[(size_t)t * p.cap * 128 + entry * 128 + half * 64 + b * 32 + lane] = v;
                if (lane == 0)
                    p.a_scales[((size_t)(t >> 7) * p.cap + entry) * kMxTileBytes + (t & 31) * 16 + ((t & 127) >> 5) * 4 + half * 2 + b] = (uint8_t)byte;
            }
        }
        if (cs > 1) cluster_sync_all();      // peers are done with this CTA's tile
    }
    mx_teardown(&bars, cols);
}

// Grid (cluster, d / 128, token tiles): the CTAs of a cluster split the list.
__global__ void __launch_bounds__(kMxThreads)
mx_down_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const MxArgs p) {
    __shared__ MxBars bars;
    const int cs = gridDim.x, rank = blockIdx.x, z = blockIdx.z, cols = mx_tmem_cols(p.tile, p.stages);
    uint8_t *smem = mx_setup(&bars, p.stages, cols);
    pdl_wait();
    pdl_launch_dependents();
    const int n = ld_dep(p.count);
    const int columns = min(p.tile, (p.B - z * p.tile + 15) & ~15);
    const MxRange r = {n * rank / cs, n * (rank + 1) / cs - n * rank / cs};
    mx_mainloop<true>(&wmap, &xmap, p, smem, &bars, (int64_t)blockIdx.y * p.G, r, z, columns);
    if (cs > 1) cluster_sync_all();
    const int e = (int)(threadIdx.x >> 5) - 2, lane = threadIdx.x & 31;
    if (e >= 0) {
        if (cs == 1) epilogue_sync();
        const uint32_t base = smem_u32(smem);
        for (int c = e * cs + rank; c < columns && z * p.tile + c < p.B; c += kMxEpiWarps * cs) {
            const uint32_t at = base + (uint32_t)(c * 128 + lane * 4) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            if (cs == 1) {
                v = *reinterpret_cast<const float4 *>(smem + (size_t)(c * 128 + lane * 4) * 4);
            } else {
                for (int q = 0; q < cs; ++q) {
                    const float4 u = ld_cluster4(map_to_cta(at, q));
                    v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
                }
            }
            const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
            *reinterpret_cast<uint2 *>(p.out + (size_t)(z * p.tile + c) * p.d + blockIdx.y * 128 + lane * 4) =
                make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
        }
    }
    if (cs > 1) cluster_sync_all();
    mx_teardown(&bars, cols);
}

// Matrix of bytes [rows, inner]: boxes of 128 bytes x box_rows, 128-byte swizzle.
bool make_map_bytes(CUtensorMap *map, const void *base, uint64_t inner, uint64_t rows, uint32_t box_rows) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {inner, rows}, strides[1] = {inner};
    const cuuint32_t box[2] = {128, box_rows}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Packed weight tiles, seen as rows of 128 four-bit elements: a box is a tile.
bool make_map_tiles(CUtensorMap *map, const void *base, uint64_t tiles) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {128, tiles * 128}, strides[1] = {64};
    const cuuint32_t box[2] = {128, 128}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_clusters(void (*kernel)(const CUtensorMap, const CUtensorMap, const MxArgs), dim3 grid, size_t smem, cudaStream_t st,
                            const CUtensorMap &w, const CUtensorMap &x, const MxArgs &p) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = dim3(kMxThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = grid.x; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, w, x, p);
}

constexpr int kMxSmemOne = 226 * 1024, kMxSmemTwo = 112 * 1024;   // a CTA's shared memory, alone on its SM or with another

}  // namespace

cs_status prepare_mx_ffn(cs_plan *plan) {
    for (auto *k : {mx_gateup_kernel, mx_down_kernel})
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMxSmemOne) != cudaSuccess || prefer_shared(k) != cudaSuccess)
            return CS_ERR_CUDA;
    return prefer_shared(mx_list_kernel) == cudaSuccess ? CS_OK : CS_ERR_CUDA;
}

cs_status launch_mx_ffn(cs_plan *plan, const cs_mx_layer *L, const uint8_t *q, const uint8_t *s, const int32_t *support, bool shared,
                        int B, void *out, cudaStream_t st) {
    const int d = plan->cfg.d, k = plan->cfg.k, G = plan->G, kb = d / 128;
    const int cap = shared ? k : (int)min((int64_t)G, (int64_t)B * k);
    const int rows = shared ? 1 : B;
    const int tile = min(kMxMaxTile, (B + 15) / 16 * 16), tiles = (B + tile - 1) / tile;
    const bool two = tile <= 128;                        // two CTAs on an SM
    const int room = (two ? kMxSmemTwo : kMxSmemOne) - 1024 - (int)sizeof(MxBars) - 64;
    const int stages = max(2, min(kMxMaxStages, room / mx_stage_bytes(tile)));
    const size_t smem = 1024 + (size_t)max(stages * mx_stage_bytes(tile), tile * 512);
    const int slots = plan->sm_count * (two ? 2 : 1);
    CUtensorMap wg, wd, xm, am;
    if (!make_map_tiles(&wg, L->gate_up_codes, (uint64_t)2 * G * kb) || !make_map_tiles(&wd, L->down_codes, (uint64_t)kb * G) ||
        !make_map_bytes(&xm, q, d, B, tile) || !make_map_bytes(&am, plan->mx_a, (uint64_t)cap * 128, B, tile)) {
        snprintf(plan->cuda_error, sizeof plan->cuda_error, "cuTensorMapEncodeTiled failed");
        return CS_ERR_CUDA;
    }
    cudaError_t e = launch_pdl(true, mx_list_kernel, dim3(1), dim3((int)min((int64_t)1024, max((int64_t)128, ((int64_t)rows * k + 31) / 32 * 32))), 0, st, support, rows, k, G,
                               shared ? nullptr : plan->mask, plan->glist, plan->nu, plan->status);
    if (e != cudaSuccess) return record_cuda(plan, e, "mx_list_kernel");
    MxArgs p;
    p.w_scales = L->gate_up_scales; p.x_scales = s; p.list = plan->glist; p.count = plan->nu; p.mask = shared ? nullptr : plan->mask;
    p.a = plan->mx_a; p.a_scales = plan->mx_a_scales; p.out = static_cast<__nv_bfloat16 *>(out); p.status = plan->status;
    p.B = B; p.d = d; p.G = G; p.cap = cap; p.tile = tile; p.stages = stages; p.w_once = tiles == 1;
    int cs = 1;
    while (cs < kMxMaxCluster && 2 * cap * tiles * cs * 2 <= slots && kb / (cs * 2) >= 4) cs *= 2;
    e = launch_clusters(mx_gateup_kernel, dim3(cs, 2 * cap, tiles), smem, st, wg, xm, p);
    if (e != cudaSuccess) return record_cuda(plan, e, "mx_gateup_kernel");
    p.w_scales = L->down_scales; p.x_scales = plan->mx_a_scales;
    cs = max(1, min(min(kMxMaxCluster, cap), slots / (kb * tiles)));
    e = launch_clusters(mx_down_kernel, dim3(cs, kb, tiles), smem, st, wd, am, p);
    if (e != cudaSuccess) return record_cuda(plan, e, "mx_down_kernel");
    plan->launches += 3;
    return CS_OK;
}

}  // namespace cs
