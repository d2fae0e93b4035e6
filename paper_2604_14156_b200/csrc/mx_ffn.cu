// Actuator on microscaled operands: the SwiGLU FFN over the groups of the supports, weights in blocks of e2m1, activations in blocks of e4m3.
//
//   mx_list_kernel     the union of the supports, and each token's membership bits
//   mx_gateup_kernel   a[t, c] = silu(Wg_c . n_t) (Wu_c . n_t), rounded to blocks of 32 channels in e4m3; blocks of groups outside the
//                      token's support are zero
//   mx_down_kernel     out[t, :] = sum_c a[t, c] Wd[:, c] over the union's channels, rounded to bf16
//
// Both products are tcgen05.mma kind::mxf8f6f4 with block scales: the tensor core multiplies the two block scales into every partial product of 32
// and adds in f32, so neither operand is ever widened.  Weights are the M side: a tile is 128 rows x 128 columns, 8 KB in memory and 16 KB in
// shared memory (TMA spreads 16 codes over 16 bytes, the form the instruction wants).  Tokens are the N side, 16 to 160 columns.  In
// gate/up 64 channels of W_gate and the same 64 of W_up share a tile: one accumulator holds both, and 172 tiles for 86 groups spread better over
// 148 SMs than 86.  The scales go from shared memory to tensor memory with tcgen05.cp, in a place of their own per stage of the ring.
//
// What bounds it: HBM's 6.5 TB/s want 42 KB of weights in flight on every SM (a load takes 0.4 us from L2 and 0.9 from HBM, and 0.6 pass from the
// end of a stage's products to the next load's issue and back), and weights take twice their size in shared memory: four stages of 25 KB, two CTAs to an SM
// where there are that many, stream 5.0 TB/s at 64 tokens.  At one token the chain of latencies is all there is: list, first loads, products, exchange,
// and again.  (Two warps issuing the products, loads asked of L2 ahead of the ring, and waits that poll gained nothing; one CTA with eight stages to
// an SM was slower, but with 172 tiles on 148 SMs that is two rounds, and says nothing about the ring's depth.)
// 7B layer, 22 of 86 groups: 1 token 13.0 us, 3 tokens 17.2, 64 tokens 29.4, against 18.4, 48.6 and 72.3 MB of weights (a captured graph, 14 layers in turn, so
// that weights come from HBM; one layer again and again 12.4, 17.1 and 27.3).
//
// Work is split over a cluster where there are fewer tiles than SMs: each CTA of a cluster takes a part of the k blocks, and the
// accumulators are added over distributed shared memory in a fixed order.
#include <stdio.h>

#include <atomic>

#include "mx_core.cuh"

namespace cs {

namespace {

constexpr int kMxEpiWarps = 8;
constexpr int kMxThreads = 128 + 32 * kMxEpiWarps;   // weight loads, MMA, token loads, one idle warp; epilogue
constexpr int kMxMaxStages = 8;
constexpr int kMxMaxCluster = 8;
constexpr int kMxReadyPolls = 16;
constexpr int kMxPitch = 132;                        // floats from column to column of the spilled tile: float4 reads of 8 columns hit all banks
constexpr int kMxNarrowTokens = 128, kMxNarrowFew = 160, kMxMaxTile = 160;   // larger batches take the pairs of mx_wide.cu, see launch_mx_ffn

struct MxBars {
    uint64_t full[kMxMaxStages], empty[kMxMaxStages], acc;
    uint32_t tmem, aborted;
    uint32_t all[4];                // the union
    int32_t list[kMaxG], count;
    uint32_t bits[kMxMaxTile / 32]; // fold: which tokens of the tile use this CTA's group
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
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ void epilogue_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kMxEpiWarps) : "memory"); }
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
    mx_list_of(all, list, count);
}

struct MxRange { int first, n; };

// Three warps feed and run the products of k blocks [r.first, r.first + r.n) against the batch.  Weight tile of k block j: wtile + 2 j, or with DOWN
// wtile + (d / 128) list[j].
template <bool DOWN>
__device__ __forceinline__ void mx_load_weights(const CUtensorMap *map, const MxArgs &p, uint8_t *smem, MxBars *bars, int wtile, MxRange r) {
    const uint64_t policy = policy_evict_first();
    const int stage_bytes = mx_stage_bytes(p.tile), scales = kMxWBytes + p.tile * 128;
    MxRing ring;
    for (int i = 0; i < r.n; ++i) {
        if (i >= p.stages && !mx_wait(&bars->empty[ring.stage], ring.phase ^ 1, &bars->aborted, p.status)) return;
        uint8_t *w = smem + ring.stage * stage_bytes;
        uint64_t *full = &bars->full[ring.stage];
        const int tile = DOWN ? wtile + bars->list[r.first + i] * (p.d >> 7) : wtile + 2 * (r.first + i);
        mbar_expect_tx(full, kMxWLoad + kMxTileBytes);
        tma_load_2d(w, map, 0, tile * 128, full, policy);
        bulk_load(w + scales, p.w_scales + (size_t)tile * kMxTileBytes, kMxTileBytes, full);
        ring.next(p.stages);
    }
}
__device__ __forceinline__ void mx_load_tokens(const CUtensorMap *map, const MxArgs &p, uint8_t *smem, MxBars *bars, MxRange r, int kpitch) {
    const int stage_bytes = mx_stage_bytes(p.tile), chunks = mx_chunks(p.tile);
    const uint8_t *s0 = p.x_scales, *s1 = s0 + (p.B > 128 ? (size_t)kpitch * kMxTileBytes : 0);      // a tile of 144 has a second tile of scales
    MxRing ring;
    for (int i = 0; i < r.n; ++i) {
        if (i >= p.stages && !mx_wait(&bars->empty[ring.stage], ring.phase ^ 1, &bars->aborted, p.status)) return;
        uint8_t *x = smem + ring.stage * stage_bytes + kMxWBytes;
        uint64_t *full = &bars->full[ring.stage];
        const int j = r.first + i;
        mbar_expect_tx(full, p.tile * 128 + kMxTileBytes * chunks);
        tma_load_2d(x, map, j * 128, 0, full);
        uint8_t *sc = x + p.tile * 128 + kMxTileBytes;
        bulk_load(sc, s0 + (size_t)j * kMxTileBytes, kMxTileBytes, full);
        if (chunks > 1) bulk_load(sc + kMxTileBytes, s1 + (size_t)j * kMxTileBytes, kMxTileBytes, full);
        ring.next(p.stages);
    }
}
__device__ __forceinline__ void mx_products(const MxArgs &p, uint8_t *smem, MxBars *bars, MxRange r) {
    const int stage_bytes = mx_stage_bytes(p.tile), chunks = mx_chunks(p.tile);
    uint32_t idesc[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) idesc[kk] = mx_idesc(p.tile, kk);
    const uint32_t base = smem_u32(smem), tmem = bars->tmem;
    MxRing ring;
    for (int i = 0; i < r.n; ++i) {
        if (!mx_wait(&bars->full[ring.stage], ring.phase, &bars->aborted, p.status)) break;
        tc_fence_after();
        const uint32_t w = base + ring.stage * stage_bytes, x = w + kMxWBytes, sc = x + p.tile * 128;
        const uint32_t sa = tmem + p.tile + ring.stage * 4 * (1 + chunks), sb = sa + 4;
        tc_copy_scales(sa, sc);
        tc_copy_scales(sb, sc + kMxTileBytes);
        if (chunks > 1) tc_copy_scales(sb + 4, sc + 2 * kMxTileBytes);
        const uint64_t ad = desc_sw128(w, 0), bd = desc_sw128(x, 0);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) tc_mma_mx(tmem, ad + 2 * kk, bd + 2 * kk, idesc[kk], sa, sb, (i | kk) != 0);
        tc_commit(&bars->empty[ring.stage]);
        ring.next(p.stages);
    }
    if (r.n > 0) tc_commit(&bars->acc);
}
// The accumulators of the tile's valid tokens to shared memory, [column][kMxPitch], over the drained ring; zeros where there was no k block.
__device__ __forceinline__ void mx_spill(const MxArgs &p, uint8_t *smem, MxBars *bars, MxRange r) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quarter = warp & 3;
    float *tile = reinterpret_cast<float *>(smem) + quarter * 32 + lane;
    const bool ok = r.n > 0 && mx_wait(&bars->acc, 0, &bars->aborted, p.status);
    tc_fence_after();
    for (int c = 16 * ((warp >> 2) - 1); c < p.B; c += 32) {
        uint32_t v[16];
        if (ok) { tc_ld16(bars->tmem + ((uint32_t)quarter << 21) + c, v); tc_wait_ld(); }
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (c + j < p.B) tile[(c + j) * kMxPitch] = ok ? __uint_as_float(v[j]) : 0.f;
    }
}

// Four floats at this shared-memory offset in each of the cluster's CTAs, added in rank order; all loads are in flight together.
__device__ __forceinline__ float4 sum_ranks(uint32_t addr, int cs) {
    float4 u[kMxMaxCluster];
#pragma unroll
    for (int q = 0; q < kMxMaxCluster; ++q)
        if (q < cs) u[q] = ld_cluster4(map_to_cta(addr, q));
    float4 v = u[0];
#pragma unroll
    for (int q = 1; q < kMxMaxCluster; ++q)
        if (q < cs) { v.x += u[q].x; v.y += u[q].y; v.z += u[q].z; v.w += u[q].w; }
    return v;
}

__device__ __forceinline__ uint8_t *mx_setup(MxBars *bars, int stages, int cols, const CUtensorMap *a, const CUtensorMap *b) {
    extern __shared__ uint8_t raw[];
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) { mbar_init(&bars->full[s], 2); mbar_init(&bars->empty[s], 1); }
        mbar_init(&bars->acc, 1);
        bars->aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(a) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(b) : "memory");
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
    mx_settle(&bars->aborted);
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x >> 5 == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(bars->tmem), "r"(cols) : "memory");
    }
}

// Grid (cluster, 2 cap): tile y is one half (64 channels) of list entry y / 2; the CTAs of a cluster split d.
__global__ void __launch_bounds__(kMxThreads)
mx_gateup_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const MxArgs p) {
    __shared__ MxBars bars;
    const int cs = gridDim.x, rank = blockIdx.x, entry = blockIdx.y >> 1, half = blockIdx.y & 1;
    const int kb = p.d >> 7, cols = mx_tmem_cols(p.tile, p.stages), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *smem = mx_setup(&bars, p.stages, cols, &wmap, &xmap);
    pdl_wait();
    pdl_launch_dependents();
    const bool first = blockIdx.x + blockIdx.y == 0;
    if (p.fold) {
        if (threadIdx.x < 4 + kMxMaxTile / 32) (threadIdx.x < 4 ? bars.all[threadIdx.x] : bars.bits[threadIdx.x - 4]) = 0;
        __syncthreads();
        mx_mark(p.support, p.entries, p.G, bars.all, kMxThreads);
        __syncthreads();
        mx_list_of(bars.all, bars.list, &bars.count);
    } else if (threadIdx.x == 0) {
        bars.count = ld_dep(p.count);
        bars.list[entry] = ld_dep(p.list + entry);
    }
    __syncthreads();
    if (first && warp == 3) {      // beside the products: the list for the down product, which may read it once `ready` is set
        if (p.fold) {
            for (int i = lane; i < bars.count; i += 32) p.list[i] = bars.list[i];
            if (lane == 0) *p.count = bars.count;
            __threadfence();
            __syncwarp();
        }
        if (lane == 0) asm volatile("st.release.gpu.global.u32 [%0], 1;" ::"l"(p.ready) : "memory");
    }
    if (p.fold && warp == 3 && blockIdx.x == 0) mx_check(p.support, p.entries, p.k, p.G, blockIdx.y, gridDim.y, p.status);
    if (entry < bars.count) {      // the same in every CTA of a cluster
        const int g = bars.list[entry];
        const MxRange r = {kb * rank / cs, kb * (rank + 1) / cs - kb * rank / cs};
        if (warp == 0) {
            if (elect_one()) mx_load_weights<false>(&wmap, p, smem, &bars, 2 * g * kb + half, r);
        } else if (warp == 1) {
            if (elect_one()) mx_products(p, smem, &bars, r);
        } else if (warp == 2) {
            if (elect_one()) mx_load_tokens(&xmap, p, smem, &bars, r, kb);
        } else if (warp >= 4) {
            if (p.fold && !p.shared)      // while the products run: who uses this group
                for (int t = threadIdx.x - 128; t < p.entries; t += 32 * kMxEpiWarps)
                    if (ld_dep(p.support + t) == g) atomicOr(&bars.bits[t / p.k >> 5], 1u << (t / p.k & 31));
            mx_spill(p, smem, &bars, r);
        }
        __syncwarp();
        if (cs > 1) cluster_sync_all();
        if (warp >= 4) {
            if (cs > 1)      // this CTA's columns, every cs-th, summed in place: no other CTA reads them
                for (int c = (warp - 4) * cs + rank; c < p.B; c += kMxEpiWarps * cs) {
                    const uint32_t at = (uint32_t)(c * kMxPitch + lane * 4) * 4;
                    *reinterpret_cast<float4 *>(smem + at) = sum_ranks(smem_u32(smem) + at, cs);
                }
            __syncwarp();
            if (cs > 1) cluster_arrive();      // this warp is done with its peers' tiles
            epilogue_sync();
            // four threads to a column, sixteen channels each: a block of 32 is two neighbours'
            for (int i = threadIdx.x - 128;; i += 32 * kMxEpiWarps) {
                const int c = (i >> 2) * cs + rank, part = i & 3;
                if (__all_sync(0xffffffffu, c >= p.B)) break;
                const bool in = c < p.B;
                const bool member = in && (p.shared || (p.fold ? bars.bits[c >> 5] >> (c & 31) & 1 : p.mask[4 * c + (g >> 5)] >> (g & 31) & 1));
                const float4 *gate = reinterpret_cast<const float4 *>(smem) + (in ? c * (kMxPitch / 4) : 0) + part * 4, *up = gate + 16;
                float a[16], m = 0.f;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 x = gate[j], y = up[j];
                    a[4 * j] = swiglu(x.x, y.x); a[4 * j + 1] = swiglu(x.y, y.y); a[4 * j + 2] = swiglu(x.z, y.z); a[4 * j + 3] = swiglu(x.w, y.w);
                }
#pragma unroll
                for (int j = 0; j < 16; ++j) m = max_abs(m, a[j]);
                m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, 1));
                const uint32_t byte = member ? mx_scale_byte<true>(__float_as_uint(m)) : 0u;
                const float inv = mx_inverse(byte);
                uint32_t o[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    o[j] = !member || byte == 255 ? 0u : pack_e4m3(a[4 * j] * inv, a[4 * j + 1] * inv, a[4 * j + 2] * inv, a[4 * j + 3] * inv);
                const uint32_t other = __shfl_down_sync(0xffffffffu, byte, 2);
                if (in) {
                    *reinterpret_cast<uint4 *>(p.a + (size_t)c * p.cap * 128 + entry * 128 + half * 64 + part * 16) = make_uint4(o[0], o[1], o[2], o[3]);
                    uint8_t *to = p.a_scales + ((size_t)(c >> 7) * p.cap + entry) * kMxTileBytes + (c & 31) * 16 + ((c & 127) >> 5) * 4 + half * 2;
                    if (part == 0) *reinterpret_cast<uint16_t *>(to) = (uint16_t)(byte | other << 8);
                }
            }
        }
        if (cs > 1) {      // until its peers are done with this CTA's
            __syncwarp();
            if (warp < 4) cluster_arrive();
            cluster_wait();
        }
    }
    mx_teardown(&bars, cols);
}

// Grid (cluster, d / 128): the CTAs of a cluster split the list.  Weights depend on the list alone: where gate/up, which is still
// running, has said that it stands, their loads start before the wait for gate/up's result.
__global__ void __launch_bounds__(kMxThreads)
mx_down_kernel(const __grid_constant__ CUtensorMap wmap, const __grid_constant__ CUtensorMap xmap, const MxArgs p) {
    __shared__ MxBars bars;
    const int cs = gridDim.x, rank = blockIdx.x, cols = mx_tmem_cols(p.tile, p.stages), warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint8_t *smem = mx_setup(&bars, p.stages, cols, &wmap, &xmap);
    if (threadIdx.x == 0) {
        // gate/up is running (this launch began on its trigger) and says so a microsecond in; a CTA that starts later sees it at once
        unsigned ready = 0;
        for (int poll = 0; poll < kMxReadyPolls && ready == 0; ++poll)
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(ready) : "l"(p.ready) : "memory");
        bars.all[0] = ready;
    }
    __syncthreads();
    if (bars.all[0] == 0) pdl_wait();
    if (threadIdx.x == 0) bars.count = ld_dep(p.count);
    if (threadIdx.x < kMaxG) bars.list[threadIdx.x] = ld_dep(p.list + threadIdx.x);
    __syncthreads();
    const int n = bars.count;
    const MxRange r = {n * rank / cs, n * (rank + 1) / cs - n * rank / cs};
    if (warp == 0) {
        if (elect_one()) mx_load_weights<true>(&wmap, p, smem, &bars, blockIdx.y, r);
        __syncwarp();
        pdl_wait();
    } else {
        pdl_wait();
        pdl_launch_dependents();
        if (warp == 3 && lane == 0 && blockIdx.x + blockIdx.y == 0) *p.ready = 0;
        if (warp == 1) {
            if (elect_one()) mx_products(p, smem, &bars, r);
        } else if (warp == 2) {
            if (elect_one()) mx_load_tokens(&xmap, p, smem, &bars, r, p.cap);
        } else if (warp >= 4) {
            mx_spill(p, smem, &bars, r);
        }
        __syncwarp();
    }
    if (cs > 1) cluster_sync_all();
    if (warp >= 4) {
        if (cs == 1) epilogue_sync();
#pragma unroll 2
        for (int c = (warp - 4) * cs + rank; c < p.B; c += kMxEpiWarps * cs) {
            const uint32_t at = (uint32_t)(c * kMxPitch + lane * 4) * 4;
            const float4 v = cs == 1 ? *reinterpret_cast<const float4 *>(smem + at) : sum_ranks(smem_u32(smem) + at, cs);
            const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
            *reinterpret_cast<uint2 *>(p.out + (size_t)c * p.d + blockIdx.y * 128 + lane * 4) =
                make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
        }
    }
    if (cs > 1) cluster_sync_all();
    mx_teardown(&bars, cols);
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

constexpr int kMxSmemOne = 226 * 1024, kMxSmemTwo = 112 * 1024;   // a CTA's shared memory, alone on its SM or with another of its kind ...
constexpr int kMxSmemGateUp = 102 * 1024, kMxSmemDown = 61 * 1024;   // ... or a gate/up CTA's beside two down CTAs'

}  // namespace

cs_status prepare_mx_ffn(cs_plan *plan) {
    for (auto *k : {mx_gateup_kernel, mx_down_kernel})
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kMxSmemOne) != cudaSuccess || prefer_shared(k) != cudaSuccess)
            return CS_ERR_CUDA;
    // Clusters stand within a part of the device, so fewer of them fit than its SMs suggest (of 8 CTAs 15, not 18), and one more is another round.
    // (Asked once per device: a property of it, and 0.1 ms of a plan's creation.  Threads that create plans at once may each ask, and get the same answer.)
    static std::atomic<int> clusters[64][kMxMaxCluster + 1];      // 0: not asked yet
    for (int cs = 1; cs <= kMxMaxCluster; ++cs) {
        if (plan->device < 64) plan->mx_clusters[cs] = clusters[plan->device][cs].load(std::memory_order_relaxed);
        if (plan->mx_clusters[cs] != 0) continue;
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        cfg.gridDim = dim3(cs, 1024); cfg.blockDim = dim3(kMxThreads); cfg.dynamicSmemBytes = kMxSmemOne - 2048;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = cs; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&plan->mx_clusters[cs], mx_gateup_kernel, &cfg) != cudaSuccess) return CS_ERR_CUDA;
        if (plan->device < 64) clusters[plan->device][cs].store(plan->mx_clusters[cs], std::memory_order_relaxed);
    }
    return prefer_shared(mx_list_kernel) == cudaSuccess ? prepare_mx_wide(plan) : CS_ERR_CUDA;
}

cs_status launch_mx_ffn(cs_plan *plan, const cs_mx_layer *L, const uint8_t *q, const uint8_t *s, const int32_t *support, bool shared,
                        int B, void *out, cudaStream_t st) {
    const int d = plan->cfg.d, k = plan->cfg.k, G = plan->G, kb = d / 128;
    const int cap = shared ? k : (int)min((int64_t)G, (int64_t)B * k);
    const int rows = shared ? 1 : B;
    // Which kernels.  Pairs take 256 tokens for the price of one, but a group to an item: few groups leave most pairs without one.  Narrow against wide, us:
    // 22 of 86 groups of d = 4096, own supports, 100 tokens 37.6 and 44.0, 128 39.7 and 45.6, 129 (one CTA to an SM) 48.7 and 45.6, 160 49.5 and 46.1; a shared
    // support, 44 of 86, 128 26.9 and 31.0, 144 29.2 and 31.0, 160 30.0 and 30.9: there 128 is early.  Where gate/up's tiles fit the SMs once, own supports: 16
    // of 60 of 4096, 128 tokens 28.7 and 33.2, 144 33.8 and 33.5, 160 34.2 and 33.7; 12 of 48 of 2048, 144 24.5 and 25.8, 160 25.0 and 25.6.  Shared: 22 of 4096
    // 24.0 and 28.7 at 144 and at 160; 54 of 5120 33.7 and 36.5, 34.0 and 37.0: still ahead where the narrow kernels' tile ends.
    const bool wide = B > (2 * cap <= plan->sm_count ? kMxNarrowFew : kMxNarrowTokens);
    const int tile = min(kMxMaxTile, (B + 15) / 16 * 16);
    // Shared memory.  Where the weights are few (gate/up's tiles leave room for clusters of two on an SM each), one CTA of gate/up and two of down share an
    // SM, so that down's CTAs start, and load their weights, while gate/up runs; otherwise two CTAs of a product, or one where a tile has more than 128 tokens.
    const bool beside = tile <= 32 && 4 * cap <= plan->sm_count, two = !beside && tile <= 128;
    auto ring = [&](int bytes) { return max(2, min(kMxMaxStages, (bytes - 1024 - (int)sizeof(MxBars) - 64) / mx_stage_bytes(tile))); };
    const int stages = ring(beside ? kMxSmemGateUp : two ? kMxSmemTwo : kMxSmemOne), down_stages = beside ? ring(kMxSmemDown) : stages;
    auto smem_of = [&](int n) { return 1024 + (size_t)max(n * mx_stage_bytes(tile), tile * kMxPitch * 4); };
    CUtensorMap wg, wd, xm, am;
    if (!wide && (!make_map_tiles(&wg, L->gate_up_codes, (uint64_t)2 * G * kb) || !make_map_tiles(&wd, L->down_codes, (uint64_t)kb * G) ||
        !make_map_bytes(&xm, q, d, B, tile) || !make_map_bytes(&am, plan->mx_a, (uint64_t)cap * 128, B, tile))) {
        snprintf(plan->cuda_error, sizeof plan->cuda_error, "cuTensorMapEncodeTiled failed");
        return CS_ERR_CUDA;
    }
    MxArgs p;
    p.support = support; p.list = plan->glist; p.count = plan->nu; p.ready = plan->mask_count; p.mask = plan->mask;
    p.w_scales = L->gate_up_scales; p.x_scales = s;
    p.a = plan->mx_a; p.a_scales = plan->mx_a_scales; p.out = static_cast<__nv_bfloat16 *>(out); p.status = plan->status;
    p.B = B; p.d = d; p.G = G; p.k = k; p.cap = cap; p.tile = tile; p.stages = stages; p.shared = shared;
    p.entries = (int)min((int64_t)rows * k, (int64_t)1 << 30);
    p.fold = p.entries <= (wide ? kWideFoldEntries : kMxFoldEntries);
    cudaError_t e;
    if (!p.fold) {
        e = launch_pdl(true, mx_list_kernel, dim3(1), dim3(1024), 0, st, support, rows, k, G, plan->mask, plan->glist, plan->nu, plan->status);
        if (e != cudaSuccess) return record_cuda(plan, e, "mx_list_kernel");
        plan->launches += 1;
    }
    if (wide) return launch_mx_wide(plan, L, q, p, st);
    // Gate/up's clusters: as many CTAs as fill the SMs once, or, for long rows and few tokens, twice; where the k blocks that a CTA is spared (0.31 us
    // each, 0.42 with the shorter rings beyond 64 tokens) are worth more than the exchange (1.4 us and 0.04 a token).  d = 4096, whole calls by CTAs to a
    // cluster 1, 2, 3, 4 (8): 44 tiles, 1 token 16.9, 14.3, 13.8, 13.9 (17.9) us; 132, 3 tokens 19.4, 18.0, 23.0; 120, 16 tokens 20.0, 19.0, 24.4; 64 tokens
    // 23.5, 24.9, 30.0; 64, 64 tokens 20.5, 18.5, 20.8, 128 tokens 26.9, 23.9.  d = 2048, 96 tiles, 16 tokens 13.8, 14.3,
    // 17.9; d = 1024, 48 tiles, 16 tokens 10.2, 10.8, 11.3.
    int cs = max(1, min(min(kMxMaxCluster, kb / 2), plan->sm_count / (2 * cap)));
    if (cs == 1 && tile <= 32 && 20 * cap <= 9 * plan->sm_count) cs = 2;
    while (beside && cs > 1 && 2 * cap > plan->mx_clusters[cs]) --cs;
    if ((tile <= 64 ? 31 : 42) * (kb - (kb + cs - 1) / cs) <= 140 + 4 * B) cs = 1;
    e = launch_clusters(mx_gateup_kernel, dim3(cs, 2 * cap), smem_of(stages), st, wg, xm, p);
    if (e != cudaSuccess) return record_cuda(plan, e, "mx_gateup_kernel");
    p.w_scales = L->down_scales; p.x_scales = plan->mx_a_scales; p.stages = down_stages;
    cs = max(1, min(min(kMxMaxCluster, cap), plan->sm_count * (beside ? 2 : 1) / kb));
    while (!beside && cs > 1 && kb > plan->mx_clusters[cs]) --cs;
    e = launch_clusters(mx_down_kernel, dim3(cs, kb), smem_of(down_stages), st, wd, am, p);
    if (e != cudaSuccess) {
        cudaMemsetAsync(plan->mask_count, 0, sizeof(unsigned), st);      // what the down launch would have taken back
        return record_cuda(plan, e, "mx_down_kernel");
    }
    plan->launches += 2;
    return CS_OK;
}

}  // namespace cs
