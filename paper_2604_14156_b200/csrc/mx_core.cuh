// What the FFN kernels on microscaled operands share (mx_ffn.cu: batches whose tokens fit the N side of one instruction; mx_wide.cu: larger ones).
#pragma once

#include "mma_core.cuh"
#include "mx.cuh"

namespace cs {

// What a launch needs to know beside its tensor maps.
struct MxArgs {
    const uint8_t *w_scales, *x_scales;
    const int32_t *support;         // [B, k], or with `shared` [k]
    int32_t *list, *count;          // groups of the union, ascending
    unsigned *ready;                // set while a call's list stands, before its gate/up is complete
    const uint32_t *mask;           // [B, 4] membership bits, unless folded
    uint8_t *a, *a_scales;          // gate/up's result
    __nv_bfloat16 *out;             // down's
    DeviceStatus *status;
    int B, d, G, k;
    int cap;                        // groups the list can hold: pitch of a and its scales
    int tile, stages;               // tokens of a tile, ring stages
    int entries;                    // of the support
    int shared, fold;               // one support for all tokens; the products' launch makes the list, else mx_list_kernel has
};

// A batch on CTA pairs (mx_wide.cu).
cs_status launch_mx_wide(cs_plan *plan, const cs_mx_layer *L, const uint8_t *q, const MxArgs &p, cudaStream_t st);
cs_status prepare_mx_wide(cs_plan *plan);

namespace {

// Up to this many support entries (narrow, wide) the products' launch makes the list itself; beyond, mx_list_kernel does and leaves membership bits.  With a list
// kernel and without, us, 22 of 86 groups of d = 4096: 64 tokens (1408 entries) 28.7 and 27.3, 93 (2046) 35.6 and 34.2, 94 35.7 and 34.2, 128 (2816) 39.7 and
// 38.0; wide: 200 tokens (4400) 48.5 and 46.5, 372 (8184) 68.2 and 64.9, 400 (8800) 69.2 and 65.5, 2000 (44000) 206 and 192: for rows this long both limits
// are early.  What speaks for one is the wide launch's search of a token's own entries, once a group, where rows are short: 32 of 64 of d = 1024, 200
// tokens (6400) 27.7 and 30.3, 300 (9600) 33.6 and 33.9.
constexpr int kMxFoldEntries = 2048, kWideFoldEntries = 8192;
constexpr int kMxWBytes = 128 * 128;                 // a weight tile in shared memory
constexpr int kMxWLoad = 128 * 64;                   // ... and in memory, which is what the barrier counts
// One thread of a converged warp.  The compiler knows that an elect.sync branch is taken by a single thread; behind `lane == 0` it
// wraps every instruction that takes its operands from uniform registers (tcgen05.mma, TMA) in a loop over the active threads: 95 cycles to issue
// an MMA against 46.
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(one));
    return one != 0;
}
// Marks the groups of `n` support entries in `all` (cleared before), with all `threads` threads of a CTA.
__device__ __forceinline__ void mx_mark(const int32_t *support, int n, int G, uint32_t *all, int threads) {
    for (int i0 = threadIdx.x; i0 < n; i0 += 8 * threads) {
        int g[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) g[u] = i0 + u * threads < n ? ld_dep(support + i0 + u * threads) : -1;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = i0 + u * threads;
            if (i >= n) break;
            if (g[u] >= 0 && g[u] < G) {
                const uint32_t bit = 1u << (g[u] & 31);
                if (!(*reinterpret_cast<volatile uint32_t *>(&all[g[u] >> 5]) & bit)) atomicOr(&all[g[u] >> 5], bit);
            }
        }
    }
}
// Reports entries that are not ascending within rows of k, or outside [0, G): beside the products, by one warp of each of `parts` CTAs.
__device__ __forceinline__ void mx_check(const int32_t *support, int n, int k, int G, int part, int parts, DeviceStatus *status) {
    bool bad = false;
    for (int i = part * 32 + (threadIdx.x & 31); i < n; i += 32 * parts) {
        const int g = ld_dep(support + i);
        bad |= g >= G || g <= (i % k != 0 ? ld_dep(support + i - 1) : -1);
    }
    if (bad) atomicCAS(&status->code, 0, (int)CS_ERR_SUPPORT);
}
// The marked groups in ascending order, and their number (threads 0..127 of the CTA).
__device__ __forceinline__ void mx_list_of(const uint32_t (&all)[4], int32_t *list, int32_t *count) {
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
// Ring position without divisions: the issue of a k block's copies is what a CTA's weight stream waits for first.
struct MxRing {
    int stage = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++stage == stages) { stage = 0; phase ^= 1; }
    }
};
// PEER: what the barrier stands for was written, or read, by the other CTA of a pair.
template <bool PEER = false>
__device__ __forceinline__ bool mx_wait(uint64_t *bar, uint32_t parity, uint32_t *aborted, DeviceStatus *status) {
    const uint32_t addr = smem_u32(bar);
    for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
        uint32_t done;
        if (PEER)
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                         : "=r"(done) : "r"(addr), "r"(parity) : "memory");
        else
            asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                         : "=r"(done) : "r"(addr), "r"(parity) : "memory");
        if (done) return true;
        if (*reinterpret_cast<volatile uint32_t *>(aborted)) return false;
    }
    *reinterpret_cast<volatile uint32_t *>(aborted) = 1;
    atomicCAS(&status->code, 0, (int)CS_ERR_TIMEOUT);
    return false;
}
// After a wait that gave up: copies may still be on their way into this CTA's shared memory; they land within microseconds.
__device__ __forceinline__ void mx_settle(const uint32_t *aborted) {
    if (*reinterpret_cast<const volatile uint32_t *>(aborted))
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);
}
__device__ __forceinline__ void bulk_load(void *dst, const void *src, uint32_t bytes, uint64_t *bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
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
// Packed weight tiles, seen as rows of 128 four-bit elements: a box is a tile, or some rows of one.
bool make_map_tiles(CUtensorMap *map, const void *base, uint64_t tiles, uint32_t box_rows = 128) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {128, tiles * 128}, strides[1] = {64};
    const cuuint32_t box[2] = {128, box_rows}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_16U4_ALIGN16B, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

}  // namespace cs
