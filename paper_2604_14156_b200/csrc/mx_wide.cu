// The FFN on microscaled operands for batches beyond one tile of mx_ffn.cu and for prompts, on pairs of CTAs.
//
//   mx_wide_kernel      both products: first every gate/up item (256 tokens x one group: 128 channels of W_gate and of W_up), then every down item (256
//                       tokens x 256 or 192 columns of the output, or a part of the list of it)
//   mx_wide_sum_kernel  adds the parts
//
// Here the tensor pipe is the bound, and before it what an SM can draw from L2: a single CTA of 128 weight rows x 256 tokens takes 41 KB for 512
// cycles of products.  A cluster of two CTAs issues one instruction of 256 x 256 (cta_group::2): each brings 128 tokens and 128 weight
// rows, 25 KB for the same 512 cycles.  Tokens are the M side, so a tensor-memory lane is a token and a row of 32 neighbouring columns in it a
// block of channels: the epilogue finds a block's largest element, silu's two factors and the bytes it writes in one thread's registers.  A packed
// gate/up tile (64 rows of W_gate, the same 64 of W_up) is one CTA's half of the columns.
//
// The kernel is persistent, one pair of CTAs on two SMs.  Pairs claim items in order from a counter, the next one shortly before the loads of the last
// end (not earlier, so that pairs that start first leave items to the others), and the ring of loads runs on across items.  One accumulator of 256
// columns (the scales need some of the other 256): the epilogue takes it into registers, 128 a thread, hands it back, and does its arithmetic while the
// next item's products run.  A down item's token loads wait until the epilogues of its token tile's gate/up items have counted themselves; its weights do
// not.  Gate/up items wait for nothing, come first in the order of claims, and are claimed by pairs that run; so every wait ends however few of the
// pairs the device has room for (items dealt out in advance would wait for pairs that have no SM yet).  All waits are bounded besides.  The gate/up
// phase also asks L2 for the down weights.
//
// 2048 tokens of d = 5120, 27 of 108 groups (217 GFLOP), back to back in a graph: two launches of single CTAs 160 us, pairs 103, without spilled accumulators and
// with the union of the supports inside the launch 83, one launch 79, claimed items 75 (2.9 PFLOP/s; 91 over a second of load, at the clocks of the power
// cap).  Where there are few items the first claim costs 1 us (777 tokens, 11 groups, 30.7 -> 31.5).  An item's 40 k blocks take 12 us, of which the
// products alone are 10.7, and 1 to 1.5 us pass from its last product to the next item's first.
#include <stdio.h>

#include "mx_core.cuh"

namespace cs {

namespace {

constexpr int kWideStages = 6;
constexpr int kWideStageBytes = 128 * 128 + kMxWBytes + 3 * kMxTileBytes + 512;     // tokens, weights, scales: a multiple of 1024
constexpr int kWideEpiWarps = 8;
constexpr int kWideThreads = 128 + 32 * kWideEpiWarps;    // token loads, products, weight loads, claims and the support's check; epilogue
constexpr int kWideTokens = 256;
constexpr int kWideClaims = 2;      // items a pair has claimed and not all of its warps have taken up
constexpr int kWideAhead = 8;       // k blocks (0.27 us each) before the end of an item's loads at which the next is claimed (1 to 1.5 us)
constexpr int kWideTakers = 2 * (2 + kWideEpiWarps) + 1;      // loads and epilogue of both CTAs, products of one
static_assert(kWideStageBytes % 1024 == 0, "operands stand on 1024-byte boundaries");

struct WideArgs {
    MxArgs p;
    int ztiles;        // token tiles
    int splits;        // parts of the list a down item is cut into; > 1: f32 results to `partial`
    int whole;         // the output's rows stand on 32-byte boundaries: whole sectors
    const uint8_t *down_codes, *down_scales;
    float *partial;    // [down item and part][256 tokens][256 columns]
    unsigned *done;    // [ztiles] epilogue warps that have stored their part of a token tile's activations; behind them the pairs that have ended
    unsigned *next;    // the next item; not in a line of `done`, which waiting pairs poll
};

struct WideBars {
    uint64_t full[kWideStages], empty[kWideStages], acc_full, acc_empty, claim_ask, claim_full[kWideClaims], claim_empty[kWideClaims];
    int claim[kWideClaims];
    uint32_t tmem, aborted;
    uint32_t all[4];
    int32_t list[kMaxG], count;
};

// Instruction descriptor: e4m3 (tokens) x e2m1 (weights) with block scales, M = 256 over the pair, n columns.
__device__ __forceinline__ uint32_t wide_idesc(int n, int kk) {
    return ((uint32_t)kk << 4) | (5u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | (2u << 27) | ((uint32_t)kk << 29);
}
__device__ __forceinline__ void wide_copy_scales(uint32_t taddr, uint32_t saddr) {     // the same offsets in both CTAs
    const uint64_t desc = (uint64_t)((saddr & 0x3ffff) >> 4) | ((uint64_t)(128 >> 4) << 32) | ((uint64_t)1 << 46);
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
__device__ __forceinline__ void wide_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\n"
                 "tcgen05.mma.cta_group::2.kind::mxf8f6f4.block_scale [%0], %1, %2, %3, [%5], [%6], p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(sa), "r"(sb) : "memory");
}
__device__ __forceinline__ void store32(void *p, const uint32_t (&v)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

__device__ __forceinline__ void prefetch_l2(const void *p, uint32_t bytes) {
    asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// Item i of a call: first every token tile's gate/up items, then the down items.  DB: 32-column blocks of a CTA's half of a down item.
struct WideItem {
    bool down;
    int z, col;            // token tile; list entry (gate/up) or first output column (down)
    int first, n;          // its k blocks
    int index;             // of a down item and its part
};
template <int DB> __host__ __device__ __forceinline__ int wide_across(int d) { return (d + 64 * DB - 1) / (64 * DB); }
template <int DB> __device__ __forceinline__ WideItem wide_item(const WideArgs &w, int count, int i) {
    WideItem t;
    const int gate = w.ztiles * count;
    t.down = i >= gate;
    if (!t.down) {
        t.z = i / count; t.col = i - t.z * count;
        t.first = 0; t.n = w.p.d >> 7; t.index = 0;
    } else {
        t.index = i - gate;
        const int across = wide_across<DB>(w.p.d), q = t.index / w.splits, part = t.index - q * w.splits;
        t.z = q / across; t.col = (q - t.z * across) * (64 * DB);
        t.first = count * part / w.splits; t.n = count * (part + 1) / w.splits - t.first;
    }
    return t;
}

// Until all of a token tile's activations are in memory (bounded).  They were stored by ordinary stores of other SMs and are read by TMA, so a proxy fence
// stands between the acquire and the loads.
__device__ __forceinline__ bool wide_ready(const unsigned *done, unsigned need, uint32_t *aborted, DeviceStatus *status) {
    for (uint32_t spin = 0; spin < kSpinLimit; ++spin) {
        unsigned v;
        asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(done) : "memory");
        if (v >= need) {
            asm volatile("fence.proxy.async;" ::: "memory");
            return true;
        }
        if (*reinterpret_cast<volatile uint32_t *>(aborted)) return false;
        __nanosleep(100);
    }
    *reinterpret_cast<volatile uint32_t *>(aborted) = 1;
    atomicCAS(&status->code, 0, (int)CS_ERR_TIMEOUT);
    return false;
}

// The pair's claims: one thread of its first CTA takes the next item when its token loads ask for it, and tells both CTAs, until there is none.  (Asynchronous
// stores that the barrier counts, so that nothing has to be released: 1 us a call against a store and an arrival.)
__device__ __forceinline__ void wide_tell(WideBars *bars, int slot, int item) {
#pragma unroll
    for (int cta = 0; cta < 2; ++cta) {
        const uint32_t bar = map_to_cta(smem_u32(&bars->claim_full[slot]), cta);
        asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], 4;" ::"r"(bar) : "memory");
        asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.b32 [%0], %1, [%2];"
                     ::"r"(map_to_cta(smem_u32(&bars->claim[slot]), cta)), "r"(item), "r"(bar) : "memory");
    }
}
__device__ __forceinline__ void wide_claim(WideBars *bars, unsigned *next, int first, int items, DeviceStatus *status) {
    if (first >= items) return;      // told while the list was made
    MxRing ring;
    for (int n = 1;; ++n) {
        ring.next(kWideClaims);
        if (!mx_wait(&bars->claim_ask, (n - 1) & 1, &bars->aborted, status)) return;
        if (n >= kWideClaims && !mx_wait<true>(&bars->claim_empty[ring.stage], ring.phase ^ 1, &bars->aborted, status)) return;
        const int item = (int)atomicAdd(next, 1u);
        wide_tell(bars, ring.stage, item);
        if (item >= items) return;
    }
}
// An arrival without release, which would hold the thread until its loads and stores, or the tensor core, have got that far: at 300 tokens of the 7B layer
// 10 us.  `read`: what was read before and may be overwritten after it, not negative; the address takes its sign, so that the arrival cannot go ahead.
__device__ __forceinline__ void wide_arrive(uint64_t *bar, int read) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(map_to_cta(smem_u32(bar), 0) + (uint32_t)(read >> 31)) : "memory");
}
// The next item for one of the roles, a thread or with WARP a warp; `items` or more: there is none, or a wait gave up.
template <bool WARP> __device__ __forceinline__ int wide_next(WideBars *bars, MxRing &ring, DeviceStatus *status) {
    bool ok = mx_wait<true>(&bars->claim_full[ring.stage], ring.phase, &bars->aborted, status);
    if (WARP) ok = __all_sync(0xffffffffu, ok);
    if (!ok) return 0x7fffffff;
    const int item = *reinterpret_cast<volatile int *>(&bars->claim[ring.stage]);
    if (WARP) __syncwarp();
    if (!WARP || (threadIdx.x & 31) == 0) wide_arrive(&bars->claim_empty[ring.stage], item);
    ring.next(kWideClaims);
    return item;
}

template <int DB> __global__ void __launch_bounds__(kWideThreads, 1)
mx_wide_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_xs, const __grid_constant__ CUtensorMap tm_gu,
               const __grid_constant__ CUtensorMap tm_gus, const __grid_constant__ CUtensorMap tm_a, const __grid_constant__ CUtensorMap tm_as,
               const __grid_constant__ CUtensorMap tm_d, const __grid_constant__ CUtensorMap tm_ds, const WideArgs w) {
    extern __shared__ uint8_t raw[];
    __shared__ WideBars bars;
    constexpr int kDownRows = 32 * DB;        // weight rows a CTA brings for a down item; 128 for gate/up
    const MxArgs &p = w.p;
    const uint32_t rank = cluster_ctarank();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    if (threadIdx.x == 0) {
        for (int s = 0; s < kWideStages; ++s) { mbar_init(&bars.full[s], 1); mbar_init(&bars.empty[s], 1); }
        mbar_init(&bars.acc_full, 1);
        mbar_init(&bars.acc_empty, 2 * kWideEpiWarps);
        mbar_init(&bars.claim_ask, 1);
        for (int s = 0; s < kWideClaims; ++s) { mbar_init(&bars.claim_full[s], 1); mbar_init(&bars.claim_empty[s], kWideTakers); }
        bars.aborted = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (const CUtensorMap *m : {&tm_x, &tm_xs, &tm_gu, &tm_gus, &tm_a, &tm_as, &tm_d, &tm_ds})
            asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    }
    if (warp == 1) {   // the same warp of both CTAs allocates for the pair
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&bars.tmem)), "r"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();        // the peer's barriers exist before anything signals them
    tc_fence_after();
    pdl_wait();
    pdl_launch_dependents();
    const bool claimer = rank == 0 && threadIdx.x == 96;
    unsigned first = 0;
    if (claimer) first = atomicAdd(w.next, 1u);      // on its way while the list is made
    if (p.fold) {
        if (threadIdx.x < 4) bars.all[threadIdx.x] = 0;
        __syncthreads();
        mx_mark(p.support, p.entries, p.G, bars.all, kWideThreads);
        __syncthreads();
        mx_list_of(bars.all, bars.list, &bars.count);
    } else {
        if (threadIdx.x == 0) bars.count = ld_dep(p.count);
        if (threadIdx.x < kMaxG) bars.list[threadIdx.x] = ld_dep(p.list + threadIdx.x);
    }
    if (claimer) wide_tell(&bars, 0, (int)first);
    __syncthreads();
    const int kb = p.d >> 7, count = bars.count, items = w.ztiles * (count + wide_across<DB>(p.d) * w.splits);

    if (warp == 0) {          // tokens, and the bytes both CTAs will bring
        if (elect_one()) {
            const uint32_t full0 = map_to_cta(smem_u32(&bars.full[0]), 0);
            MxRing ring, claims;
            int fill = 0, ready = -1;
            for (int i; (i = wide_next<false>(&bars, claims, p.status)) < items;) {
                const WideItem t = wide_item<DB>(w, count, i);
                if (t.n == 0) {
                    if (rank == 0) wide_arrive(&bars.claim_ask, 0);
                    continue;
                }
                const int asks = t.first + max(0, t.n - kWideAhead);
                if (t.down && t.z != ready) {
                    if (!wide_ready(w.done + t.z, (unsigned)count * 2 * kWideEpiWarps, &bars.aborted, p.status)) goto done;
                    ready = t.z;
                }
                const CUtensorMap *x = t.down ? &tm_a : &tm_x, *xs = t.down ? &tm_as : &tm_xs;
                const uint32_t bytes = 2 * (128 * 128 + (t.down ? kDownRows : 128) * 64 + 3 * kMxTileBytes);
                const int chunk = 2 * t.z + (int)rank, row = chunk * (t.down ? p.cap : kb);
                for (int j = t.first; j < t.first + t.n; ++j, ++fill) {
                    if (rank == 0 && j == asks) wide_arrive(&bars.claim_ask, 0);
                    if (fill >= kWideStages && !mx_wait(&bars.empty[ring.stage], ring.phase ^ 1, &bars.aborted, p.status)) goto done;
                    uint8_t *st = smem + ring.stage * kWideStageBytes;
                    if (rank == 0) mbar_expect_tx(&bars.full[ring.stage], bytes);
                    tma_load_2d_pair(st, x, j * 128, chunk * 128, full0 + 8u * ring.stage);
                    tma_load_2d_pair(st + 128 * 128 + kMxWBytes, xs, 0, row + j, full0 + 8u * ring.stage);
                    ring.next(kWideStages);
                }
            }
        }
    } else if (warp == 2) {   // weights
        if (elect_one()) {
            const uint32_t full0 = map_to_cta(smem_u32(&bars.full[0]), 0);
            MxRing ring, claims;
            int fill = 0, ahead = blockIdx.x;
            for (int i; (i = wide_next<false>(&bars, claims, p.status)) < items;) {
                const WideItem t = wide_item<DB>(w, count, i);
                const CUtensorMap *m = t.down ? &tm_d : &tm_gu, *ms = t.down ? &tm_ds : &tm_gus;
                // Gate/up: this CTA's half of the group.  Down: rows of W_down from where they stand, which may run into the next group's (columns
                // behind d, left out later); two tiles of scales from the one that holds the first column.
                for (int j = t.first; j < t.first + t.n; ++j, ++fill) {
                    if (fill >= kWideStages && !mx_wait(&bars.empty[ring.stage], ring.phase ^ 1, &bars.aborted, p.status)) goto done;
                    uint8_t *st = smem + ring.stage * kWideStageBytes + 128 * 128;
                    const uint32_t full = full0 + 8u * ring.stage;
                    const int tile = t.down ? bars.list[j] * kb + (t.col >> 7) : (bars.list[t.col] * kb + j) * 2;
                    tma_load_2d_pair(st, m, 0, tile * 128 + (t.down ? (t.col & 127) + (int)rank * kDownRows : (int)rank * 128), full);
                    tma_load_2d_pair(st + kMxWBytes + kMxTileBytes, ms, 0, tile, full);
                    if (!t.down && fill >= kWideStages && ahead < kb * count) {      // the down product's weights on their way to L2
                        const size_t next = (size_t)bars.list[ahead / kb] * kb + ahead % kb;
                        prefetch_l2(w.down_codes + next * kMxWLoad, kMxWLoad);
                        prefetch_l2(w.down_scales + next * kMxTileBytes, kMxTileBytes);
                        ahead += gridDim.x;
                    }
                    ring.next(kWideStages);
                }
            }
        }
    } else if (warp == 1) {
        if (rank == 0 && elect_one()) {
            const uint32_t base = smem_u32(smem), tmem = bars.tmem;
            MxRing ring, claims;
            int turn = 0;
            for (int i; (i = wide_next<false>(&bars, claims, p.status)) < items;) {
                const WideItem t = wide_item<DB>(w, count, i);
                if (t.n == 0) continue;
                uint32_t idesc[4];
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) idesc[kk] = wide_idesc(t.down ? 64 * DB : 256, kk);
                const uint32_t shift = t.down ? (uint32_t)(t.col & 127) >> 5 : 0;     // the first column's place in its tile of scales
                if (turn > 0 && !mx_wait(&bars.acc_empty, (turn - 1) & 1, &bars.aborted, p.status)) goto done;
                tc_fence_after();
                for (int j = 0; j < t.n; ++j) {
                    if (!mx_wait(&bars.full[ring.stage], ring.phase, &bars.aborted, p.status)) goto done;
                    tc_fence_after();
                    const uint32_t a = base + ring.stage * kWideStageBytes, b = a + 128 * 128, sc = b + kMxWBytes;
                    const uint32_t sa = tmem + 256 + ring.stage * 12, sb = sa + 4;
                    wide_copy_scales(sa, sc);
                    wide_copy_scales(sb, sc + kMxTileBytes);
                    wide_copy_scales(sb + 4, sc + 2 * kMxTileBytes);
                    const uint64_t ad = desc_sw128(a, 0), bd = desc_sw128(b, 0);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) wide_mma(tmem, ad + 2 * kk, bd + 2 * kk, idesc[kk], sa, sb + shift, (j | kk) != 0);
                    tc_commit_pair(&bars.empty[ring.stage]);
                    ring.next(kWideStages);
                }
                tc_commit_pair(&bars.acc_full);
                ++turn;
            }
        }
    } else if (warp == 3) {
        if (rank == 0) {
            if (claimer) wide_claim(&bars, w.next, (int)first, items, p.status);
        } else if (p.fold) {
            mx_check(p.support, p.entries, p.k, p.G, pair, pairs, p.status);
        }
    } else {
        const int quarter = warp & 3, half = (warp >> 2) - 1;      // lanes and half of the columns
        const uint32_t empty0 = map_to_cta(smem_u32(&bars.acc_empty), 0);
        const uint32_t acc = bars.tmem + ((uint32_t)(quarter * 32) << 16);
        MxRing claims;
        int turn = 0;
        for (;;) {
            __syncwarp();      // lanes without a token skip parts of an item
            const int i = wide_next<true>(&bars, claims, p.status);
            if (i >= items) break;
            const WideItem t = wide_item<DB>(w, count, i);
            const int token = t.z * kWideTokens + (int)rank * 128 + quarter * 32 + lane;
            if (!t.down) {
                bool member = p.shared;      // whether this token uses the group; found while the products run
                if (!p.shared && token < p.B) {
                    const int g = bars.list[t.col];
                    if (p.fold)
                        for (int j = 0; j < p.k; ++j) member |= ld_dep(p.support + (size_t)token * p.k + j) == g;
                    else
                        member = ld_dep(reinterpret_cast<const int32_t *>(p.mask) + 4 * (size_t)token + (g >> 5)) >> (g & 31) & 1;
                }
                __syncwarp();
                if (!__all_sync(0xffffffffu, mx_wait(&bars.acc_full, turn & 1, &bars.aborted, p.status))) break;
                tc_fence_after();
                uint32_t v[4][32];
#pragma unroll
                for (int b = 0; b < 4; ++b) tc_ld32(acc + half * 128 + 32 * b, v[b]);
                tc_wait_ld();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_cluster(empty0);
                ++turn;
                if (token < p.B) {
                    uint32_t scales = 0;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        float m = 0.f;
#pragma unroll
                        for (int c = 0; c < 32; ++c) {      // in place: the registers are what there is
                            const float a = swiglu(__uint_as_float(v[b][c]), __uint_as_float(v[b + 2][c]));
                            v[b][c] = __float_as_uint(a);
                            m = max_abs(m, a);
                        }
                        const uint32_t byte = member ? mx_scale_byte<true>(__float_as_uint(m)) : 0u;
                        const float inv = mx_inverse(byte);
                        uint32_t o[8];
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            o[c] = !member || byte == 255 ? 0u : pack_e4m3(__uint_as_float(v[b][4 * c]) * inv, __uint_as_float(v[b][4 * c + 1]) * inv,
                                                                           __uint_as_float(v[b][4 * c + 2]) * inv, __uint_as_float(v[b][4 * c + 3]) * inv);
                        store32(p.a + (size_t)token * p.cap * 128 + t.col * 128 + half * 64 + b * 32, o);
                        scales |= byte << (8 * b);
                    }
                    *reinterpret_cast<uint16_t *>(p.a_scales + ((size_t)(token >> 7) * p.cap + t.col) * kMxTileBytes + (token & 31) * 16 +
                                                  ((token & 127) >> 5) * 4 + half * 2) = (uint16_t)scales;
                }
                __syncwarp();      // one lane's release covers the warp's stores; a fence in each lane cost 3 us an item
                if (lane == 0) asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(w.done + t.z) : "memory");
            } else {
                uint32_t v[DB][32];
                if (t.n > 0) {
                    if (!__all_sync(0xffffffffu, mx_wait(&bars.acc_full, turn & 1, &bars.aborted, p.status))) break;
                    tc_fence_after();
#pragma unroll
                    for (int b = 0; b < DB; ++b) tc_ld32(acc + half * kDownRows + 32 * b, v[b]);
                    tc_wait_ld();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(empty0);
                    ++turn;
                } else {
#pragma unroll
                    for (int b = 0; b < DB; ++b)
#pragma unroll
                        for (int c = 0; c < 32; ++c) v[b][c] = 0;
                }
                if (token >= p.B) continue;
#pragma unroll
                for (int b = 0; b < DB; ++b) {
                    const int col = t.col + half * kDownRows + 32 * b;
                    if (col >= p.d) break;
                    if (w.splits > 1) {
                        float *to = w.partial + ((size_t)t.index * kWideTokens + token - t.z * kWideTokens) * 256 + half * kDownRows + 32 * b;
#pragma unroll
                        for (int h = 0; h < 4; ++h) {
                            uint32_t o[8];
#pragma unroll
                            for (int c = 0; c < 8; ++c) o[c] = v[b][8 * h + c];
                            store32(to + 8 * h, o);
                        }
                        continue;
                    }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t o[8];
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            const __nv_bfloat162 f = __floats2bfloat162_rn(__uint_as_float(v[b][16 * h + 2 * c]), __uint_as_float(v[b][16 * h + 2 * c + 1]));
                            o[c] = *reinterpret_cast<const uint32_t *>(&f);
                        }
                        __nv_bfloat16 *to = p.out + (size_t)token * p.d + col + 16 * h;
                        if (w.whole) {
                            store32(to, o);
                        } else {
                            reinterpret_cast<uint4 *>(to)[0] = make_uint4(o[0], o[1], o[2], o[3]);
                            reinterpret_cast<uint4 *>(to)[1] = make_uint4(o[4], o[5], o[6], o[7]);
                        }
                    }
                }
            }
        }
    }
done:
    __syncwarp();
    mx_settle(&bars.aborted);
    // Neither CTA leaves (or frees tensor memory) while the other may still read its shared memory or signal its barriers; every wait above
    // is bounded, so both reach this point.
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(bars.tmem), "r"(512) : "memory");
    }
    // the last pair to end clears the counters for the next call
    if (threadIdx.x == 0 && rank == 0) {
        __threadfence();
        if (atomicAdd(w.done + w.ztiles, 1u) == (unsigned)pairs - 1) {
            for (int z = 0; z <= w.ztiles; ++z) w.done[z] = 0;
            *w.next = 0;
        }
    }
}

// out[t, c] = the sum of an item's parts, in their order.  Four columns a thread.
__global__ void __launch_bounds__(256)
mx_wide_sum_kernel(const WideArgs w, int width) {
    pdl_launch_dependents();
    pdl_wait();
    const int across = (w.p.d + width - 1) / width, d4 = w.p.d >> 2;
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= w.p.B * d4) return;
    const int t = i / d4, c = (i - t * d4) * 4, z = t / kWideTokens, x = c / width;
    const float *from = w.partial + ((size_t)(z * across + x) * w.splits * kWideTokens + t - z * kWideTokens) * 256 + c - x * width;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < w.splits; ++s) {
        const float4 u = ld_dep4(from + (size_t)s * kWideTokens * 256);
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v.x, v.y), hi = __floats2bfloat162_rn(v.z, v.w);
    *reinterpret_cast<uint2 *>(w.p.out + (size_t)t * w.p.d + c) = make_uint2(*reinterpret_cast<const uint32_t *>(&lo), *reinterpret_cast<const uint32_t *>(&hi));
}

// Tiles of 512 scales, `box_tiles` to a box.
bool make_map_scales(CUtensorMap *map, const void *base, uint64_t tiles, uint32_t box_tiles) {
    EncodeTiledFn fn = encode_fn();
    if (fn == nullptr) return false;
    const cuuint64_t dims[2] = {128, tiles}, strides[1] = {kMxTileBytes};
    const cuuint32_t box[2] = {128, box_tiles}, estr[2] = {1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, const_cast<void *>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr size_t kWideSmem = 1024 + (size_t)kWideStages * kWideStageBytes;

}  // namespace

cs_status prepare_mx_wide(cs_plan *plan) {
    (void)plan;
    for (auto *k : {mx_wide_kernel<3>, mx_wide_kernel<4>})
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kWideSmem) != cudaSuccess || prefer_shared(k) != cudaSuccess)
            return CS_ERR_CUDA;
    return prefer_shared(mx_wide_sum_kernel) == cudaSuccess ? CS_OK : CS_ERR_CUDA;
}

size_t mx_wide_partial_bytes(const cs_plan *plan) {      // plans of small batches never come here
    return plan->cfg.max_tokens <= 128 ? 0 : (size_t)(plan->sm_count / 2) * kWideTokens * 256 * sizeof(float);
}

cs_status launch_mx_wide(cs_plan *plan, const cs_mx_layer *L, const uint8_t *q, const MxArgs &args, cudaStream_t st) {
    const int d = args.d, kb = d / 128, G = args.G, B = args.B, chunks = (B + 127) / 128, pairs = plan->sm_count / 2;
    WideArgs w;
    w.p = args;
    w.ztiles = (B + kWideTokens - 1) / kWideTokens;
    w.partial = plan->mx_partial; w.next = plan->mx_done; w.done = plan->mx_done + kMxDoneOffset;
    w.down_codes = L->down_codes; w.down_scales = L->down_scales;
    w.whole = reinterpret_cast<uintptr_t>(args.out) % 32 == 0;
    // Output columns of a down item: the width whose rounds over the pairs cost least (13B shape, 2048 tokens: 160 items of 256 are three rounds, 216
    // of 192 three rounds of 3/4).
    const int n256 = wide_across<4>(d) * w.ztiles, n192 = wide_across<3>(d) * w.ztiles;
    const bool narrow = (n192 + pairs - 1) / pairs * 3 < (n256 + pairs - 1) / pairs * 4;
    const int width = narrow ? 192 : 256, items = narrow ? n192 : n256;
    // Fewer items than half the pairs: cut the list, into parts of at least four k blocks
    w.splits = 2 * items <= pairs ? max(1, min(min(pairs / items, 8), args.cap / 4)) : 1;
    CUtensorMap x, xs, wg, wgs, a, as, wd, wds;
    if (!make_map_bytes(&x, q, d, B, 128) || !make_map_scales(&xs, args.x_scales, (uint64_t)chunks * kb, 1) ||
        !make_map_tiles(&wg, L->gate_up_codes, (uint64_t)2 * G * kb) || !make_map_scales(&wgs, L->gate_up_scales, (uint64_t)2 * G * kb, 2) ||
        !make_map_bytes(&a, plan->mx_a, (uint64_t)args.cap * 128, B, 128) || !make_map_scales(&as, plan->mx_a_scales, (uint64_t)chunks * args.cap, 1) ||
        !make_map_tiles(&wd, L->down_codes, (uint64_t)kb * G, width / 2) || !make_map_scales(&wds, L->down_scales, (uint64_t)kb * G, 2)) {
        snprintf(plan->cuda_error, sizeof plan->cuda_error, "cuTensorMapEncodeTiled failed");
        return CS_ERR_CUDA;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(2 * (unsigned)min((int64_t)pairs, (int64_t)w.ztiles * args.cap + (int64_t)items * w.splits));
    cfg.blockDim = dim3(kWideThreads); cfg.dynamicSmemBytes = kWideSmem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = 2;
    cudaError_t e = cudaLaunchKernelEx(&cfg, narrow ? mx_wide_kernel<3> : mx_wide_kernel<4>, x, xs, wg, wgs, a, as, wd, wds, w);
    if (e != cudaSuccess) return record_cuda(plan, e, "mx_wide_kernel");
    plan->launches += 1;
    if (w.splits > 1) {
        e = launch_pdl(true, mx_wide_sum_kernel, dim3((unsigned)(((int64_t)B * (d / 4) + 255) / 256)), dim3(256), 0, st, w, width);
        if (e != cudaSuccess) return record_cuda(plan, e, "mx_wide_sum_kernel");
        plan->launches += 1;
    }
    return CS_OK;
}

}  // namespace cs
