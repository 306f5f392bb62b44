// tile_gemm.cuh -- what the products on tcgen05 tiles share (mx_gemm.cuh, i8_gemm.cuh): bounded waits, clusters and the list of tiles over
// experts' ragged rows.
//
// A tile is kTileRowsW rows of W (the lanes of tensor memory; two CTAs' in a pair) by some tokens.  P: the kernel's parameters (M, N, E, nt,
// wtiles, wdiv_m, wdiv_s, offsets, status, wait_cycles).
#pragma once
#include <cstdint>

#include "attn_ptx.cuh"
#include "float_act.cuh"
#include "ilw_kernels.h"
#include "ilwdetr.h"

namespace ilw {

constexpr int kTileRowsW = 128;   // rows of W a CTA
// A CTA a tile; several CTAs of a cluster to a tile's K; two SMs a tile.
enum TileMode { TILE_ONE = 0, TILE_SPLIT = 1, TILE_PAIR = 2 };

struct TileExpert {
    int32_t start, row, end, width;  // first token tile, its rows [row, end), rows a tile
};

namespace {

struct Tile {
    int32_t e, row0, rows, n0;
};

// Bounded wait: false (after latching `code` and raising the abort flag) when it ran out, or when another role aborted.
template <typename P> __device__ __forceinline__ bool wait_bar(uint32_t b, uint32_t parity, volatile int *abort, const P &p, int code) {
    if (bar_try(b, parity)) return true;
    const long long t0 = clock64();
    for (uint32_t i = 0;; ++i) {
        if (bar_try(b, parity)) return true;
        if ((i & 63) == 63) {
            if (*abort) return false;
            if (clock64() - t0 > p.wait_cycles) {
                if (p.status) atomicExch(p.status, code);
                *abort = 1;
                return false;
            }
        }
    }
}
// The same for a whole warp, one answer for all lanes (the tcgen05 instructions after it are warp-wide).
template <typename P> __device__ __forceinline__ bool wait_warp(uint32_t b, uint32_t parity, volatile int *abort, const P &p, int code) {
    return __all_sync(0xffffffffu, wait_bar(b, parity, abort, p, code));
}
// The same in fewer instructions: a short loop out of line, which sleeps kSleep ns between tries where waits are long.  A try that has to wait
// comes back within some 100 clocks, and where issue slots are short 28 warps of tries, branches and counters take them from
// others (40 of 100 instructions of a large int8 product; 641 us, so 615).  The MXFP4 products wait on shorter chains and lose by
// it (8192 cubed 166 us, so 189).
__device__ __forceinline__ bool bar_try_now(uint32_t b, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n .reg .pred P;\n mbarrier.try_wait.parity.shared::cta.b64 P, [%1], %2;\n selp.b32 %0, 1, 0, P;\n}\n"
        : "=r"(ok)
        : "r"(b), "r"(parity)
        : "memory");
    return ok != 0;
}
template <int kSleep, typename P> __device__ __noinline__ bool wait_lean_long(uint32_t b, uint32_t parity, volatile int *abort, const P *p, int code) {
    const long long t0 = clock64();
    for (;;) {
#pragma unroll 1
        for (int i = 0; i < 64; ++i) {
            if (kSleep) __nanosleep(kSleep);
            if (__all_sync(0xffffffffu, bar_try_now(b, parity))) return true;
        }
        bool over = *abort;
        if (!over && clock64() - t0 > p->wait_cycles) {
            if (p->status) atomicExch(p->status, code);
            *abort = 1;
            over = true;
        }
        if (__any_sync(0xffffffffu, over)) return false;
    }
}
template <int kSleep = 0, typename P> __device__ __forceinline__ bool wait_lean(uint32_t b, uint32_t parity, volatile int *abort, const P &p, int code) {
    return __all_sync(0xffffffffu, bar_try_now(b, parity)) || wait_lean_long<kSleep>(b, parity, abort, &p, code);
}
// The same for a lane that issues loads or MMAs on its own, with the long way out of line: its loop then keeps the operands in
// uniform registers and a wait with nothing to wait for costs next to nothing (a block of K: 225 clocks for 6 copies and 4
// MMAs of 16 tokens, what they take; with a vote of the warp 395).
template <typename P> __device__ __noinline__ bool wait_long(uint32_t b, uint32_t parity, volatile int *abort, const P *p, int code) {
    return wait_bar(b, parity, abort, *p, code);
}
template <typename P> __device__ __forceinline__ bool wait_lane(uint32_t b, uint32_t parity, volatile int *abort, const P &p, int code) {
    return bar_try(b, parity) || wait_long(b, parity, abort, &p, code);
}

// This barrier's address in CTA `rank` of the cluster, and an arrival there.  What the arrivals of a pair order is read by the
// tensor core alone, through the async proxy, to which its writers hand it themselves (TMA, or fence.proxy.async
// after the stores); a release at cluster scope on top of that held each arrival up by some 1000 clocks.
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void arrive_cluster(uint32_t addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *m) {
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)m) : "memory");
}

// A value that is the same in every lane, in a uniform register: the operands of TMA loads and MMAs are uniform
// registers, and each one that has to be moved there at its instruction costs some 50 clocks (with values that the
// compiler could not know to be uniform a TMA load took 300 clocks, which was the rate of every product).
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __reduce_max_sync(0xffffffffu, v); }
// An arrival at `bar` (of a pair: in both CTAs, unless `local`) when the MMAs and copies issued so far have ended.
template <bool PAIR>
__device__ __forceinline__ void commit_mma(uint32_t bar, bool local = false) {
    if constexpr (PAIR) {
        if (!local)
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                         "h"((uint16_t)3)
                         : "memory");
        else
            asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    } else {
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    }
}
__device__ __forceinline__ void lds128(uint32_t a, uint32_t (&v)[4]) {
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                 : "r"(a)
                 : "memory");
}

// (By a whole warp.) The list of tiles: the experts that have rows, in order, `count` of them with `sum` tiles of up to p.nt rows
// (multiples of kStep), and an end.  Their ranges are held in order, apart and inside [0, M], whatever the offsets say; rows
// before `head` and from `tail` on are no expert's.
template <int kStep, typename P>
__device__ __forceinline__ void list_tiles(const P &p, TileExpert *tab, int32_t *tab_id, int lane, int32_t &sum, int32_t &count, int32_t &head, int32_t &tail) {
    const int32_t M = (int32_t)p.M;
    int32_t before = 0;  // (sum, count, before: of the experts before these 32: tiles, those with rows, end of the last range)
    sum = count = 0, head = M;
    for (int e0 = 0; e0 < p.E; e0 += 32) {
        const int e = e0 + lane;
        int32_t l = 0, h = e < p.E ? M : 0;
        if (p.offsets && e < p.E) {
            l = max(0, min(p.offsets[e], M));
            h = max(0, min(p.offsets[e + 1], M));
        }
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, h, d);
            if (lane >= d) h = max(h, y);
        }
        h = max(h, before);
        const int32_t prev = __shfl_up_sync(0xffffffffu, h, 1);
        l = min(max(l, lane ? prev : before), h);
        if (e0 == 0) head = __shfl_sync(0xffffffffu, l, 0);
        before = __shfl_sync(0xffffffffu, h, 31);
        const int32_t rows = e < p.E ? h - l : 0, tiles = (rows + p.nt - 1) / p.nt;
        int32_t x = tiles;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int32_t y = __shfl_up_sync(0xffffffffu, x, d);
            if (lane >= d) x += y;
        }
        const uint32_t with = __ballot_sync(0xffffffffu, rows > 0);
        if (rows > 0) {  // equal tiles of at most nt, multiples of 16 (a pair's: of 32)
            const int i = count + __popc(with & ((1u << lane) - 1));
            *(int4 *)(tab + i) = make_int4(sum + x - tiles, l, h, ((rows + tiles - 1) / tiles + kStep - 1) & ~(kStep - 1));
            tab_id[i] = e;
        }
        sum += __shfl_sync(0xffffffffu, x, 31);
        count += __popc(with);
    }
    if (lane == 0) tab[count].start = sum;
    tail = before;
    __syncwarp();
}

// (By a whole warp.) Tile t: the tile of W's rows runs fastest, so CTAs that run together share a token tile's rows.  tab: the
// experts that have rows, n of them (n <= 1024: two probes of 32), and an end.  (kRowsW: rows of W a tile.)
template <int MODE, int kRowsW = kTileRowsW, typename P>
__device__ __forceinline__ Tile find_tile(const P &p, const TileExpert *tab, const int32_t *id, int n, int32_t t, uint32_t rank) {
    const int lane = threadIdx.x & 31;
    const int32_t tt = (int32_t)((__umulhi((uint32_t)t, p.wdiv_m) + (uint32_t)t) >> p.wdiv_s);  // t / wtiles
    int a = 0;  // the expert with start <= tt < the next one's
    if (n > 32) a = 32 * (__popc(__ballot_sync(0xffffffffu, 32 * lane < n && tab[min(32 * lane, n)].start <= tt)) - 1);
    a += __popc(__ballot_sync(0xffffffffu, a + lane < n && tab[min(a + lane, n)].start <= tt)) - 1;
    const int4 x = *(const int4 *)(tab + a);
    Tile r;
    r.e = id[a];
    r.row0 = x.y + (tt - x.x) * x.w;
    r.rows = min(x.w, x.z - r.row0);
    r.n0 = (t - tt * p.wtiles) * (MODE == TILE_PAIR ? 2 * kRowsW : kRowsW) + (MODE == TILE_PAIR ? rank * kRowsW : 0);
    return r;
}

}  // namespace
}  // namespace ilw
