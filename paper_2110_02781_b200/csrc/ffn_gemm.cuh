// What the two product kernels share: operand order, epilogue pieces, tensor maps, launches with clusters.
#pragma once
#include <algorithm>
#include <atomic>
#include "ffn_math.cuh"
#include "gemm_tc_common.cuh"

namespace ftp {
using namespace tc;
namespace ffn {

constexpr int BK = 64;                       // reduction elements per stage: one 128-byte swizzle row
// Operand tiles arrive one plane of A and of B at a time, the smallest planes of a block first, each read from memory once;
// the products that matter are issued as soon as their planes are there:
//   plane 1: A1 B1    plane 0: A0 B2, A2 B0, A0 B1, A1 B0, A0 B0
// (those with planes that exist).  Dropped: A1 B2, A2 B1, A2 B2, below 2^-24 of the result.
//
// Float results: the tensor cores cut their accumulator instead of rounding it, an error that grows with the number of
// steps (measured 3.5e-5 of the result after 2048 steps of 16 elements).  So the products of the main planes have an
// accumulator of their own, and every CHUNK blocks both are emptied into registers, which add with rounding.
constexpr int CHUNK = 4;
// bf16 results stay in the accumulator up to LONG_SUM blocks a slice (131072 terms): for terms of one sign that costs about 2^-24
// of the result per step, 1/8 of bf16's half step at that length and twice the half step for 8M terms in eight slices.  Longer
// slices are emptied every LONG_CHUNK blocks (200000 x 2048 x 2048 weight gradient: 1411 instead of 1118 us).
constexpr int LONG_SUM = 2048, LONG_CHUNK = 64;

struct KArgs {
    Epi e[2];
    long long M;
    int N;
    int kb_part, parts_k;                    // 64-wide reduction blocks per part, parts of the reduction
    int parts_n;                             // 2: the column tiles of output 1 follow those of output 0
    int tiles_m, tiles_n;                    // column tiles of one output
    int pa, pb, np;                          // planes of A and of B, the larger of the two
    int chunk;                               // blocks per accumulation in the tensor cores (float results, long_sum)
    int long_sum;                            // a bf16 result whose slices are longer than LONG_SUM blocks
    int* err;
};

namespace {

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32_issue(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// 32 columns of an accumulator, and of its small terms `small` columns further, added to acc[0..31].  Where an operand holds an
// infinity or a NaN, its first plane alone carries it and the product of the first planes is what the operands' product is;
// the small terms beside it are that infinity times what is left of the other operand, of either sign or 0: not added.
__device__ __forceinline__ void add_acc(uint32_t taddr, uint32_t small, bool both, float* acc) {
    uint32_t r[32], q[32];
    tmem_ld32_issue(taddr, r);
    if (both) tmem_ld32_issue(taddr + small, q);
    tmem_ld_wait();
    if (both) {
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const float v = __uint_as_float(r[i]);
            acc[i] += fabsf(v) < __uint_as_float(0x7f800000u) ? v + __uint_as_float(q[i]) : v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[i] += __uint_as_float(r[i]);
    }
}
// MN-major operand: slabs of 64 reduction rows x 64 elements (128-byte rows, 128-byte swizzle), slab_bytes apart
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t slab_bytes) {
    return (uint64_t)((saddr >> 4) & 0x3FFF) | (uint64_t)((slab_bytes >> 4) & 0x3FFF) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
__device__ __forceinline__ void mbar_arrive_one(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_rank(uint32_t saddr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ uint32_t ld_cluster1(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// Eight lanes (a quarter of a warp, lane % 8 in column order) hold one 32-column block of a row, four columns each:
// write their codes and the block's scale byte.
__device__ __forceinline__ void img_store4(const Image& im, long long m, int n, const float (&v)[4], bool row_ok) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    const unsigned e = img_exp(top);
    const float inv = img_inv(e);
    if (row_ok && n < im.pitch) {
        *reinterpret_cast<unsigned*>(im.q + m * im.pitch + n) =
            pack_codes(img_code(v[0], inv), img_code(v[1], inv), img_code(v[2], inv), img_code(v[3], inv));
        if ((threadIdx.x & 7) == 0) im.e[m * (im.pitch / IMG_BLOCK) + n / IMG_BLOCK] = (uint8_t)e;
    }
}

// act of N values: the choice outside the loop, so that the values' instruction chains interleave
template <bool FAST, int N>
__device__ __forceinline__ void act_all(float (&a)[N], int act) {
    switch (act) {
        case FTP_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = act_value<FAST>(a[i], FTP_ACT_RELU);
            break;
        case FTP_ACT_RELU6:
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = act_value<FAST>(a[i], FTP_ACT_RELU6);
            break;
        case FTP_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = act_value<FAST>(a[i], FTP_ACT_GELU);
            break;
        case FTP_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) a[i] = act_value<FAST>(a[i], FTP_ACT_SILU);
            break;
        default: break;
    }
}

// Bounded wait: as mbar_wait, but the clock and the error word are looked at only once a wait has lasted for 256 tests.
__device__ __forceinline__ bool wait_for(uint32_t bar, uint32_t parity, int* err, int code) {
    unsigned long long t0 = 0;
    for (unsigned it = 1;; ++it) {
        if (mbar_test(bar, parity)) return true;
        if ((it & 255u) == 0u) {
            if (*((volatile int*)err) != 0) return false;             // another role already gave up
            const unsigned long long t = gtime();
            if (t0 == 0) t0 = t;
            else if (t - t0 > TC_WAIT_NS) { atomicCAS(err, 0, code); return false; }
        }
    }
}
// the same answer for the whole warp
__device__ __forceinline__ bool warp_wait_for(uint32_t bar, uint32_t parity, int* err, int code) {
    return __all_sync(0xffffffffu, wait_for(bar, parity, err, code));
}
// a test that does not suspend the thread
__device__ __forceinline__ bool mbar_peek(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// the same for a barrier that was tested before
__device__ __forceinline__ bool warp_ready(bool seen, uint32_t bar, uint32_t parity, int* err, int code) {
    return __all_sync(0xffffffffu, seen) || warp_wait_for(bar, parity, err, code);
}
// one thread of a converged warp
__device__ __forceinline__ bool elect_one() {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.b32 %0, 1, 0, p;\n}" : "=r"(ok));
    return ok != 0;
}

// A position in the ring of operand tiles: the slot and the parity of its use.  
template <int STAGES>
struct Slot {
    int s = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() { ahead(1); }
    __device__ __forceinline__ void ahead(int n) {                   // n <= STAGES
        s += n;
        if (s >= STAGES) { s -= STAGES; parity ^= 1; }
    }
};

// The copies are issued by PRODUCERS warps that take the slots in turn (a slot's wait, count and copies take a warp about
// 600 cycles, the MMAs of a slot 256 to 512).  Producer j's slots are those of number j, j + PRODUCERS, ... over all tiles;
// with three planes a producer always fetches the same one.
constexpr int PRODUCERS = 3;
__device__ __forceinline__ int producer_of(int warp) { return warp == 0 ? 0 : warp - 1; }           // warps 0, 2, 3

__device__ __forceinline__ void umma_bf16_pair(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// signals the barrier at this offset in the CTAs of `mask` (both of the pair) once the MMAs issued so far have completed
__device__ __forceinline__ void umma_commit_pair(uint32_t bar, uint16_t mask) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"(mask) : "memory");
}

// The MMA warp of either kernel: `blocks` 64-wide blocks per tile, one tile (tile kernel) or `tiles` of them in turn.  The
// whole warp walks the loop and one elected thread issues, so that descriptors and addresses stay in uniform registers: with the
// loop inside a single-thread branch four MMAs and a commit took 1300 cycles to issue, more than they take to run.
//   full / empty: ring barriers; accf / acce: accumulator complete / read, BUFS of them in turn.
template <int CG, int BN, int STAGES, uint32_t STAGE_BYTES, uint32_t A_BYTES, bool AMN, bool BMN, bool CHUNKED, int BUFS>
__device__ __forceinline__ bool mma_warp(uint32_t ring, uint32_t full0, uint32_t empty0, uint32_t accf0, uint32_t acce0, uint32_t tmem, int tiles, int blocks,
                                         const KArgs& p, uint16_t mask = 3) {
    constexpr uint32_t SLAB = 64 * BK * 2;
    constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (AMN ? 1u << 15 : 0u) | (BMN ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) |
                               ((uint32_t)(CG * 128 >> 4) << 24);
    const uint64_t a0 = AMN ? desc_mn(ring, SLAB) : umma_desc_k_sw128(ring), b0 = BMN ? desc_mn(ring + A_BYTES, SLAB) : umma_desc_k_sw128(ring + A_BYTES);
    Slot<STAGES> sl;
    // float results: an accumulator is BN columns for the products of the main planes and BN for all the small ones, so that
    // adding those costs the sum no accuracy
    constexpr uint32_t ACC = CHUNKED ? 2 * BN : BN;
    int chunk = 0;
    bool first = true, first_small = true, peek0 = false, peek1 = false;
    uint32_t d0 = tmem;
    auto four = [&](uint32_t d, bool& first, int sa, int sb) {       // a block of the planes in slots sa and sb; one thread
        const uint64_t ad = a0 + (uint64_t)((uint32_t)sa * (STAGE_BYTES >> 4)), bd = b0 + (uint64_t)((uint32_t)sb * (STAGE_BYTES >> 4));
#pragma unroll
        for (int k = 0; k < BK / 16; ++k) {                          // 16 elements further: 32 bytes along a K-major row, 16 rows of an MN-major slab
            const uint32_t acc = first && k == 0 ? 0u : 1u;
            if (CG == 2) umma_bf16_pair(d, ad + (uint64_t)(k * (AMN ? 128 : 2)), bd + (uint64_t)(k * (BMN ? 128 : 2)), idesc, acc);
            else umma_bf16(d, ad + (uint64_t)(k * (AMN ? 128 : 2)), bd + (uint64_t)(k * (BMN ? 128 : 2)), idesc, acc);
        }
        first = false;
    };
    auto commit = [&](uint32_t bar) { if (CG == 2) umma_commit_pair(bar, mask); else umma_commit(bar); };
    for (int t = 0; t < tiles; ++t) {
        int left = 0;
        for (int kb = 0; kb < blocks; ++kb) {
            if (left == 0) {                                         // a new accumulation
                const int b = BUFS == 1 ? 0 : chunk & 1;
                if (chunk >= BUFS && !warp_wait_for(acce0 + 8 * b, ((BUFS == 1 ? chunk : chunk >> 1) & 1) ^ 1, p.err, 4)) return false;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                d0 = tmem + (uint32_t)b * ACC;
                first = first_small = true;
                left = CHUNKED ? min(p.chunk, blocks - kb) : blocks;
            }
            --left;
            // The barriers of the slots to come are tested before this block's MMAs are issued (a test of a barrier that is
            // complete still takes over a hundred cycles), so that the wait for them usually costs a vote.
            if (!CHUNKED || p.np == 1) {
                const int s0 = sl.s;
                if (!warp_ready(peek0, full0 + 8 * s0, sl.parity, p.err, 2)) return false;
                sl.next();
                const bool two = STAGES >= 6 && left > 0;            // two blocks a trip where the ring is long
                const int s1 = sl.s;
                if (two) {
                    if (!warp_ready(peek1, full0 + 8 * s1, sl.parity, p.err, 2)) return false;
                    sl.next();
                    --left;
                    ++kb;
                }
                peek0 = mbar_peek(full0 + 8 * sl.s, sl.parity);
                if (STAGES >= 6) {
                    Slot<STAGES> then = sl;
                    then.next();
                    peek1 = mbar_peek(full0 + 8 * then.s, then.parity);
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (elect_one()) {
                    four(d0, first, s0, s0);
                    commit(empty0 + 8 * s0);
                    if (two) {
                        four(d0, first, s1, s1);
                        commit(empty0 + 8 * s1);
                    }
                    if (left == 0) commit(accf0 + 8 * (BUFS == 1 ? 0 : chunk & 1));
                }
                first = false;
            } else {
                const int s2 = sl.s;
                if (!warp_wait_for(full0 + 8 * sl.s, sl.parity, p.err, 2)) return false;
                sl.next();
                const int s1 = sl.s;
                if (!warp_wait_for(full0 + 8 * sl.s, sl.parity, p.err, 2)) return false;
                sl.next();
                const bool mid = p.pa > 1 && p.pb > 1;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (mid && elect_one()) four(d0 + BN, first_small, s1, s1);
                if (mid) first_small = false;
                const int s0 = sl.s;
                if (!warp_wait_for(full0 + 8 * sl.s, sl.parity, p.err, 2)) return false;
                sl.next();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if (elect_one()) {
                    if (p.pb > 2) four(d0 + BN, first_small, s0, s2);
                    if (p.pa > 2) four(d0 + BN, first_small, s2, s0);
                    if (p.pb > 1) four(d0 + BN, first_small, s0, s1);
                    if (p.pa > 1) four(d0 + BN, first_small, s1, s0);
                    four(d0, first, s0, s0);
                    commit(empty0 + 8 * s2);
                    commit(empty0 + 8 * s1);
                    commit(empty0 + 8 * s0);
                    if (left == 0) commit(accf0 + 8 * (BUFS == 1 ? 0 : chunk & 1));
                }
                first = first_small = false;
            }
            __syncwarp();
            if (left == 0) ++chunk;
        }
    }
    return true;
}

// Rows rank, rank + S, ... of a 128-row tile that the S CTAs `first`, `first` + stride, ... of the cluster have each staged in
// shared memory (BN columns, PITCH floats between rows), added and finished.  All threads of the block; a thread takes four
// columns of four rows at a time, so that their loads and activations overlap (a row at a time: 14.8 instead of 10.4 us for
// 1024 x 1024 x 1024 on 128 x 128 tiles).  A CTA adds its own sums first and the others' in turn from there: an order that
// depends on the row alone, and no two CTAs read the same one at a time (all from the first: 1.5 us more with S = 4).
template <typename T, int EPI, int BN, int PITCH>
__device__ __forceinline__ void finish_rows(const Epi& e, uint32_t base, uint32_t S, uint32_t rank, uint32_t first, uint32_t stride, long long m0, int n0, long long M,
                                            int N) {
    constexpr int OUTC = EPI == EPI_GATED ? BN / 2 : BN, LPR = OUTC / 4, RPW = 32 / LPR, U = 4;      // lanes per row, rows per warp
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, step = (int)(blockDim.x >> 5) * RPW;
    const int rows = (int)max(0ll, min(128ll, M - m0)), c = (lane % LPR) * 4, n = n0 + c, valid = min(4, max(0, N - n));
    float bias[4] = {0.f, 0.f, 0.f, 0.f};
    if (EPI == EPI_LINEAR && e.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i < valid) bias[i] = __ldg(e.bias + n + i);
    }
#pragma unroll 1
    for (int i0 = warp * RPW; i0 * (int)S + (int)rank < rows; i0 += step * U) {                      // whole warps: img_store4 exchanges
        int r[U];
        bool on[U];
        float a[4 * U], b[4 * U], add[4 * U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            r[u] = (i0 + u * step + lane / LPR) * (int)S + (int)rank;
            on[u] = r[u] < rows;
#pragma unroll
            for (int i = 0; i < 4; ++i) { a[4 * u + i] = b[4 * u + i] = 0.f; add[4 * u + i] = bias[i]; }
        }
        for (uint32_t k = 0; k < S; ++k) {
            const uint32_t turn = rank + k < S ? rank + k : rank + k - S;
            const uint32_t there = S > 1 ? map_rank(base, first + turn * stride) : base;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!on[u]) continue;
                const uint32_t from = there + (uint32_t)(r[u] * PITCH + c) * 4;
                const float4 v = ld_cluster4(from);
                a[4 * u] += v.x; a[4 * u + 1] += v.y; a[4 * u + 2] += v.z; a[4 * u + 3] += v.w;
                if (EPI == EPI_GATED) {
                    const float4 w = ld_cluster4(from + OUTC * 4);
                    b[4 * u] += w.x; b[4 * u + 1] += w.y; b[4 * u + 2] += w.z; b[4 * u + 3] += w.w;
                }
            }
        }
        if (EPI == EPI_LINEAR) {
#pragma unroll
            for (int i = 0; i < 4 * U; ++i) a[i] += add[i];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float add4[4] = {0.f, 0.f, 0.f, 0.f};
            if (EPI != EPI_GATED && e.add && on[u] && valid) load4(static_cast<const T*>(e.add) + (m0 + r[u]) * e.ldadd + n, valid, e.vec_add, add4);
#pragma unroll
            for (int i = 0; i < 4; ++i) add[4 * u + i] = add4[i];
        }
        if (EPI != EPI_STORE && e.stash_kind != STASH_NONE) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const long long m = m0 + r[u];
                float a4[4], b4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) { a4[i] = a[4 * u + i]; b4[i] = b[4 * u + i]; }
                if (e.stash_kind == STASH_FULL) {
                    if (!on[u] || !valid) continue;
                    store4(static_cast<T*>(e.stash[0]) + m * e.ldstash + n, valid, e.vec_stash, a4);
                    if (EPI == EPI_GATED) store4(static_cast<T*>(e.stash[1]) + m * e.ldstash + n, valid, e.vec_stash, b4);
                } else {
                    // columns past the end are zero products (their operand tiles are filled with zeros): no effect on a block's maximum
                    img_store4(e.img[0], m, n, a4, on[u]);
                    if (EPI == EPI_GATED) img_store4(e.img[1], m, n, b4, on[u]);
                }
            }
        }
        if (!e.y) continue;
        if (EPI != EPI_STORE) act_all<sizeof(T) == 2>(a, e.act);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = EPI == EPI_GATED ? a[4 * u + i] * b[4 * u + i] : a[4 * u + i] + add[4 * u + i];
            if (on[u] && valid) store4(static_cast<T*>(e.y) + (m0 + r[u]) * e.ldy + n, valid, e.vec_y, v);
        }
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------
bool make_map(CUtensorMap* map, const Operand& o, int box_x, int box_y) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.planes};
    const cuuint64_t strides[2] = {(cuuint64_t)o.ld * 2, (cuuint64_t)(o.planes > 1 ? o.plane : o.rows * o.ld) * 2};
    const cuuint32_t box[3] = {(cuuint32_t)box_x, (cuuint32_t)box_y, 1};
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(o.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct Maps { CUtensorMap a[2], b[2]; };
bool make_maps(Maps& m, const Product& p, int a_rows, int b_rows) {
    const int na = p.parts > 1 && p.cat_k ? 2 : 1, nb = p.parts > 1 ? 2 : 1;
    for (int i = 0; i < na; ++i) if (!make_map(&m.a[i], p.A[i], 64, p.a_mn ? BK : a_rows)) return false;
    for (int i = 0; i < nb; ++i) if (!make_map(&m.b[i], p.B[i], 64, p.b_mn ? BK : b_rows)) return false;
    if (na == 1) m.a[1] = m.a[0];
    if (nb == 1) m.b[1] = m.b[0];
    return true;
}

// More than 48 KB of dynamic shared memory has to be asked for, once per kernel and device (done: the kernel's, one bit per
// device).
template <typename K>
cudaError_t allow_smem(std::atomic<unsigned long long>& done, K kern, int bytes) {
    int dev = -1;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0;
    if (done.load(std::memory_order_acquire) & bit) return cudaSuccess;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}

template <typename... KA, typename... A>
cudaError_t launch_cluster(void (*kern)(KA...), dim3 grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t st, A&&... args) {
    ++launches();
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = pdl_enabled() ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...);
}


}  // namespace

// products on CTA pairs (ffn_pair.cu); wide: 256 x 256 tiles instead of 256 x 128; S > 1: pairs that share a 256 x 128 tile's
// reduction
ftp_status run_product_pair(const Product& p, const KArgs& base, bool wide, int S, cudaStream_t st, const char* who);

}  // namespace ffn
}  // namespace ftp
