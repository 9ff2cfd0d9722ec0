// Products of the feed-forward operators on the 5th-generation tensor cores: D = op(A) op(B) from bf16 planes with float
// accumulation in tensor memory and the operators' epilogues.
//
// Operands are read as they lie in memory: with the reduction contiguous (K-major) or across their rows (MN-major).  A
// float tensor comes as three bf16 planes (8 mantissa bits each, 24 together) and a product of two of them as the six
// plane products that matter; the dropped ones are below 2^-24 of the result.
//
// tile kernel: one CTA per 128 x BN tile and slice of the reduction.  Warps 0, 2 and 3 (one elected thread each) stream operand tiles
// with TMA into a ring in shared memory, warp 1 issues the MMAs, warps 4-7 move the accumulator to shared memory.
// The slices of one tile form a cluster: each CTA then adds up the rows rank, rank + S, ... of the tile over the
// cluster's shared memory, in an order that depends on the row alone, and finishes them (bias, activation, residual, kept values), so a
// product with few tiles still uses the whole GPU, needs no workspace, and gives the same bits every time.
//
// Every wait is bounded; see gemm_tc.cu for the error protocol.
#include <cmath>
#include "ffn_gemm.cuh"

namespace ftp {
namespace ffn {
namespace {

// ---- one CTA per tile and reduction slice ---------------------------------------------------------------------------
constexpr int TILE_THREADS = 256;
// DEEP: a ring that fills an SM's shared memory, for launches of one CTA an SM or fewer (a block's turn through a short ring
// takes a load's latency divided by its slots); otherwise two CTAs share an SM, one's epilogue beside the other's products.
// Float results (three operand tiles a block) always take the long one.
// AR = 32: at most 32 rows of A are loaded, into the first 32 of the 128 rows that the MMA reads.  The other rows are whatever
// lies behind them in shared memory (inside the allocation, see the 12 KB at its end); they only reach accumulator rows
// that nobody reads.  A stage is then mostly B, which is what a product of a few tokens has to stream.
template <int BN, int AR> constexpr uint32_t TILE_STAGE = AR * BK * 2 + BN * BK * 2;
template <int BN, int AR, bool DEEP> constexpr int TILE_STAGES = (DEEP ? 196608 : 98304) / TILE_STAGE<BN, AR>;
template <int BN, int AR, bool DEEP> constexpr uint32_t TILE_SMEM = TILE_STAGES<BN, AR, DEEP> * TILE_STAGE<BN, AR> + (128 - AR) * 128 + 1024;

// AMN / BMN: the operand is MN-major.  EPI_GATED: the tile's first BN / 2 columns are A B[0], the others A B[1].
template <typename T, int BN, bool AMN, bool BMN, int EPI, int AR, bool DEEP>
__global__ void __launch_bounds__(TILE_THREADS, DEEP ? 1 : 2) ffn_tile_kernel(const __grid_constant__ CUtensorMap mapA0, const __grid_constant__ CUtensorMap mapA1,
                                                                   const __grid_constant__ CUtensorMap mapB0, const __grid_constant__ CUtensorMap mapB1,
                                                                   const __grid_constant__ KArgs p) {
    constexpr bool CHUNKED = sizeof(T) == 4;
    constexpr int STAGES = TILE_STAGES<BN, AR, DEEP>;
    constexpr int BUFS = CHUNKED ? 2 : 1;                            // accumulators in tensor memory
    constexpr uint32_t ACC = CHUNKED ? 2 * BN : BN, TMEM_COLS = BUFS * ACC;
    constexpr uint32_t SLAB = 64 * BK * 2, A_BYTES = AR * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    constexpr int OUTC = EPI == EPI_GATED ? BN / 2 : BN;             // output columns of a tile
    constexpr int PITCH = BN + 4;                                    // floats between rows of the staged accumulator: 16-byte accesses of 8 lanes hit all banks
    static_assert((AR == 128 || (!AMN && !CHUNKED)) && (DEEP || !CHUNKED), "");
    static_assert(AR * PITCH * 4 <= STAGES * STAGE_BYTES, "the staged accumulator reuses the operand ring");
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) unsigned long long bars[2 * STAGES + 2 * BUFS];
    __shared__ uint32_t tmem_base, failed;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t S;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
    const uint32_t rank = cluster_rank();
    const int tile = blockIdx.x / S, tn_all = p.tiles_n * p.parts_n;
    const int tm = tile / tn_all, tn = tile % tn_all, out = tn / p.tiles_n;
    const long long m0 = (long long)tm * 128;
    const int n0 = (tn - out * p.tiles_n) * OUTC;
    // this slice's share of the 64-wide blocks
    const int all_kb = p.kb_part * p.parts_k;
    const int kb0 = (int)((long long)all_kb * rank / S), kb1 = (int)((long long)all_kb * (rank + 1) / S);
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[STAGES]), accf0 = smem_u32(&bars[2 * STAGES]), acce0 = accf0 + 8 * BUFS;

    if (threadIdx.x == 0) {
        tma_prefetch_map(&mapA0); tma_prefetch_map(&mapB0);
        if (p.parts_k > 1) tma_prefetch_map(&mapA1);
        if (p.parts_k > 1 || p.parts_n > 1 || EPI == EPI_GATED) tma_prefetch_map(&mapB1);
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int b = 0; b < BUFS; ++b) { mbar_init(accf0 + 8 * b, 1); mbar_init(acce0 + 8 * b, 4); }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    grid_dep_sync();

    if (warp < 4 && warp != 1) {
        // ---- producers ----
        Slot<STAGES> sl;
        const uint32_t ring = smem_u32(smem);
        const int me = producer_of(warp), z = p.np == 1 ? 0 : p.np - 1 - me, step = p.np == 1 ? PRODUCERS : 1;
        const uint32_t bytes = (z < p.pa ? A_BYTES : 0) + (z < p.pb ? B_BYTES : 0);
        bool ok = true, peek = false;
        sl.ahead(me);
        for (int kb = kb0 + (p.np == 1 ? me : 0); kb < kb1; kb += step, sl.ahead(PRODUCERS)) {
            const int part = kb >= p.kb_part, k = (kb - (part ? p.kb_part : 0)) * BK;
            ok = warp_ready(peek, empty0 + 8 * sl.s, sl.parity ^ 1, p.err, 1);                       // at once for a slot never used
            if (!ok) break;
            Slot<STAGES> then = sl;
            then.ahead(PRODUCERS);
            peek = mbar_peek(empty0 + 8 * then.s, then.parity ^ 1);  // of this warp's next slot, see mma_warp
            if (elect_one()) {
                const CUtensorMap* ma = part ? &mapA1 : &mapA0;
                const CUtensorMap* mb = (part || out) ? &mapB1 : &mapB0;
                const uint32_t sa = ring + (uint32_t)sl.s * STAGE_BYTES, sb = sa + A_BYTES, bar = full0 + 8 * sl.s;
                mbar_expect_tx(bar, bytes);
                if (z < p.pa) {
                    if (AMN) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) tma_load_3d(sa + t * SLAB, ma, (int)m0 + 64 * t, k, z, bar);
                    } else
                        tma_load_3d(sa, ma, k, (int)m0, z, bar);
                }
                if (z < p.pb) {
                    if (EPI == EPI_GATED) {
#pragma unroll
                        for (int t = 0; t < BN / 64; ++t)
                            tma_load_3d(sb + t * SLAB, t < BN / 128 ? &mapB0 : &mapB1, n0 + 64 * (t & (BN / 128 - 1)), k, z, bar);
                    } else if (BMN) {
#pragma unroll
                        for (int t = 0; t < BN / 64; ++t) tma_load_3d(sb + t * SLAB, mb, n0 + 64 * t, k, z, bar);
                    } else
                        tma_load_3d(sb, mb, k, n0, z, bar);
                }
            }
            __syncwarp();
        }
        if (!ok) {
            // error path: time for the copies already issued to land before the block's memory is released
            const unsigned long long t0 = gtime();
            while (gtime() - t0 < 1000000ull) __nanosleep(1000);
        }
    } else if (warp == 1) {
        mma_warp<1, BN, STAGES, STAGE_BYTES, A_BYTES, AMN, BMN, CHUNKED, BUFS>(smem_u32(smem), full0, empty0, accf0, acce0, tmem, 1, kb1 - kb0, p);
    } else if (warp >= 4 && (AR == 128 || (warp & 3) == 0)) {
        // ---- accumulator -> shared memory (the ring is free once the last MMA has completed) ----
        const int q = warp & 3;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
        float* row = reinterpret_cast<float*>(smem) + (q * 32 + lane) * PITCH;
        bool have = true;
        if (CHUNKED) {
            float acc[BN];
#pragma unroll
            for (int i = 0; i < BN; ++i) acc[i] = 0.f;
            const int chunks = (kb1 - kb0 + p.chunk - 1) / p.chunk;
            for (int c = 0; c < chunks && have; ++c) {
                const int b = c & 1;
                have = __all_sync(0xffffffffu, wait_for(accf0 + 8 * b, (c >> 1) & 1, p.err, 3));
                if (!have) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                for (int g = 0; g < BN / 32; ++g) add_acc(lanes + (uint32_t)b * ACC + g * 32, BN, p.np > 1, acc + g * 32);
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                if (lane == 0) mbar_arrive_one(acce0 + 8 * b);
            }
            if (have) {
#pragma unroll
                for (int g = 0; g < BN / 4; ++g) *reinterpret_cast<float4*>(row + g * 4) = make_float4(acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
            }
        } else {
            have = __all_sync(0xffffffffu, kb1 > kb0 ? wait_for(accf0, 0, p.err, 3) : true);
            if (have) {
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                for (int c = 0; c < BN / 32; ++c) {
                    uint32_t r[32];
                    if (kb1 > kb0) tmem_ld32(lanes + (uint32_t)(c * 32), r);
                    else {
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = 0u;
                    }
#pragma unroll
                    for (int g = 0; g < 8; ++g) *reinterpret_cast<uint4*>(row + c * 32 + g * 4) = make_uint4(r[4 * g], r[4 * g + 1], r[4 * g + 2], r[4 * g + 3]);
                }
            }
        }
        if (!have && lane == 0) failed = 1;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    if (S > 1) cluster_sync_all();

    // ---- rows rank, rank + S, ... of the tile, added over the slices ----
    bool ok = true;
    for (uint32_t k = 0; k < S; ++k) ok = ok && (S > 1 ? ld_cluster1(map_rank(smem_u32(&failed), k)) : failed) == 0;
    if (ok) finish_rows<T, EPI, BN, PITCH>(p.e[out], smem_u32(smem), S, rank, 0, 1, m0, n0, p.M, p.N);
    if (S > 1) cluster_sync_all();                                   // nobody leaves while another CTA reads its shared memory
}

// ---- host -----------------------------------------------------------------------------------------------------------
template <typename T, int BN, bool AMN, bool BMN, int EPI, int AR, bool DEEP>
ftp_status launch_tile(const Product& p, KArgs& k, int S, cudaStream_t st, const char* who) {
    Maps m;
    FTP_REQUIRE(make_maps(m, p, AR, BN), FTP_ECUDA, "%s: cannot describe an operand to the copy engine", who);
    auto kern = ffn_tile_kernel<T, BN, AMN, BMN, EPI, AR, DEEP>;
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = allow_smem(asked, kern, (int)TILE_SMEM<BN, AR, DEEP>);
    if (e == cudaSuccess) e = launch_cluster(kern, dim3((unsigned)((long long)k.tiles_m * k.tiles_n * k.parts_n * S)), TILE_THREADS, TILE_SMEM<BN, AR, DEEP>, S, st, m.a[0], m.a[1], m.b[0], m.b[1], k);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}

template <int BN, bool AMN, bool BMN, int EPI, int AR>
ftp_status tile_deep(const Product& p, KArgs& k, int S, cudaStream_t st, const char* who) {
    if ((long long)k.tiles_m * k.tiles_n * k.parts_n * S <= 148) return launch_tile<__nv_bfloat16, BN, AMN, BMN, EPI, AR, true>(p, k, S, st, who);
    return launch_tile<__nv_bfloat16, BN, AMN, BMN, EPI, AR, false>(p, k, S, st, who);
}
template <int BN, bool AMN, bool BMN, int EPI>
ftp_status tile_typed(const Product& p, KArgs& k, int S, cudaStream_t st, const char* who) {
    if (p.out_f32) return launch_tile<float, BN, AMN, BMN, EPI, 128, true>(p, k, S, st, who);
    if constexpr (!AMN)
        if (p.M <= 32) return tile_deep<BN, AMN, BMN, EPI, 32>(p, k, S, st, who);
    return tile_deep<BN, AMN, BMN, EPI, 128>(p, k, S, st, who);
}

}  // namespace

// What a form of a product takes, in microseconds, up to what all forms share.  From launches timed one form at a time
// (5..4096 tokens, 512..12288 channels, all three products, both types): c = a 64-wide block of one tile (c2 with two CTAs
// on an SM), base = launch, first loads and last epilogue, epi = a tile's epilogue where nothing hides it, share(S) = the
// cluster and its exchange, and what reading the operands from memory takes at the rate the form reaches.  A wave is 74
// pairs, 148 CTAs or twice that; clusters of four and eight do not fill every group of SMs.
struct Form { bool pair; int cols, S; double cost; };
static Form choose_form(KArgs& k, const Product& p) {
    const bool f32 = p.out_f32 && k.np > 1;
    const int gated = p.epi == EPI_GATED ? 2 : 1;
    const double blocks = (double)k.kb_part * k.parts_k;
    const double mbytes = 2e-6 * blocks * 64 * ((double)p.M * k.pa + (double)p.N * gated * k.parts_n * k.pb);
    auto tiles = [&](int rows, int cols) { return (double)((p.M + rows - 1) / rows) * ((p.N + cols / gated - 1) / (cols / gated)) * k.parts_n; };
    Form best{true, 256, 1, 1e30};
    auto take = [&](const Form& f) { if (f.cost < best.cost) best = f; };
    // rows that cannot be moved four elements at a time: of the result, and of what is read or kept beside it
    const Epi& e = k.e[0];
    const double ragged = e.vec_y ? 0 : 5.0, beside = (e.add && !e.vec_add ? 1 : 0) + (e.stash_kind == STASH_FULL && !e.vec_stash ? 1 : 0);
    static constexpr double share[9] = {0, 0, 1.5, 2.1, 2.7, 3.1, 3.4, 3.8, 4.2}, pair_share[5] = {0, 0, 2.1, 2.4, 2.8};
    auto pair = [&](int cols, double c, double base, double epi) {
        const double t = c * blocks, n = tiles(256, cols), waves = std::ceil(n / 74);
        take({true, cols, 1, base + ragged + 7 * beside + std::max(t + (waves - 1) * std::max(t, epi + 5 * beside), mbytes / std::min(4.0, 0.085 * n))});
        for (int S = 2; cols == 128 && S <= 4 && S <= blocks; ++S)   // one tile per cluster of four, six or eight CTAs
            if (tiles(256, cols) * S <= (S == 2 ? 66 : S == 3 ? 60 : 52))
                take({true, cols, S, base + pair_share[S] + ragged / S + std::max(c * std::ceil(blocks / S), mbytes / 5.2)});
    };
    if (f32 || p.out_f32) pair(128, f32 ? 0.82 : 0.2, 5.4, 3.0);
    else {
        pair(256, 0.29, 7.1, 4.0);
        pair(128, 0.15, 5.6, 2.9);
    }
    auto tile = [&](int cols, double c, double c2, double base, double epi) {
        for (int S = 1; S <= 8 && S <= blocks; ++S) {
            const double room = S <= 2 ? 148 : S <= 4 ? 132 : 104, n = tiles(128, cols) * S, len = std::ceil(blocks / S);
            double t;
            if (n <= room) t = c * len;
            else {
                const double waves = std::ceil(n / (c2 > 0 ? 2 * room : room));
                t = waves * (c2 > 0 ? c2 : c) * len + (waves - 1) * epi;
            }
            take({false, cols, S, base + share[S] + ragged / S + std::max(t, mbytes / 5.2)});
        }
    };
    if (f32) {
        tile(128, 1.3, 0, 3.6, 3.0);
        if (gated == 1) tile(64, 1.0, 0, 3.1, 2.8);
    } else if (p.out_f32) {
        tile(128, 0.4, 0, 3.6, 3.0);
        if (gated == 1) tile(64, 0.3, 0, 3.1, 2.8);
    } else {
        tile(128, 0.325, 0.6, 4.2, 6.0);
        if (gated == 1) tile(64, 0.253, 0.36, 3.8, 4.7);
    }
    if (!p.out_f32 && blocks > (double)LONG_SUM * best.S) {          // too long a sum for the accumulator: pairs that empty it
        best.cost = 1e30;
        const double n = tiles(256, 128);
        for (int S = 1; S <= 4; ++S)
            if (S == 1 || n * S <= (S == 2 ? 66 : S == 3 ? 60 : 52)) take({true, 128, S, pair_share[S] + 0.15 * std::ceil(blocks / S) * std::ceil(n * S / 74)});
        k.long_sum = 1;
        k.chunk = LONG_CHUNK;
    }
    return best;
}

ftp_status run_product(const Product& p, cudaStream_t st, const char* who) {
    KArgs k{};
    k.e[0] = p.e[0]; k.e[1] = p.e[1];
    k.M = p.M; k.N = p.N; k.err = p.err;
    k.pa = p.A[0].planes; k.pb = p.B[0].planes;
    k.np = std::max(k.pa, k.pb);
    k.kb_part = (int)((p.K + BK - 1) / BK);
    k.parts_k = (p.parts > 1 && p.cat_k) ? 2 : 1;
    k.chunk = CHUNK;
    k.parts_n = (p.parts > 1 && !p.cat_k && p.epi != EPI_GATED) ? 2 : 1;
    const Form f = choose_form(k, p);
    if (f.pair) return run_product_pair(p, k, f.cols == 256, f.S, st, who);
    k.tiles_m = (int)((p.M + 127) / 128);
    const int outc = p.epi == EPI_GATED ? f.cols / 2 : f.cols;
    k.tiles_n = (p.N + outc - 1) / outc;
    FTP_REQUIRE((long long)k.tiles_m * k.tiles_n * k.parts_n * f.S < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    const bool narrow = f.cols == 64;
    if (p.epi == EPI_GATED) return tile_typed<128, false, true, EPI_GATED>(p, k, f.S, st, who);
    if (p.epi == EPI_LINEAR) return narrow ? tile_typed<64, false, true, EPI_LINEAR>(p, k, f.S, st, who) : tile_typed<128, false, true, EPI_LINEAR>(p, k, f.S, st, who);
    if (p.a_mn) return narrow ? tile_typed<64, true, true, EPI_STORE>(p, k, f.S, st, who) : tile_typed<128, true, true, EPI_STORE>(p, k, f.S, st, who);
    return narrow ? tile_typed<64, false, false, EPI_STORE>(p, k, f.S, st, who) : tile_typed<128, false, false, EPI_STORE>(p, k, f.S, st, who);
}

}  // namespace ffn
}  // namespace ftp
