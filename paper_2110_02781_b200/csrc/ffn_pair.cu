// Products of the feed-forward operators on CTA pairs: 256 x BN tiles, persistent.
//
// Two CTAs of a cluster work on one tile: each holds 128 rows of A and half of B's columns in its shared memory and 128
// rows of the accumulator in its tensor memory, and one tcgen05.mma.cta_group::2 of 256 x BN x 16 reads both, so every
// operand byte that a CTA loads is used for twice as many products as in a tile of its own -- which is what bounds large
// products: at 256 x 256 a pair needs 64 KB per 8.4 MFLOP from L2.
//
// Warps 0, 2 and 3 (one elected thread each, in each CTA) stream the operand tiles with TMA; the bytes of both CTAs are counted on the
// first CTA's barrier.  Warp 1 of the first CTA issues the MMAs and hands stages and accumulators on with commits that
// signal both CTAs.  Warps 4-11 empty the accumulator: warp w the 32 lanes of its quarter and one half of the columns.  The
// accumulator is double (2 x BN columns), so the epilogue of a tile -- bias, activation, kept values, residual -- runs
// beside the MMAs of the next.  Finished pieces of 32 x 32 go through 4 KB of shared memory per warp, so that a global
// access covers whole 64- or 128-byte pieces of a row whatever its pitch.
//
// Float results are summed in registers chunk by chunk (see CHUNK).  Every wait is bounded; see gemm_tc.cu for the error
// protocol.
#include "ffn_gemm.cuh"

namespace ftp {
namespace ffn {
namespace {

constexpr int PAIR_THREADS = 12 * 32;
constexpr int SMS = 148;
template <int BN> constexpr int PAIR_STAGES = BN == 256 ? 6 : 8;
template <int BN> constexpr uint32_t PAIR_RING = PAIR_STAGES<BN> * (128 * BK * 2 + BN / 2 * BK * 2);
template <int BN> constexpr uint32_t PAIR_SMEM = PAIR_RING<BN> + 8 * 4096 + 1024;

// The mbarrier may be the other CTA's of the pair.
__device__ __forceinline__ void tma_load_3d_pair(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// tile number -> row tile and column tile: bands of 8 row tiles, column by column, so that the tiles in flight at one time
// share operands in L2
__device__ __forceinline__ void tile_at(int t, int tiles_m, int tiles_n, int& tm, int& tn) {
    constexpr int BAND = 8;
    const int per = BAND * tiles_n, band = t / per, in = t - band * per, rows = min(BAND, tiles_m - band * BAND);
    tn = in / rows;
    tm = band * BAND + in - tn * rows;
}

// A 32 x 32 piece in a warp's shared memory: rows of 128 (float) or 64 (bf16) bytes, 16-byte parts exchanged within the
// row so that both the per-row and the per-part accesses of a quarter-warp hit all banks.
template <typename T> __device__ __forceinline__ uint32_t piece_at(int row, int part) {
    return sizeof(T) == 4 ? row * 128 + ((part ^ (row & 7)) << 4) : row * 64 + ((part ^ ((row >> 1) & 3)) << 4);
}
template <typename T> __device__ __forceinline__ void piece_put(uint8_t* buf, int row, const float (&v)[32]) {
#pragma unroll
    for (int g = 0; g < (int)sizeof(T) * 2; ++g) {
        uint4 o;
        if (sizeof(T) == 4) o = make_uint4(__float_as_uint(v[4 * g]), __float_as_uint(v[4 * g + 1]), __float_as_uint(v[4 * g + 2]), __float_as_uint(v[4 * g + 3]));
        else {
            constexpr int W = sizeof(T) == 4 ? 0 : 8;
            o = make_uint4(bf_pack(v[(W * g) & 31], v[(W * g + 1) & 31]), bf_pack(v[(W * g + 2) & 31], v[(W * g + 3) & 31]), bf_pack(v[(W * g + 4) & 31], v[(W * g + 5) & 31]),
                           bf_pack(v[(W * g + 6) & 31], v[(W * g + 7) & 31]));
        }
        *reinterpret_cast<uint4*>(buf + piece_at<T>(row, g)) = o;
    }
}
template <typename T> __device__ __forceinline__ void piece_get(const uint8_t* buf, int row, float (&v)[32]) {
#pragma unroll
    for (int g = 0; g < (int)sizeof(T) * 2; ++g) {
        const uint4 o = *reinterpret_cast<const uint4*>(buf + piece_at<T>(row, g));
        const unsigned u[4] = {o.x, o.y, o.z, o.w};
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[(4 * g + i) & 31] = __uint_as_float(u[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) { v[(8 * g + 2 * i) & 31] = bf_lo(u[i]); v[(8 * g + 2 * i + 1) & 31] = bf_hi(u[i]); }
        }
    }
}
// The same where rows lie on fewer bytes than the accesses below, or are cut.
template <typename T, bool STORE>
__device__ __forceinline__ void piece_move_loose(uint8_t* buf, T* p, long long ld, long long m0, int n0, long long M, int N) {
    constexpr int EL = 16 / sizeof(T);
    const int lane = threadIdx.x & 31;
    if (sizeof(T) == 2 && (reinterpret_cast<uintptr_t>(p) & 3) == 0 && (ld & 1) == 0 && n0 + 32 <= N) {
        // bf16 rows on 4 bytes: two elements per lane, two rows per access
        const int pair = lane & 15, row = lane >> 4;
        T* g = p + (m0 + row) * ld + n0 + pair * 2;
        const long long left = M - m0 - row;
        unsigned v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (STORE) v[i] = *reinterpret_cast<const unsigned*>(buf + piece_at<T>(i * 2 + row, pair >> 2) + (pair & 3) * 4);
            else v[i] = i * 2 < left ? *reinterpret_cast<const unsigned*>(g + (long long)(i * 2) * ld) : 0u;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if (!STORE) *reinterpret_cast<unsigned*>(buf + piece_at<T>(i * 2 + row, pair >> 2) + (pair & 3) * 4) = v[i];
            else if (i * 2 < left) *reinterpret_cast<unsigned*>(g + (long long)(i * 2) * ld) = v[i];
        }
    } else {
        // rows anywhere, or cut: an element per lane, so that an access still covers neighbouring bytes
        const bool on = n0 + lane < N;
        T* g = p + m0 * ld + n0 + lane;
#pragma unroll 1
        for (int r0 = 0; r0 < 32; r0 += 16) {
            T v[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (STORE) v[i] = *(reinterpret_cast<const T*>(buf + piece_at<T>(r0 + i, lane / EL)) + lane % EL);
                else if (on && m0 + r0 + i < M) v[i] = g[(r0 + i) * ld];
                else v[i] = T(0.f);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                if (!STORE) *(reinterpret_cast<T*>(buf + piece_at<T>(r0 + i, lane / EL)) + lane % EL) = v[i];
                else if (on && m0 + r0 + i < M) g[(r0 + i) * ld] = v[i];
            }
        }
    }
}

// The piece against rows m0.., columns n0.. of a matrix (ld elements between rows, cut at M x N); vec as in Epi.  EVEN: rows on
// 16 bytes, and no 16-byte part of a row is cut; a kernel of its own, since the other paths cost this one registers (8192 x 64
// x 4096 bf16: 48 instead of 34 us).  All loads are begun before the first result is stored (one at a time: 233 instead of 117 us for
// 8192 x 64 x 4096 float with a residual).
template <typename T, bool STORE, bool EVEN>
__device__ __forceinline__ void piece_move(uint8_t* buf, T* p, long long ld, int vec, long long m0, int n0, long long M, int N) {
    constexpr int PARTS = sizeof(T) * 2, EL = 16 / sizeof(T), ROWS = 32 / PARTS, IT = 32 / ROWS;    // parts of a row, elements of a part, rows per access
    const int lane = threadIdx.x & 31;
    if (EVEN || (vec != 0 && n0 + 32 <= N)) {
        const int part = lane % PARTS, row = lane / PARTS, n = n0 + part * EL;
        const bool whole = EVEN || sizeof(T) == 4 || vec == 2;       // otherwise bf16 rows on 8 bytes
        const bool on = !EVEN || n < N;
        if (STORE) {
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const long long m = m0 + i * ROWS + row;
                if (on && m < M) {
                    T* g = p + m * ld + n;
                    const uint4* s = reinterpret_cast<const uint4*>(buf + piece_at<T>(i * ROWS + row, part));
                    if (whole) *reinterpret_cast<uint4*>(g) = *s;
                    else {
                        reinterpret_cast<uint2*>(g)[0] = reinterpret_cast<const uint2*>(s)[0];
                        reinterpret_cast<uint2*>(g)[1] = reinterpret_cast<const uint2*>(s)[1];
                    }
                }
            }
        } else {
            uint4 v[IT];
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const long long m = m0 + i * ROWS + row;
                const T* g = p + m * ld + n;
                if (!on || m >= M) v[i] = make_uint4(0u, 0u, 0u, 0u);
                else if (whole) v[i] = *reinterpret_cast<const uint4*>(g);
                else {
                    const uint2 x = reinterpret_cast<const uint2*>(g)[0], y = reinterpret_cast<const uint2*>(g)[1];
                    v[i] = make_uint4(x.x, x.y, y.x, y.y);
                }
            }
#pragma unroll
            for (int i = 0; i < IT; ++i) *reinterpret_cast<uint4*>(buf + piece_at<T>(i * ROWS + row, part)) = v[i];
        }
    } else
        piece_move_loose<T, STORE>(buf, p, ld, m0, n0, M, N);
}

// one row's 32 columns of an 8-bit image, all in this thread
__device__ __forceinline__ void img_store32(const Image& im, long long m, int n, const float (&v)[32]) {
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 32; ++i) top = max(top, __float_as_uint(v[i]) & 0x7fffffffu);
    const unsigned e = img_exp(top);
    const float inv = img_inv(e);
    uint4* q = reinterpret_cast<uint4*>(im.q + m * im.pitch + n);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = pack_codes(img_code(v[h * 16 + 4 * i], inv), img_code(v[h * 16 + 4 * i + 1], inv), img_code(v[h * 16 + 4 * i + 2], inv), img_code(v[h * 16 + 4 * i + 3], inv));
        q[h] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    im.e[m * (im.pitch / IMG_BLOCK) + n / IMG_BLOCK] = (uint8_t)e;
}

// The addend of a 32 x 32 bf16 piece on its way from memory, 16 bytes per access: four accesses per lane, begun before the
// piece's accumulator is read.
struct Ahead { uint4 v[4]; };
template <bool EVEN>
__device__ __forceinline__ bool ahead_ok(const Epi& e, long long m, int n, long long M, int N) {
    return e.add && m < M && (EVEN ? n < N : e.vec_add == 2 && n + 32 <= N);
}
__device__ __forceinline__ void ahead_load(Ahead& h, const Epi& e, long long m, int n, long long M, int N) {
    const int lane = threadIdx.x & 31, part = lane & 3;
    const __nv_bfloat16* p = static_cast<const __nv_bfloat16*>(e.add) + n + part * 8;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const long long r = m + k * 8 + (lane >> 2);
        h.v[k] = r < M && n + part * 8 < N ? *reinterpret_cast<const uint4*>(p + r * e.ldadd) : make_uint4(0u, 0u, 0u, 0u);
    }
}

// The epilogue on 32 columns n.. of 32 rows m.. (this thread: row m + lane); buf: the warp's 4 KB; ahead: the piece's
// addend if it was begun (bf16).
template <typename T, int EPI, bool EVEN>
__device__ __forceinline__ void finish_piece(const Epi& e, uint8_t* buf, long long m, int n, long long M, int N, float (&a)[32], float (&b)[32], bool have_ahead,
                                             const Ahead& ahead) {
    const int lane = threadIdx.x & 31;
    constexpr bool FAST = sizeof(T) == 2;
    if (n >= N || m >= M) return;                                    // the whole piece lies outside
    auto put = [&](void* p, long long ld, int vec, const float (&v)[32]) {
        piece_put<T>(buf, lane, v);
        __syncwarp();
        piece_move<T, true, EVEN>(buf, static_cast<T*>(p), ld, vec, m, n, M, N);
        __syncwarp();
    };
    if (EPI == EPI_LINEAR && e.bias) {
        if (e.vec_bias && n + 32 <= N) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float4 v = __ldg(reinterpret_cast<const float4*>(e.bias + n) + i);
                a[4 * i] += v.x; a[4 * i + 1] += v.y; a[4 * i + 2] += v.z; a[4 * i + 3] += v.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) if (n + i < N) a[i] += __ldg(e.bias + n + i);
        }
    }
    if (EPI != EPI_STORE && e.stash_kind == STASH_FULL) {
        put(e.stash[0], e.ldstash, e.vec_stash, a);
        if (EPI == EPI_GATED) put(e.stash[1], e.ldstash, e.vec_stash, b);
    } else if (EPI != EPI_STORE && e.stash_kind == STASH_8BIT && m + lane < M) {
        // columns past the end are zero products (their operand tiles are filled with zeros): no effect on a block's maximum
        img_store32(e.img[0], m + lane, n, a);
        if (EPI == EPI_GATED) img_store32(e.img[1], m + lane, n, b);
    }
    if (!e.y) return;
    if (EPI != EPI_STORE) act_all<FAST>(a, e.act);
    if (EPI == EPI_GATED) {
#pragma unroll
        for (int i = 0; i < 32; ++i) a[i] *= b[i];
    }
    if (EPI != EPI_GATED && e.add) {
        if (sizeof(T) == 2 && (EVEN || have_ahead)) {
#pragma unroll
            for (int k = 0; k < 4; ++k) *reinterpret_cast<uint4*>(buf + piece_at<T>(k * 8 + (lane >> 2), lane & 3)) = ahead.v[k];
        } else
            piece_move<T, false, EVEN>(buf, const_cast<T*>(static_cast<const T*>(e.add)), e.ldadd, e.vec_add, m, n, M, N);
        __syncwarp();
        float r[32];
        piece_get<T>(buf, lane, r);
#pragma unroll
        for (int i = 0; i < 32; ++i) a[i] += r[i];
        __syncwarp();
    }
    put(e.y, e.ldy, e.vec_y, a);
}

// EPI_GATED: the tile's first BN / 2 columns are A B[0] (the first CTA's half of B), the others A B[1].
template <typename T, int BN, bool AMN, bool BMN, int EPI, bool EVEN>
__global__ void __launch_bounds__(PAIR_THREADS, 1) ffn_pair_kernel(const __grid_constant__ CUtensorMap mapA0, const __grid_constant__ CUtensorMap mapA1,
                                                                   const __grid_constant__ CUtensorMap mapB0, const __grid_constant__ CUtensorMap mapB1,
                                                                   const __grid_constant__ KArgs p) {
    constexpr int STAGES = PAIR_STAGES<BN>;
    constexpr bool CHUNKED = sizeof(T) == 4;
    constexpr uint32_t SLAB = 64 * BK * 2, A_BYTES = 128 * BK * 2, B_BYTES = BN / 2 * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    constexpr int OUTC = EPI == EPI_GATED ? BN / 2 : BN;             // output columns of a tile
    constexpr int WC = BN / 2;                                       // accumulator columns of an epilogue warp
    constexpr uint32_t ACC = CHUNKED ? 2 * BN : BN, TMEM_COLS = 2 * ACC;
    static_assert(TMEM_COLS <= 512, "tensor memory");
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) unsigned long long bars[2 * STAGES + 4];
    __shared__ uint32_t tmem_base;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    const int cluster = blockIdx.x >> 1, clusters = gridDim.x >> 1;
    const int tn_all = p.tiles_n * p.parts_n, tiles = p.tiles_m * tn_all, all_kb = p.kb_part * p.parts_k;
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[STAGES]), accf0 = smem_u32(&bars[2 * STAGES]), acce0 = accf0 + 16;

    if (threadIdx.x == 0) {
        tma_prefetch_map(&mapA0); tma_prefetch_map(&mapB0);
        if (p.parts_k > 1) tma_prefetch_map(&mapA1);
        if (p.parts_k > 1 || p.parts_n > 1 || EPI == EPI_GATED) tma_prefetch_map(&mapB1);
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(accf0 + 8 * b, 1); mbar_init(acce0 + 8 * b, 16); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                              // the barriers of both CTAs exist
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    grid_dep_sync();

    bool ok = true;
    if (warp < 4 && warp != 1) {
        // ---- producers ----
        Slot<STAGES> sl;
        const uint32_t lead_full0 = map_rank(full0, 0), ring = smem_u32(smem);
        const int me = producer_of(warp), z = p.np == 1 ? 0 : p.np - 1 - me, step = p.np == 1 ? PRODUCERS : 1;
        const uint32_t bytes = (z < p.pa ? 2 * A_BYTES : 0) + (z < p.pb ? 2 * B_BYTES : 0);
        int kb = p.np == 1 ? me : 0;                                 // runs on over the tiles: slots are numbered through
        bool peek = false;
        sl.ahead(me);
        for (int t = cluster; t < tiles && ok; t += clusters, kb -= all_kb) {
            int tm, tn;
            tile_at(t, p.tiles_m, tn_all, tm, tn);
            const int out = tn / p.tiles_n;
            const int m0 = tm * 256 + (int)rank * 128, n0 = (tn - out * p.tiles_n) * OUTC + (EPI == EPI_GATED ? 0 : (int)rank * (BN / 2));
            for (; kb < all_kb; kb += step, sl.ahead(PRODUCERS)) {
                const int part = kb >= p.kb_part, k = (kb - (part ? p.kb_part : 0)) * BK;
                ok = warp_ready(peek, empty0 + 8 * sl.s, sl.parity ^ 1, p.err, 1);                       // at once for a slot never used
                if (!ok) break;
                Slot<STAGES> then = sl;
                then.ahead(PRODUCERS);
                peek = mbar_peek(empty0 + 8 * then.s, then.parity ^ 1);  // of this warp's next slot, see mma_warp
                if (elect_one()) {
                    const CUtensorMap* ma = part ? &mapA1 : &mapA0;
                    const CUtensorMap* mb = (EPI == EPI_GATED ? rank != 0 : (part || out)) ? &mapB1 : &mapB0;
                    const uint32_t sa = ring + (uint32_t)sl.s * STAGE_BYTES, sb = sa + A_BYTES, bar = lead_full0 + 8 * sl.s;
                    if (rank == 0) mbar_expect_tx(full0 + 8 * sl.s, bytes);
                    if (z < p.pa) {
                        if (AMN) {
#pragma unroll
                            for (int u = 0; u < 2; ++u) tma_load_3d_pair(sa + u * SLAB, ma, m0 + 64 * u, k, z, bar);
                        } else
                            tma_load_3d_pair(sa, ma, k, m0, z, bar);
                    }
                    if (z < p.pb) {
                        if (BMN) {
#pragma unroll
                            for (int u = 0; u < BN / 128; ++u) tma_load_3d_pair(sb + u * SLAB, mb, n0 + 64 * u, k, z, bar);
                        } else
                            tma_load_3d_pair(sb, mb, k, n0, z, bar);
                    }
                }
                __syncwarp();
            }
        }
    } else if (warp == 1) {
        if (rank == 0) {
            const int mine = cluster < tiles ? (tiles - cluster + clusters - 1) / clusters : 0;
            ok = mma_warp<2, BN, STAGES, STAGE_BYTES, A_BYTES, AMN, BMN, CHUNKED, 2>(smem_u32(smem), full0, empty0, accf0, acce0, tmem, mine, all_kb, p);
        }
    } else if (warp >= 4) {
        // ---- epilogue ----
        const int q = warp & 3, half = (warp - 4) >> 2;
        uint8_t* buf = smem + PAIR_RING<BN> + (warp - 4) * 4096;
        const uint32_t lead_acce0 = map_rank(acce0, 0), lanes = tmem + ((uint32_t)(q * 32) << 16);
        // accumulator columns of this warp: linear and plain half * WC ..; gated: half * WC / 2 .. of either product
        const int col0 = EPI == EPI_GATED ? half * (WC / 2) : half * WC;
        constexpr int PIECES = (EPI == EPI_GATED ? WC / 2 : WC) / 32;
        int chunk = 0;
        for (int t = cluster; t < tiles && ok; t += clusters) {
            int tm, tn;
            tile_at(t, p.tiles_m, tn_all, tm, tn);
            const int out = tn / p.tiles_n;
            const long long m0 = (long long)tm * 256 + rank * 128 + q * 32;
            const int n0 = (tn - out * p.tiles_n) * OUTC + col0;
            if (CHUNKED) {
                float acc[WC];
#pragma unroll
                for (int i = 0; i < WC; ++i) acc[i] = 0.f;
                const int chunks = (all_kb + p.chunk - 1) / p.chunk;
                for (int c = 0; c < chunks; ++c, ++chunk) {
                    const int b = chunk & 1;
                    ok = warp_wait_for(accf0 + 8 * b, (chunk >> 1) & 1, p.err, 3);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
                    for (int g = 0; g < WC / 32; ++g) {
                        const int col = EPI == EPI_GATED ? (g < WC / 64 ? col0 + g * 32 : BN / 2 + col0 + (g - WC / 64) * 32) : col0 + g * 32;
                        add_acc(lanes + (uint32_t)b * ACC + col, BN, p.np > 1, acc + g * 32);
                    }
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive_cluster(lead_acce0 + 8 * b);
                }
                if (!ok) break;
#pragma unroll
                for (int g = 0; g < PIECES; ++g) {
                    float a[32], b2[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) { a[i] = acc[g * 32 + i]; b2[i] = EPI == EPI_GATED ? acc[(WC / 2 + g * 32 + i) % WC] : 0.f; }
                    finish_piece<T, EPI, EVEN>(p.e[out], buf, m0, n0 + g * 32, p.M, p.N, a, b2, false, Ahead());
                }
            } else {
                const int b = chunk & 1;
                const Epi& e = p.e[out];
                Ahead ahead;
                bool have = EPI != EPI_GATED && ahead_ok<EVEN>(e, m0, n0, p.M, p.N);
                if (have) ahead_load(ahead, e, m0, n0, p.M, p.N);
                ok = warp_wait_for(accf0 + 8 * b, (chunk >> 1) & 1, p.err, 3);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                for (int g = 0; g < PIECES; ++g) {
                    float a[32], b2[32];
                    uint32_t r[32], r2[32];
                    tmem_ld32_issue(lanes + (uint32_t)(b * BN + col0 + g * 32), r);
                    if (EPI == EPI_GATED) tmem_ld32_issue(lanes + (uint32_t)(b * BN + BN / 2 + col0 + g * 32), r2);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 32; ++i) { a[i] = __uint_as_float(r[i]); b2[i] = EPI == EPI_GATED ? __uint_as_float(r2[i]) : 0.f; }
                    if (g == PIECES - 1) {                           // the accumulator is in registers: the tile after next may overwrite it
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0) mbar_arrive_cluster(lead_acce0 + 8 * b);
                    }
                    const Ahead now = ahead;
                    const bool have_now = have;
                    have = EPI != EPI_GATED && g + 1 < PIECES && ahead_ok<EVEN>(e, m0, n0 + (g + 1) * 32, p.M, p.N);
                    if (have) ahead_load(ahead, e, m0, n0 + (g + 1) * 32, p.M, p.N);
                    finish_piece<T, EPI, EVEN>(e, buf, m0, n0 + g * 32, p.M, p.N, a, b2, have_now, now);
                }
                ++chunk;
            }
        }
    }
    if (!ok) {
        // error path: time for the copies and MMAs already issued, which touch both CTAs, before either may leave
        const unsigned long long t0 = gtime();
        while (gtime() - t0 < 1000000ull) __nanosleep(1000);
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync_all();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
}

// Several pairs of a cluster share a 256 x 128 tile's reduction, for products with too few tiles for all pairs: every CTA
// leaves its 128 rows of partial sums in shared memory (the ring is free by then), and the CTAs that hold the same rows add
// and finish every S-th of them each (finish_rows): 1024 x 1024 x 1024 float 22 instead of 28 us, 512 x 11008 x 512 bf16 15
// instead of 30.  CHUNKED: the accumulator is emptied into registers every p.chunk blocks: float results, and long reductions of
// bf16 ones (see LONG_SUM).
template <typename T, bool AMN, bool BMN, int EPI, bool CHUNKED>
__global__ void __launch_bounds__(PAIR_THREADS, 1) ffn_split_kernel(const __grid_constant__ CUtensorMap mapA0, const __grid_constant__ CUtensorMap mapA1,
                                                                    const __grid_constant__ CUtensorMap mapB0, const __grid_constant__ CUtensorMap mapB1,
                                                                    const __grid_constant__ KArgs p) {
    constexpr int BN = 128, STAGES = PAIR_STAGES<BN>, WC = BN / 2, PITCH = BN + 4;
    constexpr int BUFS = CHUNKED ? 2 : 1;
    constexpr uint32_t SLAB = 64 * BK * 2, A_BYTES = 128 * BK * 2, B_BYTES = BN / 2 * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    constexpr uint32_t ACC = CHUNKED ? 2 * BN : BN, TMEM_COLS = BUFS * ACC;
    constexpr int OUTC = EPI == EPI_GATED ? BN / 2 : BN;
    static_assert(128 * PITCH * 4 <= STAGES * STAGE_BYTES, "the staged sums reuse the operand ring");
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) unsigned long long bars[2 * STAGES + 2 * BUFS];
    __shared__ uint32_t tmem_base, failed;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t C;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(C));
    const uint32_t cta = cluster_rank(), side = cta & 1, slice = cta >> 1, S = C >> 1;
    const int tn_all = p.tiles_n * p.parts_n, all_kb = p.kb_part * p.parts_k;
    int tm, tn;
    tile_at((int)(blockIdx.x / C), p.tiles_m, tn_all, tm, tn);
    const int out = tn / p.tiles_n;
    const long long m0 = (long long)tm * 256 + side * 128;
    const int n0 = (tn - out * p.tiles_n) * OUTC;
    const int kb0 = (int)((long long)all_kb * slice / S), kb1 = (int)((long long)all_kb * (slice + 1) / S);
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[STAGES]), accf0 = smem_u32(&bars[2 * STAGES]), acce0 = accf0 + 8 * BUFS;

    if (threadIdx.x == 0) {
        tma_prefetch_map(&mapA0); tma_prefetch_map(&mapB0);
        if (p.parts_k > 1) tma_prefetch_map(&mapA1);
        if (p.parts_k > 1 || p.parts_n > 1 || EPI == EPI_GATED) tma_prefetch_map(&mapB1);
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        for (int b = 0; b < BUFS; ++b) { mbar_init(accf0 + 8 * b, 1); mbar_init(acce0 + 8 * b, 16); }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync_all();                                              // the barriers of all CTAs exist
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    grid_dep_sync();

    bool ok = true;
    if (warp < 4 && warp != 1) {
        // ---- producers ----
        Slot<STAGES> sl;
        const uint32_t lead_full0 = map_rank(full0, cta & ~1u), ring = smem_u32(smem);
        const int me = producer_of(warp), z = p.np == 1 ? 0 : p.np - 1 - me, step = p.np == 1 ? PRODUCERS : 1;
        const uint32_t bytes = (z < p.pa ? 2 * A_BYTES : 0) + (z < p.pb ? 2 * B_BYTES : 0);
        const int nb = n0 + (EPI == EPI_GATED ? 0 : (int)side * (BN / 2));
        bool peek = false;
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
                const CUtensorMap* mb = (EPI == EPI_GATED ? side != 0 : (part || out)) ? &mapB1 : &mapB0;
                const uint32_t sa = ring + (uint32_t)sl.s * STAGE_BYTES, sb = sa + A_BYTES, bar = lead_full0 + 8 * sl.s;
                if (side == 0) mbar_expect_tx(full0 + 8 * sl.s, bytes);
                if (z < p.pa) {
                    if (AMN) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) tma_load_3d_pair(sa + u * SLAB, ma, (int)m0 + 64 * u, k, z, bar);
                    } else
                        tma_load_3d_pair(sa, ma, k, (int)m0, z, bar);
                }
                if (z < p.pb) {
                    if (BMN) tma_load_3d_pair(sb, mb, nb, k, z, bar);
                    else tma_load_3d_pair(sb, mb, k, nb, z, bar);
                }
            }
            __syncwarp();
        }
    } else if (warp == 1) {
        if (side == 0)
            ok = mma_warp<2, BN, STAGES, STAGE_BYTES, A_BYTES, AMN, BMN, CHUNKED, BUFS>(smem_u32(smem), full0, empty0, accf0, acce0, tmem, 1, kb1 - kb0, p,
                                                                                     (uint16_t)(3u << (cta & ~1u)));
    } else if (warp >= 4) {
        // ---- partial sums -> shared memory ----
        const int q = warp & 3, col0 = ((warp - 4) >> 2) * WC;
        const uint32_t lead_acce0 = map_rank(acce0, cta & ~1u), lanes = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)col0;
        float* row = reinterpret_cast<float*>(smem) + (q * 32 + lane) * PITCH + col0;
        float acc[WC];
#pragma unroll
        for (int i = 0; i < WC; ++i) acc[i] = 0.f;
        const int chunks = CHUNKED ? (kb1 - kb0 + p.chunk - 1) / p.chunk : 1;
        for (int c = 0; c < chunks; ++c) {
            const int b = CHUNKED ? c & 1 : 0;
            ok = warp_wait_for(accf0 + 8 * b, CHUNKED ? (c >> 1) & 1 : 0, p.err, 3);
            if (!ok) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
            for (int g = 0; g < WC / 32; ++g) add_acc(lanes + (uint32_t)b * ACC + g * 32, BN, CHUNKED && p.np > 1, acc + g * 32);
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            if (CHUNKED && lane == 0) mbar_arrive_cluster(lead_acce0 + 8 * b);
        }
        if (ok) {                                                    // the last MMA of the tile has completed: the ring is free
#pragma unroll
            for (int g = 0; g < WC / 4; ++g) *reinterpret_cast<float4*>(row + g * 4) = make_float4(acc[4 * g], acc[4 * g + 1], acc[4 * g + 2], acc[4 * g + 3]);
        }
    }
    if (!ok) {
        if (lane == 0) failed = 1;
        // error path: time for the copies and MMAs already issued, which touch both CTAs, before either may leave
        const unsigned long long t0 = gtime();
        while (gtime() - t0 < 1000000ull) __nanosleep(1000);
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    cluster_sync_all();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    bool all = true;
    for (uint32_t k = 0; k < C; ++k) all = all && ld_cluster1(map_rank(smem_u32(&failed), k)) == 0;
    if (all) finish_rows<T, EPI, BN, PITCH>(p.e[out], smem_u32(smem), S, slice, side, 2, m0, n0, p.M, p.N);
    cluster_sync_all();                                              // nobody leaves while another CTA reads its shared memory
}

template <typename T, int BN, bool AMN, bool BMN, int EPI, bool EVEN>
ftp_status launch_pair(const Product& p, const KArgs& k, cudaStream_t st, const char* who) {
    Maps m;
    FTP_REQUIRE(make_maps(m, p, 128, BN / 2), FTP_ECUDA, "%s: cannot describe an operand to the copy engine", who);
    auto kern = ffn_pair_kernel<T, BN, AMN, BMN, EPI, EVEN>;
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = allow_smem(asked, kern, (int)PAIR_SMEM<BN>);
    const long long tiles = (long long)k.tiles_m * k.tiles_n * k.parts_n;
    FTP_REQUIRE(tiles < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    if (e == cudaSuccess) e = launch_cluster(kern, dim3(2 * (unsigned)std::min<long long>(tiles, SMS / 2)), PAIR_THREADS, PAIR_SMEM<BN>, 2, st, m.a[0], m.a[1], m.b[0], m.b[1], k);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, int BN, bool AMN, bool BMN, int EPI>
ftp_status launch_either(const Product& p, const KArgs& k, cudaStream_t st, const char* who) {
    bool even = p.N % (16 / (int)sizeof(T)) == 0;
    for (int i = 0; i < k.parts_n; ++i) {
        const Epi& e = k.e[i];
        constexpr int need = sizeof(T) == 4 ? 1 : 2;                 // four floats, eight bf16
        even = even && (!e.y || e.vec_y >= need) && (!e.add || e.vec_add >= need) && (e.stash_kind != STASH_FULL || e.vec_stash >= need);
    }
    return even ? launch_pair<T, BN, AMN, BMN, EPI, true>(p, k, st, who) : launch_pair<T, BN, AMN, BMN, EPI, false>(p, k, st, who);
}
template <typename T, bool AMN, bool BMN, int EPI, bool CHUNKED = sizeof(T) == 4>
ftp_status launch_split(const Product& p, const KArgs& k, int S, cudaStream_t st, const char* who) {
    Maps m;
    FTP_REQUIRE(make_maps(m, p, 128, 64), FTP_ECUDA, "%s: cannot describe an operand to the copy engine", who);
    auto kern = ffn_split_kernel<T, AMN, BMN, EPI, CHUNKED>;
    constexpr uint32_t SMEM = PAIR_RING<128> + 1024;
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = allow_smem(asked, kern, (int)SMEM);
    const long long tiles = (long long)k.tiles_m * k.tiles_n * k.parts_n;
    FTP_REQUIRE(tiles * 2 * S < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    if (e == cudaSuccess) e = launch_cluster(kern, dim3((unsigned)(tiles * 2 * S)), PAIR_THREADS, SMEM, 2 * S, st, m.a[0], m.a[1], m.b[0], m.b[1], k);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <int BN, bool AMN, bool BMN, int EPI>
ftp_status pair_typed(const Product& p, const KArgs& k, int S, cudaStream_t st, const char* who) {
    if constexpr (BN == 128) {                                       // 256 float sums per thread row do not fit into registers
        if (p.out_f32) return S > 1 ? launch_split<float, AMN, BMN, EPI>(p, k, S, st, who) : launch_either<float, BN, AMN, BMN, EPI>(p, k, st, who);
        if (k.long_sum) return launch_split<__nv_bfloat16, AMN, BMN, EPI, true>(p, k, S, st, who);
        if (S > 1) return launch_split<__nv_bfloat16, AMN, BMN, EPI>(p, k, S, st, who);
    }
    return launch_either<__nv_bfloat16, BN, AMN, BMN, EPI>(p, k, st, who);
}
template <int BN>
ftp_status pair_kind(const Product& p, const KArgs& k, int S, cudaStream_t st, const char* who) {
    if (p.epi == EPI_GATED) return pair_typed<BN, false, true, EPI_GATED>(p, k, S, st, who);
    if (p.epi == EPI_LINEAR) return pair_typed<BN, false, true, EPI_LINEAR>(p, k, S, st, who);
    if (p.a_mn) return pair_typed<BN, true, true, EPI_STORE>(p, k, S, st, who);
    return pair_typed<BN, false, false, EPI_STORE>(p, k, S, st, who);
}

}  // namespace

ftp_status run_product_pair(const Product& p, const KArgs& base, bool wide, int S, cudaStream_t st, const char* who) {
    KArgs k = base;
    wide = wide && !p.out_f32;
    const int bn = wide ? 256 : 128, outc = p.epi == EPI_GATED ? bn / 2 : bn;
    k.tiles_m = (int)((p.M + 255) / 256);
    k.tiles_n = (p.N + outc - 1) / outc;
    return wide ? pair_kind<256>(p, k, 1, st, who) : pair_kind<128>(p, k, S, st, who);
}

}  // namespace ffn
}  // namespace ftp
