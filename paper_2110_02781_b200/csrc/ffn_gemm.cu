// Products of the feed-forward operators on the 5th-generation tensor cores: D = op(A) op(B) from bf16 planes with float
// accumulation in tensor memory and the operators' epilogues.
//
// Operands are read as they lie in memory: with the reduction contiguous (K-major) or across their rows (MN-major).  A
// float tensor comes as three bf16 planes (8 mantissa bits each, 24 together) and a product of two of them as the six
// plane products that matter; the dropped ones are below 2^-24 of the result.
//
// tile kernel: one CTA per 128 x BN tile and slice of the reduction.  Warp 0 (one thread) streams operand tiles with TMA
// into a ring in shared memory, warp 1 (one thread) issues the MMAs, warps 2-5 move the accumulator to shared memory.
// The slices of one tile form a cluster: each CTA then adds up the rows rank, rank + S, ... of the tile over the
// cluster's shared memory, always in rank order, and finishes them (bias, activation, residual, kept values), so a
// product with few tiles still uses the whole GPU, needs no workspace, and gives the same bits every time.
//
// Every wait is bounded; see gemm_tc.cu for the error protocol.
#include <algorithm>
#include <cstring>
#include "ffn_math.cuh"
#include "gemm_tc_common.cuh"

namespace ftp {
using namespace tc;
namespace ffn {
namespace {

constexpr int BK = 64;                       // reduction elements per stage: one 128-byte swizzle row

// The plane pairs of a product, small terms first.
struct Pairs { int n; unsigned char a[6], b[6]; };
inline Pairs plane_pairs(int pa, int pb) {
    Pairs r{};
    for (int s = 4; s >= 0; --s)             // s = sum of the plane indices: terms of relative size 2^-8s
        for (int i = 0; i < pa; ++i) {
            const int j = s - i;
            if (j < 0 || j >= pb || s > 2) continue;
            r.a[r.n] = (unsigned char)i; r.b[r.n] = (unsigned char)j; ++r.n;
        }
    return r;
}

struct KArgs {
    Epi e[2];
    long long M;
    int N;
    int kb_part, parts_k;                    // 64-wide reduction blocks per part, parts of the reduction
    int parts_n;                             // 2: the column tiles of output 1 follow those of output 0
    int tiles_m, tiles_n;                    // column tiles of one output
    Pairs pairs;
    int* err;
};

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// MN-major operand: slabs of 64 reduction rows x 64 elements (128-byte rows, 128-byte swizzle), slab_bytes apart
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t slab_bytes) {
    return (uint64_t)((saddr >> 4) & 0x3FFF) | (uint64_t)((slab_bytes >> 4) & 0x3FFF) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
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

// The epilogue on four columns n.. of row m; a whole warp calls it (row_ok: this lane's row exists).
template <typename T, int EPI>
__device__ __forceinline__ void finish4(const Epi& e, long long m, int n, int N, bool row_ok, float (&a)[4], float (&b)[4]) {
    const int valid = row_ok ? min(4, max(0, N - n)) : 0;
    T* y = static_cast<T*>(e.y);
    constexpr bool FAST = sizeof(T) == 2;
    float add[4] = {0.f, 0.f, 0.f, 0.f};
    if (EPI != EPI_GATED && e.add && valid) load4(static_cast<const T*>(e.add) + m * e.ldadd + n, valid, e.vec_add, add);
    if (EPI == EPI_STORE) {
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] += add[i];
        if (valid) store4(y + m * e.ldy + n, valid, e.vec_y, a);
        return;
    }
    if (EPI == EPI_LINEAR && e.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) if (i < valid) a[i] += __ldg(e.bias + n + i);
    }
    if (e.stash_kind == STASH_FULL && valid) {
        store4(static_cast<T*>(e.stash[0]) + m * e.ldstash + n, valid, e.vec_stash, a);
        if (EPI == EPI_GATED) store4(static_cast<T*>(e.stash[1]) + m * e.ldstash + n, valid, e.vec_stash, b);
    } else if (e.stash_kind == STASH_8BIT) {
        // columns past the end are zero products (their operand tiles are filled with zeros): no effect on a block's maximum
        img_store4(e.img[0], m, n, a, row_ok);
        if (EPI == EPI_GATED) img_store4(e.img[1], m, n, b, row_ok);
    }
    if (valid && y) {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float f = act_value<FAST>(a[i], e.act);
            v[i] = EPI == EPI_GATED ? f * b[i] : f + add[i];
        }
        store4(y + m * e.ldy + n, valid, e.vec_y, v);
    }
}

// ---- one CTA per tile and reduction slice ---------------------------------------------------------------------------
constexpr int TILE_THREADS = 192;
template <int BN> constexpr int TILE_STAGES = BN == 128 ? 6 : 8;
template <int BN> constexpr uint32_t TILE_SMEM = TILE_STAGES<BN> * (128 * BK * 2 + BN * BK * 2) + 1024;

// AMN / BMN: the operand is MN-major.  EPI_GATED: the tile's first BN / 2 columns are A B[0], the others A B[1].
template <typename T, int BN, bool AMN, bool BMN, int EPI>
__global__ void __launch_bounds__(TILE_THREADS, 1) ffn_tile_kernel(const __grid_constant__ CUtensorMap mapA0, const __grid_constant__ CUtensorMap mapA1,
                                                                   const __grid_constant__ CUtensorMap mapB0, const __grid_constant__ CUtensorMap mapB1,
                                                                   const __grid_constant__ KArgs p) {
    constexpr int STAGES = TILE_STAGES<BN>;
    constexpr uint32_t SLAB = 64 * BK * 2, A_BYTES = 128 * BK * 2, B_BYTES = BN * BK * 2, STAGE_BYTES = A_BYTES + B_BYTES;
    constexpr int OUTC = EPI == EPI_GATED ? BN / 2 : BN;             // output columns of a tile
    constexpr int PITCH = BN + 4;                                    // floats between rows of the staged accumulator: 16-byte accesses of 8 lanes hit all banks
    static_assert(128 * PITCH * 4 <= STAGES * STAGE_BYTES, "the staged accumulator reuses the operand ring");
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ __align__(8) unsigned long long bars[2 * STAGES + 1];
    __shared__ uint32_t tmem_base, failed;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t S;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
    const uint32_t rank = cluster_rank();
    const int tile = blockIdx.x / S, tn_all = p.tiles_n * p.parts_n;
    const int tm = tile / tn_all, tn = tile % tn_all, out = tn / p.tiles_n;
    const long long m0 = (long long)tm * 128;
    const int n0 = (tn - out * p.tiles_n) * OUTC;
    // this slice's share of the 64-wide blocks; a block is done for every pair of planes before the next (its tiles are
    // read from L2 again, not from memory)
    const int all_kb = p.kb_part * p.parts_k;
    const int kb0 = (int)((long long)all_kb * rank / S), kb1 = (int)((long long)all_kb * (rank + 1) / S);
    const int its = (kb1 - kb0) * p.pairs.n;
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[STAGES]), accum = smem_u32(&bars[2 * STAGES]);

    if (threadIdx.x == 0) {
        tma_prefetch_map(&mapA0); tma_prefetch_map(&mapB0);
        if (p.parts_k > 1) tma_prefetch_map(&mapA1);
        if (p.parts_k > 1 || p.parts_n > 1 || EPI == EPI_GATED) tma_prefetch_map(&mapB1);
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, 1); }
        mbar_init(accum, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "r"((uint32_t)BN) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = tmem_base;
    grid_dep_sync();

    if (warp == 0) {
        if (lane == 0) {
            // ---- producer ----
            int it = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1 && ok; ++kb) {
                const int part = kb / p.kb_part, k = (kb - part * p.kb_part) * BK;
                const CUtensorMap* ma = part ? &mapA1 : &mapA0;
                const CUtensorMap* mb = (part || out) ? &mapB1 : &mapB0;
                for (int pr = 0; pr < p.pairs.n; ++pr, ++it) {
                    const int s = it % STAGES;
                    if (it >= STAGES && !mbar_wait(empty0 + 8 * s, ((it / STAGES) & 1) ^ 1, p.err, 1)) { ok = false; break; }
                    const uint32_t sa = smem_u32(smem + s * STAGE_BYTES), sb = sa + A_BYTES, bar = full0 + 8 * s;
                    const int za = p.pairs.a[pr], zb = p.pairs.b[pr];
                    mbar_expect_tx(bar, STAGE_BYTES);
                    if (AMN) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) tma_load_3d(sa + t * SLAB, ma, (int)m0 + 64 * t, k, za, bar);
                    } else
                        tma_load_3d(sa, ma, k, (int)m0, za, bar);
                    if (EPI == EPI_GATED) {
#pragma unroll
                        for (int t = 0; t < BN / 64; ++t)
                            tma_load_3d(sb + t * SLAB, t < BN / 128 ? &mapB0 : &mapB1, n0 + 64 * (t & (BN / 128 - 1)), k, zb, bar);
                    } else if (BMN) {
#pragma unroll
                        for (int t = 0; t < BN / 64; ++t) tma_load_3d(sb + t * SLAB, mb, n0 + 64 * t, k, zb, bar);
                    } else
                        tma_load_3d(sb, mb, k, n0, zb, bar);
                }
            }
            if (!ok || *((volatile int*)p.err) != 0) {
                // error path: let the copies already issued land before the block's memory is released
                for (int k = max(0, it - STAGES); k < it; ++k) {
                    const unsigned long long t0 = gtime();
                    while (!mbar_test(full0 + 8 * (k % STAGES), (k / STAGES) & 1) && gtime() - t0 < 1000000ull) __nanosleep(128);
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            // ---- MMA issuer ----
            constexpr uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | (AMN ? 1u << 15 : 0u) | (BMN ? 1u << 16 : 0u) | ((uint32_t)(BN >> 3) << 17) |
                                       ((uint32_t)(128 >> 4) << 24);
            bool ok = true;
            for (int it = 0; it < its && ok; ++it) {
                const int s = it % STAGES;
                ok = mbar_wait(full0 + 8 * s, (it / STAGES) & 1, p.err, 2);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t sa = smem_u32(smem + s * STAGE_BYTES), sb = sa + A_BYTES;
                const uint64_t ad = AMN ? desc_mn(sa, SLAB) : umma_desc_k_sw128(sa), bd = BMN ? desc_mn(sb, SLAB) : umma_desc_k_sw128(sb);
#pragma unroll
                for (int k = 0; k < BK / 16; ++k)            // 16 elements further: 32 bytes along a K-major row, 16 rows of an MN-major slab
                    umma_bf16(tmem, ad + (uint64_t)(k * (AMN ? 128 : 2)), bd + (uint64_t)(k * (BMN ? 128 : 2)), idesc, (it > 0 || k > 0) ? 1u : 0u);
                umma_commit(empty0 + 8 * s);
            }
            if (ok && its > 0) umma_commit(accum);
        }
    } else {
        // ---- accumulator -> shared memory (the ring is free once the last MMA has completed) ----
        const int q = warp & 3;
        const bool have = __all_sync(0xffffffffu, its > 0 ? mbar_wait(accum, 0, p.err, 3) : true);
        if (have) {
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            float* row = reinterpret_cast<float*>(smem) + (q * 32 + lane) * PITCH;
#pragma unroll 1
            for (int c = 0; c < BN / 32; ++c) {
                uint32_t r[32];
                if (its > 0) tmem_ld32(tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(c * 32), r);
                else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) r[i] = 0u;
                }
#pragma unroll
                for (int g = 0; g < 8; ++g) *reinterpret_cast<uint4*>(row + c * 32 + g * 4) = make_uint4(r[4 * g], r[4 * g + 1], r[4 * g + 2], r[4 * g + 3]);
            }
        } else if (lane == 0)
            failed = 1;
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)BN) : "memory");
    if (S > 1) cluster_sync_all();

    // ---- rows rank, rank + S, ... of the tile, added over the slices in rank order ----
    bool ok = true;
    for (uint32_t k = 0; k < S; ++k) ok = ok && (S > 1 ? ld_cluster1(map_rank(smem_u32(&failed), k)) : failed) == 0;
    if (ok) {
        constexpr int LPR = OUTC / 4, RPW = 32 / LPR;                // lanes per row, rows per warp
        const int rows = (int)min(128ll, p.M - m0), c = (lane % LPR) * 4;
        const uint32_t base = smem_u32(smem);
        for (int i = warp * RPW; i * (int)S + (int)rank < rows; i += (TILE_THREADS / 32) * RPW) {
            const int r = (i + lane / LPR) * (int)S + (int)rank;
            const bool row_ok = r < rows;
            const uint32_t at = base + (uint32_t)((row_ok ? r : 0) * PITCH + c) * 4;
            float a[4] = {0.f, 0.f, 0.f, 0.f}, b[4] = {0.f, 0.f, 0.f, 0.f};
            for (uint32_t k = 0; k < S; ++k) {
                const uint32_t from = S > 1 ? map_rank(at, k) : at;
                const float4 u = ld_cluster4(from);
                a[0] += u.x; a[1] += u.y; a[2] += u.z; a[3] += u.w;
                if (EPI == EPI_GATED) {
                    const float4 w = ld_cluster4(from + OUTC * 4);
                    b[0] += w.x; b[1] += w.y; b[2] += w.z; b[3] += w.w;
                }
            }
            finish4<T, EPI>(p.e[out], m0 + r, n0 + c, p.N, row_ok, a, b);
        }
    }
    if (S > 1) cluster_sync_all();                                   // nobody leaves while another CTA reads its shared memory
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
    for (int i = 0; i < 2; ++i) {
        const Operand& A = p.A[(p.parts > 1 && p.cat_k) ? i : 0];
        const Operand& B = p.B[p.parts > 1 ? i : 0];
        if (!make_map(&m.a[i], A, 64, p.a_mn ? BK : a_rows) || !make_map(&m.b[i], B, 64, p.b_mn ? BK : b_rows)) return false;
    }
    return true;
}

template <typename... KA, typename... A>
cudaError_t launch_cluster(void (*kern)(KA...), unsigned grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t st, A&&... args) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(grid);
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

template <typename T, int BN, bool AMN, bool BMN, int EPI>
ftp_status launch_tile(const Product& p, KArgs& k, int S, cudaStream_t st, const char* who) {
    Maps m;
    FTP_REQUIRE(make_maps(m, p, 128, BN), FTP_ECUDA, "%s: cannot describe an operand to the copy engine", who);
    auto kern = ffn_tile_kernel<T, BN, AMN, BMN, EPI>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)TILE_SMEM<BN>);
    if (e == cudaSuccess) e = launch_cluster(kern, (unsigned)((long long)k.tiles_m * k.tiles_n * k.parts_n * S), TILE_THREADS, TILE_SMEM<BN>, S, st, m.a[0], m.a[1], m.b[0], m.b[1], k);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}

template <int BN, bool AMN, bool BMN, int EPI>
ftp_status tile_typed(const Product& p, KArgs& k, int S, cudaStream_t st, const char* who) {
    return p.out_f32 ? launch_tile<float, BN, AMN, BMN, EPI>(p, k, S, st, who) : launch_tile<__nv_bfloat16, BN, AMN, BMN, EPI>(p, k, S, st, who);
}

}  // namespace

ftp_status run_product(const Product& p, cudaStream_t st, const char* who) {
    constexpr int SMS = 148;
    KArgs k{};
    k.e[0] = p.e[0]; k.e[1] = p.e[1];
    k.M = p.M; k.N = p.N; k.err = p.err;
    k.pairs = plane_pairs(p.A[0].planes, p.B[0].planes);
    k.kb_part = (int)((p.K + BK - 1) / BK);
    k.parts_k = (p.parts > 1 && p.cat_k) ? 2 : 1;
    k.parts_n = (p.parts > 1 && !p.cat_k && p.epi != EPI_GATED) ? 2 : 1;
    k.tiles_m = (int)((p.M + 127) / 128);
    auto tiles = [&](int outc) { return (long long)k.tiles_m * ((p.N + outc - 1) / outc) * k.parts_n; };
    const int outc128 = p.epi == EPI_GATED ? 64 : 128;
    const bool narrow = p.epi != EPI_GATED && tiles(outc128) < SMS && p.N > 64 ? true : (p.epi != EPI_GATED && p.N <= 64);
    const int outc = narrow ? 64 : outc128;
    k.tiles_n = (p.N + outc - 1) / outc;
    // slices of the reduction: as many as fill the SMs once, each at least four blocks long
    const long long t = tiles(outc), blocks = (long long)k.kb_part * k.parts_k * k.pairs.n;
    int S = 1;
    while (S < 8 && t * S * 2 <= SMS && blocks / (S * 2) >= 4 && (long long)k.kb_part * k.parts_k >= S * 2) S *= 2;
    FTP_REQUIRE(t * S < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    if (p.epi == EPI_GATED) return tile_typed<128, false, true, EPI_GATED>(p, k, S, st, who);
    if (p.epi == EPI_LINEAR) return narrow ? tile_typed<64, false, true, EPI_LINEAR>(p, k, S, st, who) : tile_typed<128, false, true, EPI_LINEAR>(p, k, S, st, who);
    if (p.a_mn) return narrow ? tile_typed<64, true, true, EPI_STORE>(p, k, S, st, who) : tile_typed<128, true, true, EPI_STORE>(p, k, S, st, who);
    return narrow ? tile_typed<64, false, false, EPI_STORE>(p, k, S, st, who) : tile_typed<128, false, false, EPI_STORE>(p, k, S, st, who);
}

}  // namespace ffn
}  // namespace ftp
