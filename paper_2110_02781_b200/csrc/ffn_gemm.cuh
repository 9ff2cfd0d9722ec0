// What the two product kernels share: operand order, epilogue pieces, tensor maps, launches with clusters.
#pragma once
#include <algorithm>
#include "ffn_math.cuh"
#include "gemm_tc_common.cuh"

namespace ftp {
using namespace tc;
namespace ffn {

constexpr int BK = 64;                       // reduction elements per stage: one 128-byte swizzle row
// Operand tiles arrive one plane of A and of B at a time, the smallest planes of a block first; once the main planes are
// there, the products of the block that matter are issued small terms first, each plane read from memory once:
//   plane 1: A1 B1    plane 0: A0 B2, A2 B0, A0 B1, A1 B0, A0 B0
// (those with planes that exist).  Dropped: A1 B2, A2 B1, A2 B2, below 2^-24 of the result.
//
// Float results: the tensor cores cut their accumulator instead of rounding it, an error that grows with the number of
// steps (measured 3.5e-5 of the result after 2048 steps of 16 elements).  So it is emptied into registers, which add with
// rounding, after every block of a product of planes and every CHUNK blocks of a product of bf16 tensors.
constexpr int CHUNK = 4;

struct KArgs {
    Epi e[2];
    long long M;
    int N;
    int kb_part, parts_k;                    // 64-wide reduction blocks per part, parts of the reduction
    int parts_n;                             // 2: the column tiles of output 1 follow those of output 0
    int tiles_m, tiles_n;                    // column tiles of one output
    int pa, pb, np;                          // planes of A and of B, the larger of the two
    int chunk;                               // blocks per accumulation in the tensor cores (float results)
    int* err;
};

namespace {

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
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

// The MMAs of a block that its plane z completes; ad / bd: descriptors of the operand tiles of plane 0, 1, 2.
// mma(ad, bd) issues the four 16-element steps.
template <typename F>
__device__ __forceinline__ void plane_products(int z, const KArgs& p, F&& mma) {
    if (p.np == 1) { mma(0, 0); return; }
    if (z == 1 && p.pa > 1 && p.pb > 1) mma(1, 1);
    if (z == 0) {
        if (p.pb > 2) mma(0, 2);
        if (p.pa > 2) mma(2, 0);
        if (p.pb > 1) mma(0, 1);
        if (p.pa > 1) mma(1, 0);
        mma(0, 0);
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


}  // namespace

// products on CTA pairs (ffn_pair.cu); wide: 256 x 256 tiles instead of 256 x 128
ftp_status run_product_pair(const Product& p, const KArgs& base, bool wide, cudaStream_t st, const char* who);

}  // namespace ffn
}  // namespace ftp
