// Feed-forward products of a few tokens (a decoding step): y = act(x w + b) + r and h = act(x wg) * (x wu).
//
// The weights are read once and everything else is small, so the kernels are a stream of w through the SIMT pipes: a CTA
// takes a strip of columns 128 bytes wide, eight neighbouring lanes a row of it, and every thread keeps one sum per token
// and column.  The rows of w are divided among the CTAs of a cluster when the strips alone do not fill the GPU; the parts
// are added in float in a fixed order: lanes, warps, CTAs.  Floor: the bytes of w at the memory's rate.
#include <algorithm>
#include "ffn_gemm.cuh"

namespace ftp {
namespace ffn {
namespace {

constexpr int FEW_THREADS = 256, FEW_WARPS = 8, FEW_STEP = 32;       // rows of w per step of a block

__device__ __forceinline__ void prefetch_2d(const CUtensorMap* map, int x, int y) {
    asm volatile("cp.async.bulk.prefetch.tensor.2d.L2.global [%0, {%1, %2}];" ::"l"(map), "r"(x), "r"(y) : "memory");
}

struct FewArgs {
    const void* x; long long ldx;
    const void* w[2]; long long ldw;
    int vec_w, vec_x, ring;                                          // rows of w / of x on 16 bytes; both
    Span all[2];                                                     // the bytes of w
    Epi e;
    int* err;
    int rows, K, N, kper;                                            // kper: rows of w per CTA of a cluster
};

template <typename T> struct Wide;
template <> struct Wide<__nv_bfloat16> { static constexpr int V = 8; };
template <> struct Wide<float> { static constexpr int V = 4; };

__device__ __forceinline__ uint4 ld_stream(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
template <typename T> __device__ __forceinline__ uint4 ld_partial(const T* p, int valid) {         // element by element, zeros behind
    uint4 v = make_uint4(0u, 0u, 0u, 0u);
    T* e = reinterpret_cast<T*>(&v);
#pragma unroll
    for (int i = 0; i < Wide<T>::V; ++i) if (i < valid) e[i] = p[i];
    return v;
}
template <typename T> __device__ __forceinline__ void unpack(const uint4& q, float (&v)[Wide<T>::V]) {
    const unsigned u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (sizeof(T) == 4) v[i] = __uint_as_float(u[i]);
        else { v[(2 * i) % Wide<T>::V] = bf_lo(u[i]); v[(2 * i + 1) % Wide<T>::V] = bf_hi(u[i]); }
    }
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void put1(float* p, float v) { *p = v; }
__device__ __forceinline__ void put1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }
__device__ __forceinline__ float ld_cluster_f(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// floats between the tokens' values of neighbouring rows of w in shared memory: four tokens are read at a time
template <int MR> constexpr int FEW_PITCH = MR <= 4 ? MR : MR + 4;

// a CTA's strip of columns, share of the reduction and tokens (groups of MR along the grid's second axis, which find the
// same lines of w in L2)
struct Part { int n0, k0, klen, m0, rows; uint32_t S, rank; };
template <int CW, int MR>
__device__ __forceinline__ Part my_part(const FewArgs& p) {
    Part t;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(t.S));
    t.rank = cluster_rank();
    t.n0 = (int)(blockIdx.x / t.S) * CW;
    t.k0 = (int)t.rank * p.kper;
    t.klen = max(0, min(p.K - t.k0, p.kper));
    t.m0 = blockIdx.y * MR;
    t.rows = min(MR, p.rows - t.m0);
    return t;
}

// x of the CTA's share into shared memory, [k][token]; `threads` threads, this one being `t`
template <typename T, int MR>
__device__ __forceinline__ void stage_x(float* xs, const FewArgs& p, const Part& q, int t, int threads) {
    constexpr int V = Wide<T>::V, XP = FEW_PITCH<MR>;
    const T* x = static_cast<const T*>(p.x) + q.m0 * p.ldx + q.k0;
    // neighbouring lanes take neighbouring tokens: their stores fall into different banks
    const int items = (q.klen + V - 1) / V * MR;
    for (int i0 = t; i0 < items; i0 += threads * 4) {
        uint4 v[4];
        int at[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {                                // loads of four items in flight
            const int i = i0 + j * threads, m = i % MR, k = i / MR * V;
            at[j] = i < items ? k * XP + m : -1;
            v[j] = make_uint4(0u, 0u, 0u, 0u);
            if (i < items && m < q.rows) v[j] = p.vec_x && k + V <= q.klen ? ld_stream(x + m * p.ldx + k) : ld_partial<T>(x + m * p.ldx + k, q.klen - k);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (at[j] >= 0) {
                float f[V];
                unpack<T>(v[j], f);
#pragma unroll
                for (int e = 0; e < V; ++e) xs[at[j] + e * XP] = f[e];        // kper is a multiple of V: room for the zeros behind klen
            }
        }
    }
}

// acc += x[k] w[k]: one row of w, V columns, MR tokens
template <int V, int MR, int P>
__device__ __forceinline__ void multiply(float (&acc)[P][MR][V], const float* xk, const float (&f)[P][V]) {
    constexpr int G = MR < 4 ? MR : 4;
#pragma unroll
    for (int m0 = 0; m0 < MR; m0 += G) {
        float xv[G];
        if (G == 4) {
            const float4 t = *reinterpret_cast<const float4*>(xk + m0);
            xv[0] = t.x; xv[1 % G] = t.y; xv[2 % G] = t.z; xv[3 % G] = t.w;
        } else {
#pragma unroll
            for (int m = 0; m < G; ++m) xv[m] = xk[m0 + m];
        }
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int m = 0; m < G; ++m)
#pragma unroll
                for (int j = 0; j < V; ++j) acc[q][m0 + m][j] = fmaf(xv[m], f[q][j], acc[q][m0 + m][j]);
    }
}

// Sums of the eight warps 0..7 (lanes 8 and 16 apart hold other rows of the same columns) into `part`, through `red`.  All
// threads of the block call it.
template <int V, int MR, int P>
__device__ __forceinline__ void block_sums(float (&acc)[P][MR][V], float* red, float* part) {
    constexpr int CW = 8 * V;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (warp < FEW_WARPS) {
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int m = 0; m < MR; ++m)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float v = acc[q][m][j];
                    v += __shfl_xor_sync(0xffffffffu, v, 8);
                    v += __shfl_xor_sync(0xffffffffu, v, 16);
                    if (lane < 8) red[((warp * P + q) * MR + m) * CW + lane * V + j] = v;
                }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < P * MR * CW; i += blockDim.x) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) v += red[w * P * MR * CW + i];
        part[i] = v;
    }
}

// What the epilogue adds to this thread's first output, loaded ahead of the cluster's barrier
template <typename T, int MR, int P>
__device__ __forceinline__ float2 ahead_few(const FewArgs& p, const Part& t) {
    constexpr int CW = 8 * Wide<T>::V;
    const int i = threadIdx.x, n = t.n0 + i % CW;
    float2 v = make_float2(0.f, 0.f);
    if (P == 1 && t.rank == 0 && i < MR * CW && i / CW < t.rows && n < p.N) {
        if (p.e.bias) v.x = __ldg(p.e.bias + n);
        if (p.e.add) v.y = to_f(static_cast<const T*>(p.e.add)[(t.m0 + i / CW) * p.e.ldadd + n]);
    }
    return v;
}

// The cluster's parts added in rank order and finished by its first CTA.  Whole warps: CW is 32 or 64, a warp holds 32
// columns of a row.
template <typename T, int MR, int P>
__device__ __forceinline__ void finish_few(const FewArgs& p, const Part& t, float* part, const float2& ahead) {
    constexpr int CW = 8 * Wide<T>::V;
    constexpr bool FAST = sizeof(T) == 2;
    const int lane = threadIdx.x & 31;
    const Epi& e = p.e;
    T* y = static_cast<T*>(e.y);
    for (int i = threadIdx.x; i < MR * CW; i += blockDim.x) {
        const int n = t.n0 + i % CW;
        const long long m = t.m0 + i / CW;
        float z[2] = {0.f, 0.f};
#pragma unroll
        for (int q = 0; q < P; ++q) {
            const uint32_t at = smem_u32(part) + (uint32_t)(q * MR * CW + i) * 4;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = k < (int)t.S ? ld_cluster_f(t.S > 1 ? map_rank(at, k) : at) : 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) z[q] += v[k];
        }
        const bool row_ok = i / CW < t.rows, on = row_ok && n < p.N;
        const bool first = i == (int)threadIdx.x;
        if (P == 1 && e.bias && on) z[0] += first ? ahead.x : __ldg(e.bias + n);
        if (e.stash_kind == STASH_FULL && on) {
#pragma unroll
            for (int q = 0; q < P; ++q) put1(static_cast<T*>(e.stash[q]) + m * e.ldstash + n, z[q]);
        } else if (e.stash_kind == STASH_8BIT) {
#pragma unroll
            for (int q = 0; q < P; ++q) {
                unsigned top = __float_as_uint(z[q]) & 0x7fffffffu;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
                const unsigned ex = img_exp(top);
                if (row_ok && n < e.img[q].pitch) {
                    e.img[q].q[m * e.img[q].pitch + n] = (int8_t)img_code(z[q], img_inv(ex));
                    if (lane == 0) e.img[q].e[m * (e.img[q].pitch / IMG_BLOCK) + n / IMG_BLOCK] = (uint8_t)ex;
                }
            }
        }
        if (on && y) {
            float v = act_value<FAST>(z[0], e.act);
            if (P == 2) v *= z[1];
            else if (e.add) v += first ? ahead.y : to_f(static_cast<const T*>(e.add)[m * e.ldadd + n]);
            put1(y + m * e.ldy + n, v);
        }
    }
}

// MR: tokens (rounded up); P: products (2: gated).
// Rows of w and of x on 16 bytes: one thread streams boxes of 128 rows x 128 bytes of w (gated: 64 of either), and the tokens'
// values for those rows, with TMA into a ring in shared memory; eight warps multiply, an eighth of the rows each.  The ring keeps 96 KB per CTA, two
// CTAs an SM, on their way from memory all the time, which loads into registers do not (4.0 TB/s of 6.5 with eight in flight
// per thread).
constexpr int RING_BYTES = 96 * 1024, RING_THREADS = FEW_THREADS + 32;
template <int P> constexpr int RING_ROWS = 128 / P;                  // rows of a box: 16 KB of weights a stage (8 KB: 25 us instead of 20 for 4096 x 12288)
template <typename T, int MR, int P>
__global__ void __launch_bounds__(RING_THREADS, MR * P * Wide<T>::V <= 32 ? 2 : 1)
ffn_few_ring_kernel(const __grid_constant__ CUtensorMap map0, const __grid_constant__ CUtensorMap map1, const __grid_constant__ CUtensorMap mapx,
                    const __grid_constant__ FewArgs p) {
    constexpr int V = Wide<T>::V, CW = 8 * V;
    constexpr int ROWS = RING_ROWS<P>, STEPS = ROWS / 32;            // a warp takes ROWS / 8 rows, four a step
    constexpr uint32_t BOX = ROWS * 128, XBOX = MR * ROWS * sizeof(T), STAGE = P * BOX + (XBOX + 127) / 128 * 128;
    constexpr int STAGES = RING_BYTES / STAGE;
    extern __shared__ __align__(16) uint8_t smem_raw[];
    uint8_t* ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 127) & ~uintptr_t(127));   // at the end [FEW_WARPS][P][MR][CW]
    __shared__ __align__(8) unsigned long long bars[2 * STAGES];
    __shared__ float part[P * MR * CW];
    __shared__ int failed;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Part t = my_part<CW, MR>(p);
    const int boxes = (t.klen + ROWS - 1) / ROWS;
    const uint32_t full0 = smem_u32(&bars[0]), empty0 = smem_u32(&bars[STAGES]);
    if (threadIdx.x == 0) {
        tma_prefetch_map(&map0); tma_prefetch_map(&mapx);
        if (P == 2) tma_prefetch_map(&map1);
        for (int s = 0; s < STAGES; ++s) { mbar_init(full0 + 8 * s, 1); mbar_init(empty0 + 8 * s, FEW_WARPS); }
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // The first boxes of w on their way into L2 while the kernel before this one still runs (a hint: nothing is read yet)
    if (warp == FEW_WARPS && elect_one())
        for (int b = 0; b < min(boxes, STAGES); ++b) {
            prefetch_2d(&map0, t.n0, t.k0 + b * ROWS);
            if (P == 2) prefetch_2d(&map1, t.n0, t.k0 + b * ROWS);
        }
    __syncthreads();
    grid_dep_sync();

    float acc[P][MR][V];
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[q][m][j] = 0.f;
    bool ok = true;
    if (warp == FEW_WARPS) {
        // ---- producer ----
        Slot<STAGES> sl;
        for (int b = 0; b < boxes; ++b, sl.next()) {
            ok = warp_wait_for(empty0 + 8 * sl.s, sl.parity ^ 1, p.err, 11);
            if (!ok) break;
            if (elect_one()) {
                const uint32_t dst = smem_u32(ring) + (uint32_t)sl.s * STAGE, bar = full0 + 8 * sl.s;
                const int k = t.k0 + b * ROWS;
                mbar_expect_tx(bar, P * BOX + XBOX);
                tma_load_2d(dst, &map0, t.n0, k, bar);
                if (P == 2) tma_load_2d(dst + BOX, &map1, t.n0, k, bar);
                tma_load_2d(dst + P * BOX, &mapx, k, t.m0, bar);
            }
            __syncwarp();
        }
    } else {
        Slot<STAGES> sl;
        for (int b = 0; b < boxes; ++b, sl.next()) {
            ok = warp_wait_for(full0 + 8 * sl.s, sl.parity, p.err, 12);
            if (!ok) break;
            // rows behind the end of the reduction are zeros in w and in x; shares are whole boxes
            const uint8_t* stage = ring + (uint32_t)sl.s * STAGE;
            const int row = warp * (ROWS / 8) + (lane >> 3);
            const T* xk = reinterpret_cast<const T*>(stage + P * BOX) + row;
#pragma unroll
            for (int u = 0; u < STEPS; ++u) {
                float f[P][V];
#pragma unroll
                for (int q = 0; q < P; ++q) unpack<T>(*reinterpret_cast<const uint4*>(stage + q * BOX + (row + 4 * u) * 128 + (lane & 7) * 16), f[q]);
#pragma unroll
                for (int m = 0; m < MR; ++m) {
                    const float xv = to_f(xk[m * ROWS + 4 * u]);
#pragma unroll
                    for (int q = 0; q < P; ++q)
#pragma unroll
                        for (int j = 0; j < V; ++j) acc[q][m][j] = fmaf(xv, f[q][j], acc[q][m][j]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_one(empty0 + 8 * sl.s);
        }
    }
    if (!ok) {
        if (lane == 0) failed = 1;
        const unsigned long long t0 = gtime();                       // time for the copies already issued to land
        while (gtime() - t0 < 1000000ull) __nanosleep(1000);
    }
    __syncthreads();                                                 // every box has been read: the ring is free
    block_sums<V, MR, P>(acc, reinterpret_cast<float*>(ring), part);
    const float2 ahead = ahead_few<T, MR, P>(p, t);
    if (t.S > 1) cluster_sync_all(); else __syncthreads();
    if (t.rank == 0) {
        bool all = true;
        for (uint32_t k = 0; k < t.S; ++k) all = all && (t.S > 1 ? ld_cluster1(map_rank(smem_u32(&failed), k)) : (uint32_t)failed) == 0;
        if (all) finish_few<T, MR, P>(p, t, part, ahead);
    }
    if (t.S > 1) cluster_sync_all();                                 // nobody leaves while the first CTA reads its shared memory
}

// Any other rows of w: loads into registers, a batch of U steps ahead.
// Sixteen bytes of a row of w: EVEN: rows on 16 bytes, a strip's last columns element by element; otherwise the parts that cover
// them (3952 x 12063 bf16, one token: 64 us element by element, 42 so).
template <typename T, bool EVEN> struct Row16 {
    uint4 q;
    __device__ __forceinline__ void begin(const T* at, int valid, const Span&) {
        q = valid <= 0 ? make_uint4(0u, 0u, 0u, 0u) : valid >= Wide<T>::V ? ld_stream(at) : ld_partial<T>(at, valid);
    }
    __device__ __forceinline__ uint4 end(int) const { return q; }
};
template <typename T> struct Row16<T, false> {
    Words<T, 4> r;
    __device__ __forceinline__ void begin(const T* at, int valid, const Span& all) { r.begin(at, valid, all); }
    __device__ __forceinline__ uint4 end(int valid) const {
        unsigned u[4];
        r.end(valid, u);
        return make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <typename T, int MR, int P, bool EVEN>
__global__ void __launch_bounds__(FEW_THREADS) ffn_few_kernel(const __grid_constant__ FewArgs p) {
    constexpr int V = Wide<T>::V, CW = 8 * V, XP = FEW_PITCH<MR>;    // columns of a thread and of a block
    constexpr int U = P * MR * V >= 128 || !EVEN ? 2 : 4;
    extern __shared__ __align__(16) float xs[];                      // [kper][XP], at the end [FEW_WARPS][P][MR][CW] in its place
    __shared__ float part[P * MR * CW];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Part t = my_part<CW, MR>(p);
    const int c = t.n0 + (lane & 7) * V, valid = p.N - c, row = warp * 4 + (lane >> 3);
    grid_dep_sync();

    auto load = [&](Row16<T, EVEN> (&w)[U][P], int kb) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = kb + u * FEW_STEP + row;
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const T* at = static_cast<const T*>(p.w[q]) + (long long)(t.k0 + k) * p.ldw + c;
                w[u][q].begin(at, k < t.klen ? valid : 0, p.all[q]);
            }
        }
    };
    Row16<T, EVEN> w[U][P], next[U][P];
    load(w, 0);
    stage_x<T, MR>(xs, p, t, threadIdx.x, FEW_THREADS);
    __syncthreads();

    float acc[P][MR][V];
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[q][m][j] = 0.f;
    for (int kb = 0; kb < t.klen; kb += FEW_STEP * U) {
        load(next, kb + FEW_STEP * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int k = kb + u * FEW_STEP + row;
            if (k < t.klen) {
                float f[P][V];
#pragma unroll
                for (int q = 0; q < P; ++q) unpack<T>(w[u][q].end(valid), f[q]);
                multiply<V, MR, P>(acc, xs + k * XP, f);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int q = 0; q < P; ++q) w[u][q] = next[u][q];
    }
    __syncthreads();
    block_sums<V, MR, P>(acc, xs, part);
    const float2 ahead = ahead_few<T, MR, P>(p, t);
    if (t.S > 1) cluster_sync_all(); else __syncthreads();
    if (t.rank == 0) finish_few<T, MR, P>(p, t, part, ahead);
    if (t.S > 1) cluster_sync_all();                                 // nobody leaves while the first CTA reads its shared memory
}

template <typename T>
bool make_ring_map(CUtensorMap* map, const void* base, long long cols, long long rows, long long ld, int box_x, int box_y) {
    EncodeTiledFn fn = encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld * sizeof(T)};
    const cuuint32_t box[2] = {(cuuint32_t)box_x, (cuuint32_t)box_y}, estr[2] = {1, 1};
    return fn(map, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, estr,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int MR, int CW>
dim3 few_grid(const FewArgs& a, int S) { return dim3((unsigned)((a.N + CW - 1) / CW * S), (unsigned)((a.rows + MR - 1) / MR)); }

template <typename T, int MR, int P>
ftp_status launch_ring(const FewArgs& a, int S, cudaStream_t st, const char* who) {
    constexpr int CW = 8 * Wide<T>::V, V = 16 / (int)sizeof(T), B = 128 / (int)sizeof(T);
    CUtensorMap m0, m1, mx;
    const long long ldx = a.rows == 1 ? (a.K + V - 1) / V * V : a.ldx;       // one row: never stepped over
    FTP_REQUIRE(make_ring_map<T>(&m0, a.w[0], a.N, a.K, a.ldw, B, RING_ROWS<P>) && (P == 1 || make_ring_map<T>(&m1, a.w[1], a.N, a.K, a.ldw, B, RING_ROWS<P>)) &&
                    make_ring_map<T>(&mx, a.x, a.K, a.rows, ldx, RING_ROWS<P>, MR), FTP_ECUDA, "%s: cannot describe an operand to the copy engine", who);
    if (P == 1) m1 = m0;
    static_assert(FEW_WARPS * P * MR * CW * 4 <= RING_BYTES / 2, "the warps' sums reuse the ring");
    auto kern = ffn_few_ring_kernel<T, MR, P>;
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = allow_smem(asked, kern, RING_BYTES + 128);
    if (e == cudaSuccess) e = launch_cluster(kern, few_grid<MR, CW>(a, S), RING_THREADS, RING_BYTES + 128, S, st, m0, m1, mx, a);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}

template <typename T, int MR, int P>
ftp_status launch_few(const FewArgs& a, int S, cudaStream_t st, const char* who) {
    if constexpr (sizeof(T) == 4 || MR <= 2)                         // four bf16 tokens come with at most 4 MB of w (few_tokens)
        if (a.ring) return launch_ring<T, MR, P>(a, S, st, who);
    constexpr int CW = 8 * Wide<T>::V;
    const size_t x_bytes = (size_t)FEW_PITCH<MR> * a.kper * 4, red_bytes = (size_t)FEW_WARPS * P * MR * CW * 4;
    auto kern = a.vec_w ? ffn_few_kernel<T, MR, P, true> : ffn_few_kernel<T, MR, P, false>;
    static std::atomic<unsigned long long> asked[2] = {};
    cudaError_t e = allow_smem(asked[a.vec_w ? 1 : 0], kern, FEW_SMEM);
    if (e == cudaSuccess) e = launch_cluster(kern, few_grid<MR, CW>(a, S), FEW_THREADS, std::max(x_bytes, red_bytes), S, st, a);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, int P>
ftp_status few_rows(const FewArgs& a, int S, cudaStream_t st, const char* who) {
    if (a.rows == 1) return launch_few<T, 1, P>(a, S, st, who);
    if (a.rows == 2) return launch_few<T, 2, P>(a, S, st, who);
    if constexpr (sizeof(T) == 4) {
        if constexpr (P == 1)
            if (a.rows > 8) return launch_few<T, 16, P>(a, S, st, who);
        if (a.rows > 4) return launch_few<T, 8, P>(a, S, st, who);
    }
    if constexpr (sizeof(T) == 4 || P == 1) return launch_few<T, 4, P>(a, S, st, who);
    return fail(FTP_EUNSUPPORTED, "%s: no few-token form for %d tokens", who, a.rows);   // few_tokens sends none
}

// bytes of shared memory that the tokens of a group take beside `k` rows of w
long long few_smem(long long rows, long long k, bool f32, int products) {
    const int group = rows <= 2 ? (int)rows : rows <= 4 || !f32 ? 4 : rows <= 8 || products == 2 ? 8 : 16;
    return (k + 2 * FEW_STEP) * (group <= 4 ? group : group + 4) * 4;
}

}  // namespace

// The tokens of a CTA's share of the reduction (an eighth at least) have to fit into its shared memory.  bf16: two tokens, or
// four of a small linear op; beyond that the tensor cores are faster (four tokens, 4096 x 12288: 28.0 against 21.2 us).
// float: up to 32 tokens (gated: 16), since the tensor cores would first need the planes of w, five times its bytes (16
// tokens, 4096 x 4096: 30 against 55 us).
bool few_tokens(long long rows, long long cin, long long cout, bool f32, int products) {
    const long long most = f32 ? (products == 2 ? 16 : 32) : (products == 1 && cin * cout <= 2 << 20 ? 4 : 2);
    return rows <= most && few_smem(rows, (cin + 7) / 8, f32, products) <= FEW_SMEM;
}

ftp_status run_few(const void* x, long long ldx, const void* const* w, long long ldw, int products, int rows, int K, int N, bool f32, const Epi& e, int* err,
                   cudaStream_t st, const char* who) {
    constexpr int SMS = 148;
    FewArgs a{};
    a.x = x; a.ldx = ldx; a.ldw = ldw;
    for (int i = 0; i < products; ++i) a.w[i] = w[i];
    a.vec_w = aligned(w[0], 16) && (products == 1 || aligned(w[1], 16)) && ldw * (f32 ? 4 : 2) % 16 == 0;
    a.vec_x = aligned(x, 16) && (rows == 1 || ldx * (f32 ? 4 : 2) % 16 == 0);
    a.e = e;
    a.err = err;
    for (int i = 0; i < products; ++i) a.all[i] = f32 ? span_of<float>(w[i], K, N, ldw) : span_of<__nv_bfloat16>(w[i], K, N, ldw);
    a.rows = rows; a.K = K; a.N = N;
    // Up to 4 MB of w the loads into registers are quicker, whose kernel begins and ends faster (one token, 1024 x 1024 bf16:
    // 3.6 against 4.6 us; 4096 x 4096 float: 14.2 against 13.1; the gated 4096 x 12288 bf16: 45 against 34.6)
    a.ring = a.vec_w && a.vec_x && (long long)K * N * products * (f32 ? 4 : 2) > 4 << 20;
    // CTAs per strip of columns: one wave of two CTAs an SM, of one where the sums need more registers, of four small ones
    // without a ring; two boxes each at least
    const long long strips = (N + (f32 ? 32 : 64) - 1) / (f32 ? 32 : 64), groups = rows <= 4 ? 1 : rows <= 8 || products == 2 ? (rows + 7) / 8 : (rows + 15) / 16;
    const int room = !a.ring ? 4 : (f32 && rows * products > 8 ? 1 : 2);
    int S = (int)std::max<long long>(1, std::min<long long>(8, room * SMS / (strips * groups)));
    const int box = a.ring ? 128 / products : FEW_STEP * 2;
    while (S > 1 && K / S < 128) --S;
    if (!a.ring)
        while (S < 8 && few_smem(rows, (K + S - 1) / S, f32, products) > FEW_SMEM) ++S;
    a.kper = ((K + S - 1) / S + box - 1) / box * box;
    if (f32) return products == 2 ? few_rows<float, 2>(a, S, st, who) : few_rows<float, 1>(a, S, st, who);
    return products == 2 ? few_rows<__nv_bfloat16, 2>(a, S, st, who) : few_rows<__nv_bfloat16, 1>(a, S, st, who);
}

}  // namespace ffn
}  // namespace ftp
