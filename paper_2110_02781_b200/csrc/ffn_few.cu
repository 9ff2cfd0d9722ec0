// Feed-forward products of one to eight tokens (a decoding step): y = act(x w + b) + r and h = act(x wg) * (x wu).
//
// The weights are read once and everything else is small, so the kernel is a stream of w through the SIMT pipes: eight
// neighbouring lanes read a 128-byte line of a row of w, a warp four rows, a block 32 rows a step with several steps' loads
// in flight, and every thread keeps one sum per token and column.  The rows of w are divided among the CTAs of a cluster
// when the strips of columns alone do not fill the GPU; the parts are added in float in a fixed order: lanes, warps, CTAs.
// Floor: cin cout bytes at the memory's rate.
#include <algorithm>
#include "ffn_gemm.cuh"

namespace ftp {
namespace ffn {
namespace {

constexpr int FEW_THREADS = 256, FEW_WARPS = 8, FEW_STEP = 32;       // rows of w per step of a block

struct FewArgs {
    const void* x; long long ldx;
    const void* w[2]; long long ldw;
    int vec_w;
    Epi e;
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

// MR: tokens (rounded up); P: products (2: gated)
template <typename T, int MR, int P>
__global__ void __launch_bounds__(FEW_THREADS) ffn_few_kernel(const __grid_constant__ FewArgs p) {
    constexpr int V = Wide<T>::V, CW = 8 * V;                        // columns of a thread and of a block
    constexpr int U = P * MR >= 8 ? 4 : 8;                           // steps in flight
    constexpr bool FAST = sizeof(T) == 2;
    extern __shared__ float xs[];                                    // [MR][kper]
    __shared__ float red[FEW_WARPS][P][MR][CW];
    __shared__ float part[P][MR][CW];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t S;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(S));
    const uint32_t rank = cluster_rank();
    const int n0 = (int)(blockIdx.x / S) * CW, k0 = (int)rank * p.kper, klen = max(0, min(p.K - k0, p.kper));
    const int c = n0 + (lane & 7) * V, valid = p.N - c, row = warp * 4 + (lane >> 3);
    const bool whole = p.vec_w && valid >= V;
    grid_dep_sync();

    for (int i = threadIdx.x; i < MR * klen; i += FEW_THREADS) {
        const int m = i / klen, k = i - m * klen;
        xs[m * p.kper + k] = m < p.rows ? to_f(static_cast<const T*>(p.x)[m * p.ldx + k0 + k]) : 0.f;
    }
    __syncthreads();

    float acc[P][MR][V];
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int j = 0; j < V; ++j) acc[q][m][j] = 0.f;
    if (valid > 0) {
        for (int kb = 0; kb < klen; kb += FEW_STEP * U) {
            uint4 w[U][P];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = kb + u * FEW_STEP + row;
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    const T* at = static_cast<const T*>(p.w[q]) + (long long)(k0 + k) * p.ldw + c;
                    w[u][q] = k >= klen ? make_uint4(0u, 0u, 0u, 0u) : whole ? ld_stream(at) : ld_partial<T>(at, valid);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int k = kb + u * FEW_STEP + row;
                if (k < klen) {
#pragma unroll
                    for (int q = 0; q < P; ++q) {
                        float f[V];
                        unpack<T>(w[u][q], f);
#pragma unroll
                        for (int m = 0; m < MR; ++m) {
                            const float xv = xs[m * p.kper + k];
#pragma unroll
                            for (int j = 0; j < V; ++j) acc[q][m][j] = fmaf(xv, f[j], acc[q][m][j]);
                        }
                    }
                }
            }
        }
    }
    // lanes 8 and 16 apart hold other rows of the same columns
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                float v = acc[q][m][j];
                v += __shfl_xor_sync(0xffffffffu, v, 8);
                v += __shfl_xor_sync(0xffffffffu, v, 16);
                if (lane < 8) red[warp][q][m][lane * V + j] = v;
            }
    __syncthreads();
    for (int i = threadIdx.x; i < P * MR * CW; i += FEW_THREADS) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < FEW_WARPS; ++w) v += (&red[w][0][0][0])[i];
        (&part[0][0][0])[i] = v;
    }
    if (S > 1) cluster_sync_all(); else __syncthreads();
    if (rank == 0) {
        const Epi& e = p.e;
        T* y = static_cast<T*>(e.y);
        for (int i = threadIdx.x; i < MR * CW; i += FEW_THREADS) {   // whole warps: CW is 32 or 64, a warp holds 32 columns of a row
            const int m = i / CW, n = n0 + i % CW;
            float z[2] = {0.f, 0.f};
#pragma unroll
            for (int q = 0; q < P; ++q) {
                const uint32_t at = smem_u32(&part[0][0][0]) + (uint32_t)(q * MR * CW + i) * 4;
                for (uint32_t k = 0; k < S; ++k) z[q] += ld_cluster_f(S > 1 ? map_rank(at, k) : at);
            }
            const bool on = m < p.rows && n < p.N;
            if (P == 1 && e.bias && on) z[0] += __ldg(e.bias + n);
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
                    if (m < p.rows && n < e.img[q].pitch) {
                        e.img[q].q[m * e.img[q].pitch + n] = (int8_t)img_code(z[q], img_inv(ex));
                        if (lane == 0) e.img[q].e[m * (e.img[q].pitch / IMG_BLOCK) + n / IMG_BLOCK] = (uint8_t)ex;
                    }
                }
            }
            if (on && y) {
                float v = act_value<FAST>(z[0], e.act);
                if (P == 2) v *= z[1];
                else if (e.add) v += to_f(static_cast<const T*>(e.add)[m * e.ldadd + n]);
                put1(y + m * e.ldy + n, v);
            }
        }
    }
    if (S > 1) cluster_sync_all();                                   // nobody leaves while rank 0 reads its shared memory
}

template <typename T, int MR, int P>
ftp_status launch_few(const FewArgs& a, int S, cudaStream_t st, const char* who) {
    constexpr int CW = 8 * Wide<T>::V;
    auto kern = ffn_few_kernel<T, MR, P>;
    const size_t smem = (size_t)MR * a.kper * 4;
    static std::atomic<unsigned long long> asked{0};
    cudaError_t e = allow_smem(asked, kern, FEW_SMEM);
    if (e == cudaSuccess) e = launch_cluster(kern, (unsigned)((a.N + CW - 1) / CW * S), FEW_THREADS, smem, S, st, a);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, int P>
ftp_status few_rows(const FewArgs& a, int S, cudaStream_t st, const char* who) {
    if (a.rows == 1) return launch_few<T, 1, P>(a, S, st, who);
    if (a.rows == 2) return launch_few<T, 2, P>(a, S, st, who);
    if (a.rows <= 4) return launch_few<T, 4, P>(a, S, st, who);
    return launch_few<T, 8, P>(a, S, st, who);
}

}  // namespace

// the tokens of a CTA's share of the reduction (an eighth at least) have to fit into its shared memory
bool few_tokens(long long rows, long long cin) { return rows <= FEW_ROWS && ((cin + 7) / 8 + FEW_STEP) * FEW_ROWS * 4 <= FEW_SMEM; }

ftp_status run_few(const void* x, long long ldx, const void* const* w, long long ldw, int products, int rows, int K, int N, bool f32, const Epi& e, cudaStream_t st,
                   const char* who) {
    constexpr int SMS = 148;
    FewArgs a{};
    a.x = x; a.ldx = ldx; a.ldw = ldw;
    for (int i = 0; i < products; ++i) a.w[i] = w[i];
    a.vec_w = aligned(w[0], 16) && (products == 1 || aligned(w[1], 16)) && ldw * (f32 ? 4 : 2) % 16 == 0;
    a.e = e;
    a.rows = rows; a.K = K; a.N = N;
    // CTAs per strip of columns: enough for two or three CTAs on every SM, and a few steps for each
    const long long strips = (N + (f32 ? 32 : 64) - 1) / (f32 ? 32 : 64);
    int S = 1;
    while (S < 8 && strips * S < 2 * SMS && K / (S * 2) >= 2 * FEW_STEP) S *= 2;
    while (S < 8 && (long long)((K + S - 1) / S + FEW_STEP) * FEW_ROWS * 4 > FEW_SMEM) S *= 2;
    a.kper = ((K + S - 1) / S + FEW_STEP - 1) / FEW_STEP * FEW_STEP;
    if (f32) return products == 2 ? few_rows<float, 2>(a, S, st, who) : few_rows<float, 1>(a, S, st, who);
    return products == 2 ? few_rows<__nv_bfloat16, 2>(a, S, st, who) : few_rows<__nv_bfloat16, 1>(a, S, st, who);
}

}  // namespace ffn
}  // namespace ftp
