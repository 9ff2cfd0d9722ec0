// Shared by the operators around the feed-forward products (join.cu, recurrence.cu, logprob.cu): rows seen as groups of 16
// bytes per thread, sums over a row's threads, the counter-based generator of the dropout masks, launches.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "ffn_math.cuh"
#include "launch.cuh"
#include "op_checks.h"

namespace ftp {
namespace token {

typedef __nv_bfloat16 bf16;
using ffn::bf_hi;
using ffn::bf_lo;
using ffn::bf_pack;
constexpr int SMS = 148;

template <typename... A> void launch(A&&... args) {
    ++ffn::launches();
    ftp::launch(std::forward<A>(args)...);
}
template <typename... KA, typename... A>
cudaError_t launch_cluster(void (*kern)(KA...), dim3 grid, unsigned block, size_t smem, unsigned cluster, cudaStream_t st, A&&... args) {
    ++ffn::launches();
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

__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned cluster_rank() { unsigned r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ unsigned smem_at(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ unsigned on_rank(unsigned at, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}

// ---- a row's columns on its threads ----
// A thread holds groups of V columns (16 bytes).  VEC: V neighbours, one access (every row starts on 16 bytes and holds
// whole groups).  Otherwise the V columns lie `threads` apart, so that a warp's accesses are still neighbours.
template <typename T> constexpr int V = 16 / (int)sizeof(T);
template <typename T, bool VEC> __device__ __forceinline__ int column(int t, int threads, int g, int j) {
    return VEC ? (g * threads + t) * V<T> + j : (g * V<T> + j) * threads + t;
}
template <typename T> __device__ __forceinline__ void decode(const uint4& r, float (&v)[V<T>]) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) v[i] = __uint_as_float(w[i]);
        else { v[2 * i] = bf_lo(w[i]); v[2 * i + 1] = bf_hi(w[i]); }
    }
}
template <typename T> __device__ __forceinline__ uint4 encode(const float (&v)[V<T>]) {
    if constexpr (sizeof(T) == 4) return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    else return make_uint4(bf_pack(v[0], v[1]), bf_pack(v[2], v[3]), bf_pack(v[4], v[5]), bf_pack(v[6], v[7]));
}
__device__ __forceinline__ unsigned bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ unsigned bits_of(bf16 v) { return __bfloat16_as_ushort(v); }
__device__ __forceinline__ void from_bits(float* p, unsigned b) { *p = __uint_as_float(b); }
__device__ __forceinline__ void from_bits(bf16* p, unsigned b) { *p = __ushort_as_bfloat16((unsigned short)b); }

template <typename T, bool VEC> __device__ __forceinline__ uint4 fetch(const T* row, int t, int threads, int g, int cols) {
    if constexpr (VEC) {
        const int c = column<T, true>(t, threads, g, 0);
        return c < cols ? *reinterpret_cast<const uint4*>(row + c) : make_uint4(0u, 0u, 0u, 0u);
    } else {
        unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int c = column<T, false>(t, threads, g, j);
            if (c < cols) w[j * (int)sizeof(T) / 4] |= bits_of(row[c]) << (sizeof(T) == 4 ? 0 : 16 * (j & 1));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void put(T* row, int t, int threads, int g, int cols, const uint4& r) {
    if constexpr (VEC) {
        const int c = column<T, true>(t, threads, g, 0);
        if (c < cols) *reinterpret_cast<uint4*>(row + c) = r;
    } else {
        const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int c = column<T, false>(t, threads, g, j);
            if (c < cols) from_bits(row + c, w[j * (int)sizeof(T) / 4] >> (sizeof(T) == 4 ? 0 : 16 * (j & 1)));
        }
    }
}
// the same columns of a float vector; `other` where there is none, and behind the last column
template <typename T, bool VEC> __device__ __forceinline__ void fetch_vector(const float* w, float other, int t, int threads, int g, int cols, float (&v)[V<T>]) {
#pragma unroll
    for (int j = 0; j < V<T>; ++j) v[j] = other;
    if (!w) return;
    if constexpr (VEC) {
        const int c = column<T, true>(t, threads, g, 0);
        if (c < cols) {
#pragma unroll
            for (int q = 0; q < V<T> / 4; ++q) {
                const float4 f = *reinterpret_cast<const float4*>(w + c + 4 * q);
                v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int c = column<T, false>(t, threads, g, j);
            if (c < cols) v[j] = w[c];
        }
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void put_vector(float* w, int t, int threads, int g, int cols, const float (&v)[V<T>]) {
    if constexpr (VEC) {
        const int c = column<T, true>(t, threads, g, 0);
        if (c < cols) {
#pragma unroll
            for (int q = 0; q < V<T> / 4; ++q) *reinterpret_cast<float4*>(w + c + 4 * q) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int c = column<T, false>(t, threads, g, j);
            if (c < cols) w[c] = v[j];
        }
    }
}

// Sums over the `threads` (32 or a multiple) threads of a row; `red`: two places for a pair of floats per warp, used in turn, so
// that one barrier a sum is enough.  The whole block takes part.  The order of additions depends on the thread alone.
struct RowSum {
    float2* red;
    int threads, turn;
    __device__ __forceinline__ float2 operator()(float a, float b) {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, d);
            b += __shfl_xor_sync(0xffffffffu, b, d);
        }
        if (threads == 32) return make_float2(a, b);
        const int w = threadIdx.x >> 5, n = threads >> 5, first = w & ~(n - 1);
        float2* at = red + turn * 16;
        turn ^= 1;
        if ((threadIdx.x & 31) == 0) at[w] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
        for (int i = 0; i < n; ++i) { a += at[first + i].x; b += at[first + i].y; }
        return make_float2(a, b);
    }
};

// ---- dropout ----
// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011).
__device__ __forceinline__ uint4 philox(uint4 c, unsigned k0, unsigned k1) {
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned h0 = __umulhi(c.x, 0xD2511F53u), l0 = c.x * 0xD2511F53u, h1 = __umulhi(c.z, 0xCD9E8D57u), l1 = c.z * 0xCD9E8D57u;
        c = make_uint4(h1 ^ c.y ^ k0, l1, h0 ^ c.w ^ k1, l0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return c;
}
// One call gives the eight columns 8 i .. 8 i + 7 of a row 16 bits each, lowest first; a column stays where its bits are at
// least `cut`.
struct Drop {
    const unsigned long long* rng;           // key, step
    unsigned long long key, step;
    unsigned cut, site;
    float factor;
    int64_t row0;
    __device__ __forceinline__ void begin() { if (cut) { key = rng[0]; step = rng[1]; } }
    __device__ __forceinline__ unsigned keep8(unsigned long long group) const {
        const uint4 r = philox(make_uint4((unsigned)group, (unsigned)(group >> 32) | site << 8, (unsigned)step, (unsigned)(step >> 32)), (unsigned)key,
                               (unsigned)(key >> 32));
        const unsigned w[4] = {r.x, r.y, r.z, r.w};
        unsigned m = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) m |= ((w[i] & 0xffffu) >= cut ? 1u : 0u) << (2 * i) | ((w[i] >> 16) >= cut ? 2u : 0u) << (2 * i);
        return m;
    }
    // bit j: column j of group g stays.  Whole warps, which hold columns of one row.
    template <typename T, bool VEC> __device__ __forceinline__ unsigned keep(int64_t row, int t, int threads, int g, int cols) const {
        const unsigned long long first = (unsigned long long)(row0 + row) * (unsigned)((cols + 7) / 8);
        if constexpr (VEC) {
            const int c = column<T, true>(t, threads, g, 0);
            const unsigned m = keep8(first + (unsigned)(c >> 3));
            return V<T> == 8 ? m : m >> (c & 4);
        } else {
            // the warp's columns are V runs of 32, four groups of eight each: a lane makes one of these 4 V groups
            const int l = t & 31, base = t - l, lj = (l >> 2) & (V<T> - 1);
            const unsigned mine = keep8(first + (unsigned)(((g * V<T> + lj) * threads + base) >> 3) + (l & 3));
            unsigned m = 0;
#pragma unroll
            for (int j = 0; j < V<T>; ++j) m |= (__shfl_sync(0xffffffffu, mine, j * 4 + (l >> 3)) >> (l & 7) & 1u) << j;
            return m;
        }
    }
};

inline ftp_status drop_of(Drop* d, double p, const void* rng, int32_t site, int64_t row0, int64_t rows, int64_t cols, const char* who) {
    FTP_REQUIRE(p >= 0.0 && p <= 1.0, FTP_EINVAL, "%s: dropout must be in 0..1", who);
    *d = Drop{};
    d->cut = (unsigned)(p * 65536.0 + 0.5);
    d->factor = d->cut < 65536 ? 65536.f / (float)(65536 - d->cut) : 0.f;
    d->site = (unsigned)site;
    d->row0 = row0;
    d->rng = static_cast<const unsigned long long*>(rng);
    if (!d->cut) return FTP_OK;
    FTP_REQUIRE(site >= 0 && site < (1 << 24), FTP_ERANGE, "%s: site must be in 0..2^24-1", who);
    FTP_REQUIRE(row0 >= 0 && row0 < (1ll << 38) && (row0 + rows) * (double)((cols + 7) / 8) < 1099511627776.0, FTP_ERANGE, "%s: rows beyond the generator's range", who);
    FTP_REQUIRE(rows == 0 || rng, FTP_EINVAL, "%s: dropout without the generator's words", who);
    FTP_REQUIRE(on_bytes(rng, 8), FTP_ERANGE, "%s: the generator's words must start on an 8-byte boundary", who);
    return FTP_OK;
}

// threads of a row (32..512) and groups per thread for `cols` columns
inline void row_shape(int cols, int v, int* threads, int* groups) {
    *threads = 32;
    while (*threads < 512 && *threads * v < cols) *threads *= 2;
    *groups = 1;
    while ((int64_t)*threads * v * *groups < cols) *groups *= 2;
}

}  // namespace token
}  // namespace ftp
