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
// An error that the caller reports by itself: not left behind for the next call's check of its own launches.
inline cudaError_t told(cudaError_t e) {
    if (e != cudaSuccess) cudaGetLastError();
    return e;
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
    return told(cudaLaunchKernelEx(&cfg, kern, std::forward<A>(args)...));
}

__device__ __forceinline__ void cluster_sync() { asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ unsigned cluster_rank() { unsigned r; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ unsigned smem_at(const void* p) { return (unsigned)__cvta_generic_to_shared(p); }
__device__ __forceinline__ unsigned on_rank(unsigned at, unsigned rank) {
    unsigned r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(at), "r"(rank));
    return r;
}

// An attribute of a kernel, told to the driver once per kernel, device and thread (1.5 us a call otherwise)
template <cudaFuncAttribute WHAT> bool kernel_may(const void* kern, int value) {
    static thread_local const void* known[64] = {};
    static thread_local int devices[64] = {};
    int dev = -1;
    if (told(cudaGetDevice(&dev)) != cudaSuccess) return false;
    const size_t at = (reinterpret_cast<uintptr_t>(kern) >> 4) % 64;
    if (known[at] == kern && devices[at] == dev) return true;
    if (told(cudaFuncSetAttribute(kern, WHAT, value)) != cudaSuccess) return false;
    known[at] = kern;
    devices[at] = dev;
    return true;
}
// `bytes` of dynamic shared memory, the same for every call with a kernel
inline bool more_shared(const void* kern, size_t bytes) { return kernel_may<cudaFuncAttributeMaxDynamicSharedMemorySize>(kern, (int)bytes); }
// clusters of more than eight blocks
inline bool large_clusters(const void* kern) { return kernel_may<cudaFuncAttributeNonPortableClusterSizeAllowed>(kern, 1); }

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

// Loads: a thread whose columns lie behind the last one gets others of the row (no load is conditional).
template <typename T, bool VEC> __device__ __forceinline__ int column_in(int t, int threads, int g, int j, int cols) {
    return min(column<T, VEC>(t, threads, g, j), VEC ? cols - V<T> + j : cols - 1);
}
template <typename T, bool VEC> __device__ __forceinline__ uint4 fetch(const T* row, int t, int threads, int g, int cols) {
    if constexpr (VEC) {
        // read once: kept out of the first cache, which is for the vectors that every row needs
        uint4 r;
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w)
                     : "l"(reinterpret_cast<const char*>(row) + (unsigned)column_in<T, true>(t, threads, g, 0, cols) * (unsigned)sizeof(T)) : "memory");
        return r;
    }
    else {
        unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < V<T>; ++j) w[j * (int)sizeof(T) / 4] |= bits_of(row[column_in<T, false>(t, threads, g, j, cols)]) << (sizeof(T) == 4 ? 0 : 16 * (j & 1));
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void put(T* row, int t, int threads, int g, int cols, const uint4& r) {
    if constexpr (VEC) {
        const int c = column<T, true>(t, threads, g, 0);
        if (c < cols) *reinterpret_cast<uint4*>(reinterpret_cast<char*>(row) + (unsigned)c * (unsigned)sizeof(T)) = r;
    } else {
        const unsigned w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int c = column<T, false>(t, threads, g, j);
            if (c < cols) from_bits(row + c, w[j * (int)sizeof(T) / 4] >> (sizeof(T) == 4 ? 0 : 16 * (j & 1)));
        }
    }
}
// the same columns of a float vector
template <typename T, bool VEC> __device__ __forceinline__ void fetch_vector(const float* w, int t, int threads, int g, int cols, float (&v)[V<T>]) {
    if constexpr (VEC) {
        const char* at = reinterpret_cast<const char*>(w) + (unsigned)column_in<T, true>(t, threads, g, 0, cols) * 4u;
#pragma unroll
        for (int q = 0; q < V<T> / 4; ++q) {
            const float4 f = reinterpret_cast<const float4*>(at)[q];
            v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V<T>; ++j) v[j] = w[column_in<T, false>(t, threads, g, j, cols)];
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

// Two floats at a time: the packed forms of sm_100 do an addition, product or fused product of both in one instruction.
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float a, float b) { F2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ F2 f2(float a) { return f2(a, a); }
__device__ __forceinline__ float2 parts(F2 v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }
__device__ __forceinline__ float sum2(F2 v) { const float2 p = parts(v); return p.x + p.y; }
template <typename T> constexpr int P = V<T> / 2;                    // pairs of a group
template <typename T> __device__ __forceinline__ void decode(const uint4& r, F2 (&v)[P<T>]) {
    const unsigned w[4] = {r.x, r.y, r.z, r.w};
    if constexpr (sizeof(T) == 4) {
        v[0] = f2(__uint_as_float(w[0]), __uint_as_float(w[1]));
        v[1] = f2(__uint_as_float(w[2]), __uint_as_float(w[3]));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = f2(bf_lo(w[i]), bf_hi(w[i]));
    }
}
template <typename T> __device__ __forceinline__ uint4 encode(const F2 (&v)[P<T>]) {
    unsigned w[4];
    if constexpr (sizeof(T) == 4) {
        const float2 a = parts(v[0]), b = parts(v[1]);
        return make_uint4(__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(b.x), __float_as_uint(b.y));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) { const float2 a = parts(v[i]); w[i] = bf_pack(a.x, a.y); }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <typename T, bool VEC> __device__ __forceinline__ void fetch_vector(const float* w, int t, int threads, int g, int cols, F2 (&v)[P<T>]) {
    float f[V<T>];
    fetch_vector<T, VEC>(w, t, threads, g, cols, f);
#pragma unroll
    for (int j = 0; j < P<T>; ++j) v[j] = f2(f[2 * j], f[2 * j + 1]);
}

// Sums over the threads of a block (32 to 512, whole warps) that holds one row, through one place per warp; `red` holds two sets of
// 16 places, used in turn, so that one barrier a sum is enough.  The order of additions depends on the thread alone.
__device__ __forceinline__ int halves(int warps) { return 1 << (31 - __clz(warps - 1)); }   // half of the power of two that holds 2 to 16 warps
struct RowSum {
    float* red;
    int turn;
    __device__ __forceinline__ float operator()(float a) {
#pragma unroll
        for (int d = 16; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
        const int n = blockDim.x >> 5, lane = threadIdx.x & 31;
        if (n == 1) return a;
        float* at = red + turn * 16;
        turn ^= 1;
        if (lane == 0) at[threadIdx.x >> 5] = a;
        __syncthreads();
        const int h = halves(n), k = lane & (2 * h - 1);
        a = k < n ? at[k] : 0.f;
        for (int d = h; d; d >>= 1) a += __shfl_xor_sync(0xffffffffu, a, d);
        return a;
    }
};
// N such sums at once; `red`: two sets of 16 N floats
template <int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* red, int& turn) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int d = 16; d; d >>= 1) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    const int n = blockDim.x >> 5, lane = threadIdx.x & 31;
    if (n == 1) return;
    float* at = red + turn * 16 * N;
    turn ^= 1;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) at[(threadIdx.x >> 5) * N + i] = v[i];
    }
    __syncthreads();
    const int h = halves(n), k = lane & (2 * h - 1);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = k < n ? at[k * N + i] : 0.f;
    for (int d = h; d; d >>= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], d);
    }
}

// ---- dropout ----
// Philox 4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; SC 2011).
// A round: (x, y, z, w) -> (hi(z M1) ^ y ^ k0, lo(z M1), hi(x M0) ^ w ^ k1, lo(x M0)); the keys grow by a constant each.
struct Rounds { uint4 k[5]; };                                       // the keys of two rounds each
__device__ __forceinline__ void philox_keys(Rounds& r, int i, unsigned k0, unsigned k1) {   // those of rounds 2 i and 2 i + 1
    k0 += 0x9E3779B9u * (2 * i);
    k1 += 0xBB67AE85u * (2 * i);
    r.k[i] = make_uint4(k0, k1, k0 + 0x9E3779B9u, k1 + 0xBB67AE85u);
}
__device__ __forceinline__ uint4 philox(uint4 c, const Rounds& r) {
#pragma unroll
    for (int i = 0; i < 5; ++i) {
        const uint4 k = r.k[i];
        unsigned long long p0 = (unsigned long long)c.x * 0xD2511F53u, p1 = (unsigned long long)c.z * 0xCD9E8D57u;
        c = make_uint4((unsigned)(p1 >> 32) ^ c.y ^ k.x, (unsigned)p1, (unsigned)(p0 >> 32) ^ c.w ^ k.y, (unsigned)p0);
        p0 = (unsigned long long)c.x * 0xD2511F53u;
        p1 = (unsigned long long)c.z * 0xCD9E8D57u;
        c = make_uint4((unsigned)(p1 >> 32) ^ c.y ^ k.z, (unsigned)p1, (unsigned)(p0 >> 32) ^ c.w ^ k.w, (unsigned)p0);
    }
    return c;
}
// One call gives the eight columns 8 i .. 8 i + 7 of a row 16 bits each, lowest first; a column stays where its bits are at
// least `cut`.
struct Drop {
    const unsigned long long* rng;           // key, step
    unsigned cut, site;
    float factor;
    int64_t row0;
};
// What a kernel makes of it: the rounds' keys wait in shared memory, where a call fetches them two rounds at a time (an addition
// less per key than making them anew).
struct Dropping {
    const Rounds* keys;
    unsigned long long step;
    int64_t row0;
    unsigned cut, site;
    // the whole block takes part
    __device__ __forceinline__ Dropping(const Drop& d, Rounds& shared) : keys(&shared), step(0), row0(d.row0), cut(d.cut), site(d.site << 8) {
        if (!cut) return;
        const unsigned long long key = d.rng[0];
        step = d.rng[1];
        if (threadIdx.x < 5) philox_keys(shared, threadIdx.x, (unsigned)key, (unsigned)(key >> 32));
        __syncthreads();
    }
    __device__ __forceinline__ uint4 bits(unsigned long long group) const {
        return philox(make_uint4((unsigned)group, (unsigned)(group >> 32) | site, (unsigned)step, (unsigned)(step >> 32)), *keys);
    }
    // the number of a row's first group
    __device__ __forceinline__ unsigned long long first_of(int64_t row, int cols) const { return (unsigned long long)(row0 + row) * (unsigned)((cols + 7) / 8); }
    // v's columns of group g of the row whose first group of eight is number `first`: those that do not stay become 0.  Whole warps, which hold columns of one row.
    template <typename T, bool VEC> __device__ __forceinline__ void operator()(unsigned long long first, int t, int threads, int g, F2 (&v)[P<T>]) const {
        const unsigned high = cut << 16;                             
        if (cut >> 16) {
#pragma unroll
            for (int j = 0; j < P<T>; ++j) v[j] = 0ull;
            return;
        }
        if constexpr (VEC) {
            const int c = column<T, true>(t, threads, g, 0);
            const uint4 r = bits(first + (unsigned)(c >> 3));
            unsigned w[4] = {r.x, r.y, r.z, r.w};
            if (V<T> == 4 && (c & 4)) { w[0] = r.z; w[1] = r.w; }
#pragma unroll
            for (int j = 0; j < P<T>; ++j) {
                const float2 p = parts(v[j]);
                v[j] = f2((w[j] << 16) >= high ? p.x : 0.f, w[j] >= high ? p.y : 0.f);
            }
        } else {
            // the warp's columns are V runs of 32, four groups of eight each: a lane makes one of these 4 V groups
            const int l = t & 31, base = t - l, lj = (l >> 2) & (V<T> - 1);
            const uint4 r = bits(first + (unsigned)(((g * V<T> + lj) * threads + base) >> 3) + (l & 3));
            const unsigned w[4] = {r.x, r.y, r.z, r.w};
            unsigned mine = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) mine |= ((w[i] << 16) >= high ? 1u : 0u) << (2 * i) | (w[i] >= high ? 2u : 0u) << (2 * i);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) {
                const unsigned a = __shfl_sync(0xffffffffu, mine, 8 * j + (l >> 3)), b = __shfl_sync(0xffffffffu, mine, 8 * j + 4 + (l >> 3));
                const float2 p = parts(v[j]);
                v[j] = f2(a >> (l & 7) & 1 ? p.x : 0.f, b >> (l & 7) & 1 ? p.y : 0.f);
            }
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

// threads of a row (whole warps, 512 at most) and groups per thread (a power of two, `most` at most while that needs no more than 512 threads)
inline void row_shape(int cols, int v, int most, int* threads, int* groups) {
    int t = 32;
    while (t < 512 && (int64_t)t * v * most < cols) t *= 2;
    *groups = 1;
    while ((int64_t)t * v * *groups < cols) *groups *= 2;
    *threads = ((cols + v * *groups - 1) / (v * *groups) + 31) / 32 * 32;
}

}  // namespace token
}  // namespace ftp
