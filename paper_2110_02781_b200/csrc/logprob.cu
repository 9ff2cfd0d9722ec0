// Log probabilities of given tokens under rows of logits, the rows' entropies and their likeliest tokens; and the logits' gradient.
//
// Bound by memory: the forward pass reads every logit once, the backward pass reads them once more and writes the gradient.
// Forward: a block per row, a cluster of up to eight where there are few rows, a warp where they are many and short; a thread keeps the largest of its
// logits, m, and with it sum e^(z - m) and sum e^(z - m) (z - m), from which the entropy is log sum - (second / first).  The sums are rescaled only where
// four groups of 16 bytes hold a new largest logit.  Rows that do not start on 16 bytes are read from the boundary before them, the two partial groups
// element by element.
// The k likeliest tokens come from the same pass: every warp gives its 32 / warps largest thread maxima, the k-th largest of these 32 is a bound that k
// logits of the row reach, and only the groups of threads whose maximum reaches it are looked at again (about k of up to 512 threads; in registers where a
// thread has no more than four).  What reaches the bound is ranked by (value, lowest token).
// 4096 x 50021 bf16 with entropies: 73-83 us (5.0-5.6 TB/s; the exponentials use two thirds of their pipe); 16 x 128000 with 20 top tokens: 9.1 us, a
// chain of eight exchanges between threads, warps and blocks; 16000 x 12000 with a warp a row 64 us (6.0 TB/s); backward, 8192 x 32000: 182-191 us (5.5-5.8 TB/s).
#include <algorithm>
#include <type_traits>
#include "token.cuh"

namespace ftp {
namespace token {
namespace {

constexpr int MOST_THREADS = 512, MOST_TOP = 32, CAND = 2048, ROWS = 4, ROWS_CAND = 512;
constexpr float LOW = -1e4f;                                         // stands for the logarithm of 0 where it meets a factor 0

struct LogpArgs {
    const void* x;
    const int32_t* target;
    float *logp, *entropy, *lse, *top_logp;
    int32_t* top;
    int64_t rows, ld;
    int vocab, k, room;                                              // room: candidates that fit into shared memory
    float scale, scale2, near;                                       // scale2: scale * log2(e); near: see near_of
};

// a float's place in the order of floats (NaN above infinity)
__device__ __forceinline__ unsigned order_of(float v) {
    const unsigned u = __float_as_uint(v + 0.f);                     // -0 counts as 0
    return v != v ? ~0u : u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float from_order(unsigned u) { return __uint_as_float(u >> 31 ? u & 0x7fffffffu : ~u); }
typedef unsigned long long Key;
__device__ __forceinline__ Key key_of(float v, int c) { return (Key)order_of(v) << 32 | (unsigned)~c; }

template <typename T> __device__ __forceinline__ float power(float t2) {   // 2^t2
    return sizeof(T) == 4 ? exp2f(t2) : ffn::ex2_fast(t2);
}

// A row seen in whole groups of 16 bytes: group i holds columns i V - off .. i V - off + V - 1
template <typename T> struct Row {
    const T* p;                                                      // at the boundary before the row
    int off, vocab, first, end, all;                                 // whole groups first .. end - 1 of `all`
    __device__ __forceinline__ Row(const void* x, int64_t row, int64_t ld, int n) {
        const T* at = static_cast<const T*>(x) + row * ld;
        off = (int)((reinterpret_cast<uintptr_t>(at) & 15) / sizeof(T));
        p = at - off;
        vocab = n;
        first = off ? 1 : 0;
        end = (int)(((int64_t)n + off) / V<T>);
        all = (int)(((int64_t)n + off + V<T> - 1) / V<T>);
    }
    __device__ __forceinline__ uint4 whole(int i) const { return reinterpret_cast<const uint4*>(p)[i]; }
    // any group; -infinity beyond the row
    __device__ __forceinline__ uint4 any(int i) const {
        if (i >= first && i < end) return whole(i);
        unsigned w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int64_t c = (int64_t)i * V<T> + j - off;
            w[j * (int)sizeof(T) / 4] |= (c >= 0 && c < vocab ? bits_of(p[(int64_t)i * V<T> + j]) : sizeof(T) == 4 ? 0xff800000u : 0xff80u) << (sizeof(T) == 4 ? 0 : 16 * (j & 1));
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    __device__ __forceinline__ void values(int i, float (&v)[V<T>]) const { decode<T>(any(i), v); }
};

__device__ __forceinline__ unsigned max_bf2(unsigned a, unsigned b) { unsigned r; asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b)); return r; }   // NaN only if both are
// Logits far below any that counts are raised to this, so that their distance to the largest stays finite where it meets the factor 0.  That holds while
// the largest lies between FAR / 10 and `near_of`; other rows clamp the distances one by one.
constexpr float FAR = -1e18f;
inline float near_of(float scale2) { return (float)std::min(3.4e38, 3e38 / scale2 + FAR); }
template <typename T> __device__ __forceinline__ uint4 raised(uint4 q) {   // a NaN stays one
    if constexpr (sizeof(T) == 2)
        asm("max.NaN.bf16x2 %0, %0, %4;\nmax.NaN.bf16x2 %1, %1, %4;\nmax.NaN.bf16x2 %2, %2, %4;\nmax.NaN.bf16x2 %3, %3, %4;"
            : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w) : "r"(bf_pack(FAR, FAR)));
    else
        asm("{\n.reg .f32 f;\nmov.b32 f, %4;\n.reg .f32 a, b, c, d;\nmov.b32 a, %0;\nmov.b32 b, %1;\nmov.b32 c, %2;\nmov.b32 d, %3;\n"
            "max.NaN.f32 a, a, f;\nmax.NaN.f32 b, b, f;\nmax.NaN.f32 c, c, f;\nmax.NaN.f32 d, d, f;\nmov.b32 %0, a;\nmov.b32 %1, b;\nmov.b32 %2, c;\nmov.b32 %3, d;\n}"
            : "+r"(q.x), "+r"(q.y), "+r"(q.z), "+r"(q.w) : "r"(__float_as_uint(FAR)));
    return q;
}
template <typename T> __device__ __forceinline__ uint4 nothing() {         // a group of -infinity
    const unsigned w = sizeof(T) == 4 ? 0xff800000u : 0xff80ff80u;
    return make_uint4(w, w, w, w);
}
// the largest of a group; with a NaN in it, that of the others
template <typename T> __device__ __forceinline__ float top_of(const uint4& q) {
    if constexpr (sizeof(T) == 4) return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
    else {
        const unsigned w = max_bf2(max_bf2(q.x, q.y), max_bf2(q.z, q.w));
        return fmaxf(bf_lo(w), bf_hi(w));
    }
}
template <typename T, bool ENTROPY> struct Sums {
    float m = -INFINITY, at = 0.f;                                   // at: m, or 0 while there is none
    F2 s0 = 0ull, s1 = 0ull;
    __device__ __forceinline__ void rescale(float to, float c2) {
        const float d = m == -INFINITY ? 0.f : (at - to) * c2;       // no logit so far: the sums are 0
        const F2 f = f2(power<T>(d));
        if (ENTROPY) s1 = mul2(f, fma2(f2(fmaxf(d, LOW)), s0, s1));
        s0 = mul2(s0, f);
        m = at = to;
    }
    // N groups of logits; what is not there is -infinity
    template <int N> __device__ __forceinline__ void add(const uint4 (&q)[N], float c2, float near) {
        float top;                                                   // the largest; with a NaN among them, that of the others
        if constexpr (sizeof(T) == 2) {
            unsigned w = max_bf2(max_bf2(q[0].x, q[0].y), max_bf2(q[0].z, q[0].w));
#pragma unroll
            for (int u = 1; u < N; ++u) w = max_bf2(w, max_bf2(max_bf2(q[u].x, q[u].y), max_bf2(q[u].z, q[u].w)));
            top = fmaxf(bf_lo(w), bf_hi(w));
        } else {
            top = __uint_as_float(q[0].x);
#pragma unroll
            for (int u = 0; u < N; ++u)
                top = fmaxf(fmaxf(top, __uint_as_float(q[u].x)), fmaxf(__uint_as_float(q[u].y), fmaxf(__uint_as_float(q[u].z), __uint_as_float(q[u].w))));
        }
        if (top > m) rescale(top, c2);
        const F2 less = f2(-at), c = f2(c2);
        if (!ENTROPY || (at > 0.1f * FAR && at < near)) {
#pragma unroll
            for (int u = 0; u < N; ++u) {
                F2 v[P<T>];
                decode<T>(ENTROPY ? raised<T>(q[u]) : q[u], v);
#pragma unroll
                for (int j = 0; j < P<T>; ++j) {
                    const F2 t = mul2(add2(v[j], less), c);
                    const float2 p = parts(t);
                    const F2 e = f2(power<T>(p.x), power<T>(p.y));
                    s0 = add2(s0, e);
                    if (ENTROPY) s1 = fma2(e, t, s1);
                }
            }
        } else                                                       // even the largest logit is that far down, or it is that large
            for (int u = 0; u < N; ++u) {
                F2 v[P<T>];
                decode<T>(q[u], v);
#pragma unroll
                for (int j = 0; j < P<T>; ++j) {
                    const float2 p = parts(mul2(add2(v[j], less), c));
                    const F2 e = f2(power<T>(p.x), power<T>(p.y));
                    s0 = add2(s0, e);
                    s1 = fma2(e, f2(fmaxf(p.x, LOW), fmaxf(p.y, LOW)), s1);
                }
            }
    }
};

// The 32 largest of two lists of 32 distinct keys (or 0), each in descending order along a warp, in descending order: the larger of
// each pair from both ends, which rise and fall once, then sorted by halves.
__device__ __forceinline__ Key merge(Key a, Key b) {
    const int lane = threadIdx.x & 31;
    b = __shfl_sync(0xffffffffu, b, 31 - lane);
    a = a > b ? a : b;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const Key o = __shfl_xor_sync(0xffffffffu, a, d);
        a = (a > o) == ((lane & d) == 0) ? a : o;
    }
    return a;
}

// What the threads of a row share
template <bool TOP, bool WARP> struct Shared {
    float red[3][16], part[3], total[3];
    unsigned bound[32];
    Key best[MOST_TOP], joined[WARP ? 1 : 4][MOST_TOP];
    int hit[TOP ? (WARP ? 32 : MOST_THREADS) : 1], hits, found;
};

// WARP: a row to a warp instead of a block or a cluster
template <typename T, bool ENTROPY, bool TOP, bool WARP>
__device__ __forceinline__ void logprob_row(const LogpArgs& a, int64_t row, unsigned ranks, unsigned rank) {
    extern __shared__ Key candidates[];
    __shared__ Shared<TOP, WARP> shared[WARP ? ROWS : 1];
    const int threads = WARP ? 32 : blockDim.x, tid = WARP ? threadIdx.x & 31 : threadIdx.x, lane = tid & 31, w = tid >> 5, warps = threads >> 5;
    const int mine_at = WARP ? threadIdx.x >> 5 : 0;
    Shared<TOP, WARP>& sh = shared[mine_at];
    Key* const cand = candidates + mine_at * a.room;
    const auto sync = [] { if constexpr (WARP) __syncwarp(); else __syncthreads(); };
    const Row<T> x(a.x, row, a.ld, a.vocab);
    const int me = (int)rank * threads + tid, stride = (int)ranks * threads;
    Sums<T, ENTROPY> s;
    // the given token's logit, on its way meanwhile
    int target = -1;
    float given = 0.f;
    if (me == 0 && a.logp) {
        target = a.target[row];
        if (target >= 0 && target < a.vocab) given = (float)x.p[x.off + (int64_t)target];
    }
    // The first groups of a thread stay in registers: with no more than these, nothing is read again for the likeliest tokens.
    uint4 held[4];
    // four groups in flight; the partial groups at both ends go to the first and the last thread
    const bool head = me == 0 && x.first == 1, tail = me == stride - 1 && x.end < x.all && x.all - 1 >= x.first;
#pragma unroll
    for (int u = 0; u < 4; ++u) held[u] = x.first + me + u * stride < x.end ? x.whole(x.first + me + u * stride) : nothing<T>();
    int i = x.first + me + 4 * stride;
    if constexpr (TOP) {
        s.add(held, a.scale2, a.near);
        for (; i + 3 * stride < x.end; i += 4 * stride) {
            uint4 q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u] = x.whole(i + u * stride);
            s.add(q, a.scale2, a.near);
        }
    } else {                                                         // the next four are on their way meanwhile
        for (; i + 3 * stride < x.end; i += 4 * stride) {
            uint4 q[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) q[u] = x.whole(i + u * stride);
            s.add(held, a.scale2, a.near);
#pragma unroll
            for (int u = 0; u < 4; ++u) held[u] = q[u];
        }
        s.add(held, a.scale2, a.near);
    }
    if (i < x.end) {
        uint4 q[4];
        q[3] = nothing<T>();
#pragma unroll
        for (int u = 0; u < 3; ++u) q[u] = i + u * stride < x.end ? x.whole(i + u * stride) : nothing<T>();
        s.add(q, a.scale2, a.near);
    }
    if (head || tail) {
        const uint4 ends[2] = {head ? x.any(0) : nothing<T>(), tail ? x.any(x.all - 1) : nothing<T>()};
        s.add(ends, a.scale2, a.near);
    }
    const float mine = s.m;
    // the block's sums
    float m = s.m;
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (!WARP && lane == 0) sh.red[0][w] = m;
    if (TOP && tid == 0) sh.hits = sh.found = 0;
    if (TOP && tid < MOST_TOP) sh.best[tid] = 0;
    if constexpr (!WARP) {
        __syncthreads();
        m = sh.red[0][lane & (warps - 1)];
        for (int d = warps >> 1; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    }
    if (m > s.m) s.rescale(m, a.scale2);
    float s0 = sum2(s.s0), s1 = sum2(s.s1);
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        s0 += __shfl_xor_sync(0xffffffffu, s0, d);
        s1 += __shfl_xor_sync(0xffffffffu, s1, d);
    }
    if (!WARP && lane == 0) { sh.red[1][w] = s0; sh.red[2][w] = s1; }
    if constexpr (TOP) {
        // the warp's largest thread maxima
        unsigned o = order_of(mine);
        const int each = 32 / warps;
        if (warps == 1) sh.bound[lane] = o;
        else for (int k = 0; k < each; ++k) {
            const unsigned top = __reduce_max_sync(0xffffffffu, o);
            const unsigned who = __ballot_sync(0xffffffffu, o == top);
            if (lane == __ffs(who) - 1) o = 0;
            if (lane == 0) sh.bound[w * each + k] = top;
        }
    }
    if (TOP || !WARP) sync();
    if (!WARP && w == 0) {
        s0 = sh.red[1][lane & (warps - 1)]; s1 = sh.red[2][lane & (warps - 1)];
        for (int d = warps >> 1; d; d >>= 1) { s0 += __shfl_xor_sync(0xffffffffu, s0, d); s1 += __shfl_xor_sync(0xffffffffu, s1, d); }
        if (lane == 0) { sh.part[0] = m; sh.part[1] = s0; sh.part[2] = s1; }
    }
    if constexpr (TOP) {
        const unsigned b = sh.bound[lane];
        int above = 0;                                               // places are distinct: ties by lane
#pragma unroll
        for (int k = 0; k < 32; ++k) { const unsigned o = __shfl_sync(0xffffffffu, b, k); above += o > b || (o == b && k < lane); }
        const unsigned kth = __shfl_sync(0xffffffffu, b, __ffs(__ballot_sync(0xffffffffu, above == a.k - 1)) - 1);
        const float least = from_order(kth);                         // comparisons let a NaN pass
        const auto offer = [&](int g, const uint4& q) {
            if (top_of<T>(q) < least) return;
            float v[V<T>];
            decode<T>(q, v);
#pragma unroll
            for (int j = 0; j < V<T>; ++j) {
                if (v[j] < least) continue;
                const int c = g * V<T> + j - x.off;
                if (c < 0 || c >= a.vocab) continue;
                const int at = atomicAdd(&sh.found, 1);
                if (at < a.room) cand[at] = key_of(v[j], c);
            }
        };
        if (x.first + 4 * stride >= x.end) {
            if (order_of(mine) >= kth) {
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (x.first + me + u * stride < x.end) offer(x.first + me + u * stride, held[u]);
                if (head) offer(0, x.any(0));
                if (tail) offer(x.all - 1, x.any(x.all - 1));
            }
        } else {
            if (order_of(mine) >= kth) sh.hit[atomicAdd(&sh.hits, 1)] = tid;
            sync();
            for (int h = w; h < sh.hits; h += warps) {               // a thread's groups read again by a warp
                const int owner = (int)rank * threads + sh.hit[h];
                for (int g = x.first + owner + lane * stride; g < x.end; g += 32 * stride) offer(g, x.whole(g));
                if (lane == 0 && owner == 0 && x.first == 1) offer(0, x.any(0));
                if (lane == 0 && owner == stride - 1 && x.end < x.all && x.all - 1 >= x.first) offer(x.all - 1, x.any(x.all - 1));
            }
        }
        sync();
        const int n = sh.found;
        if (n <= a.room) {                                             // how many are larger: a warp per candidate
            for (int k = w; k < n; k += warps) {
                const Key mykey = cand[k];
                int rnk = 0;
                for (int q = lane; q - lane < n; q += 32) rnk += __popc(__ballot_sync(0xffffffffu, q < n && cand[q] > mykey));
                if (lane == 0 && rnk < a.k) sh.best[rnk] = mykey;
            }
        } else {                                                     // too many equal ones: one after another, over the whole part of the row
            Key last = ~0ull;
            for (int k = 0; k < a.k; ++k) {
                Key top = 0;
                const auto look = [&](int g) {
                    float v[V<T>];
                    x.values(g, v);
#pragma unroll
                    for (int j = 0; j < V<T>; ++j) {
                        const int c = g * V<T> + j - x.off;
                        if (c >= 0 && c < a.vocab) { const Key q = key_of(v[j], c); if (q < last && q > top) top = q; }
                    }
                };
                for (int g = x.first + me; g < x.end; g += stride) look(g);
                if (me == 0 && x.first == 1) look(0);
                if (me == stride - 1 && x.end < x.all && x.all - 1 >= x.first) look(x.all - 1);
                sync();                                              // cand: the warps' largest
#pragma unroll
                for (int d = 16; d; d >>= 1) { const Key q = __shfl_xor_sync(0xffffffffu, top, d); top = q > top ? q : top; }
                if (lane == 0) cand[w] = top;
                sync();
                for (int q = 0; q < warps; ++q) top = cand[q] > top ? cand[q] : top;
                if (tid == 0) sh.best[k] = top;
                last = top;
            }
        }
    }
    if (ranks > 1) cluster_sync(); else if (TOP || !WARP) sync();
    if (rank == 0) {
        if (ranks > 1) {
            if (w == 0) {                                            // a lane per block
                const unsigned from = on_rank(smem_at(sh.part), min((unsigned)lane, ranks - 1));
                float pm, p0, p1;
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(pm) : "r"(from) : "memory");
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p0) : "r"(from + 4) : "memory");
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p1) : "r"(from + 8) : "memory");
                float top = pm;
#pragma unroll
                for (int d = 4; d; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                if (pm != -INFINITY) {                               // else p0 is 0, or NaN
                    const float d = (pm - top) * a.scale2, f = power<T>(d);
                    p1 = f * fmaf(fmaxf(d, LOW), p0, p1);
                    p0 *= f;
                }
                if (lane >= (int)ranks) p0 = p1 = 0.f;
#pragma unroll
                for (int d = 4; d; d >>= 1) { p0 += __shfl_xor_sync(0xffffffffu, p0, d); p1 += __shfl_xor_sync(0xffffffffu, p1, d); }
                if (lane == 0) { sh.total[0] = top; sh.total[1] = p0; sh.total[2] = p1; }
            }
            if (TOP && w < (int)ranks / 2) {                         // a warp for two blocks' tokens
                Key two[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(two[i]) : "r"(on_rank(smem_at(sh.best + lane), (unsigned)(2 * w + i))) : "memory");
                sh.joined[w][lane] = merge(two[0], two[1]);
            }
            sync();
        }
        const float* const all = ranks > 1 ? sh.total : sh.part;
        const float top = WARP ? m : all[0], all0 = WARP ? s0 : all[1], all1 = WARP ? s1 : all[2];
        const float log_sum = logf(all0);
        const bool none = all0 == 0.f;                               // no token can occur
        if (tid == 0) {
            if (a.logp) a.logp[row] = target < 0 || target >= a.vocab ? 0.f : none ? -INFINITY : a.scale * (given - top) - log_sum;
            if (a.lse) { a.lse[2 * row] = top; a.lse[2 * row + 1] = log_sum; }
            if (ENTROPY) a.entropy[row] = none ? 0.f : log_sum - all1 / all0 * 0.69314718055994531f;
        }
        if constexpr (TOP) {
            const auto give = [&](int place, Key q) {
                a.top[row * a.k + place] = (int32_t)~(unsigned)q;
                if (a.top_logp) a.top_logp[row * a.k + place] = none ? -INFINITY : a.scale * (from_order((unsigned)(q >> 32)) - top) - log_sum;
            };
            if (w == 0) {
                Key q = ranks > 1 ? sh.joined[0][lane] : sh.best[lane];
                if (ranks > 2) q = merge(q, sh.joined[1][lane]);
                if (ranks > 4) q = merge(q, merge(sh.joined[2][lane], sh.joined[3][lane]));
                if (lane < a.k) give(lane, q);
            }
        }
    }
    if (ranks > 1) cluster_sync();                                   // nobody leaves while the first block reads its shared memory
}

// (A block that walks over several rows is slower, 85 instead of 78 us for 16000 x 120 bf16: nothing hides the end of a row.)
template <typename T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(MOST_THREADS, 2) logprob_forward_kernel(const LogpArgs a) {
    grid_dep_sync();
    unsigned ranks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    logprob_row<T, ENTROPY, TOP, false>(a, blockIdx.x / ranks, ranks, cluster_rank());
}
// Short rows, a warp each
template <typename T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(32 * ROWS, 8) logprob_rows_kernel(const LogpArgs a) {
    grid_dep_sync();
    const int64_t row = (int64_t)blockIdx.x * ROWS + (threadIdx.x >> 5);
    if (row < a.rows) logprob_row<T, ENTROPY, TOP, true>(a, row, 1, 0);
}

struct LogpBack {
    const void* x;
    void* dx;
    const int32_t* target;
    const float *lse, *entropy, *dlogp, *dentropy;
    int64_t rows, ld, ldd;
    int vocab;
    float scale;
};

// d = scale (dlogp (1 at the target - p) - dentropy p (log p + H)).  A warp takes 128 groups of 16 bytes of a row, four to a lane.
template <typename T, bool ENTROPY>
__global__ void __launch_bounds__(256) logprob_backward_kernel(const LogpBack a) {
    grid_dep_sync();
    const int lane = threadIdx.x & 31;
    const int64_t per_row = ((int64_t)a.vocab + 2 * V<T> - 2) / V<T> / 128 + 1, total = a.rows * per_row;      // whatever the row's offset
    for (int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); n < total; n += (int64_t)gridDim.x * 8) {
        const int64_t row = n / per_row;
        const Row<T> x(a.x, row, a.ld, a.vocab);
        T* out = static_cast<T*>(a.dx) + row * a.ldd - x.off;
        const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
        const int g0 = (int)(n - row * per_row) * 128 + lane;
        uint4 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int g = g0 + 32 * u;
            q[u] = g >= x.first && g < x.end ? x.whole(g) : nothing<T>();
        }
        const int t = a.target ? a.target[row] : -1;
        const float m = a.lse[2 * row], log_sum = a.lse[2 * row + 1];
        const bool none = m == -INFINITY && log_sum == -INFINITY, given = t >= 0 && t < a.vocab && !none;
        const float dl = given && a.dlogp ? a.dlogp[row] * a.scale : 0.f, dh = ENTROPY ? a.dentropy[row] * a.scale : 0.f;
        // log probabilities of raised logits, and dentropy times them, stay finite: elsewhere what meets the factor 0 is left out
        const bool near = m > 0.1f * FAR && (m - FAR) * a.scale * fmaxf(1.f, fabsf(dh)) < 1e38f;
        const float plus = ENTROPY ? -fmaf(dh, a.entropy[row], dl) : -dl;
        const F2 less = f2(-m), c = f2(a.scale), sum = f2(-log_sum), b = f2(-dh), k = f2(plus);
        const int at = given ? (t + x.off) / V<T> : -1, j_at = given ? (t + x.off) % V<T> : 0;     // the target's group, and its place in it
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int g = g0 + 32 * u;
            if (g >= x.all) break;
            const bool whole = g >= x.first && g < x.end;
            if (!whole) q[u] = x.any(g);
            F2 v[P<T>];
            const auto gradient = [&](auto far) {
                decode<T>(ENTROPY && !far.value ? raised<T>(q[u]) : q[u], v);
#pragma unroll
                for (int j = 0; j < P<T>; ++j) {
                    const F2 lp = fma2(add2(v[j], less), c, sum);
                    const float2 l = parts(lp);
                    F2 p;
                    if (sizeof(T) == 4) p = f2(expf(l.x), expf(l.y));
                    else {
                        const float2 z = parts(mul2(lp, f2(ffn::LOG2E)));
                        p = f2(ffn::ex2_fast(z.x), ffn::ex2_fast(z.y));
                    }
                    v[j] = mul2(p, ENTROPY ? fma2(b, lp, k) : k);
                    if (far.value) {
                        const float2 e = parts(p), d = parts(v[j]);
                        v[j] = f2(e.x == 0.f ? 0.f : d.x, e.y == 0.f ? 0.f : d.y);
                    }
                }
            };
            if (!ENTROPY || near) gradient(std::false_type{}); else gradient(std::true_type{});
            if (none)
#pragma unroll
                for (int j = 0; j < P<T>; ++j) v[j] = 0ull;
            if (g == at)
#pragma unroll
                for (int j = 0; j < P<T>; ++j) {
                    if (j_at == 2 * j) v[j] = add2(v[j], f2(dl, 0.f));
                    if (j_at == 2 * j + 1) v[j] = add2(v[j], f2(0.f, dl));
                }
            const uint4 r = encode<T>(v);
            if (whole && same) reinterpret_cast<uint4*>(out)[g] = r;
            else {
                const unsigned w[4] = {r.x, r.y, r.z, r.w};
                const int64_t c0 = (int64_t)g * V<T> - x.off;
#pragma unroll
                for (int j = 0; j < V<T>; ++j)
                    if (c0 + j >= 0 && c0 + j < a.vocab) from_bits(out + (int64_t)g * V<T> + j, w[j * (int)sizeof(T) / 4] >> (sizeof(T) == 4 ? 0 : 16 * (j & 1)));
            }
        }
    }
}

ftp_status check(const void* logits, int64_t rows, int32_t vocab, int64_t* ld, int32_t precision, float scale, const char* who) {
    FTP_REQUIRE(precision == FTP_FP32 || precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, precision);
    FTP_REQUIRE(rows >= 0 && vocab >= 1, FTP_EINVAL, "%s: rows must not be negative, vocab must be positive", who);
    FTP_REQUIRE(rows < (1ll << 28) && vocab < (1 << 30), FTP_ERANGE, "%s: tensor too large", who);
    FTP_REQUIRE(scale > 0.f && scale <= 1e18f, FTP_EINVAL, "%s: scale must be positive, 1e18 at most", who);
    if (ftp_status s = check_pitches({*ld}, vocab, who)) return s;
    if (!*ld) *ld = vocab;
    FTP_REQUIRE(rows == 0 || logits, FTP_EINVAL, "%s: null buffer", who);
    return check_elements({logits}, precision == FTP_FP32 ? 4 : 2, who);
}

template <typename T> cudaError_t forward_of(LogpArgs& a, cudaStream_t st) {
    // Few rows: four groups and more to a thread.  Otherwise a warp a row while that leaves enough warps (16000 x 20001 bf16: 104 us, 145 with 64 threads,
    // 116 with 128; but 1500 x 20001: 29, 21, 16), and 128 threads above (8000 x 32000: 94, 102, 85 us; 4096 x 50021: 79, 85, 71, 101 with 512), or more while
    // these do not fill the GPU (800 x 50000: 23 us with 128 threads, 19 with 256).  The choice does not depend on k, so that the log probabilities do not.
    const int groups = (a.vocab + V<T> - 1) / V<T>;
    int threads = 32, ranks = 1;
    if (a.rows < SMS) while (threads < MOST_THREADS && threads * 4 < groups) threads *= 2;
    else if (groups > (a.rows >= SMS * 64 ? 3200 : a.rows >= SMS * 16 ? 1600 : 128)) {
        threads = 128;
        while (threads < MOST_THREADS && a.rows * threads < SMS * 1024 && threads * 32 < groups) threads *= 2;
    }
    while (ranks < 8 && a.rows * ranks * 2 <= 2 * SMS && ranks * 2 * threads * 2 <= groups) ranks *= 2;
    // Rows of one warp: four to a block, because a multiprocessor starts a block every 0.27 us (8192 x 192 bf16: 16 us with a block a row, 4.6 here).
    if (threads == 32 && ranks == 1 && a.rows >= SMS * ROWS) {
        a.room = std::min(a.room, ROWS_CAND);
        auto kern = a.k ? (a.entropy ? logprob_rows_kernel<T, true, true> : logprob_rows_kernel<T, false, true>)
                        : (a.entropy ? logprob_rows_kernel<T, true, false> : logprob_rows_kernel<T, false, false>);
        launch(kern, dim3((unsigned)((a.rows + ROWS - 1) / ROWS)), dim3(32 * ROWS), a.k ? ROWS * a.room * sizeof(Key) : 0, st, a);
        return cudaSuccess;
    }
    auto kern = a.k ? (a.entropy ? logprob_forward_kernel<T, true, true> : logprob_forward_kernel<T, false, true>)
                    : (a.entropy ? logprob_forward_kernel<T, true, false> : logprob_forward_kernel<T, false, false>);
    return launch_cluster(kern, dim3((unsigned)(a.rows * ranks)), threads, a.k ? a.room * sizeof(Key) : 0, ranks, st, a);
}

}  // namespace
}  // namespace token
}  // namespace ftp

using namespace ftp;
using namespace ftp::token;

extern "C" {

ftp_status ftp_logprob_forward(const void* logits, int64_t rows, int32_t vocab, int64_t ldl, int32_t precision, float scale, const int32_t* targets, float* logp,
                               float* entropy, float* lse, int32_t* top, float* top_logp, int32_t k, void* stream) {
    const char* who = "logprob_forward";
    if (ftp_status s = check(logits, rows, vocab, &ldl, precision, scale, who)) return s;
    FTP_REQUIRE(k >= 0 && k <= MOST_TOP && k <= vocab, FTP_EINVAL, "%s: k must be in 0..%d and at most vocab", who, MOST_TOP);
    FTP_REQUIRE(rows == 0 || ((top != nullptr) == (k > 0) && (k > 0 || !top_logp)), FTP_EINVAL, "%s: k and the places for the top tokens disagree", who);
    FTP_REQUIRE(rows == 0 || !logp || targets, FTP_EINVAL, "%s: log probabilities of no tokens", who);
    if (ftp_status s = check_elements({targets, logp, entropy, lse, top, top_logp}, 4, who)) return s;
    if (ftp_status s = check_addresses({logp, entropy, lse, top, top_logp}, {logits, targets}, who)) return s;
    if (rows == 0) return FTP_OK;
    LogpArgs a{logits, targets, logp, entropy, lse, top_logp, top, rows, ldl, vocab, k, std::max(32, std::min(CAND, vocab)), scale, scale * 1.44269504088896341f, near_of(scale * 1.44269504088896341f)};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = precision == FTP_FP32 ? forward_of<float>(a, st) : forward_of<bf16>(a, st);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return launched(who);
}

ftp_status ftp_logprob_backward(const void* logits, int64_t rows, int32_t vocab, int64_t ldl, int32_t precision, float scale, const int32_t* targets, const float* lse,
                                const float* entropy, const float* dlogp, const float* dentropy, void* dlogits, int64_t ldd, void* stream) {
    const char* who = "logprob_backward";
    if (ftp_status s = check(logits, rows, vocab, &ldl, precision, scale, who)) return s;
    if (ftp_status s = check_pitches({ldd}, vocab, who)) return s;
    if (!ldd) ldd = vocab;
    FTP_REQUIRE(rows == 0 || (lse && dlogits && (dlogp || dentropy)), FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(rows == 0 || ((!dlogp || targets) && (!dentropy || entropy)), FTP_EINVAL, "%s: a gradient without its targets or entropies", who);
    if (ftp_status s = check_elements({dlogits}, precision == FTP_FP32 ? 4 : 2, who)) return s;
    if (ftp_status s = check_elements({targets, lse, entropy, dlogp, dentropy}, 4, who)) return s;
    if (ftp_status s = check_addresses({dlogits}, {targets, lse, entropy, dlogp, dentropy}, who)) return s;
    if (ftp_status s = check_in_place(logits, dlogits, ldl, ldd, rows, vocab, who)) return s;
    if (rows == 0) return FTP_OK;
    const LogpBack a{logits, dlogits, targets, lse, entropy, dlogp, dentropy, rows, ldl, ldd, vocab, scale};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int v = precision == FTP_FP32 ? 4 : 8;
    const int64_t pieces = rows * (((int64_t)vocab + 2 * v - 2) / v / 128 + 1);
    const dim3 grid((unsigned)std::min<int64_t>((pieces + 7) / 8, SMS * 64));
    if (precision == FTP_FP32) launch(dentropy ? logprob_backward_kernel<float, true> : logprob_backward_kernel<float, false>, grid, dim3(256), 0, st, a);
    else launch(dentropy ? logprob_backward_kernel<bf16, true> : logprob_backward_kernel<bf16, false>, grid, dim3(256), 0, st, a);
    return launched(who);
}

}  // extern "C"
