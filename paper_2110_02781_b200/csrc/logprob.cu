// Log probabilities of given tokens under rows of logits, the rows' entropies and their likeliest tokens; and the logits' gradient.
//
// Bound by memory: the forward pass reads every logit once, the backward pass reads them once more and writes the gradient.
// Forward: a block per row (a cluster of up to eight where there are few rows); a thread keeps the largest of its logits, m, and
// with it sum e^(z - m) and sum e^(z - m) (z - m), from which the entropy is log sum - (second / first).  The sums are rescaled
// only where a group of 16 bytes holds a new largest logit.  Rows that do not start on 16 bytes are read from the boundary before
// them, the two partial groups element by element.
// The k likeliest tokens come from the same pass: every warp gives its 32 / warps largest thread maxima, the k-th largest of
// these 32 is a bound that k logits of the row reach, and only the groups of threads whose maximum reaches it are read again (about k
// of up to 512 threads).  What reaches the bound is ranked by (value, lowest token) in shared memory.
#include <algorithm>
#include "token.cuh"

namespace ftp {
namespace token {
namespace {

constexpr int MOST_THREADS = 512, MOST_TOP = 32, CAND = 2048;
constexpr float LOW = -1e4f;                                         // stands for the logarithm of 0 where it meets a factor 0

struct LogpArgs {
    const void* x;
    const int32_t* target;
    float *logp, *entropy, *lse, *top_logp;
    int32_t* top;
    int64_t rows, ld;
    int vocab, k;
    float scale, scale2;                                             // scale2: scale * log2(e)
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
    __device__ __forceinline__ void values(int i, float (&v)[V<T>]) const {
        if (i >= first && i < end) { decode<T>(whole(i), v); return; }
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const int64_t c = (int64_t)i * V<T> + j - off;
            v[j] = c >= 0 && c < vocab ? (float)p[(int64_t)i * V<T> + j] : -INFINITY;
        }
    }
};

template <typename T, bool ENTROPY> struct Sums {
    float m = -INFINITY, at = 0.f, s0 = 0.f, s1 = 0.f;               // at: m, or 0 while there is none
    __device__ __forceinline__ void rescale(float to, float c2) {
        const float d = m == -INFINITY ? 0.f : (at - to) * c2, f = power<T>(d);                // no logit so far: the sums are 0
        if (ENTROPY) s1 = f * fmaf(fmaxf(d, LOW), s0, s1);
        s0 *= f;
        m = at = to;
    }
    __device__ __forceinline__ void add(const float (&v)[V<T>], float c2) {
        float top = v[0];
#pragma unroll
        for (int j = 1; j < V<T>; ++j) top = fmaxf(top, v[j]);
        if (top > m) rescale(top, c2);
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const float t = (v[j] - at) * c2, e = power<T>(t);
            s0 += e;
            if (ENTROPY) s1 = fmaf(e, fmaxf(t, LOW), s1);
        }
    }
};

template <typename T, bool ENTROPY, bool TOP>
__global__ void __launch_bounds__(MOST_THREADS, 2) logprob_forward_kernel(const LogpArgs a) {
    extern __shared__ Key cand[];                                    // TOP: CAND candidates
    __shared__ float red[3][16];
    __shared__ float part[3];
    __shared__ unsigned bound[32];
    __shared__ Key best[MOST_TOP], joined[8 * MOST_TOP];
    __shared__ int hit[MOST_THREADS], hits, found;
    grid_dep_sync();
    unsigned ranks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const unsigned rank = cluster_rank();
    const int threads = blockDim.x, tid = threadIdx.x, lane = tid & 31, w = tid >> 5, warps = threads >> 5;
    const int64_t row = blockIdx.x / ranks;
    const Row<T> x(a.x, row, a.ld, a.vocab);
    const int me = (int)rank * threads + tid, stride = (int)ranks * threads;
    Sums<T, ENTROPY> s;
    int i = x.first + me;
    for (; i + 3 * stride < x.end; i += 4 * stride) {
        uint4 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) q[u] = x.whole(i + u * stride);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            float v[V<T>];
            decode<T>(q[u], v);
            s.add(v, a.scale2);
        }
    }
    for (; i < x.end; i += stride) {
        float v[V<T>];
        decode<T>(x.whole(i), v);
        s.add(v, a.scale2);
    }
    // the partial groups at both ends go to the first threads
    if (me == 0 && x.first == 1) {
        float v[V<T>];
        x.values(0, v);
        s.add(v, a.scale2);
    }
    if (me == stride - 1 && x.end < x.all && x.all - 1 >= x.first) {
        float v[V<T>];
        x.values(x.all - 1, v);
        s.add(v, a.scale2);
    }
    const float mine = s.m;
    // the block's sums
    float m = s.m;
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    if (lane == 0) red[0][w] = m;
    if (TOP && tid == 0) { hits = 0; found = 0; }
    if (TOP && tid < MOST_TOP) best[tid] = 0;
    __syncthreads();
    m = red[0][0];
    for (int k = 1; k < warps; ++k) m = fmaxf(m, red[0][k]);
    if (m > s.m) s.rescale(m, a.scale2);
    float s0 = s.s0, s1 = s.s1;
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        s0 += __shfl_xor_sync(0xffffffffu, s0, d);
        s1 += __shfl_xor_sync(0xffffffffu, s1, d);
    }
    if (lane == 0) { red[1][w] = s0; red[2][w] = s1; }
    if constexpr (TOP) {
        // the warp's largest thread maxima
        unsigned o = order_of(mine);
        const int each = 32 / warps;
        for (int k = 0; k < each; ++k) {
            const unsigned top = __reduce_max_sync(0xffffffffu, o);
            const unsigned who = __ballot_sync(0xffffffffu, o == top);
            if (lane == __ffs(who) - 1) o = 0;
            if (lane == 0) bound[w * each + k] = top;
        }
    }
    __syncthreads();
    if (tid == 0) {
        s0 = red[1][0]; s1 = red[2][0];
        for (int k = 1; k < warps; ++k) { s0 += red[1][k]; s1 += red[2][k]; }
        part[0] = m; part[1] = s0; part[2] = s1;
    }
    if constexpr (TOP) {
        const unsigned b = bound[lane];
        int above = 0;                                               // places are distinct: ties by lane
#pragma unroll
        for (int k = 0; k < 32; ++k) { const unsigned o = __shfl_sync(0xffffffffu, b, k); above += o > b || (o == b && k < lane); }
        const unsigned kth = __shfl_sync(0xffffffffu, b, __ffs(__ballot_sync(0xffffffffu, above == a.k - 1)) - 1);
        if (order_of(mine) >= kth) hit[atomicAdd(&hits, 1)] = tid;
        __syncthreads();
        const auto offer = [&](int g) {
            float v[V<T>];
            x.values(g, v);
#pragma unroll
            for (int j = 0; j < V<T>; ++j) {
                const int c = g * V<T> + j - x.off;
                if (c >= 0 && c < a.vocab && order_of(v[j]) >= kth) {
                    const int at = atomicAdd(&found, 1);
                    if (at < CAND) cand[at] = key_of(v[j], c);
                }
            }
        };
        for (int h = w; h < hits; h += warps) {
            const int owner = (int)rank * threads + hit[h];
            for (int g = x.first + owner + lane * stride; g < x.end; g += 32 * stride) offer(g);
            if (lane == 0 && owner == 0 && x.first == 1) offer(0);
            if (lane == 0 && owner == stride - 1 && x.end < x.all && x.all - 1 >= x.first) offer(x.all - 1);
        }
        __syncthreads();
        const int n = found;
        if (n <= CAND) {
            for (int k = tid; k < n; k += threads) {
                const Key mykey = cand[k];
                int rnk = 0;
                for (int q = 0; q < n; ++q) rnk += cand[q] > mykey;
                if (rnk < a.k) best[rnk] = mykey;
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
                __syncthreads();                                     // cand: the warps' largest
#pragma unroll
                for (int d = 16; d; d >>= 1) { const Key q = __shfl_xor_sync(0xffffffffu, top, d); top = q > top ? q : top; }
                if (lane == 0) cand[w] = top;
                __syncthreads();
                for (int q = 0; q < warps; ++q) top = cand[q] > top ? cand[q] : top;
                if (tid == 0) best[k] = top;
                last = top;
            }
        }
    }
    if (ranks > 1) cluster_sync(); else __syncthreads();
    if (rank == 0 && (TOP || w == 0)) {
        float top = part[0], all0 = part[1], all1 = part[2];
        if (ranks > 1) {
            float pm[8], p0[8], p1[8];
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const unsigned from = on_rank(smem_at(part), min((unsigned)r, ranks - 1));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(pm[r]) : "r"(from) : "memory");
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p0[r]) : "r"(from + 4) : "memory");
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(p1[r]) : "r"(from + 8) : "memory");
            }
#pragma unroll
            for (int r = 1; r < 8; ++r) top = fmaxf(top, pm[r]);
            all0 = all1 = 0.f;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                if (r >= (int)ranks || pm[r] == -INFINITY) { if (r < (int)ranks) all0 += p0[r]; continue; }   // p0 is 0, or NaN
                const float d = (pm[r] - top) * a.scale2, f = power<T>(d);
                all1 += f * fmaf(fmaxf(d, LOW), p0[r], p1[r]);
                all0 = fmaf(f, p0[r], all0);
            }
        }
        const float log_sum = logf(all0);
        if (tid == 0) {
            const bool none = all0 == 0.f;                           // no token can occur
            if (a.logp) {
                const int t = a.target[row];
                float v = 0.f;
                if (t >= 0 && t < a.vocab) v = none ? -INFINITY : a.scale * ((float)x.p[x.off + (int64_t)t] - top) - log_sum;
                a.logp[row] = v;
            }
            if (a.lse) { a.lse[2 * row] = top; a.lse[2 * row + 1] = log_sum; }
            if (ENTROPY) a.entropy[row] = none ? 0.f : log_sum - all1 / all0 * 0.69314718055994531f;
        }
        if constexpr (TOP) {
            Key* from = best;
            if (ranks > 1) {
                for (int k = tid; k < (int)ranks * a.k; k += threads) {
                    const unsigned at = on_rank(smem_at(best), (unsigned)(k / a.k)) + 8u * (unsigned)(k % a.k);
                    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(joined[k]) : "r"(at) : "memory");
                }
                __syncthreads();
                for (int k = tid; k < (int)ranks * a.k; k += threads) {
                    const Key q = joined[k];
                    int rnk = 0;
                    for (int z = 0; z < (int)ranks * a.k; ++z) rnk += joined[z] > q;
                    if (q && rnk < a.k) {
                        a.top[row * a.k + rnk] = (int32_t)~(unsigned)q;
                        if (a.top_logp) { const float v = from_order((unsigned)(q >> 32)); a.top_logp[row * a.k + rnk] = all0 == 0.f ? -INFINITY : a.scale * (v - top) - log_sum; }
                    }
                }
            } else if (tid < a.k) {
                const Key q = from[tid];
                a.top[row * a.k + tid] = (int32_t)~(unsigned)q;
                if (a.top_logp) { const float v = from_order((unsigned)(q >> 32)); a.top_logp[row * a.k + tid] = all0 == 0.f ? -INFINITY : a.scale * (v - top) - log_sum; }
            }
        }
    }
    if (ranks > 1) cluster_sync();                                   // nobody leaves while the first block reads its shared memory
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
template <typename T>
__global__ void __launch_bounds__(256) logprob_backward_kernel(const LogpBack a) {
    grid_dep_sync();
    const int lane = threadIdx.x & 31;
    const int64_t per_row = ((int64_t)a.vocab + 2 * V<T> - 2) / V<T> / 128 + 1, total = a.rows * per_row;      // whatever the row's offset
    for (int64_t n = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); n < total; n += (int64_t)gridDim.x * 8) {
        const int64_t row = n / per_row;
        const Row<T> x(a.x, row, a.ld, a.vocab);
        T* out = static_cast<T*>(a.dx) + row * a.ldd - x.off;
        const bool same = (reinterpret_cast<uintptr_t>(out) & 15) == 0;
        const int64_t g0 = (n - row * per_row) * 128 + lane;
        uint4 q[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t g = g0 + 32 * u;
            q[u] = g >= x.first && g < x.end ? x.whole((int)g) : make_uint4(0u, 0u, 0u, 0u);
        }
        const int t = a.target ? a.target[row] : -1;
        const float m = a.lse[2 * row], log_sum = a.lse[2 * row + 1];
        const bool none = m == -INFINITY && log_sum == -INFINITY, given = t >= 0 && t < a.vocab && !none;
        const float dl = given && a.dlogp ? a.dlogp[row] * a.scale : 0.f, dh = a.dentropy ? a.dentropy[row] * a.scale : 0.f, entropy = a.dentropy ? a.entropy[row] : 0.f;
        const float plus = fmaf(dh, entropy, dl);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t g = g0 + 32 * u;
            if (g >= x.all) break;
            const bool whole = g >= x.first && g < x.end;
            float v[V<T>];
            if (whole) decode<T>(q[u], v); else x.values((int)g, v);
#pragma unroll
            for (int j = 0; j < V<T>; ++j) {
                const float lp = (v[j] - m) * a.scale - log_sum;
                const float p = sizeof(T) == 4 ? expf(lp) : ffn::ex2_fast(lp * ffn::LOG2E);
                v[j] = none ? 0.f : -p * fmaf(dh, fmaxf(lp, LOW), plus);
            }
            const int64_t c0 = g * V<T> - x.off;
            if (given && t >= c0 && t < c0 + V<T>) {
#pragma unroll
                for (int j = 0; j < V<T>; ++j) if (t == c0 + j) v[j] += dl;
            }
            if (whole && same) reinterpret_cast<uint4*>(out)[g] = encode<T>(v);
            else {
                const uint4 r = encode<T>(v);
                const unsigned b[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int j = 0; j < V<T>; ++j)
                    if (c0 + j >= 0 && c0 + j < a.vocab) from_bits(out + g * V<T> + j, b[j * (int)sizeof(T) / 4] >> (sizeof(T) == 4 ? 0 : 16 * (j & 1)));
            }
        }
    }
}

ftp_status check(const void* logits, int64_t rows, int32_t vocab, int64_t* ld, int32_t precision, float scale, const char* who) {
    FTP_REQUIRE(precision == FTP_FP32 || precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, precision);
    FTP_REQUIRE(rows >= 0 && vocab >= 1, FTP_EINVAL, "%s: rows must not be negative, vocab must be positive", who);
    FTP_REQUIRE(rows < (1ll << 28) && vocab < (1 << 30), FTP_ERANGE, "%s: tensor too large", who);
    FTP_REQUIRE(scale > 0.f && scale <= 3e38f, FTP_EINVAL, "%s: scale must be positive and finite", who);
    if (ftp_status s = check_pitches({*ld}, vocab, who)) return s;
    if (!*ld) *ld = vocab;
    FTP_REQUIRE(rows == 0 || logits, FTP_EINVAL, "%s: null buffer", who);
    return check_elements({logits}, precision == FTP_FP32 ? 4 : 2, who);
}

template <typename T> cudaError_t forward_of(const LogpArgs& a, cudaStream_t st) {
    // a thread takes four groups and more; blocks of 512 share a row while that gives every multiprocessor no more than two
    const int groups = (a.vocab + V<T> - 1) / V<T>;
    int threads = 32, ranks = 1;
    while (threads < MOST_THREADS && threads * 4 < groups) threads *= 2;
    while (ranks < 8 && a.rows * ranks * 2 <= 2 * SMS && ranks * 2 * threads * 2 <= groups) ranks *= 2;
    auto kern = a.k ? (a.entropy ? logprob_forward_kernel<T, true, true> : logprob_forward_kernel<T, false, true>)
                    : (a.entropy ? logprob_forward_kernel<T, true, false> : logprob_forward_kernel<T, false, false>);
    return launch_cluster(kern, dim3((unsigned)(a.rows * ranks)), threads, a.k ? CAND * sizeof(Key) : 0, ranks, st, a);
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
    const LogpArgs a{logits, targets, logp, entropy, lse, top_logp, top, rows, ldl, vocab, k, scale, scale * 1.44269504088896341f};
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
    if (precision == FTP_FP32) launch(logprob_backward_kernel<float>, grid, dim3(256), 0, st, a);
    else launch(logprob_backward_kernel<bf16>, grid, dim3(256), 0, st, a);
    return launched(who);
}

}  // extern "C"
