// A block's result joins the residual stream: s = alpha x + beta gate drop(post(u)), and the next block's input y = pre(s), in one
// pass over the tokens each way; and dropout by itself.
//
// Bound by memory in principle: the forward pass reads u, x and writes s, y; the backward pass reads u, s, dy, ds and writes du, dx.  A row lies in
// the registers of a block of 32 to 512 threads, which take 16 bytes of columns one to eight times; a sum over a row is five shuffles, one exchange
// between its warps and up to four shuffles more.  Forward: up to 32 columns a thread make these cheap and leave more rows in flight, the next row's
// loads start as soon as a row's values are taken; a single row is spread over more threads.  The column sums of the backward pass (gradients of
// the norms' weights and of a gate that many rows share) grow in shared memory, each thread its own columns, over at most 64 rows, and a second
// kernel adds the blocks' sums in double, in a fixed order.
// What sets the time is latency at 16 warps a multiprocessor, which the registers allow, over as many instructions as there are: 1.8 of 4 a cycle forward
// (34 an element), 2.2 backward (76), no pipe over 39 %; packed float arithmetic halved them.  8192 x 4096 bf16 forward with dropout and a gate
// 65 us (4.1 TB/s), without both 46, 8192 x 8192 without both 93 (5.7 TB/s); backward 131 us with dropout, a gate and three column sums (3.1 TB/s), 118
// without dropout, 106 without the gate too, 88-91 for the second norm alone.  8192 x 2048 float: 48 forward, 90 backward, without both.
// A call that leaves out u, ds or a weight's gradient goes through the kernel for any (8192 x 4096 bf16: 140-162 us, floors 31 to 62).
// Rows off 16 bytes: a thread's columns lie a block's width apart, single elements (8000 x 4001 bf16: 157 us forward, 247 backward).
#include <algorithm>
#include "token.cuh"

namespace ftp {
namespace token {
namespace {

enum { SUM_W_PRE, SUM_B_PRE, SUM_W_POST, SUM_B_POST, SUM_GATE, SUMS };

struct JoinArgs {
    const void *u, *x, *gate, *dy, *ds;
    void *s, *y, *du, *dx, *dgate;           // s: written by the forward pass, read by the backward pass
    const float *w_post, *b_post, *w_pre, *b_pre;
    float* stats;                            // four planes of `rows`: mean and 1 / deviation of u, of s
    int64_t rows, ldu, ldx, lds, ldy, ldg, lddu, ldds, lddx, lddg, gate_rows;
    int cols, threads, groups, post, pre, full;  // full: no thread has columns behind the last one
    float eps, alpha, beta, per_col;         // per_col: 1 / cols
    Drop drop;
    // backward
    float *sums, *gate_sums, *spill;         // blocks' column sums; a shared gate's sums; the running sums where shared memory is too small
    float* out[SUMS];                        // where the column sums go when there is one block
    int at[SUMS], nsums, run;                // place of each sum or -1; rows of a run (the rows that one row's threads walk)
};

// A row; its number is the same in all threads of a block, so that its address stays in uniform registers.
template <typename T> __device__ __forceinline__ const T* in_row(const void* base, int64_t ld, int64_t row) { return static_cast<const T*>(base) + row * ld; }
template <typename T> __device__ __forceinline__ T* out_row(void* base, int64_t ld, int64_t row) { return static_cast<T*>(base) + row * ld; }
// a row of the gate: a float vector, or a row of the tensors' type for every gate_rows rows
template <typename T, bool VEC> __device__ __forceinline__ void gate_of(const JoinArgs& a, int64_t row, int t, int g, F2 (&v)[P<T>]) {
    if (a.gate_rows == 0) fetch_vector<T, VEC>(static_cast<const float*>(a.gate), t, a.threads, g, a.cols, v);
    else decode<T>(fetch<T, VEC>(static_cast<const T*>(a.gate) + (int64_t)((unsigned)row / (unsigned)a.gate_rows) * a.ldg, t, a.threads, g, a.cols), v);
}

// What lies behind the last column becomes 0.
template <typename T, bool VEC> __device__ __forceinline__ void clip(int t, int threads, int g, int cols, F2 (&v)[P<T>]) {
    if constexpr (VEC) {
        if (column<T, true>(t, threads, g, 0) >= cols)
#pragma unroll
            for (int j = 0; j < P<T>; ++j) v[j] = 0ull;
    } else {
#pragma unroll
        for (int j = 0; j < P<T>; ++j) {
            const float2 p = parts(v[j]);
            v[j] = f2(column<T, false>(t, threads, g, 2 * j) < cols ? p.x : 0.f, column<T, false>(t, threads, g, 2 * j + 1) < cols ? p.y : 0.f);
        }
    }
}

template <typename T, int G, bool VEC> __device__ __forceinline__ void clip_row(const JoinArgs& a, int t, F2 (&v)[G][P<T>]) {
    if (a.full) return;
#pragma unroll
    for (int g = 0; g < G; ++g) clip<T, VEC>(t, a.threads, g, a.cols, v[g]);
}

// mean and 1 / deviation of the rows in v (0 behind the last column)
template <typename T, int G, bool VEC> __device__ __forceinline__ float2 moments(const JoinArgs& a, int kind, const F2 (&v)[G][P<T>], int t, RowSum& sum) {
    float mean = 0.f;
    F2 q = 0ull;
    if (kind == FTP_NORM_LAYER) {
        F2 p = 0ull;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < P<T>; ++j) p = add2(p, v[g][j]);
        mean = sum(sum2(p)) * a.per_col;
        const F2 less = f2(-mean);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            F2 d[P<T>];
#pragma unroll
            for (int j = 0; j < P<T>; ++j) d[j] = add2(v[g][j], less);
            if (!a.full) clip<T, VEC>(t, a.threads, g, a.cols, d);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) q = fma2(d[j], d[j], q);
        }
    } else {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < P<T>; ++j) q = fma2(v[g][j], v[g][j], q);
    }
    return make_float2(mean, 1.f / sqrtf(fmaf(sum(sum2(q)), a.per_col, a.eps)));
}
// v * c or v + c over all groups of a row
template <typename T, int G, bool VEC> __device__ __forceinline__ void scale_by(const JoinArgs& a, const float* w, int t, F2 (&v)[G][P<T>]) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
        F2 c[P<T>];
        fetch_vector<T, VEC>(w, t, a.threads, g, a.cols, c);
#pragma unroll
        for (int j = 0; j < P<T>; ++j) v[g][j] = mul2(v[g][j], c[j]);
    }
}
template <typename T, int G, bool VEC> __device__ __forceinline__ void shift_by(const JoinArgs& a, const float* b, int t, F2 (&v)[G][P<T>]) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
        F2 c[P<T>];
        fetch_vector<T, VEC>(b, t, a.threads, g, a.cols, c);
#pragma unroll
        for (int j = 0; j < P<T>; ++j) v[g][j] = add2(v[g][j], c[j]);
    }
}
template <typename T, int G, bool VEC> __device__ __forceinline__ void gate_by(const JoinArgs& a, int64_t row, int t, F2 (&v)[G][P<T>]) {
#pragma unroll
    for (int g = 0; g < G; ++g) {
        F2 c[P<T>];
        gate_of<T, VEC>(a, row, t, g, c);
#pragma unroll
        for (int j = 0; j < P<T>; ++j) v[g][j] = mul2(v[g][j], c[j]);
    }
}
// (v - mean) / deviation * w + b
template <typename T, int G, bool VEC>
__device__ __forceinline__ void apply(const JoinArgs& a, float2 m, const float* w, const float* b, int t, F2 (&v)[G][P<T>]) {
    const F2 r = f2(m.y), less = f2(-m.x * m.y);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < P<T>; ++j) v[g][j] = fma2(v[g][j], r, less);
    if (w) scale_by<T, G, VEC>(a, w, t, v);
    if (b) shift_by<T, G, VEC>(a, b, t, v);
}
template <typename T, int G, bool VEC>
__device__ __forceinline__ void fetch_row(const JoinArgs& a, const T* row, int t, uint4 (&r)[G]) {
#pragma unroll
    for (int g = 0; g < G; ++g) r[g] = fetch<T, VEC>(row, t, a.threads, g, a.cols);
}
template <typename T, int G, bool VEC>
__device__ __forceinline__ void put_row(const JoinArgs& a, T* row, int t, const F2 (&v)[G][P<T>]) {
#pragma unroll
    for (int g = 0; g < G; ++g) put<T, VEC>(row, t, a.threads, g, a.cols, encode<T>(v[g]));
}
template <typename T, int G> __device__ __forceinline__ void decode_row(const uint4 (&r)[G], F2 (&v)[G][P<T>]) {
#pragma unroll
    for (int g = 0; g < G; ++g) decode<T>(r[g], v[g]);
}

// Threads resident on a multiprocessor, by the columns of a thread: what their registers leave (64, 80 and 128 a thread).
constexpr int forward_threads(int columns) { return columns <= 8 ? 1024 : columns <= 16 ? 768 : 512; }
constexpr int BACKWARD_THREADS = 512;

// Rows that the backward pass takes at a time where the usual gradients are asked for: the vectors that all rows share, and the running sums, are then
// read half as often (8192 x 4096 bf16: 130 us; a row at a time 138, the first cache's bandwidth three quarters used).  With the eight sums of a layer norm a
// row at a time is faster (8192 x 2048 float 171 instead of 206 us).
constexpr int PAIR = 2;

template <typename T, int G, bool VEC>
__global__ void __launch_bounds__(forward_threads(G * V<T>)) join_forward_kernel(const JoinArgs a) {
    __shared__ float red[32];
    __shared__ Rounds keys;
    grid_dep_sync();
    const Dropping drop(a.drop, keys);
    RowSum sum{red, 0};
    const int t = threadIdx.x;
    const F2 f = f2(drop.cut ? a.beta * a.drop.factor : a.beta), alpha = f2(a.alpha);
    int64_t row = blockIdx.x;
    const int64_t step = gridDim.x;
    uint4 ru[G], rx[G];
    if (a.u) fetch_row<T, G, VEC>(a, in_row<T>(a.u, a.ldu, row), t, ru);
    if (a.x) fetch_row<T, G, VEC>(a, in_row<T>(a.x, a.ldx, row), t, rx);
    for (; row < a.rows; row += step) {
        F2 v[G][P<T>];
        const bool more = row + step < a.rows;                       // the next row's loads start as soon as this one's values are taken
        if (a.u) {
            decode_row<T, G>(ru, v);
            if (more) fetch_row<T, G, VEC>(a, in_row<T>(a.u, a.ldu, row + step), t, ru);
            clip_row<T, G, VEC>(a, t, v);
            if (a.post != FTP_NORM_NONE) {
                const float2 m = moments<T, G, VEC>(a, a.post, v, t, sum);
                if (a.stats && t == 0) { a.stats[row] = m.x; a.stats[a.rows + row] = m.y; }
                apply<T, G, VEC>(a, m, a.w_post, a.b_post, t, v);
            }
            if (a.gate) gate_by<T, G, VEC>(a, row, t, v);
            if (drop.cut) {
                const unsigned long long first = drop.first_of(row, a.cols);
#pragma unroll
                for (int g = 0; g < G; ++g) drop.template operator()<T, VEC>(first, t, a.threads, g, v[g]);
            }
            if (a.x) {
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    F2 r[P<T>];
                    decode<T>(rx[g], r);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) v[g][j] = fma2(v[g][j], f, mul2(r[j], alpha));
                }
                if (more) fetch_row<T, G, VEC>(a, in_row<T>(a.x, a.ldx, row + step), t, rx);
            } else {
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) v[g][j] = mul2(v[g][j], f);
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint4 to = encode<T>(v[g]);                    // the stream goes on in the tensors' type, here too
                put<T, VEC>(out_row<T>(a.s, a.lds, row), t, a.threads, g, a.cols, to);
                decode<T>(to, v[g]);
            }
        } else {
            decode_row<T, G>(rx, v);
            if (more) fetch_row<T, G, VEC>(a, in_row<T>(a.x, a.ldx, row + step), t, rx);
        }
        if (a.pre != FTP_NORM_NONE) {
            clip_row<T, G, VEC>(a, t, v);
            const float2 m = moments<T, G, VEC>(a, a.pre, v, t, sum);
            if (a.stats && t == 0) { a.stats[2 * a.rows + row] = m.x; a.stats[3 * a.rows + row] = m.y; }
            apply<T, G, VEC>(a, m, a.w_pre, a.b_pre, t, v);
            put_row<T, G, VEC>(a, out_row<T>(a.y, a.ldy, row), t, v);
        }
    }
}

// A thread's running sum number `i` (of V columns): float4s that lie a block's width apart.
template <typename T> struct Running {
    float4* at;
    __device__ __forceinline__ float4& q(int i, int k) const { return at[(unsigned)(i * (V<T> / 4) + k) * blockDim.x]; }
    __device__ __forceinline__ void add(int i, const F2 (&v)[P<T>]) const {
#pragma unroll
        for (int k = 0; k < V<T> / 4; ++k) {
            const float4 f = q(i, k);
            const float2 x = parts(add2(f2(f.x, f.y), v[2 * k])), y = parts(add2(f2(f.z, f.w), v[2 * k + 1]));
            q(i, k) = make_float4(x.x, x.y, y.x, y.y);
        }
    }
    __device__ __forceinline__ void get(int i, float (&v)[V<T>]) const {
#pragma unroll
        for (int k = 0; k < V<T> / 4; ++k) { const float4 f = q(i, k); v[4 * k] = f.x; v[4 * k + 1] = f.y; v[4 * k + 2] = f.z; v[4 * k + 3] = f.w; }
    }
    __device__ __forceinline__ void clear(int i) const {
#pragma unroll
        for (int k = 0; k < V<T> / 4; ++k) q(i, k) = make_float4(0.f, 0.f, 0.f, 0.f);
    }
};

// With x^ and u^ the normalised rows of s and u, g = dy w_pre, K = beta gate mask / (1 - p), r the 1 / deviation of s and r' that of u:
//
//   e = ds + r g;   c1 = - r mean(g) (layer norm only), c2 = - r mean(g x^);   D = e + c1 + c2 x^
//   dx = alpha D;   dv = K D;   du = r' (dv w_post - mean(dv w_post) - u^ mean(dv w_post u^));   dgate = (K / gate) D (u^ w_post + b_post)
//
// A dropped element adds nothing, whatever u and D hold there: its terms are cleared, where a product with 0 could be NaN (1 % of the time; a
// gate, which multiplies what is left, has to be finite everywhere: clearing behind it too took 3 to 5 %).
// The sums over a row that du needs are sums of K w_post (e + c1 + c2 x^) and of that times u^: linear in c1 and c2, so all sums of a row
// go through one exchange, and its values are decoded once.
// KIND: what is known when compiled, because a question per group of columns costs three instructions.  BOTH: both norms with weights; PRE_ONLY: the second
// norm alone; with weights and their gradients, biases only where a norm is a layer norm, a u, ds, dx and du.
enum { ANY = 0, BOTH = 1, PRE_ONLY = 2 };
template <typename T, int G, bool VEC, bool LAYER, int KIND>
__global__ void __launch_bounds__(BACKWARD_THREADS) join_backward_kernel(const JoinArgs a) {
    constexpr bool USUAL = KIND != ANY, AHEAD = USUAL && VEC;
    constexpr int NS = LAYER ? 8 : 3, R = USUAL && !LAYER && G * V<T> <= 8 ? PAIR : 1;
    const bool pre = USUAL || a.pre != FTP_NORM_NONE, post = USUAL ? KIND == BOTH : a.post != FTP_NORM_NONE, w_pre = USUAL || a.w_pre,
               w_post = USUAL ? KIND == BOTH : a.w_post != nullptr, b_post = USUAL && (!LAYER || KIND != BOTH) ? false : a.b_post != nullptr;
    const bool gated = a.gate, graded = a.dgate;
    // places of the running sums
    const int at_w_pre = USUAL ? 0 : a.at[SUM_W_PRE], at_b_pre = USUAL && !LAYER ? -1 : a.at[SUM_B_PRE],
              at_w_post = !USUAL || LAYER ? a.at[SUM_W_POST] : KIND == BOTH ? 1 : -1, at_b_post = USUAL && !LAYER ? -1 : a.at[SUM_B_POST],
              at_gate = !USUAL || LAYER ? a.at[SUM_GATE] : KIND == BOTH ? 2 : 1;
    extern __shared__ float4 dynamic[];
    __shared__ float red[2 * 16 * NS * R];
    __shared__ Rounds keys;
    grid_dep_sync();
    const Dropping drop(a.drop, keys);
    const int t = threadIdx.x;
    int turn = 0;
    Running<T> run{dynamic + t};
    for (int i = 0; i < a.nsums * G; ++i) run.clear(i);
    const int64_t mine = blockIdx.x, first = mine * a.run, last = min(first + a.run, a.rows);
    int64_t group = a.gate_rows > 1 ? first / a.gate_rows : 0, next = a.gate_rows > 1 ? (group + 1) * a.gate_rows : 0;   // next: first row of the next group
    const F2 f = f2(drop.cut ? a.beta * a.drop.factor : a.beta), alpha = f2(a.alpha);
    // AHEAD: the next rows are on their way while these are worked on; a thread copies its own columns into shared memory and reads them itself
    const unsigned staged = smem_at(dynamic) + a.nsums * (G * (V<T> / 4)) * blockDim.x * 16 + t * 16;
    const int64_t lds[4] = {a.lds, a.ldy, a.ldds, a.ldu};
    const void* const bases[4] = {a.s, a.dy, a.ds, a.u};
    const auto ahead = [&](int64_t from) {
#pragma unroll
        for (int q = 0; q < R; ++q)
            if (from + q < last)
#pragma unroll
                for (int n = 0; n < 4; ++n)
#pragma unroll
                    for (int g = 0; g < G; ++g)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" :: "r"(staged + ((q * 4 + n) * G + g) * blockDim.x * 16),
                                     "l"(reinterpret_cast<const char*>(in_row<T>(bases[n], lds[n], from + q)) + (unsigned)column_in<T, true>(t, a.threads, g, 0, a.cols) * (unsigned)sizeof(T)) : "memory");
    };
    const auto arrived = [&](int q, int n, uint4 (&r)[G]) {
#pragma unroll
        for (int g = 0; g < G; ++g)
            asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r[g].x), "=r"(r[g].y), "=r"(r[g].z), "=r"(r[g].w) : "r"(staged + ((q * 4 + n) * G + g) * blockDim.x * 16) : "memory");
    };
    if constexpr (AHEAD) ahead(first);
    for (int64_t row = first; row < last;) {
        if (a.gate_sums && row == next) {                            // another group: its predecessor's sum is complete as far as this run goes
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float v[V<T>];
                run.get(at_gate * G + g, v);
                put_vector<T, VEC>(a.gate_sums + (mine + group) * a.cols, t, a.threads, g, a.cols, v);
                run.clear(at_gate * G + g);
            }
            ++group;
            next += a.gate_rows;
        }
        const int64_t end = a.gate_sums ? min(last, next) : last;    // the rows of an iteration share a group
        bool on[R];
#pragma unroll
        for (int q = 0; q < R; ++q) on[q] = row + q < end;
        uint4 ru[R][G], rs[R][G], rdy[R][G], rds[R][G];
        if constexpr (AHEAD) asm volatile("cp.async.wait_all;" ::: "memory");
#pragma unroll
        for (int q = 0; q < R; ++q) {
            if (!on[q]) {                                            // zeros, which add nothing
#pragma unroll
                for (int g = 0; g < G; ++g) ru[q][g] = rs[q][g] = rdy[q][g] = rds[q][g] = make_uint4(0u, 0u, 0u, 0u);
                continue;
            }
            if constexpr (AHEAD) {
                arrived(q, 0, rs[q]);
                arrived(q, 1, rdy[q]);
                arrived(q, 2, rds[q]);
                arrived(q, 3, ru[q]);
                continue;
            }
            if (pre) fetch_row<T, G, VEC>(a, in_row<T>(a.s, a.lds, row + q), t, rs[q]);
            if (USUAL || a.dy) fetch_row<T, G, VEC>(a, in_row<T>(a.dy, a.ldy, row + q), t, rdy[q]);
            if (USUAL || a.ds) fetch_row<T, G, VEC>(a, in_row<T>(a.ds, a.ldds, row + q), t, rds[q]);
            if (USUAL || a.u) fetch_row<T, G, VEC>(a, in_row<T>(a.u, a.ldu, row + q), t, ru[q]);
        }
        if constexpr (AHEAD) ahead(min(row + R, end));
        float r[R];
        F2 rp[R], lp[R], rn[R], ln[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            float ms = 0.f, mu = 0.f, ri = 1.f;
            r[q] = 0.f;
            if (pre && on[q]) { ms = a.stats[2 * a.rows + row + q]; r[q] = a.stats[3 * a.rows + row + q]; }
            if (post && on[q]) { mu = a.stats[row + q]; ri = a.stats[a.rows + row + q]; }
            rp[q] = f2(r[q]);
            lp[q] = f2(-ms * r[q]);
            rn[q] = f2(ri);
            ln[q] = f2(-mu * ri);
        }
        F2 e[R][G][P<T>], xh[R][G][P<T>], kept[R][G][P<T>], uh[R][G][P<T>], sum[R][NS];   // kept: all bits of what is not dropped
#pragma unroll
        for (int q = 0; q < R; ++q) {
#pragma unroll
            for (int i = 0; i < NS; ++i) sum[q][i] = 0ull;
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int j = 0; j < P<T>; ++j) kept[q][g][j] = on[q] ? ~0ull : 0ull;
            if (drop.cut) {
                const unsigned long long n = drop.first_of(row + q, a.cols);
#pragma unroll
                for (int g = 0; g < G; ++g) drop.template operator()<T, VEC>(n, t, a.threads, g, kept[q][g]);
            }
            clip_row<T, G, VEC>(a, t, kept[q]);
            if (USUAL || a.ds) decode_row<T, G>(rds[q], e[q]);
            else
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) e[q][g][j] = 0ull;
        }
        if (pre) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                F2 w[P<T>], h[P<T>], b[P<T>];
                if (w_pre) fetch_vector<T, VEC>(a.w_pre, t, a.threads, g, a.cols, w);
#pragma unroll
                for (int q = 0; q < R; ++q) {
                    F2 d[P<T>];
                    decode<T>(rdy[q][g], d);
                    if (!a.full) clip<T, VEC>(t, a.threads, g, a.cols, d);
                    decode<T>(rs[q][g], xh[q][g]);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) {
                        xh[q][g][j] = fma2(xh[q][g][j], rp[q], lp[q]);
                        h[j] = q ? fma2(xh[q][g][j], d[j], h[j]) : mul2(xh[q][g][j], d[j]);
                        b[j] = q ? add2(b[j], d[j]) : d[j];
                        if (w_pre) d[j] = mul2(d[j], w[j]);
                        sum[q][0] = fma2(d[j], xh[q][g][j], sum[q][0]);
                        if (LAYER) sum[q][3] = add2(sum[q][3], d[j]);
                        e[q][g][j] = fma2(rp[q], d[j], e[q][g][j]);
                    }
                }
                if (at_b_pre >= 0) run.add(at_b_pre * G + g, b);
                if (at_w_pre >= 0) run.add(at_w_pre * G + g, h);
            }
        }
        if (USUAL || a.u) {
#pragma unroll
            for (int q = 0; q < R; ++q) decode_row<T, G>(ru[q], uh[q]);
            if (post) {
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    F2 w[P<T>], gate[P<T>];
                    if (w_post) fetch_vector<T, VEC>(a.w_post, t, a.threads, g, a.cols, w);
#pragma unroll
                    for (int q = 0; q < R; ++q) {
                        if (gated && (q == 0 || (a.gate_rows && on[q]))) gate_of<T, VEC>(a, row + q, t, g, gate);
#pragma unroll
                        for (int j = 0; j < P<T>; ++j) {
                            F2& x = uh[q][g][j];
                            x = fma2(x, rn[q], ln[q]);
                            F2 k = f;
                            if (gated) k = mul2(k, gate[j]);
                            if (w_post) k = mul2(k, w[j]);
                            const F2 z = mul2(k, x) & kept[q][g][j], d = e[q][g][j] & kept[q][g][j];
                            if (LAYER) k &= kept[q][g][j];
                            sum[q][1] = fma2(z, d, sum[q][1]);
                            if (pre) sum[q][2] = fma2(z, xh[q][g][j], sum[q][2]);
                            if (LAYER) {
                                sum[q][4] = add2(sum[q][4], z);
                                sum[q][5] = fma2(k, d, sum[q][5]);
                                if (pre) sum[q][6] = fma2(k, xh[q][g][j], sum[q][6]);
                                sum[q][7] = add2(sum[q][7], k);
                            }
                        }
                    }
                }
            }
        }
        float all[R * NS];
#pragma unroll
        for (int q = 0; q < R; ++q)
#pragma unroll
            for (int i = 0; i < NS; ++i) all[q * NS + i] = sum2(sum[q][i]);
        row_sums<R * NS>(all, red, turn);
        F2 c1[R], c2[R], e1[R], e2[R];
#pragma unroll
        for (int q = 0; q < R; ++q) {
            const float* s = all + q * NS;
            const float c2f = -s[0] * a.per_col * r[q], c1f = LAYER && a.pre == FTP_NORM_LAYER ? -s[LAYER ? 3 : 0] * a.per_col * r[q] : 0.f;
            c1[q] = f2(c1f);
            c2[q] = f2(c2f);
            e1[q] = e2[q] = 0ull;
            if (post) {
                e2[q] = f2(-fmaf(c2f, s[2], LAYER ? fmaf(c1f, s[LAYER ? 4 : 0], s[1]) : s[1]) * a.per_col);
                if (LAYER && a.post == FTP_NORM_LAYER) e1[q] = f2(-fmaf(c2f, s[LAYER ? 6 : 0], fmaf(c1f, s[LAYER ? 7 : 0], s[LAYER ? 5 : 0])) * a.per_col);
            }
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            F2 w[P<T>], b[P<T>], gate[P<T>], of_gate[P<T>], of_w[P<T>], of_b[P<T>];
            if (w_post) fetch_vector<T, VEC>(a.w_post, t, a.threads, g, a.cols, w);
            if (graded && b_post) fetch_vector<T, VEC>(a.b_post, t, a.threads, g, a.cols, b);
#pragma unroll
            for (int q = 0; q < R; ++q) {
                F2 (&d)[P<T>] = e[q][g];
                F2 (&x)[P<T>] = uh[q][g];
                if (pre) {
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) {
                        d[j] = fma2(c2[q], xh[q][g][j], d[j]);
                        if (LAYER) d[j] = add2(d[j], c1[q]);
                    }
                }
                if ((USUAL || a.dx) && on[q]) {
                    F2 p[P<T>];
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) p[j] = mul2(alpha, d[j]);
                    put<T, VEC>(out_row<T>(a.dx, a.lddx, row + q), t, a.threads, g, a.cols, encode<T>(p));
                }
#pragma unroll
                for (int j = 0; j < P<T>; ++j) d[j] = mul2(d[j], f) & kept[q][g][j];
                if (graded) {
                    F2 p[P<T>];
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) {
                        p[j] = w_post ? mul2(x[j], w[j]) : x[j];
                        if (b_post) p[j] = add2(p[j], b[j]);
                        p[j] = mul2(p[j], d[j]);
                        if (!post) p[j] &= kept[q][g][j];            // u as it came
                        of_gate[j] = q ? add2(of_gate[j], p[j]) : p[j];
                    }
                    if (a.gate_rows == 1 && on[q]) put<T, VEC>(out_row<T>(a.dgate, a.lddg, row + q), t, a.threads, g, a.cols, encode<T>(p));
                }
                if (gated) {
                    if (q == 0 || (a.gate_rows && on[q])) gate_of<T, VEC>(a, row + q, t, g, gate);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) d[j] = mul2(d[j], gate[j]);
                }
#pragma unroll
                for (int j = 0; j < P<T>; ++j) {
                    of_b[j] = q ? add2(of_b[j], d[j]) : d[j];
                    of_w[j] = q ? fma2(d[j], x[j], of_w[j]) : mul2(d[j], x[j]);
                }
                if ((USUAL || a.du) && on[q]) {
                    if (post) {
#pragma unroll
                        for (int j = 0; j < P<T>; ++j) {
                            if (w_post) d[j] = mul2(d[j], w[j]);
                            if (LAYER) d[j] = add2(d[j], e1[q]);
                            d[j] = mul2(rn[q], fma2(e2[q], x[j], d[j]));
                        }
                    }
                    put<T, VEC>(out_row<T>(a.du, a.lddu, row + q), t, a.threads, g, a.cols, encode<T>(d));
                }
            }
            if (graded && a.gate_rows != 1) run.add(at_gate * G + g, of_gate);
            if (at_b_post >= 0) run.add(at_b_post * G + g, of_b);
            if (at_w_post >= 0) run.add(at_w_post * G + g, of_w);
        }
        row = min(row + R, end);
    }
    if (a.gate_sums && first < a.rows) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float v[V<T>];
            run.get(at_gate * G + g, v);
            put_vector<T, VEC>(a.gate_sums + (mine + group) * a.cols, t, a.threads, g, a.cols, v);
        }
    }
    const int n = a.gate_sums ? a.nsums - 1 : a.nsums;               // a shared gate's sum comes last
    for (int k = 0; k < n; ++k) {
        float* to = a.sums + ((size_t)blockIdx.x * n + k) * a.cols;
        if (gridDim.x == 1) {
#pragma unroll
            for (int o = 0; o < SUMS; ++o) if (a.at[o] == k) to = a.out[o];
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float v[V<T>];
            run.get(k * G + g, v);
            put_vector<T, VEC>(to, t, a.threads, g, a.cols, v);
        }
    }
}

// The same for rows of more than 16 columns a thread, whose values do not fit into registers: a group of columns at a time, every group read twice (the
// second time from the second cache: 2000 x 16384 bf16 with all terms 1090 us with the values spilled to local memory, and 500 so).
template <typename T, bool VEC, bool LAYER>
__global__ void __launch_bounds__(BACKWARD_THREADS) join_backward_wide_kernel(const JoinArgs a) {
    constexpr int NS = LAYER ? 8 : 3;
    extern __shared__ float4 dynamic[];
    __shared__ float red[2 * 16 * NS];
    __shared__ Rounds keys;
    grid_dep_sync();
    const Dropping drop(a.drop, keys);
    const bool pre = a.pre != FTP_NORM_NONE, post = a.post != FTP_NORM_NONE;
    const int t = threadIdx.x, G = a.groups;
    int turn = 0;
    Running<T> run{(a.spill ? reinterpret_cast<float4*>(a.spill) + (size_t)blockIdx.x * a.nsums * G * (V<T> / 4) * blockDim.x : dynamic) + t};
    for (int i = 0; i < a.nsums * G; ++i) run.clear(i);
    const int64_t mine = blockIdx.x, first = mine * a.run, last = min(first + a.run, a.rows);
    int64_t group = a.gate_rows > 1 ? first / a.gate_rows : 0, next = a.gate_rows > 1 ? (group + 1) * a.gate_rows : 0;
    const F2 f = f2(drop.cut ? a.beta * a.drop.factor : a.beta), alpha = f2(a.alpha);
    const auto flush = [&](int64_t slot, bool again) {
        for (int g = 0; g < G; ++g) {
            float v[V<T>];
            run.get(a.at[SUM_GATE] * G + g, v);
            put_vector<T, VEC>(a.gate_sums + slot * a.cols, t, a.threads, g, a.cols, v);
            if (again) run.clear(a.at[SUM_GATE] * G + g);
        }
    };
    for (int64_t row = first; row < last; ++row) {
        if (a.gate_sums && row == next) {
            flush(mine + group, true);
            ++group;
            next += a.gate_rows;
        }
        float ms = 0.f, r = 0.f, mu = 0.f, ri = 1.f;
        if (pre) { ms = a.stats[2 * a.rows + row]; r = a.stats[3 * a.rows + row]; }
        if (post) { mu = a.stats[row]; ri = a.stats[a.rows + row]; }
        const F2 rp = f2(r), lp = f2(-ms * r), rn = f2(ri), ln = f2(-mu * ri);
        const unsigned long long number = drop.cut ? drop.first_of(row, a.cols) : 0;
        // e, x^, what is not dropped, u^ and dy of a group
        const auto load = [&](int g, F2 (&e)[P<T>], F2 (&xh)[P<T>], F2 (&kept)[P<T>], F2 (&uh)[P<T>], F2 (&dy)[P<T>]) {
            uint4 rs, rdy, rds, ru;
            if (pre) rs = fetch<T, VEC>(in_row<T>(a.s, a.lds, row), t, a.threads, g, a.cols);
            if (a.dy) rdy = fetch<T, VEC>(in_row<T>(a.dy, a.ldy, row), t, a.threads, g, a.cols);
            if (a.ds) rds = fetch<T, VEC>(in_row<T>(a.ds, a.ldds, row), t, a.threads, g, a.cols);
            if (a.u) ru = fetch<T, VEC>(in_row<T>(a.u, a.ldu, row), t, a.threads, g, a.cols);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) { e[j] = xh[j] = uh[j] = dy[j] = 0ull; kept[j] = ~0ull; }
            if (drop.cut) drop.template operator()<T, VEC>(number, t, a.threads, g, kept);
            clip<T, VEC>(t, a.threads, g, a.cols, kept);
            if (a.ds) decode<T>(rds, e);
            if (a.u) decode<T>(ru, uh);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) uh[j] = fma2(uh[j], rn, ln);
            if (!pre) return;
            F2 w[P<T>];
            decode<T>(rdy, dy);
            clip<T, VEC>(t, a.threads, g, a.cols, dy);
            decode<T>(rs, xh);
            if (a.w_pre) fetch_vector<T, VEC>(a.w_pre, t, a.threads, g, a.cols, w);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) {
                xh[j] = fma2(xh[j], rp, lp);
                e[j] = fma2(rp, a.w_pre ? mul2(dy[j], w[j]) : dy[j], e[j]);
            }
        };
        // K and K w_post
        const auto factors = [&](int g, const F2 (&kept)[P<T>], F2 (&k)[P<T>], F2 (&kw)[P<T>]) {
            F2 w[P<T>];
            if (a.gate) gate_of<T, VEC>(a, row, t, g, w);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) k[j] = (a.gate ? mul2(f, w[j]) : f) & kept[j];
            if (a.w_post) fetch_vector<T, VEC>(a.w_post, t, a.threads, g, a.cols, w);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) kw[j] = a.w_post ? mul2(k[j], w[j]) : k[j];
        };
        F2 sum[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) sum[i] = 0ull;
        if (pre || post)
#pragma unroll 1
            for (int g = 0; g < G; ++g) {
                F2 e[P<T>], xh[P<T>], kept[P<T>], uh[P<T>], dy[P<T>], k[P<T>], kw[P<T>];
                load(g, e, xh, kept, uh, dy);
                if (a.at[SUM_B_PRE] >= 0) run.add(a.at[SUM_B_PRE] * G + g, dy);
                if (a.at[SUM_W_PRE] >= 0) {
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) k[j] = mul2(xh[j], dy[j]);
                    run.add(a.at[SUM_W_PRE] * G + g, k);
                }
                if (pre) {
                    F2 w[P<T>];
                    if (a.w_pre) fetch_vector<T, VEC>(a.w_pre, t, a.threads, g, a.cols, w);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) {
                        const F2 d = a.w_pre ? mul2(dy[j], w[j]) : dy[j];
                        sum[0] = fma2(d, xh[j], sum[0]);
                        if (LAYER) sum[3] = add2(sum[3], d);
                    }
                }
                if (post) {
                    factors(g, kept, k, kw);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) {
                        const F2 z = mul2(kw[j], uh[j]);
                        e[j] &= kept[j];
                        sum[1] = fma2(z, e[j], sum[1]);
                        sum[2] = fma2(z, xh[j], sum[2]);
                        if (LAYER) {
                            sum[4] = add2(sum[4], z);
                            sum[5] = fma2(kw[j], e[j], sum[5]);
                            sum[6] = fma2(kw[j], xh[j], sum[6]);
                            sum[7] = add2(sum[7], kw[j]);
                        }
                    }
                }
            }
        float s[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) s[i] = sum2(sum[i]);
        row_sums<NS>(s, red, turn);
        const float c2f = -s[0] * a.per_col * r, c1f = LAYER && a.pre == FTP_NORM_LAYER ? -s[LAYER ? 3 : 0] * a.per_col * r : 0.f;
        float e1 = 0.f, e2 = 0.f;
        if (post) {
            e2 = -fmaf(c2f, s[2], LAYER ? fmaf(c1f, s[LAYER ? 4 : 0], s[1]) : s[1]) * a.per_col;
            if (LAYER && a.post == FTP_NORM_LAYER) e1 = -fmaf(c2f, s[LAYER ? 6 : 0], fmaf(c1f, s[LAYER ? 7 : 0], s[LAYER ? 5 : 0])) * a.per_col;
        }
        // dx may lie on ds: a thread reads its columns of a group before it writes them
#pragma unroll 1
        for (int g = 0; g < G; ++g) {
            F2 d[P<T>], xh[P<T>], kept[P<T>], uh[P<T>], dy[P<T>], k[P<T>], kw[P<T>];
            load(g, d, xh, kept, uh, dy);
            factors(g, kept, k, kw);
#pragma unroll
            for (int j = 0; j < P<T>; ++j) {
                d[j] = fma2(f2(c2f), xh[j], d[j]);
                if (LAYER) d[j] = add2(d[j], f2(c1f));
                dy[j] = mul2(alpha, d[j]);
                d[j] &= kept[j];
            }
            if (a.dx) put<T, VEC>(out_row<T>(a.dx, a.lddx, row), t, a.threads, g, a.cols, encode<T>(dy));
            if (a.dgate) {
                F2 w[P<T>], p[P<T>];
#pragma unroll
                for (int j = 0; j < P<T>; ++j) p[j] = uh[j];
                if (a.w_post) {
                    fetch_vector<T, VEC>(a.w_post, t, a.threads, g, a.cols, w);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) p[j] = mul2(p[j], w[j]);
                }
                if (a.b_post) {
                    fetch_vector<T, VEC>(a.b_post, t, a.threads, g, a.cols, w);
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) p[j] = add2(p[j], w[j]);
                }
#pragma unroll
                for (int j = 0; j < P<T>; ++j) p[j] = mul2(p[j], mul2(d[j], f)) & kept[j];
                if (a.gate_rows == 1) put<T, VEC>(out_row<T>(a.dgate, a.lddg, row), t, a.threads, g, a.cols, encode<T>(p));
                else run.add(a.at[SUM_GATE] * G + g, p);
            }
#pragma unroll
            for (int j = 0; j < P<T>; ++j) {
                k[j] = mul2(k[j], d[j]);
                d[j] = mul2(kw[j], d[j]);
            }
            if (a.at[SUM_B_POST] >= 0) run.add(a.at[SUM_B_POST] * G + g, k);
            if (a.at[SUM_W_POST] >= 0) {
#pragma unroll
                for (int j = 0; j < P<T>; ++j) k[j] = mul2(k[j], uh[j]);
                run.add(a.at[SUM_W_POST] * G + g, k);
            }
            if (a.du) {
                if (post)
#pragma unroll
                    for (int j = 0; j < P<T>; ++j) d[j] = mul2(rn, fma2(f2(e2), uh[j], add2(d[j], f2(e1))));
                put<T, VEC>(out_row<T>(a.du, a.lddu, row), t, a.threads, g, a.cols, encode<T>(d));
            }
        }
    }
    if (a.gate_sums && first < a.rows) flush(mine + group, false);
    const int n = a.gate_sums ? a.nsums - 1 : a.nsums;
    for (int k = 0; k < n; ++k) {
        float* to = a.sums + ((size_t)blockIdx.x * n + k) * a.cols;
        if (gridDim.x == 1) {
#pragma unroll
            for (int o = 0; o < SUMS; ++o) if (a.at[o] == k) to = a.out[o];
        }
        for (int g = 0; g < G; ++g) {
            float v[V<T>];
            run.get(k * G + g, v);
            put_vector<T, VEC>(to, t, a.threads, g, a.cols, v);
        }
    }
}

// Blocks' column sums joined in double: a warp per 32 columns and 32nd of the blocks, eight loads in flight.
struct JoinSums { const float* part; float* out[SUMS]; int n, cols; int64_t blocks; };
__global__ void __launch_bounds__(1024) join_sums_kernel(const JoinSums a) {
    constexpr int W = 32, U = 8;
    __shared__ double part[W][33];
    grid_dep_sync();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    double s = 0.0;
    if (c < a.cols) {
        const int64_t step = (int64_t)a.n * a.cols;
        const float* p = a.part + (int64_t)blockIdx.y * a.cols + c;
        for (int64_t b = w; b < a.blocks; b += W * U) {
            float v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) v[u] = b + u * W < a.blocks ? p[(b + u * W) * step] : 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) s += v[u];
        }
    }
    part[w][lane] = s;
    __syncthreads();
    for (int n = W / 2; n; n >>= 1) {
        if (w < n) part[w][lane] = s += part[w + n][lane];
        __syncthreads();
    }
    if (w == 0 && c < a.cols) a.out[blockIdx.y][c] = (float)s;
}
// A group's gate gradient: the sums of the runs that hold rows of it, one after another (long groups take long: 8192 x 512 bf16 with 4096 rows a group 78 us
// for the whole call, 31 with a gate vector).
template <typename T>
__global__ void __launch_bounds__(128) join_gate_kernel(const float* part, int64_t groups, int64_t gate_rows, int64_t rows, int run, int cols, T* out, int64_t ld) {
    grid_dep_sync();
    const int c = blockIdx.x * 128 + threadIdx.x;
    if (c >= cols) return;
    for (int64_t g = blockIdx.y; g < groups; g += gridDim.y) {
        const int64_t last = min(rows, (g + 1) * gate_rows) - 1;
        double s = 0.0;
        for (int64_t r = g * gate_rows / run; r <= last / run; ++r) s += part[(r + g) * cols + c];
        if constexpr (sizeof(T) == 4) out[g * ld + c] = (float)s;
        else out[g * ld + c] = __float2bfloat16((float)s);
    }
}

// A warp per 32 V columns of a row, four such pieces in flight.  16384 x 4096 bf16: 61 us, 4.4 TB/s, 2.6 instructions a cycle and the integer pipe over half
// used: 22 instructions an element, a quarter of them the generator's products and exclusive ors, the others masks, conversions and 64-bit indexes; one
// piece in flight 69 us, two 60, eight 70.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dropout_kernel(const T* x, T* y, int64_t rows, int cols, int64_t ldx, int64_t ldy, const Drop d) {
    __shared__ Rounds keys;
    grid_dep_sync();
    const Dropping drop(d, keys);
    const int t = threadIdx.x & 31;
    const unsigned per_row = (unsigned)((cols + 32 * V<T> - 1) / (32 * V<T>));           // pieces of a warp
    const int64_t total = rows * per_row;
    constexpr int U = 4;                                                                // in flight
    for (int64_t i0 = ((int64_t)blockIdx.x * 8 + (threadIdx.x >> 5)) * U; i0 < total; i0 += (int64_t)gridDim.x * 8 * U) {
        uint4 q[U];
        int64_t row[U];
        int at[U];
        row[0] = i0 / per_row;
        at[0] = (int)(i0 - row[0] * per_row);
#pragma unroll
        for (int u = 1; u < U; ++u) {
            const bool wrap = at[u - 1] + 1 == (int)per_row;
            row[u] = row[u - 1] + wrap;
            at[u] = wrap ? 0 : at[u - 1] + 1;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (row[u] < rows) q[u] = fetch<T, VEC>(x + row[u] * ldx, t, 32, at[u], cols);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= rows) break;
            F2 v[P<T>];
            decode<T>(q[u], v);
            if (drop.cut) {
#pragma unroll
                for (int j = 0; j < P<T>; ++j) v[j] = mul2(v[j], f2(d.factor));
                drop.template operator()<T, VEC>(drop.first_of(row[u], cols), t, 32, at[u], v);
            }
            put<T, VEC>(y + row[u] * ldy, t, 32, at[u], cols, encode<T>(v));
        }
    }
}

// ---- host ----
ftp_status check_desc(const ftp_join_desc* d, const char* who) {
    FTP_REQUIRE(d, FTP_EINVAL, "%s: null descriptor", who);
    FTP_REQUIRE(d->precision == FTP_FP32 || d->precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, d->precision);
    FTP_REQUIRE(d->post >= FTP_NORM_NONE && d->post <= FTP_NORM_LAYER && d->pre >= FTP_NORM_NONE && d->pre <= FTP_NORM_LAYER, FTP_EINVAL, "%s: unknown norm", who);
    FTP_REQUIRE(d->rows >= 0 && d->cols >= 1 && d->gate_rows >= 0, FTP_EINVAL, "%s: rows and gate_rows must not be negative, cols must be positive", who);
    FTP_REQUIRE(d->cols <= 16384, FTP_EUNSUPPORTED, "%s: rows of more than 16384 columns", who);
    FTP_REQUIRE(d->rows < (1ll << 31) && d->gate_rows < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    FTP_REQUIRE(d->eps >= 0.f && d->eps <= 3e38f && d->alpha - d->alpha == 0.f && d->beta - d->beta == 0.f, FTP_EINVAL, "%s: eps, alpha and beta must be finite, eps not negative", who);
    Drop drop;
    if (ftp_status s = drop_of(&drop, d->dropout, reinterpret_cast<const void*>(8), d->site, d->row0, d->rows, d->cols, who)) return s;
    return check_pitches({d->ldu, d->ldx, d->lds, d->ldy, d->ldg, d->lddu, d->ldds, d->lddx, d->lddg}, d->cols, who);
}

void fill(JoinArgs& a, const ftp_join_desc* d) {
    const auto ld = [&](int64_t v) { return v ? v : (int64_t)d->cols; };
    a.rows = d->rows; a.cols = d->cols; a.post = d->post; a.pre = d->pre;
    a.eps = d->eps; a.alpha = d->alpha; a.beta = d->beta; a.per_col = (float)(1.0 / d->cols);
    a.ldu = ld(d->ldu); a.ldx = ld(d->ldx); a.lds = ld(d->lds); a.ldy = ld(d->ldy); a.ldg = ld(d->ldg);
    a.lddu = ld(d->lddu); a.ldds = ld(d->ldds); a.lddx = ld(d->lddx); a.lddg = ld(d->lddg);
    a.gate_rows = d->gate_rows;
}
template <typename T> bool fills(const JoinArgs& a, int groups) { return (int64_t)a.threads * V<T> * groups == a.cols; }
// every row of it starts on 16 bytes
template <typename T> bool wide(const void* p, int64_t ld, int64_t rows) { return !p || (on_bytes(p, 16) && (rows <= 1 || ld * (int64_t)sizeof(T) % 16 == 0)); }
bool wide_vectors(std::initializer_list<const void*> all) {
    for (const void* p : all) if (!on_bytes(p, 16)) return false;
    return true;
}

template <typename T, int G>
void forward_of(const JoinArgs& a, bool vec, cudaStream_t st) {
    const dim3 grid((unsigned)std::min<int64_t>(a.rows, SMS * std::min(32, forward_threads(G * V<T>) / a.threads)));
    launch(vec ? join_forward_kernel<T, G, true> : join_forward_kernel<T, G, false>, grid, dim3(a.threads), 0, st, a);
}
// columns of a thread: as many groups as leave every multiprocessor 512 threads, up to 32 columns
inline int groups_for(int64_t rows, int cols, int v) {
    int most = 1;
    while (most < 32 / v && rows * cols >= (int64_t)SMS * 512 * v * most * 2) most *= 2;
    return most;
}
template <typename T>
void run_forward(JoinArgs& a, cudaStream_t st) {
    int groups;
    row_shape(a.cols, V<T>, groups_for(a.rows, a.cols, V<T>), &a.threads, &groups);
    const bool vec = a.cols % V<T> == 0 && wide<T>(a.u, a.ldu, a.rows) && wide<T>(a.x, a.ldx, a.rows) && wide<T>(a.s, a.lds, a.rows) && wide<T>(a.y, a.ldy, a.rows) &&
                     (a.gate_rows ? wide<T>(a.gate, a.ldg, 2) : on_bytes(a.gate, 16)) && wide_vectors({a.w_post, a.b_post, a.w_pre, a.b_pre});
    a.full = fills<T>(a, groups);
    switch (groups) {
        case 1: forward_of<T, 1>(a, vec, st); break;
        case 2: forward_of<T, 2>(a, vec, st); break;
        case 4: forward_of<T, 4>(a, vec, st); break;
        default: if constexpr (sizeof(T) == 4) forward_of<T, 8>(a, vec, st);
    }
}

// The backward pass's work on its rows: runs of up to 64 rows (the float additions of a running sum), as long as give all blocks that the GPU
// holds the same, once or more often (12000 x 3584 bf16 with runs of 64: 250 us, 173 with 41).  Eight columns a thread, two rows at a time, or
// sixteen.  Up to 2048 columns eight (12000 x 2048 bf16, 8 and 16: both rms 95 and 107 us, layer norms 146 and 196, the second norm alone 67 and 71).  bf16
// above: sixteen, except for both rms over 2560.  Up to 2560 columns these are 160 threads, of which three blocks fit and of the other kind one (12000 x 2560
// 140 and 127 us); from there on two and one (2568: 144 and 153, 2624: 147 and 156, 3328: 175 and 177, 4096: 193 and 195).  Layer norms take a row
// at a time anyway (2176: 226 and 172, 3328: 278 and 247; but 4096 with gate and dropout 310 and 332), the second norm alone is bound by memory sooner (2176: 89 and
// 75, 4096: 130 and 126).  Float up to 4096: eight (8000 x 2176 both rms 128 and 154, 4096 212 and 237, layer norms 220 and 251).
struct JoinPlan { int threads, groups, run; int64_t blocks; };
JoinPlan plan_backward(const ftp_join_desc* d) {
    JoinPlan p;
    const int v = d->precision == FTP_FP32 ? 4 : 8;
    const bool layer = d->post == FTP_NORM_LAYER || d->pre == FTP_NORM_LAYER, few = d->cols <= 2048 || (d->cols <= 4096 && (v == 4 || (d->post && !layer && d->cols > 2560)));
    row_shape(d->cols, v, (few ? 8 : 16) / v, &p.threads, &p.groups);
    const int64_t each = (int64_t)SMS * std::min(16, BACKWARD_THREADS / p.threads);
    const int64_t turns = std::max<int64_t>(1, (d->rows + 64 * each - 1) / (64 * each));                  // of the GPU's blocks: whole ones
    p.run = (int)std::max<int64_t>(4, (d->rows + each * turns - 1) / (each * turns));
    p.blocks = (d->rows + p.run - 1) / p.run;
    return p;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
constexpr size_t MOST_SMEM = 200 * 1024, KERNEL_SMEM = 220 * 1024;  // for the running sums, and with the rows ahead
struct JoinSpace { size_t sums, gate, spill, total; };
JoinSpace space_of(const ftp_join_desc* d, const JoinPlan& p, int nsums) {
    const int v = d->precision == FTP_FP32 ? 4 : 8;
    const size_t running = (size_t)nsums * p.groups * v * p.threads * 4;
    JoinSpace s{};
    s.sums = p.blocks > 1 ? up256((size_t)p.blocks * nsums * d->cols * 4) : 0;
    if (d->gate_rows > 1) s.gate = up256((size_t)(p.blocks + (d->rows + d->gate_rows - 1) / d->gate_rows) * d->cols * 4);
    s.spill = running > MOST_SMEM ? up256((size_t)p.blocks * running) : 0;
    s.total = s.sums + s.gate + s.spill;
    return s;
}

template <typename T, int G, int KIND> void (*backward_kernel(bool vec, bool layer))(JoinArgs) {
    return layer ? (vec ? join_backward_kernel<T, G, true, true, KIND> : join_backward_kernel<T, G, false, true, KIND>)
                 : (vec ? join_backward_kernel<T, G, true, false, KIND> : join_backward_kernel<T, G, false, false, KIND>);
}
template <typename T, int G>
ftp_status backward_of(JoinArgs& a, const JoinPlan& p, bool vec, int kind, cudaStream_t st, const char* who) {
    size_t smem = (size_t)a.nsums * G * V<T> * p.threads * 4;           // 160 KB at most: only rows of more columns a thread spill their sums
    const bool layer = a.post == FTP_NORM_LAYER || a.pre == FTP_NORM_LAYER;
    void (*kern)(JoinArgs) = nullptr;
    size_t staged = 0;
    if constexpr (G * V<T> <= 16) {
        if (kind == BOTH) kern = backward_kernel<T, G, BOTH>(vec, layer);
        else if (kind == PRE_ONLY) kern = backward_kernel<T, G, PRE_ONLY>(vec, layer);
        if (kern && vec) staged = (size_t)(!layer && G * V<T> <= 8 ? PAIR : 1) * 4 * G * 16 * p.threads;
        if (smem + staged > KERNEL_SMEM) { kern = nullptr; staged = 0; }                                      // five sums beside the rows ahead: bf16 over 7680 columns, float over 6144
    }
    if (!kern) kern = backward_kernel<T, G, ANY>(vec, layer);
    smem += staged;
    // 48 KB with what the kernel holds beside it
    if (smem > 40 * 1024) FTP_REQUIRE(more_shared(reinterpret_cast<const void*>(kern), KERNEL_SMEM), FTP_ECUDA, "%s: no shared memory", who);
    launch(kern, dim3((unsigned)p.blocks), dim3(p.threads), smem, st, a);
    return FTP_OK;
}
template <typename T> bool wide_rows(const JoinArgs& a) {
    return a.cols % V<T> == 0 && wide<T>(a.u, a.ldu, a.rows) && wide<T>(a.s, a.lds, a.rows) && wide<T>(a.dy, a.ldy, a.rows) && wide<T>(a.ds, a.ldds, a.rows) &&
           wide<T>(a.du, a.lddu, a.rows) && wide<T>(a.dx, a.lddx, a.rows) && (a.gate_rows ? wide<T>(a.gate, a.ldg, 2) : on_bytes(a.gate, 16)) &&
           (a.gate_rows != 1 || wide<T>(a.dgate, a.lddg, a.rows)) && wide_vectors({a.w_post, a.b_post, a.w_pre, a.out[0], a.out[1], a.out[2], a.out[3], a.out[4]});
}
template <typename T>
ftp_status run_backward(JoinArgs& a, const JoinPlan& p, int kind, cudaStream_t st, const char* who) {
    a.threads = p.threads;
    a.groups = p.groups;
    a.full = fills<T>(a, p.groups);
    const bool vec = wide_rows<T>(a);
    if (p.groups * V<T> > 16) {
        const bool layer = a.post == FTP_NORM_LAYER || a.pre == FTP_NORM_LAYER;
        auto kern = layer ? (vec ? join_backward_wide_kernel<T, true, true> : join_backward_wide_kernel<T, false, true>)
                          : (vec ? join_backward_wide_kernel<T, true, false> : join_backward_wide_kernel<T, false, false>);
        const size_t smem = a.spill ? 0 : (size_t)a.nsums * p.groups * V<T> * p.threads * 4;
        FTP_REQUIRE(more_shared(reinterpret_cast<const void*>(kern), KERNEL_SMEM), FTP_ECUDA, "%s: no shared memory", who);
        launch(kern, dim3((unsigned)p.blocks), dim3(p.threads), smem, st, a);
        return FTP_OK;
    }
    switch (p.groups) {
        case 1: return backward_of<T, 1>(a, p, vec, kind, st, who);
        case 2: return backward_of<T, 2>(a, p, vec, kind, st, who);
        case 4: if constexpr (sizeof(T) == 4) return backward_of<T, 4>(a, p, vec, kind, st, who);
    }
    return FTP_OK;
}

ftp_status zero_vectors(std::initializer_list<float*> all, int cols, cudaStream_t st, const char* who) {
    for (float* p : all)
        if (p) FTP_REQUIRE(told(cudaMemsetAsync(p, 0, (size_t)cols * 4, st)) == cudaSuccess, FTP_ECUDA, "%s: memset failed", who);
    return FTP_OK;
}

}  // namespace
}  // namespace token
}  // namespace ftp

using namespace ftp;
using namespace ftp::token;

extern "C" {

ftp_status ftp_join_forward(const ftp_join_desc* d, const void* u, const void* x, const float* w_post, const float* b_post, const void* gate, const float* w_pre,
                            const float* b_pre, const void* rng, void* s, void* y, float* stats, void* stream) {
    const char* who = "join_forward";
    if (ftp_status e = check_desc(d, who)) return e;
    if (d->rows == 0) return FTP_OK;
    FTP_REQUIRE(u || x, FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE((y != nullptr) == (d->pre != FTP_NORM_NONE), FTP_EINVAL, "%s: y is the result of the second norm, and only of that", who);
    FTP_REQUIRE((s != nullptr) == (u != nullptr), FTP_EINVAL, "%s: s is the sum with u, and only that", who);
    FTP_REQUIRE(u || (d->post == FTP_NORM_NONE && !gate && d->dropout == 0.0 && d->alpha == 1.f), FTP_EINVAL, "%s: without u there is the second norm of x alone", who);
    FTP_REQUIRE(d->post != FTP_NORM_NONE || (!w_post && !b_post), FTP_EINVAL, "%s: weights of a norm that is not there", who);
    FTP_REQUIRE(d->pre != FTP_NORM_NONE || (!w_pre && !b_pre), FTP_EINVAL, "%s: weights of a norm that is not there", who);
    FTP_REQUIRE(gate || d->gate_rows == 0, FTP_EINVAL, "%s: gate_rows without a gate", who);
    const size_t e = d->precision == FTP_FP32 ? 4 : 2;
    if (ftp_status r = check_elements({u, x, s, y, d->gate_rows ? gate : nullptr}, e, who)) return r;
    if (ftp_status r = check_elements({w_post, b_post, w_pre, b_pre, stats, d->gate_rows ? nullptr : gate}, 4, who)) return r;
    if (ftp_status r = check_addresses({s, y, stats}, {u, w_post, b_post, gate, w_pre, b_pre, rng}, who)) return r;
    if (ftp_status r = check_addresses({y, stats}, {x}, who)) return r;
    if (ftp_status r = check_in_place(x, s, d->ldx, d->lds, d->rows, d->cols, who)) return r;
    JoinArgs a{};
    fill(a, d);
    if (ftp_status r = drop_of(&a.drop, u ? d->dropout : 0.0, rng, d->site, d->row0, d->rows, d->cols, who)) return r;
    a.u = u; a.x = x; a.gate = gate; a.s = s; a.y = y; a.stats = stats;
    a.w_post = w_post; a.b_post = b_post; a.w_pre = w_pre; a.b_pre = b_pre;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (d->precision == FTP_FP32) run_forward<float>(a, st); else run_forward<bf16>(a, st);
    return launched(who);
}

ftp_status ftp_join_workspace_bytes(const ftp_join_desc* d, size_t* bytes) {
    if (ftp_status e = check_desc(d, "join_workspace_bytes")) return e;
    FTP_REQUIRE(bytes, FTP_EINVAL, "join_workspace_bytes: null argument");
    *bytes = d->rows ? space_of(d, plan_backward(d), SUMS).total : 0;
    return FTP_OK;
}

ftp_status ftp_join_backward(const ftp_join_desc* d, const void* u, const void* s, const float* w_post, const float* b_post, const void* gate, const float* w_pre,
                             const float* stats, const void* rng, const void* dy, const void* ds, void* du, void* dx, float* dw_post, float* db_post,
                             float* dw_pre, float* db_pre, void* dgate, void* ws, size_t ws_bytes, void* stream) {
    const char* who = "join_backward";
    if (ftp_status e = check_desc(d, who)) return e;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    FTP_REQUIRE(d->post != FTP_NORM_NONE || (!w_post && !b_post && !dw_post && !db_post), FTP_EINVAL, "%s: weights of a norm that is not there", who);
    FTP_REQUIRE(d->pre != FTP_NORM_NONE || (!w_pre && !dw_pre && !db_pre && !dy), FTP_EINVAL, "%s: weights or gradients of a norm that is not there", who);
    FTP_REQUIRE((gate || d->gate_rows == 0) && (gate || !dgate), FTP_EINVAL, "%s: a gate's rows or gradient without a gate", who);
    const size_t e = d->precision == FTP_FP32 ? 4 : 2;
    if (ftp_status r = check_elements({w_post, b_post, w_pre, stats, dw_post, db_post, dw_pre, db_pre, d->gate_rows ? nullptr : gate, d->gate_rows ? nullptr : dgate}, 4, who)) return r;
    if (ftp_status r = check_addresses({du, dx, dw_post, db_post, dw_pre, db_pre, dgate}, {u, s, w_post, b_post, gate, w_pre, stats, rng, dy}, who)) return r;
    if (ftp_status r = check_addresses({du, dw_post, db_post, dw_pre, db_pre, dgate}, {ds}, who)) return r;
    if (d->rows == 0) return zero_vectors({dw_post, db_post, dw_pre, db_pre, d->gate_rows ? nullptr : static_cast<float*>(dgate)}, d->cols, st, who);
    FTP_REQUIRE(dy || d->pre == FTP_NORM_NONE, FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(dy || ds, FTP_EINVAL, "%s: no gradient comes in", who);
    FTP_REQUIRE(s || d->pre == FTP_NORM_NONE, FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(u || (d->post == FTP_NORM_NONE && !dgate), FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(stats || (d->post == FTP_NORM_NONE && d->pre == FTP_NORM_NONE), FTP_EINVAL, "%s: a norm's backward pass needs its statistics", who);
    if (ftp_status r = check_elements({u, s, dy, ds, du, dx, d->gate_rows ? gate : nullptr, d->gate_rows ? dgate : nullptr}, e, who)) return r;
    if (ftp_status r = check_in_place(ds, dx, d->ldds, d->lddx, d->rows, d->cols, who)) return r;
    const JoinPlan p = plan_backward(d);
    const size_t need = space_of(d, p, SUMS).total;
    FTP_REQUIRE(need == 0 || (ws && ws_bytes >= need), FTP_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need);
    FTP_REQUIRE(need == 0 || on_bytes(ws, 256), FTP_ERANGE, "%s: workspace must start on a 256-byte boundary", who);
    JoinArgs a{};
    fill(a, d);
    if (ftp_status r = drop_of(&a.drop, d->dropout, rng, d->site, d->row0, d->rows, d->cols, who)) return r;
    a.u = u; a.s = const_cast<void*>(s); a.gate = gate; a.dy = dy; a.ds = ds; a.du = du; a.dx = dx; a.dgate = dgate;
    a.w_post = w_post; a.b_post = b_post; a.w_pre = w_pre; a.stats = const_cast<float*>(stats);
    a.run = p.run;
    const bool shared_gate = dgate && d->gate_rows > 1;
    float* out[SUMS] = {dw_pre, db_pre, dw_post, db_post, d->gate_rows ? nullptr : static_cast<float*>(dgate)};
    JoinSums j{};
    for (int i = 0; i < SUMS; ++i) {
        a.out[i] = out[i];
        a.at[i] = out[i] || (i == SUM_GATE && shared_gate) ? a.nsums : -1;
        if (out[i]) j.out[a.nsums] = out[i];
        if (a.at[i] >= 0) ++a.nsums;
    }
    // what the kernels for the usual calls take as known
    const bool layer = d->post == FTP_NORM_LAYER || d->pre == FTP_NORM_LAYER;
    int kind = ANY;
    if (d->pre != FTP_NORM_NONE && w_pre && dw_pre && u && ds && dx && du && (layer || (!b_post && !db_post && !db_pre))) {
        if (d->post == FTP_NORM_NONE) kind = PRE_ONLY;
        else if (w_post && dw_post) kind = BOTH;
    }
    const JoinSpace sp = space_of(d, p, SUMS), now = space_of(d, p, a.nsums);
    char* base = static_cast<char*>(ws);
    a.sums = reinterpret_cast<float*>(base);
    if (shared_gate) a.gate_sums = reinterpret_cast<float*>(base + sp.sums);
    if (now.spill) a.spill = reinterpret_cast<float*>(base + sp.sums + sp.gate);
    if (ftp_status r = d->precision == FTP_FP32 ? run_backward<float>(a, p, kind, st, who) : run_backward<bf16>(a, p, kind, st, who)) return r;
    const int n = a.nsums - shared_gate;
    if (n && p.blocks > 1) {
        j.part = a.sums; j.n = n; j.cols = d->cols; j.blocks = p.blocks;
        launch(join_sums_kernel, dim3((d->cols + 31) / 32, n), dim3(1024), 0, st, j);
    }
    if (shared_gate) {
        const int64_t groups = (d->rows + d->gate_rows - 1) / d->gate_rows;
        const dim3 grid((d->cols + 127) / 128, (unsigned)std::min<int64_t>(groups, 32768));
        if (d->precision == FTP_FP32) launch(join_gate_kernel<float>, grid, dim3(128), 0, st, (const float*)a.gate_sums, groups, a.gate_rows, a.rows, a.run, a.cols, static_cast<float*>(dgate), a.lddg);
        else launch(join_gate_kernel<bf16>, grid, dim3(128), 0, st, (const float*)a.gate_sums, groups, a.gate_rows, a.rows, a.run, a.cols, static_cast<bf16*>(dgate), a.lddg);
    }
    return launched(who);
}

ftp_status ftp_dropout(const void* x, void* y, int64_t rows, int32_t cols, int64_t ldx, int64_t ldy, int32_t precision, double dropout, const void* rng, int32_t site,
                       int64_t row0, void* stream) {
    const char* who = "dropout";
    FTP_REQUIRE(precision == FTP_FP32 || precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, precision);
    FTP_REQUIRE(rows >= 0 && cols >= 1, FTP_EINVAL, "%s: rows must not be negative, cols must be positive", who);
    FTP_REQUIRE(rows < (1ll << 38) && cols < (1 << 30) && rows * (double)cols <= 274877906944.0, FTP_ERANGE, "%s: tensor too large", who);
    if (ftp_status r = check_pitches({ldx, ldy}, cols, who)) return r;
    Drop drop;
    if (ftp_status r = drop_of(&drop, dropout, rng, site, row0, rows, cols, who)) return r;
    if (rows == 0) return FTP_OK;
    FTP_REQUIRE(x && y, FTP_EINVAL, "%s: null buffer", who);
    if (ftp_status r = check_elements({x, y}, precision == FTP_FP32 ? 4 : 2, who)) return r;
    if (ftp_status r = check_addresses({y}, {rng}, who)) return r;
    if (ftp_status r = check_in_place(x, y, ldx, ldy, rows, cols, who)) return r;
    if (!ldx) ldx = cols;
    if (!ldy) ldy = cols;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const auto go = [&](auto one) {
        typedef decltype(one) T;
        const int64_t pieces = rows * ((cols + 32 * V<T> - 1) / (32 * V<T>));
        const dim3 grid((unsigned)std::min<int64_t>((pieces + 31) / 32, SMS * 64));
        const bool vec = cols % V<T> == 0 && wide<T>(x, ldx, rows) && wide<T>(y, ldy, rows);
        launch(vec ? dropout_kernel<T, true> : dropout_kernel<T, false>, grid, dim3(256), 0, st, static_cast<const T*>(x), static_cast<T*>(y), rows, cols, ldx, ldy, drop);
    };
    if (precision == FTP_FP32) go(float{}); else go(bf16{});
    return launched(who);
}

}  // extern "C"
