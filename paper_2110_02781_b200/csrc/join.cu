// A block's result joins the residual stream: s = alpha x + beta gate drop(post(u)), and the next block's input y = pre(s), in one
// pass over the tokens each way; and dropout by itself.
//
// Bound by memory: the forward pass reads u, x and writes s, y; the backward pass reads u, s, dy, ds and writes du, dx.  A row lies
// in the registers of 32 to 512 threads (16 bytes of columns each, one to eight times), a block of 512 threads holds one row or
// several; every sum over a row is one exchange between its warps.  The column sums of the backward pass (gradients of the norms'
// weights and of a gate that many rows share) grow in shared memory, each thread its own columns, over at most 64 rows, and a
// second kernel adds the blocks' sums in double, in a fixed order.
#include <algorithm>
#include "token.cuh"

namespace ftp {
namespace token {
namespace {

constexpr int THREADS = 512;
enum { SUM_W_PRE, SUM_B_PRE, SUM_W_POST, SUM_B_POST, SUM_GATE, SUMS };

struct JoinArgs {
    const void *u, *x, *gate, *dy, *ds;
    void *s, *y, *du, *dx, *dgate;           // s: written by the forward pass, read by the backward pass
    const float *w_post, *b_post, *w_pre, *b_pre;
    float* stats;                            // four planes of `rows`: mean and 1 / deviation of u, of s
    int64_t rows, ldu, ldx, lds, ldy, ldg, lddu, ldds, lddx, lddg, gate_rows;
    int cols, threads, post, pre;
    float eps, alpha, beta, per_col;         // per_col: 1 / cols
    Drop drop;
    // backward
    float *sums, *gate_sums, *spill;         // blocks' column sums; a shared gate's sums; the running sums where shared memory is too small
    float* out[SUMS];                        // where the column sums go when there is one block
    int at[SUMS], nsums, run;                // place of each sum or -1; rows of a run (the rows that one row's threads walk)
    int64_t runs;
};

// a row of the gate: a float vector, or a row of the tensors' type for every gate_rows rows
template <typename T, bool VEC> __device__ __forceinline__ void gate_of(const JoinArgs& a, int64_t row, int t, int g, float (&v)[V<T>]) {
    if (!a.gate || a.gate_rows == 0) fetch_vector<T, VEC>(static_cast<const float*>(a.gate), 1.f, t, a.threads, g, a.cols, v);
    else decode<T>(fetch<T, VEC>(static_cast<const T*>(a.gate) + row / a.gate_rows * a.ldg, t, a.threads, g, a.cols), v);
}

// 1 / deviation and mean of the rows in v; what lies behind the last column is 0 and stays out of the sums
template <typename T, int G, bool VEC> __device__ __forceinline__ float2 moments(const JoinArgs& a, int kind, const float (&v)[G][V<T>], int t, RowSum& sum) {
    float mean = 0.f, q = 0.f;
    if (kind == FTP_NORM_LAYER) {
        float p = 0.f;
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
            for (int j = 0; j < V<T>; ++j) p += v[g][j];
        mean = sum(p, 0.f).x * a.per_col;
    }
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int j = 0; j < V<T>; ++j) {
            const float d = VEC ? (column<T, VEC>(t, a.threads, g, 0) < a.cols ? v[g][j] - mean : 0.f) : (column<T, VEC>(t, a.threads, g, j) < a.cols ? v[g][j] - mean : 0.f);
            q = fmaf(d, d, q);
        }
    return make_float2(mean, 1.f / sqrtf(fmaf(sum(q, 0.f).x, a.per_col, a.eps)));
}

template <typename T, int G, bool VEC>
__global__ void __launch_bounds__(THREADS, G == 1 ? 3 : G == 2 ? 2 : 1) join_forward_kernel(const JoinArgs a) {
    __shared__ float2 red[32];
    grid_dep_sync();
    Drop drop = a.drop;
    drop.begin();
    RowSum sum{red, a.threads, 0};
    const int t = threadIdx.x & (a.threads - 1), slot = threadIdx.x / a.threads, slots = THREADS / a.threads;
    for (int64_t r0 = (int64_t)blockIdx.x * slots; r0 < a.rows; r0 += (int64_t)gridDim.x * slots) {
        const bool on = r0 + slot < a.rows;
        const int64_t row = on ? r0 + slot : a.rows - 1;
        float v[G][V<T>];
        uint4 x[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            x[g] = a.x ? fetch<T, VEC>(static_cast<const T*>(a.x) + row * a.ldx, t, a.threads, g, a.cols) : make_uint4(0u, 0u, 0u, 0u);
            decode<T>(a.u ? fetch<T, VEC>(static_cast<const T*>(a.u) + row * a.ldu, t, a.threads, g, a.cols) : x[g], v[g]);
        }
        if (a.u) {
            if (a.post != FTP_NORM_NONE) {
                const float2 m = moments<T, G, VEC>(a, a.post, v, t, sum);
                if (a.stats && on && t == 0) { a.stats[row] = m.x; a.stats[a.rows + row] = m.y; }
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    float w[V<T>], b[V<T>];
                    fetch_vector<T, VEC>(a.w_post, 1.f, t, a.threads, g, a.cols, w);
                    fetch_vector<T, VEC>(a.b_post, 0.f, t, a.threads, g, a.cols, b);
#pragma unroll
                    for (int j = 0; j < V<T>; ++j) v[g][j] = fmaf((v[g][j] - m.x) * m.y, w[j], b[j]);
                }
            }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float w[V<T>], r[V<T>];
                gate_of<T, VEC>(a, row, t, g, w);
                const unsigned keep = drop.cut ? drop.keep<T, VEC>(row, t, a.threads, g, a.cols) : ~0u;
                const float f = drop.cut ? drop.factor : 1.f;
                decode<T>(x[g], r);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) {
                    const float d = keep >> j & 1 ? v[g][j] * f : 0.f;
                    v[g][j] = fmaf(a.beta, d * w[j], a.alpha * r[j]);
                }
                x[g] = encode<T>(v[g]);                              // the stream goes on in the tensors' type, here too
                if (on) put<T, VEC>(static_cast<T*>(a.s) + row * a.lds, t, a.threads, g, a.cols, x[g]);
                decode<T>(x[g], v[g]);
            }
        }
        if (a.pre != FTP_NORM_NONE) {
            if constexpr (VEC) {
#pragma unroll
                for (int g = 0; g < G; ++g)
                    if (column<T, VEC>(t, a.threads, g, 0) >= a.cols)
#pragma unroll
                        for (int j = 0; j < V<T>; ++j) v[g][j] = 0.f;
            } else {
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int j = 0; j < V<T>; ++j)
                        if (column<T, VEC>(t, a.threads, g, j) >= a.cols) v[g][j] = 0.f;
            }
            const float2 m = moments<T, G, VEC>(a, a.pre, v, t, sum);
            if (a.stats && on && t == 0) { a.stats[2 * a.rows + row] = m.x; a.stats[3 * a.rows + row] = m.y; }
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float w[V<T>], b[V<T>];
                fetch_vector<T, VEC>(a.w_pre, 1.f, t, a.threads, g, a.cols, w);
                fetch_vector<T, VEC>(a.b_pre, 0.f, t, a.threads, g, a.cols, b);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) w[j] = fmaf((v[g][j] - m.x) * m.y, w[j], b[j]);
                if (on) put<T, VEC>(static_cast<T*>(a.y) + row * a.ldy, t, a.threads, g, a.cols, encode<T>(w));
            }
        }
    }
}

// A thread's running sum number `i` (of V columns): float4s that lie a block's width apart
template <typename T> struct Running {
    float4* at;
    __device__ __forceinline__ float4& q(int i, int k) const { return at[(i * (V<T> / 4) + k) * THREADS]; }
    __device__ __forceinline__ void add(int i, const float (&v)[V<T>]) const {
#pragma unroll
        for (int k = 0; k < V<T> / 4; ++k) {
            float4 f = q(i, k);
            f.x += v[4 * k]; f.y += v[4 * k + 1]; f.z += v[4 * k + 2]; f.w += v[4 * k + 3];
            q(i, k) = f;
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

// D = ds + r (g - mean(g) - x^ mean(g x^)), g = dy w_pre, x^ = (s - mean) r  (mean(g) with the layer norm only)
// dx = alpha D;  dv = beta D gate mask / (1 - p);  du from dv w_post in the same way;  dgate = beta D drop(v)
template <typename T, int G, bool VEC>
__global__ void __launch_bounds__(THREADS, G == 1 ? 2 : 1) join_backward_kernel(const JoinArgs a) {
    extern __shared__ float4 dynamic[];
    __shared__ float2 red[32];
    grid_dep_sync();
    Drop drop = a.drop;
    drop.begin();
    RowSum sum{red, a.threads, 0};
    const int t = threadIdx.x & (a.threads - 1), slot = threadIdx.x / a.threads, slots = THREADS / a.threads;
    const int quads = G * (V<T> / 4);
    const Running<T> run{(a.spill ? reinterpret_cast<float4*>(a.spill) + (size_t)blockIdx.x * a.nsums * quads * THREADS : dynamic) + threadIdx.x};
    for (int i = 0; i < a.nsums * G; ++i) run.clear(i);
    const int64_t mine = (int64_t)blockIdx.x * slots + slot, first = mine * a.run;
    int64_t group = a.gate_rows > 1 ? first / a.gate_rows : 0, next = a.gate_rows > 1 ? (group + 1) * a.gate_rows : 0;   // next: first row of the next group
    for (int i = 0; i < a.run; ++i) {
        const int64_t row = first + i;
        const bool on = row < a.rows;
        const int64_t safe = on ? row : a.rows - 1;
        if (a.gate_sums && on && row == next) {                      // another group: its predecessor's sum is complete as far as this run goes
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float v[V<T>];
                run.get(a.at[SUM_GATE] * G + g, v);
                put_vector<T, VEC>(a.gate_sums + (mine + group) * a.cols, t, a.threads, g, a.cols, v);
                run.clear(a.at[SUM_GATE] * G + g);
            }
            ++group;
            next += a.gate_rows;
        }
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        uint4 ru[G], rs[G], rdy[G], rds[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            rs[g] = a.pre != FTP_NORM_NONE ? fetch<T, VEC>(static_cast<const T*>(a.s) + safe * a.lds, t, a.threads, g, a.cols) : zero;
            rdy[g] = a.dy && on ? fetch<T, VEC>(static_cast<const T*>(a.dy) + safe * a.ldy, t, a.threads, g, a.cols) : zero;
            rds[g] = a.ds && on ? fetch<T, VEC>(static_cast<const T*>(a.ds) + safe * a.ldds, t, a.threads, g, a.cols) : zero;
            ru[g] = a.u ? fetch<T, VEC>(static_cast<const T*>(a.u) + safe * a.ldu, t, a.threads, g, a.cols) : zero;
        }
        float2 ms = make_float2(0.f, 0.f), mu = make_float2(0.f, 1.f), c = make_float2(0.f, 0.f);
        if (a.post != FTP_NORM_NONE) mu = make_float2(a.stats[safe], a.stats[a.rows + safe]);
        if (a.pre != FTP_NORM_NONE) {
            ms = make_float2(a.stats[2 * a.rows + safe], a.stats[3 * a.rows + safe]);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                float s[V<T>], dy[V<T>], w[V<T>];
                decode<T>(rs[g], s);
                decode<T>(rdy[g], dy);
                fetch_vector<T, VEC>(a.w_pre, 1.f, t, a.threads, g, a.cols, w);
                if (a.at[SUM_B_PRE] >= 0 && on) run.add(a.at[SUM_B_PRE] * G + g, dy);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) {
                    s[j] = (s[j] - ms.x) * ms.y;
                    const float p = dy[j] * w[j];
                    c.x += p;
                    c.y = fmaf(p, s[j], c.y);
                    s[j] *= dy[j];
                }
                if (a.at[SUM_W_PRE] >= 0 && on) run.add(a.at[SUM_W_PRE] * G + g, s);
            }
            c = sum(c.x, c.y);
            c.x = a.pre == FTP_NORM_LAYER ? c.x * a.per_col : 0.f;
            c.y *= a.per_col;
        }
        float dv[G][V<T>];
        float2 e = make_float2(0.f, 0.f);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float d[V<T>], p[V<T>], q[V<T>];
            decode<T>(rds[g], d);
            if (a.pre != FTP_NORM_NONE) {
                float w[V<T>];
                decode<T>(rs[g], p);
                decode<T>(rdy[g], q);
                fetch_vector<T, VEC>(a.w_pre, 1.f, t, a.threads, g, a.cols, w);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) d[j] = fmaf(ms.y, fmaf(q[j], w[j], -c.x) - (p[j] - ms.x) * ms.y * c.y, d[j]);
            }
            if (a.dx && on) {
#pragma unroll
                for (int j = 0; j < V<T>; ++j) p[j] = a.alpha * d[j];
                put<T, VEC>(static_cast<T*>(a.dx) + row * a.lddx, t, a.threads, g, a.cols, encode<T>(p));
            }
            const unsigned keep = drop.cut ? drop.keep<T, VEC>(safe, t, a.threads, g, a.cols) : ~0u;
            const float f = drop.cut ? a.beta * drop.factor : a.beta;
#pragma unroll
            for (int j = 0; j < V<T>; ++j) d[j] = keep >> j & 1 ? d[j] * f : 0.f;      // beta D mask / (1 - p)
            decode<T>(ru[g], q);
#pragma unroll
            for (int j = 0; j < V<T>; ++j) q[j] = (q[j] - mu.x) * mu.y;
            if (a.dgate) {
                float w[V<T>], b[V<T>];
                fetch_vector<T, VEC>(a.w_post, 1.f, t, a.threads, g, a.cols, w);
                fetch_vector<T, VEC>(a.b_post, 0.f, t, a.threads, g, a.cols, b);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) p[j] = keep >> j & 1 ? d[j] * fmaf(q[j], w[j], b[j]) : 0.f;
                if (a.gate_rows == 1) {
                    if (on) put<T, VEC>(static_cast<T*>(a.dgate) + row * a.lddg, t, a.threads, g, a.cols, encode<T>(p));
                } else if (on) run.add(a.at[SUM_GATE] * G + g, p);
            }
            gate_of<T, VEC>(a, safe, t, g, p);
#pragma unroll
            for (int j = 0; j < V<T>; ++j) d[j] *= p[j];
            if (a.at[SUM_B_POST] >= 0 && on) run.add(a.at[SUM_B_POST] * G + g, d);
            if (a.at[SUM_W_POST] >= 0 && on) {
#pragma unroll
                for (int j = 0; j < V<T>; ++j) p[j] = d[j] * q[j];
                run.add(a.at[SUM_W_POST] * G + g, p);
            }
            if (a.post != FTP_NORM_NONE) {
                fetch_vector<T, VEC>(a.w_post, 1.f, t, a.threads, g, a.cols, p);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) {
                    d[j] *= p[j];
                    e.x += d[j];
                    e.y = fmaf(d[j], q[j], e.y);
                }
            }
#pragma unroll
            for (int j = 0; j < V<T>; ++j) dv[g][j] = d[j];
        }
        if (a.post != FTP_NORM_NONE && a.du) {
            e = sum(e.x, e.y);
            e.x = a.post == FTP_NORM_LAYER ? e.x * a.per_col : 0.f;
            e.y *= a.per_col;
        }
        if (a.du && on) {
#pragma unroll
            for (int g = 0; g < G; ++g) {
                if (a.post != FTP_NORM_NONE) {
                    float q[V<T>];
                    decode<T>(ru[g], q);
#pragma unroll
                    for (int j = 0; j < V<T>; ++j) dv[g][j] = mu.y * (dv[g][j] - e.x - (q[j] - mu.x) * mu.y * e.y);
                }
                put<T, VEC>(static_cast<T*>(a.du) + row * a.lddu, t, a.threads, g, a.cols, encode<T>(dv[g]));
            }
        }
    }
    if (a.gate_sums && first < a.rows) {
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float v[V<T>];
            run.get(a.at[SUM_GATE] * G + g, v);
            put_vector<T, VEC>(a.gate_sums + (mine + group) * a.cols, t, a.threads, g, a.cols, v);
        }
    }
    const int n = a.gate_sums ? a.nsums - 1 : a.nsums;               // a shared gate's sum comes last
    if (!n) return;
    __syncthreads();
    // the block's rows joined: the threads of a row's slot take every slots-th piece
    for (int i = slot; i < n * G; i += slots) {
        float all[V<T>] = {};
        for (int s = 0; s < slots; ++s) {
            float v[V<T>];
            Running<T>{run.at - threadIdx.x + s * a.threads + t}.get(i, v);
#pragma unroll
            for (int j = 0; j < V<T>; ++j) all[j] += v[j];
        }
        const int k = i / G;
        float* to = a.sums + ((size_t)blockIdx.x * n + k) * a.cols;
        if (gridDim.x == 1) {
#pragma unroll
            for (int o = 0; o < SUMS; ++o) if (a.at[o] == k) to = a.out[o];
        }
        put_vector<T, VEC>(to, t, a.threads, i - k * G, a.cols, all);
    }
}

// Blocks' column sums joined in double, 16 threads a column.
struct JoinSums { const float* part; float* out[SUMS]; int n, cols; int64_t blocks; };
__global__ void __launch_bounds__(512) join_sums_kernel(const JoinSums a) {
    __shared__ double part[16][33];
    grid_dep_sync();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    double s = 0.0;
    if (c < a.cols)
        for (int64_t b = w; b < a.blocks; b += 16) s += a.part[((size_t)b * a.n + blockIdx.y) * a.cols + c];
    part[w][lane] = s;
    __syncthreads();
    if (w == 0 && c < a.cols) {
        for (int i = 1; i < 16; ++i) s += part[i][lane];
        a.out[blockIdx.y][c] = (float)s;
    }
}
// A group's gate gradient: the sums of the runs that hold rows of it.
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

template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dropout_kernel(const T* x, T* y, int64_t rows, int cols, int64_t ldx, int64_t ldy, Drop drop) {
    grid_dep_sync();
    drop.begin();
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
            float v[V<T>];
            decode<T>(q[u], v);
            if (drop.cut) {
                const unsigned keep = drop.keep<T, VEC>(row[u], t, 32, at[u], cols);
#pragma unroll
                for (int j = 0; j < V<T>; ++j) v[j] = keep >> j & 1 ? v[j] * drop.factor : 0.f;
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
// every row of it starts on 16 bytes
template <typename T> bool wide(const void* p, int64_t ld, int64_t rows) { return !p || (on_bytes(p, 16) && (rows <= 1 || ld * (int64_t)sizeof(T) % 16 == 0)); }
bool wide_vectors(std::initializer_list<const void*> all) {
    for (const void* p : all) if (!on_bytes(p, 16)) return false;
    return true;
}

template <typename T, int G>
void forward_of(const JoinArgs& a, bool vec, cudaStream_t st) {
    const int slots = THREADS / a.threads, per_sm = G == 1 ? 3 : G == 2 ? 2 : 1;
    const dim3 grid((unsigned)std::min<int64_t>((a.rows + slots - 1) / slots, SMS * per_sm));
    if (vec) launch(join_forward_kernel<T, G, true>, grid, dim3(THREADS), 0, st, a);
    else launch(join_forward_kernel<T, G, false>, grid, dim3(THREADS), 0, st, a);
}
template <typename T>
void run_forward(JoinArgs& a, cudaStream_t st) {
    int groups;
    row_shape(a.cols, V<T>, &a.threads, &groups);
    const bool vec = a.cols % V<T> == 0 && wide<T>(a.u, a.ldu, a.rows) && wide<T>(a.x, a.ldx, a.rows) && wide<T>(a.s, a.lds, a.rows) && wide<T>(a.y, a.ldy, a.rows) &&
                     (a.gate_rows ? wide<T>(a.gate, a.ldg, 2) : on_bytes(a.gate, 16)) && wide_vectors({a.w_post, a.b_post, a.w_pre, a.b_pre});
    switch (groups) {
        case 1: forward_of<T, 1>(a, vec, st); break;
        case 2: forward_of<T, 2>(a, vec, st); break;
        case 4: forward_of<T, 4>(a, vec, st); break;
        default: if constexpr (sizeof(T) == 4) forward_of<T, 8>(a, vec, st);
    }
}

// The backward pass's work on its rows: runs of up to 64 rows (the float additions of a running sum), short ones while there are
// fewer than two blocks for every multiprocessor.
struct JoinPlan { int threads, groups, slots, run; int64_t runs, blocks; };
JoinPlan plan_backward(const ftp_join_desc* d) {
    JoinPlan p;
    row_shape(d->cols, d->precision == FTP_FP32 ? 4 : 8, &p.threads, &p.groups);
    p.slots = THREADS / p.threads;
    const int64_t want = (d->rows + (int64_t)p.slots * 2 * SMS - 1) / ((int64_t)p.slots * 2 * SMS);
    p.run = (int)std::min<int64_t>(64, std::max<int64_t>(4, want));
    p.runs = (d->rows + p.run - 1) / p.run;
    p.blocks = (p.runs + p.slots - 1) / p.slots;
    return p;
}
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
constexpr size_t MOST_SMEM = 200 * 1024;
struct JoinSpace { size_t sums, gate, spill, total; };
JoinSpace space_of(const ftp_join_desc* d, const JoinPlan& p, int nsums) {
    const int v = d->precision == FTP_FP32 ? 4 : 8;
    const size_t running = (size_t)nsums * p.groups * v * THREADS * 4;
    JoinSpace s{};
    s.sums = p.blocks > 1 ? up256((size_t)p.blocks * nsums * d->cols * 4) : 0;
    if (d->gate_rows > 1) s.gate = up256((size_t)(p.blocks * p.slots + (d->rows + d->gate_rows - 1) / d->gate_rows) * d->cols * 4);
    s.spill = running > MOST_SMEM ? up256((size_t)p.blocks * running) : 0;
    s.total = s.sums + s.gate + s.spill;
    return s;
}

template <typename T, int G>
ftp_status backward_of(const JoinArgs& a, const JoinPlan& p, bool vec, cudaStream_t st, const char* who) {
    const size_t smem = a.spill ? 0 : (size_t)a.nsums * G * V<T> * THREADS * 4;
    auto kern = vec ? join_backward_kernel<T, G, true> : join_backward_kernel<T, G, false>;
    if (smem > 40 * 1024)                                            // 48 KB with what the kernel holds beside it
        FTP_REQUIRE(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST_SMEM) == cudaSuccess, FTP_ECUDA, "%s: no shared memory", who);
    launch(kern, dim3((unsigned)p.blocks), dim3(THREADS), smem, st, a);
    return FTP_OK;
}
template <typename T>
ftp_status run_backward(JoinArgs& a, const JoinPlan& p, cudaStream_t st, const char* who) {
    a.threads = p.threads;
    const bool vec = a.cols % V<T> == 0 && wide<T>(a.u, a.ldu, a.rows) && wide<T>(a.s, a.lds, a.rows) && wide<T>(a.dy, a.ldy, a.rows) && wide<T>(a.ds, a.ldds, a.rows) &&
                     wide<T>(a.du, a.lddu, a.rows) && wide<T>(a.dx, a.lddx, a.rows) && (a.gate_rows ? wide<T>(a.gate, a.ldg, 2) : on_bytes(a.gate, 16)) &&
                     (a.gate_rows != 1 || wide<T>(a.dgate, a.lddg, a.rows)) && wide_vectors({a.w_post, a.b_post, a.w_pre, a.out[0], a.out[1], a.out[2], a.out[3], a.out[4]});
    switch (p.groups) {
        case 1: return backward_of<T, 1>(a, p, vec, st, who);
        case 2: return backward_of<T, 2>(a, p, vec, st, who);
        case 4: return backward_of<T, 4>(a, p, vec, st, who);
        default: if constexpr (sizeof(T) == 4) return backward_of<T, 8>(a, p, vec, st, who);
    }
    return FTP_OK;
}

ftp_status zero_vectors(std::initializer_list<float*> all, int cols, cudaStream_t st, const char* who) {
    for (float* p : all)
        if (p) FTP_REQUIRE(cudaMemsetAsync(p, 0, (size_t)cols * 4, st) == cudaSuccess, FTP_ECUDA, "%s: memset failed", who);
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
    a.run = p.run; a.runs = p.runs;
    const bool shared_gate = dgate && d->gate_rows > 1;
    float* out[SUMS] = {dw_pre, db_pre, dw_post, db_post, d->gate_rows ? nullptr : static_cast<float*>(dgate)};
    JoinSums j{};
    for (int i = 0; i < SUMS; ++i) {
        a.out[i] = out[i];
        a.at[i] = out[i] || (i == SUM_GATE && shared_gate) ? a.nsums : -1;
        if (out[i]) j.out[a.nsums] = out[i];
        if (a.at[i] >= 0) ++a.nsums;
    }
    const JoinSpace sp = space_of(d, p, SUMS), now = space_of(d, p, a.nsums);
    char* base = static_cast<char*>(ws);
    a.sums = reinterpret_cast<float*>(base);
    if (shared_gate) a.gate_sums = reinterpret_cast<float*>(base + sp.sums);
    if (now.spill) a.spill = reinterpret_cast<float*>(base + sp.sums + sp.gate);
    if (ftp_status r = d->precision == FTP_FP32 ? run_backward<float>(a, p, st, who) : run_backward<bf16>(a, p, st, who)) return r;
    const int n = a.nsums - shared_gate;
    if (n && p.blocks > 1) {
        j.part = a.sums; j.n = n; j.cols = d->cols; j.blocks = p.blocks;
        launch(join_sums_kernel, dim3((d->cols + 31) / 32, n), dim3(512), 0, st, j);
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
