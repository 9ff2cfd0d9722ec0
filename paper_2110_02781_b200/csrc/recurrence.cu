// Gated linear recurrence over the steps of a sequence: h_t = a_t h_(t-1) + b_t with a = 1 / (1 + e^-f), b = (1 - a) v or v, and
// y = act(o) h; every channel for itself.
//
// Bound by memory: one pass over f, v, o and y (backward: f, v, o, dy in, df, dv, do out).  A step is the map h -> a h + b, and the maps of a run of
// steps compose to one, h -> A h + B.  A thread holds a run of 16 steps of two neighbouring channels (bf16; one float channel) in registers; a warp 32
// threads of one run; a block up to eight runs after one another (four backward), and a cluster of up to sixteen blocks the runs after those, so that
// a long sequence of few channels still fills the GPU.  The runs' maps go through shared memory, the blocks' through the cluster's, and are applied in
// the order of time, whatever finishes first: one read of the data and the same bits every time.  The state and the maps are float.
// Rows on 16 bytes come and go as tiles through the copy engine (below): 65536 x 2048 bf16 forward with a gate 279 us (4.0 TB/s; four
// exponentials and reciprocals an element use half of their pipe, 256 blocks leave a seventh of the GPU idle), 24 ragged sequences of up to 4096 x 1536
// 166 forward and 262 us backward (4.3 TB/s; latency at 12 warps a multiprocessor, which the registers allow).  Float, 32000 x 1000: 137 and
// 315 us, without a gate 91 and 203.  Other rows through registers: 32000 x 2001 bf16 209 us forward, 599 backward.
// The backward pass starts every run from the state that the forward pass kept in front of it, walks it forward once and then, with
// q_t = a_t (g_t + q_(t+1)) (g: dy act(o), q_(t+1): what reaches h_t from behind), backward in the same way.
#include <algorithm>
#include <type_traits>
#include "gemm_tc_common.cuh"
#include "token.cuh"

namespace ftp {
namespace token {
namespace {

constexpr int RUN = 16, WARPS = 8, BACK_WARPS = 4, MOST_RANKS = 16;   // runs of a block forward and backward; blocks of a cluster at most
template <typename T> constexpr int LANES = 4 / (int)sizeof(T);      // channels of a thread
template <typename T> constexpr int TILE = 32 * LANES<T>;            // of a block

struct RecArgs {
    const void *f, *v, *o, *dy;
    void *y, *df, *dv, *dout;
    const float *h0, *dh1;
    float *h1, *dh0, *states;
    const int32_t* offsets;
    int64_t seqs, len, rows, ldf, ldv, ldo, ldy, lddf, lddv, lddo;
    int cols, tiles, act, coupled;
};

// A thread's channels of one row.  VEC: neighbours; otherwise 32 apart.
template <typename T, bool VEC> struct Lane {
    int c;
    __device__ __forceinline__ Lane(int tile) : c(tile * TILE<T> + (threadIdx.x & 31) * (VEC ? LANES<T> : 1)) {}
    __device__ __forceinline__ int at(int j) const { return c + (VEC ? j : 32 * j); }
    __device__ __forceinline__ unsigned get(const T* row, int cols) const {
        if constexpr (sizeof(T) == 4) return c < cols ? __float_as_uint(row[c]) : 0u;
        else if constexpr (VEC) return c < cols ? *reinterpret_cast<const unsigned*>(row + c) : 0u;
        else return (c < cols ? bits_of(row[c]) : 0u) | (c + 32 < cols ? bits_of(row[c + 32]) << 16 : 0u);
    }
    __device__ __forceinline__ void put(T* row, int cols, const float (&v)[LANES<T>]) const {
        if constexpr (sizeof(T) == 4) { if (c < cols) row[c] = v[0]; }
        else if constexpr (VEC) { if (c < cols) *reinterpret_cast<unsigned*>(row + c) = bf_pack(v[0], v[1]); }
        else {
            if (c < cols) row[c] = __float2bfloat16(v[0]);
            if (c + 32 < cols) row[c + 32] = __float2bfloat16(v[1]);
        }
    }
    // the word of two neighbours, of which the second may lie behind the last column
    __device__ __forceinline__ void put_word(T* row, int cols, unsigned v) const {
        if (c < cols) from_bits(row + c, v);
        if (sizeof(T) == 2 && c + 1 < cols) from_bits(row + c + 1, v >> 16);
    }
    __device__ __forceinline__ void get_state(const float* row, int cols, float (&v)[LANES<T>]) const {
#pragma unroll
        for (int j = 0; j < LANES<T>; ++j) v[j] = row && at(j) < cols ? row[at(j)] : 0.f;
    }
    __device__ __forceinline__ void put_state(float* row, int cols, const float (&v)[LANES<T>]) const {
#pragma unroll
        for (int j = 0; j < LANES<T>; ++j) if (at(j) < cols) row[at(j)] = v[j];
    }
};
template <typename T> __device__ __forceinline__ void split(unsigned w, float (&v)[LANES<T>]) {
    if constexpr (sizeof(T) == 4) v[0] = __uint_as_float(w);
    else { v[0] = bf_lo(w); v[1] = bf_hi(w); }
}

// a = 1 / (1 + e^-f) and 1 - a, each to a few roundings of itself, next to 1 and to 0 alike.  f below -79 counts as -79 (a 5e-35, 1 - a exactly
// 1 in float), so that 0 times infinity does not arise.  bf16: hardware exponential and reciprocal, 2^-21 relative, and 2^-24 |f| for the rounding of the
// exponent (a gate of 20 in bf16 is itself known to 2^-9 of it).
__device__ __forceinline__ float above(float f) { asm("max.NaN.f32 %0, %0, %1;" : "+f"(f) : "f"(-79.f)); return f; }
template <typename T> __device__ __forceinline__ float exp_of_minus(float f) { return sizeof(T) == 4 ? expf(-f) : ffn::ex2_fast(f * -ffn::LOG2E); }
template <typename T> __device__ __forceinline__ void gate(float f, float& a, float& other) {
    const float e = exp_of_minus<T>(above(f));
    a = sizeof(T) == 4 ? 1.f / (1.f + e) : ffn::rcp_fast(1.f + e);
    other = e * a;
}
// act(o): FORM 0 none, 1 SILU, 2 as `act` says
template <typename T, int FORM> __device__ __forceinline__ float act_of(float o, int act) {
    if (FORM == 0) return 1.f;
    return FORM == 1 ? o * ffn::sigmoid_t<sizeof(T) == 2>(o) : ffn::act_value<sizeof(T) == 2>(o, act);
}

// ---- the streamed kernels: two bf16 channels of a thread in one register pair, or a float channel ----
template <typename T> using Two = std::conditional_t<sizeof(T) == 4, float, F2>;
using token::add2;
using token::fma2;
using token::mul2;
__device__ __forceinline__ float add2(float a, float b) { return a + b; }
__device__ __forceinline__ float mul2(float a, float b) { return a * b; }
__device__ __forceinline__ float fma2(float a, float b, float c) { return fmaf(a, b, c); }
template <typename T> __device__ __forceinline__ Two<T> splat(float v) { if constexpr (sizeof(T) == 4) return v; else return f2(v); }
template <typename T> __device__ __forceinline__ Two<T> two_of(unsigned w) { if constexpr (sizeof(T) == 4) return __uint_as_float(w); else return f2(bf_lo(w), bf_hi(w)); }
template <typename T> __device__ __forceinline__ unsigned word_of(Two<T> v) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(v);
    else { const float2 p = parts(v); return bf_pack(p.x, p.y); }
}
template <typename T, typename F> __device__ __forceinline__ Two<T> each(Two<T> v, F&& f) {
    if constexpr (sizeof(T) == 4) return f(v);
    else { const float2 p = parts(v); return f2(f(p.x), f(p.y)); }
}
template <typename T> __device__ __forceinline__ Two<T> join_floats(const float (&v)[LANES<T>]) { if constexpr (sizeof(T) == 4) return v[0]; else return f2(v[0], v[1]); }
template <typename T> __device__ __forceinline__ void to_floats(Two<T> v, float (&o)[LANES<T>]) {
    if constexpr (sizeof(T) == 4) o[0] = v;
    else { const float2 p = parts(v); o[0] = p.x; o[1] = p.y; }
}
// 1 / (1 + e^-f), and e^-f
template <typename T> __device__ __forceinline__ void sigmoids(Two<T> f, Two<T>& a, Two<T>& e) {
    if constexpr (sizeof(T) == 4) e = expf(-f);
    else e = each<T>(mul2(f, splat<T>(-ffn::LOG2E)), [](float v) { return ffn::ex2_fast(v); });
    a = each<T>(add2(e, splat<T>(1.f)), [](float v) { return sizeof(T) == 4 ? 1.f / v : ffn::rcp_fast(v); });
}
template <typename T> __device__ __forceinline__ void gate2(Two<T> f, Two<T>& a, Two<T>& other) {
    Two<T> e;
    sigmoids<T>(each<T>(f, [](float v) { return above(v); }), a, e);
    other = mul2(e, a);
}

// rows of sequence b
struct Where { int64_t start, len; };
__device__ __forceinline__ Where where(const RecArgs& a, int64_t b) {
    if (!a.offsets) return Where{b * a.len, a.len};
    const int64_t lo = min(max((int64_t)a.offsets[b], (int64_t)0), a.rows), hi = min(max((int64_t)a.offsets[b + 1], lo), a.rows);
    return Where{lo, min(hi - lo, a.len)};
}

// Maps of the warps' runs joined: what reaches this warp's run and what leaves the cluster's last, from what reaches its first.
// REVERSE: the last run comes first.  `maps`: [2][warps][32], `parts`: [2][ranks][32] in shared memory, used in turn.  The blocks of a
// cluster send each other their part by asynchronous stores that count on the receiver's barrier (a cluster barrier waits for all
// of a block's earlier stores to global memory: a fifth of the kernel's stalls).  A part's place is written again two turns later, after
// this block's next part has been sent, which every warp precedes.
template <int N> struct __align__(8 * N) Map { float a[N], b[N]; };
__device__ __forceinline__ void send(unsigned to, unsigned bar, const Map<1>& m) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" :: "r"(to), "f"(m.a[0]), "f"(m.b[0]), "r"(bar) : "memory");
}
__device__ __forceinline__ void send(unsigned to, unsigned bar, const Map<2>& m) {
    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 :: "r"(to), "f"(m.a[0]), "f"(m.a[1]), "f"(m.b[0]), "f"(m.b[1]), "r"(bar) : "memory");
}
template <int N, bool REVERSE> struct Join {
    Map<N>*maps, *parts;
    unsigned bars, ranks, rank;                                      // bars: a barrier for each turn
    int w, warps;
    int* err;
    bool ok = true;
    int turn = 0;
    unsigned parity = 0;
    // the whole cluster takes part; `pair`: shared memory of two barriers
    __device__ __forceinline__ Join(Map<N>* at, uint64_t* pair, unsigned ranks, unsigned rank, int w, int warps, int* err)
        : maps(at), parts(at + 2 * warps * 32), bars(smem_at(pair)), ranks(ranks), rank(rank), w(w), warps(warps), err(err) {
        if (ranks == 1) return;
        if (threadIdx.x == 0) {
            tc::mbar_init(bars, 1);
            tc::mbar_init(bars + 8, 1);
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        }
        cluster_sync();
    }
    __device__ __forceinline__ void operator()(const Map<N>& mine, float (&carry)[N], float (&in)[N]) {
        const int lane = threadIdx.x & 31;
        Map<N>* m = maps + turn * warps * 32;
        m[w * 32 + lane] = mine;
        __syncthreads();
        Map<N> pre, all;
#pragma unroll
        for (int j = 0; j < N; ++j) { all.a[j] = 1.f; all.b[j] = 0.f; }
        pre = all;
        for (int i = 0; i < warps; ++i) {
            const int k = REVERSE ? warps - 1 - i : i;
            if (k == w) pre = all;
            const Map<N> n = m[k * 32 + lane];
#pragma unroll
            for (int j = 0; j < N; ++j) { all.b[j] = fmaf(n.a[j], all.b[j], n.b[j]); all.a[j] *= n.a[j]; }
        }
        if (ranks == 1) {
#pragma unroll
            for (int j = 0; j < N; ++j) { in[j] = fmaf(pre.a[j], carry[j], pre.b[j]); carry[j] = fmaf(all.a[j], carry[j], all.b[j]); }
        } else {
            Map<N>* p = parts + turn * ranks * 32;
            const unsigned bar = bars + 8 * turn;
            if (threadIdx.x == 0) tc::mbar_expect_tx(bar, ranks * 32 * (unsigned)sizeof(Map<N>));
            for (unsigned r = w; r < ranks; r += warps) send(on_rank(smem_at(p + rank * 32 + lane), r), on_rank(bar, r), all);   // every warp tells some of the blocks
            ok = tc::mbar_wait(bar, parity, err, 0x500) && ok;
            for (unsigned i = 0; i < ranks; ++i) {
                const unsigned k = REVERSE ? ranks - 1 - i : i;
                if (k == rank)
#pragma unroll
                    for (int j = 0; j < N; ++j) in[j] = fmaf(pre.a[j], carry[j], pre.b[j]);
                const Map<N> n = p[k * 32 + lane];
#pragma unroll
                for (int j = 0; j < N; ++j) carry[j] = fmaf(n.a[j], carry[j], n.b[j]);
            }
            parity ^= turn;
        }
        turn ^= 1;
    }
};

// The rows of a run.  WHOLE: all RUN of them are there.
template <typename T, bool VEC, bool WHOLE>
__device__ __forceinline__ void load_run(const void* base, int64_t row, int64_t ld, int n, const Lane<T, VEC>& lane, int cols, unsigned (&r)[RUN]) {
    const T* p = static_cast<const T*>(base) + row * ld;
#pragma unroll
    for (int i = 0; i < RUN; ++i) r[i] = WHOLE || i < n ? lane.get(p + i * ld, cols) : 0u;
}

// One run forward: from what is loaded to its map, and from the state in front of it to its outputs.
template <typename T, bool VEC, int FORM> struct Forward {
    static constexpr int N = LANES<T>;
    unsigned f[RUN], v[RUN], o[RUN];
    float a[RUN][N], b[RUN][N];
    template <bool WHOLE> __device__ __forceinline__ void load(const RecArgs& p, int64_t row, int n, const Lane<T, VEC>& lane) {
        load_run<T, VEC, WHOLE>(p.f, row, p.ldf, n, lane, p.cols, f);
        load_run<T, VEC, WHOLE>(p.v, row, p.ldv, n, lane, p.cols, v);
        if (FORM) load_run<T, VEC, WHOLE>(p.o, row, p.ldo, n, lane, p.cols, o);
    }
    template <bool WHOLE> __device__ __forceinline__ void map(const RecArgs& p, int n, Map<N>& all) {
#pragma unroll
        for (int j = 0; j < N; ++j) { all.a[j] = 1.f; all.b[j] = 0.f; }
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            float ff[N], vv[N];
            split<T>(f[i], ff);
            split<T>(v[i], vv);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float other;
                gate<T>(ff[j], a[i][j], other);
                b[i][j] = p.coupled ? other * vv[j] : vv[j];
                if (!WHOLE && i >= n) { a[i][j] = 1.f; b[i][j] = 0.f; }
                all.b[j] = fmaf(a[i][j], all.b[j], b[i][j]);
                all.a[j] *= a[i][j];
            }
        }
    }
    template <bool WHOLE> __device__ __forceinline__ void out(const RecArgs& p, int64_t row, int n, const Lane<T, VEC>& lane, float (&h)[N]) {
        T* y = static_cast<T*>(p.y) + row * p.ldy;
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            float oo[N];
            if (FORM) split<T>(o[i], oo);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                h[j] = fmaf(a[i][j], h[j], b[i][j]);
                oo[j] = FORM ? act_of<T, FORM>(oo[j], p.act) * h[j] : h[j];
            }
            if (WHOLE || i < n) lane.put(y + i * p.ldy, p.cols, oo);
        }
    }
};

// A cluster per sequence and tile of channels; `ranks` blocks of `warps` runs each walk down the sequence.
template <typename T, bool VEC, int FORM>
__global__ void __launch_bounds__(32 * WARPS, 2) recurrence_forward_kernel(const RecArgs a, int* err) {
    constexpr int N = LANES<T>;
    __shared__ Map<N> maps[2 * (WARPS + MOST_RANKS) * 32];
    __shared__ uint64_t pair[2];
    grid_dep_sync();
    const int warps = blockDim.x >> 5, w = threadIdx.x >> 5;
    unsigned ranks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const unsigned rank = cluster_rank();
    Join<N, false> join(maps, pair, ranks, rank, w, warps, err);
    const int64_t unit = blockIdx.x / ranks, b = unit / a.tiles;
    const Lane<T, VEC> lane((int)(unit - b * a.tiles));
    const Where seq = where(a, b);
    float carry[N];
    lane.get_state(a.h0 ? a.h0 + b * a.cols : nullptr, a.cols, carry);
    const int64_t stride = (int64_t)RUN * warps * ranks;
    for (int64_t t0 = (int64_t)RUN * (rank * warps + w), base = 0; base < seq.len; t0 += stride, base += stride) {
        const int n = (int)min((int64_t)RUN, max((int64_t)0, seq.len - t0));
        const int64_t row = seq.start + t0;
        Forward<T, VEC, FORM> r;
        Map<N> all;
        float h[N];
        if (n == RUN) {
            r.template load<true>(a, row, n, lane);
            r.template map<true>(a, n, all);
        } else {
            r.template load<false>(a, row, n, lane);
            r.template map<false>(a, n, all);
        }
        join(all, carry, h);
        if (!join.ok) continue;
        if (a.states && n > 0) lane.put_state(a.states + (seq.start / RUN + b + t0 / RUN) * a.cols, a.cols, h);
        if (n == RUN) r.template out<true>(a, row, n, lane, h); else r.template out<false>(a, row, n, lane, h);
    }
    if (ranks > 1) cluster_sync();                                   // nobody leaves while another block may send to it; every block has read h0, which may be h1
    if (a.h1 && w == 0 && rank == 0 && join.ok) lane.put_state(a.h1 + b * a.cols, a.cols, carry);
}

// ---- rows that start on 16 bytes: tiles through the copy engine ----
// Every warp works on its own: its runs' 16 x 128-byte tiles come into its own part of shared memory, two iterations ahead, and its results
// leave from there; loads hold no registers, addresses are constants, and the runs' compositions alone tie the warps together.  (Loads into
// registers: 618 us for 65536 x 2048 bf16, 59 instructions an element, half of them addresses.)
constexpr unsigned TILE_BYTES = RUN * 128;

__device__ __forceinline__ void tile_in(unsigned to, const CUtensorMap* map, int c, int64_t row, unsigned bar) { tc::tma_load_2d(to, map, c, (int)row, bar); }
__device__ __forceinline__ void tile_out(const CUtensorMap* map, int c, int64_t row, unsigned from) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" :: "l"(map), "r"(c), "r"((int)row), "r"(from) : "memory");
}
// Tiles are stored by the copy engine in whole 16 bytes: where the last columns are not (a pitch may be all the same), it would write what lies behind them.
template <typename T> __device__ __forceinline__ bool whole_tile(int c, int cols) { return c + TILE<T> <= cols || cols % V<T> == 0; }
__device__ __forceinline__ void tiles_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void tiles_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }       // shared memory may be written again
__device__ __forceinline__ void tiles_done() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }
__device__ __forceinline__ void tiles_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

struct Maps4 { CUtensorMap m[4]; };

template <typename T, int FORM, bool COUPLED>
__global__ void __launch_bounds__(32 * WARPS, 2) recurrence_forward_stream_kernel(const __grid_constant__ Maps4 maps_in, const __grid_constant__ CUtensorMap map_y, const RecArgs a,
                                                                                  int* err) {
    constexpr int N = LANES<T>;
    extern __shared__ unsigned char dynamic[];                       // per warp two stages of three tiles (f, v, o: where y is put); the maps
    unsigned char* const smem = dynamic + (-smem_at(dynamic) & 127);
    __shared__ uint64_t bars[WARPS][4], pair[2];
    const int warps = blockDim.x >> 5, w = threadIdx.x >> 5, l = threadIdx.x & 31;
    unsigned ranks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const unsigned rank = cluster_rank();
    unsigned char* const mine = smem + w * 6 * TILE_BYTES;
    Map<N>* const maps = reinterpret_cast<Map<N>*>(smem + warps * 6 * TILE_BYTES);
    const unsigned bar = smem_at(bars[w]), tiles = smem_at(mine);
    if (l == 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) tc::mbar_init(bar + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    grid_dep_sync();
    Join<N, false> join(maps, pair, ranks, rank, w, warps, err);
    const int64_t unit = blockIdx.x / ranks, b = unit / a.tiles;
    const int tile = (int)(unit - b * a.tiles), c = tile * TILE<T>;
    const Lane<T, true> lane(tile);
    const bool storable = whole_tile<T>(c, a.cols);
    const Where seq = where(a, b);
    float carry[N];
    lane.get_state(a.h0 ? a.h0 + b * a.cols : nullptr, a.cols, carry);
    const int64_t stride = (int64_t)RUN * warps * ranks, own = (int64_t)RUN * (rank * warps + w);
    const auto load_fv = [&](int64_t t0, int s) {
        if (l || t0 >= seq.len) return;
        tc::mbar_expect_tx(bar + 8 * s, 2 * TILE_BYTES);
        tile_in(tiles + (3 * s) * TILE_BYTES, &maps_in.m[0], c, seq.start + t0, bar + 8 * s);
        tile_in(tiles + (3 * s + 1) * TILE_BYTES, &maps_in.m[1], c, seq.start + t0, bar + 8 * s);
    };
    const auto load_o = [&](int64_t t0, int s) {
        if (!FORM || l || t0 >= seq.len) return;
        tc::mbar_expect_tx(bar + 16 + 8 * s, TILE_BYTES);
        tile_in(tiles + (3 * s + 2) * TILE_BYTES, &maps_in.m[2], c, seq.start + t0, bar + 16 + 8 * s);
    };
    load_fv(own, 0);
    load_o(own, 0);
    load_fv(own + stride, 1);
    bool ok = true;
    int s = 0;
    unsigned parity = 0;
    for (int64_t t0 = own, base = 0; base < seq.len; t0 += stride, base += stride) {
        const int n = (int)min((int64_t)RUN, max((int64_t)0, seq.len - t0));
        const unsigned char* at = mine + 3 * s * TILE_BYTES + 4 * l;
        Two<T> x[RUN], d[RUN];                                       // a and what is added
        Two<T> all_a = splat<T>(1.f), all_b = splat<T>(0.f);
        if (n > 0) {
            ok = tc::mbar_wait(bar + 8 * s, parity, err, 0x501) && ok;
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                const Two<T> f = two_of<T>(*reinterpret_cast<const unsigned*>(at + 128 * i)), v = two_of<T>(*reinterpret_cast<const unsigned*>(at + TILE_BYTES + 128 * i));
                Two<T> other;
                gate2<T>(f, x[i], other);
                d[i] = COUPLED ? mul2(other, v) : v;
            }
            if (n < RUN)
#pragma unroll
                for (int i = 0; i < RUN; ++i)
                    if (i >= n) { x[i] = splat<T>(1.f); d[i] = splat<T>(0.f); }
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                all_b = fma2(x[i], all_b, d[i]);
                all_a = mul2(all_a, x[i]);
            }
        }
        __syncwarp();
        load_fv(t0 + 2 * stride, s);
        if (l == 0) tiles_read();                                    // the other stage's results have left
        load_o(t0 + stride, s ^ 1);
        Map<N> all;
        to_floats<T>(all_a, all.a);
        to_floats<T>(all_b, all.b);
        float h0[N];
        join(all, carry, h0);
        ok = ok && join.ok;
        if (n > 0) {
            if (a.states && ok) lane.put_state(a.states + (seq.start / RUN + b + t0 / RUN) * a.cols, a.cols, h0);
            if (FORM) ok = tc::mbar_wait(bar + 16 + 8 * s, parity, err, 0x502) && ok;
            unsigned char* const to = mine + (3 * s + 2) * TILE_BYTES + 4 * l;
            Two<T> h = join_floats<T>(h0);
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                h = fma2(x[i], h, d[i]);
                Two<T> y = h;
                if (FORM) {
                    const Two<T> o = two_of<T>(*reinterpret_cast<const unsigned*>(to + 128 * i));
                    if (FORM == 1) {
                        Two<T> p, e;
                        sigmoids<T>(o, p, e);
                        y = mul2(mul2(o, p), h);
                    } else
                        y = mul2(each<T>(o, [&](float v) { return ffn::act_value<sizeof(T) == 2>(v, a.act); }), h);
                }
                *reinterpret_cast<unsigned*>(to + 128 * i) = word_of<T>(y);
            }
            tiles_fence();                                           // the copy engine reads this tile, or fills it again
            if (n == RUN && storable) {
                __syncwarp();
                if (l == 0 && ok) { tile_out(&map_y, c, seq.start + t0, tiles + (3 * s + 2) * TILE_BYTES); tiles_commit(); }
            } else if (ok)
                for (int i = 0; i < n; ++i) lane.put_word(static_cast<T*>(a.y) + (seq.start + t0 + i) * a.ldy, a.cols, *reinterpret_cast<const unsigned*>(to + 128 * i));
        }
        parity ^= s;
        s ^= 1;
    }
    if (l == 0) tiles_done();
    __syncwarp();
    if (ranks > 1) cluster_sync();                                   // nobody leaves while another block may send to it; every block has read h0, which may be h1
    if (a.h1 && w == 0 && rank == 0 && ok) lane.put_state(a.h1 + b * a.cols, a.cols, carry);
}

// The same backward.  Between its two walks a thread keeps, per step, a, 1 - a and the gradient g that reaches h from its own output in
// registers, and (1 - a) (h_(t-1) - v) (coupled) or (1 - a) h_(t-1) in the words of the tiles of f and v that it has read.
template <typename T, int FORM, bool COUPLED>
__global__ void __launch_bounds__(32 * BACK_WARPS, 3) recurrence_backward_stream_kernel(const __grid_constant__ Maps4 maps_in, const __grid_constant__ Maps4 maps_out, const RecArgs a,
                                                                                        int* err) {
    constexpr int N = LANES<T>;
    extern __shared__ unsigned char dynamic[];                       // per warp two stages of four tiles (f, v, o, dy: df, dv, do replace them); the maps
    unsigned char* const smem = dynamic + (-smem_at(dynamic) & 127);
    __shared__ uint64_t bars[BACK_WARPS][2], pair[2];
    const int warps = blockDim.x >> 5, w = threadIdx.x >> 5, l = threadIdx.x & 31;
    unsigned ranks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const unsigned rank = cluster_rank();
    unsigned char* const mine = smem + w * 8 * TILE_BYTES;
    Map<N>* const maps = reinterpret_cast<Map<N>*>(smem + warps * 8 * TILE_BYTES);
    const unsigned bar = smem_at(bars[w]), tiles = smem_at(mine);
    if (l == 0) {
        tc::mbar_init(bar, 1);
        tc::mbar_init(bar + 8, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    grid_dep_sync();
    Join<N, true> join(maps, pair, ranks, rank, w, warps, err);
    const int64_t unit = blockIdx.x / ranks, b = unit / a.tiles;
    const int tile = (int)(unit - b * a.tiles), c = tile * TILE<T>;
    const Lane<T, true> lane(tile);
    const bool storable = whole_tile<T>(c, a.cols);
    const Where seq = where(a, b);
    float carry[N];
    lane.get_state(a.dh1 ? a.dh1 + b * a.cols : nullptr, a.cols, carry);
    const int64_t stride = (int64_t)RUN * warps * ranks, own = (int64_t)RUN * (rank * warps + w), last = (seq.len + stride - 1) / stride * stride - stride;
    const auto load = [&](int64_t t0, int s) {
        if (l || t0 < 0 || t0 >= seq.len) return;
        tc::mbar_expect_tx(bar + 8 * s, (FORM ? 4 : 3) * TILE_BYTES);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (FORM || i != 2) tile_in(tiles + (4 * s + i) * TILE_BYTES, &maps_in.m[i], c, seq.start + t0, bar + 8 * s);
    };
    // only the first turn may find nothing of the sequence left for this warp: it then starts with the second
    int64_t t0 = last + own;
    int s = 0;
    unsigned parity = 0;
    const bool skip = t0 >= seq.len;
    load(t0 - (skip ? stride : 0), 0);
    load(t0 - (skip ? 2 : 1) * stride, 1);
    bool ok = true;
    for (int64_t base = last; base >= 0; base -= stride, t0 -= stride) {
        const int n = (int)min((int64_t)RUN, max((int64_t)0, seq.len - t0));
        unsigned char* const at = mine + 4 * s * TILE_BYTES + 4 * l;
        Two<T> x[RUN], other[RUN], g[RUN];
        Two<T> all_a = splat<T>(1.f), all_b = splat<T>(0.f);
        if (n > 0) {
            float h0[N];
            lane.get_state(a.states + (seq.start / RUN + b + t0 / RUN) * a.cols, a.cols, h0);
            Two<T> h = join_floats<T>(h0);
            ok = tc::mbar_wait(bar + 8 * s, parity, err, 0x503) && ok;
#pragma unroll
            for (int i = 0; i < RUN; ++i) {
                const Two<T> f = two_of<T>(*reinterpret_cast<const unsigned*>(at + 128 * i)), v = two_of<T>(*reinterpret_cast<const unsigned*>(at + TILE_BYTES + 128 * i));
                g[i] = two_of<T>(*reinterpret_cast<const unsigned*>(at + 3 * TILE_BYTES + 128 * i));
                gate2<T>(f, x[i], other[i]);
                float keep[N];
                to_floats<T>(mul2(other[i], COUPLED ? fma2(v, splat<T>(-1.f), h) : h), keep);
#pragma unroll
                for (int j = 0; j < N; ++j) *reinterpret_cast<float*>(at + j * TILE_BYTES + 128 * i) = keep[j];
                h = fma2(x[i], h, COUPLED ? mul2(other[i], v) : v);
                if (FORM) {
                    const Two<T> o = two_of<T>(*reinterpret_cast<const unsigned*>(at + 2 * TILE_BYTES + 128 * i));
                    Two<T> val, slope;
                    if (FORM == 1) {
                        // o below -79 counts as -79 in the product too: o times a's floor would not be small
                        const Two<T> oo = each<T>(o, [](float v) { return above(v); });
                        Two<T> p, q;
                        sigmoids<T>(oo, p, q);
                        q = mul2(q, p);
                        val = mul2(oo, p);
                        slope = fma2(val, q, p);
                    } else {
                        float oo[N], vv[N], ss[N];
                        to_floats<T>(o, oo);
#pragma unroll
                        for (int j = 0; j < N; ++j) ffn::act_both<sizeof(T) == 2>(oo[j], a.act, vv[j], ss[j]);
                        val = join_floats<T>(vv);
                        slope = join_floats<T>(ss);
                    }
                    *reinterpret_cast<unsigned*>(at + 2 * TILE_BYTES + 128 * i) = word_of<T>(mul2(mul2(g[i], h), slope));
                    g[i] = mul2(g[i], val);
                }
            }
            if (n < RUN)
#pragma unroll
                for (int i = 0; i < RUN; ++i)
                    if (i >= n) { x[i] = splat<T>(1.f); g[i] = splat<T>(0.f); }
#pragma unroll
            for (int i = RUN - 1; i >= 0; --i) {
                all_b = mul2(x[i], add2(g[i], all_b));
                all_a = mul2(all_a, x[i]);
            }
            if (FORM) tiles_fence();
        }
        __syncwarp();
        if (l == 0) {
            tiles_read();                                            // the other stage's results have left
            if (base < last - (skip ? stride : 0)) load(t0 - stride, s ^ 1);
            if (FORM && n == RUN && storable && ok) { tile_out(&maps_out.m[2], c, seq.start + t0, tiles + (4 * s + 2) * TILE_BYTES); tiles_commit(); }
        }
        Map<N> all;
        to_floats<T>(all_a, all.a);
        to_floats<T>(all_b, all.b);
        float q0[N];
        join(all, carry, q0);
        ok = ok && join.ok;
        if (n > 0) {
            Two<T> q = join_floats<T>(q0);
#pragma unroll
            for (int i = RUN - 1; i >= 0; --i) {
                const Two<T> e = add2(g[i], q);
                q = mul2(x[i], e);
                float keep[N];
#pragma unroll
                for (int j = 0; j < N; ++j) keep[j] = *reinterpret_cast<const float*>(at + j * TILE_BYTES + 128 * i);
                *reinterpret_cast<unsigned*>(at + 128 * i) = word_of<T>(mul2(q, join_floats<T>(keep)));
                *reinterpret_cast<unsigned*>(at + TILE_BYTES + 128 * i) = word_of<T>(COUPLED ? mul2(e, other[i]) : e);
            }
            tiles_fence();                                           // the copy engine reads these tiles, or fills them again in the next turn
            if (n == RUN && storable) {
                __syncwarp();
                if (l == 0 && ok) {
                    tile_out(&maps_out.m[0], c, seq.start + t0, tiles + (4 * s) * TILE_BYTES);
                    tile_out(&maps_out.m[1], c, seq.start + t0, tiles + (4 * s + 1) * TILE_BYTES);
                    tiles_commit();
                }
            } else if (ok)
                for (int i = 0; i < n; ++i) {
                    const int64_t row = seq.start + t0 + i;
                    lane.put_word(static_cast<T*>(a.df) + row * a.lddf, a.cols, *reinterpret_cast<const unsigned*>(at + 128 * i));
                    lane.put_word(static_cast<T*>(a.dv) + row * a.lddv, a.cols, *reinterpret_cast<const unsigned*>(at + TILE_BYTES + 128 * i));
                    if (FORM) lane.put_word(static_cast<T*>(a.dout) + row * a.lddo, a.cols, *reinterpret_cast<const unsigned*>(at + 2 * TILE_BYTES + 128 * i));
                }
            parity ^= s;
            s ^= 1;
        }
    }
    if (l == 0) tiles_done();
    __syncwarp();
    if (ranks > 1) cluster_sync();                                   // nobody leaves while another block may send to it; every block has read dh1, which may be dh0
    if (a.dh0 && w == 0 && rank == 0 && ok) lane.put_state(a.dh0 + b * a.cols, a.cols, carry);
}

// Sequences of at most one run, a warp each, a step at a time: a serving program's call.
template <typename T, bool VEC, int FORM>
__global__ void __launch_bounds__(128) recurrence_short_kernel(const RecArgs a) {
    constexpr int N = LANES<T>;
    grid_dep_sync();
    const int64_t unit = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5), b = unit / a.tiles;
    if (b >= a.seqs) return;
    const Lane<T, VEC> lane((int)(unit - b * a.tiles));
    const Where seq = where(a, b);
    float h[N];
    lane.get_state(a.h0 ? a.h0 + b * a.cols : nullptr, a.cols, h);
    if (a.states && seq.len > 0) lane.put_state(a.states + (seq.start / RUN + b) * a.cols, a.cols, h);
    for (int64_t row = seq.start; row < seq.start + seq.len; ++row) {
        float f[N], v[N], o[N];
        split<T>(lane.get(static_cast<const T*>(a.f) + row * a.ldf, a.cols), f);
        split<T>(lane.get(static_cast<const T*>(a.v) + row * a.ldv, a.cols), v);
        if (FORM) split<T>(lane.get(static_cast<const T*>(a.o) + row * a.ldo, a.cols), o);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            float x, other;
            gate<T>(f[j], x, other);
            h[j] = fmaf(x, h[j], a.coupled ? other * v[j] : v[j]);
            o[j] = FORM ? act_of<T, FORM>(o[j], a.act) * h[j] : h[j];
        }
        lane.put(static_cast<T*>(a.y) + row * a.ldy, a.cols, o);
    }
    if (a.h1) lane.put_state(a.h1 + b * a.cols, a.cols, h);
}

// One run backward.  Between its two walks it keeps, per step, a and the gradient g that reaches h from its own output in registers, and in shared memory
// (1 - a) (h_(t-1) - v) and 1 - a (coupled), or (1 - a) h_(t-1).
template <typename T, bool VEC, int FORM> struct Backward {
    static constexpr int N = LANES<T>;
    unsigned f[RUN], v[RUN], o[RUN], dy[RUN];
    float a[RUN][N], g[RUN][N];
    template <bool WHOLE> __device__ __forceinline__ void load(const RecArgs& p, int64_t row, int n, const Lane<T, VEC>& lane) {
        load_run<T, VEC, WHOLE>(p.f, row, p.ldf, n, lane, p.cols, f);
        load_run<T, VEC, WHOLE>(p.v, row, p.ldv, n, lane, p.cols, v);
        if (FORM) load_run<T, VEC, WHOLE>(p.o, row, p.ldo, n, lane, p.cols, o);
        load_run<T, VEC, WHOLE>(p.dy, row, p.ldy, n, lane, p.cols, dy);
    }
    // forward through the run, then its map of what reaches it from behind
    template <bool WHOLE> __device__ __forceinline__ void map(const RecArgs& p, int64_t row, int n, const Lane<T, VEC>& lane, float (&h)[N], float* before, Map<N>& all) {
        T* to = static_cast<T*>(p.dout) + (FORM ? row * p.lddo : 0);
#pragma unroll
        for (int i = 0; i < RUN; ++i) {
            float ff[N], vv[N], oo[N];
            split<T>(f[i], ff);
            split<T>(v[i], vv);
            if (FORM) split<T>(o[i], oo);
            split<T>(dy[i], g[i]);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                float other;
                gate<T>(ff[j], a[i][j], other);
                // what the second walk multiplies by: (1 - a) (h - v), or (1 - a) h; coupled: 1 - a besides, without cancellation
                before[(i * N + j) * (int)blockDim.x] = other * (p.coupled ? h[j] - vv[j] : h[j]);
                if (p.coupled) before[((RUN + i) * N + j) * (int)blockDim.x] = other;
                h[j] = fmaf(a[i][j], h[j], p.coupled ? other * vv[j] : vv[j]);
                if (FORM == 1) {
                    const float s = ffn::sigmoid_t<sizeof(T) == 2>(oo[j]), x = oo[j] * s;
                    oo[j] = g[i][j] * h[j] * (s == 1.f ? 1.f : fmaf(x, 1.f - s, s));
                    g[i][j] *= x;
                } else if (FORM == 2) {
                    float x, q;
                    ffn::act_both<sizeof(T) == 2>(oo[j], p.act, x, q);
                    oo[j] = g[i][j] * h[j] * q;
                    g[i][j] *= x;
                }
                if (!WHOLE && i >= n) { a[i][j] = 1.f; g[i][j] = 0.f; }
            }
            if (FORM && (WHOLE || i < n)) lane.put(to + i * p.lddo, p.cols, oo);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) { all.a[j] = 1.f; all.b[j] = 0.f; }
#pragma unroll
        for (int i = RUN - 1; i >= 0; --i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                all.b[j] = a[i][j] * (g[i][j] + all.b[j]);
                all.a[j] *= a[i][j];
            }
    }
    template <bool WHOLE> __device__ __forceinline__ void out(const RecArgs& p, int64_t row, int n, const Lane<T, VEC>& lane, const float* before, float (&q)[N]) {
        T *to_f = static_cast<T*>(p.df) + row * p.lddf, *to_v = static_cast<T*>(p.dv) + row * p.lddv;
#pragma unroll
        for (int i = RUN - 1; i >= 0; --i) {
            float df[N], dv[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = g[i][j] + q[j];
                q[j] = a[i][j] * d;
                df[j] = q[j] * before[(i * N + j) * (int)blockDim.x];
                dv[j] = p.coupled ? d * before[((RUN + i) * N + j) * (int)blockDim.x] : d;
            }
            if (WHOLE || i < n) {
                lane.put(to_f + i * p.lddf, p.cols, df);
                lane.put(to_v + i * p.lddv, p.cols, dv);
            }
        }
    }
};

template <typename T> constexpr int REG_WARPS = sizeof(T) == 2 ? BACK_WARPS : WARPS;   // as the registers allow: three blocks of four warps, two of eight
template <typename T, bool VEC, int FORM>
__global__ void __launch_bounds__(32 * REG_WARPS<T>, sizeof(T) == 2 ? 3 : 2) recurrence_backward_kernel(const RecArgs a, int* err) {
    constexpr int N = LANES<T>;
    __shared__ Map<N> maps[2 * (WARPS + MOST_RANKS) * 32];
    __shared__ uint64_t pair[2];
    extern __shared__ float kept[];                                  // per step and channel of a thread one or two values
    grid_dep_sync();
    const int warps = blockDim.x >> 5, w = threadIdx.x >> 5;
    float* const before = kept + threadIdx.x;
    unsigned ranks;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const unsigned rank = cluster_rank();
    Join<N, true> join(maps, pair, ranks, rank, w, warps, err);
    const int64_t unit = blockIdx.x / ranks, b = unit / a.tiles;
    const Lane<T, VEC> lane((int)(unit - b * a.tiles));
    const Where seq = where(a, b);
    float carry[N];
    lane.get_state(a.dh1 ? a.dh1 + b * a.cols : nullptr, a.cols, carry);
    const int64_t stride = (int64_t)RUN * warps * ranks;
    for (int64_t base = (seq.len + stride - 1) / stride * stride - stride; base >= 0; base -= stride) {
        const int64_t t0 = base + (int64_t)RUN * (rank * warps + w);
        const int n = (int)min((int64_t)RUN, max((int64_t)0, seq.len - t0));
        const int64_t row = seq.start + t0;
        Backward<T, VEC, FORM> r;
        Map<N> all;
        float h[N], q[N];
        lane.get_state(n > 0 ? a.states + (seq.start / RUN + b + t0 / RUN) * a.cols : nullptr, a.cols, h);
        if (n == RUN) {
            r.template load<true>(a, row, n, lane);
            r.template map<true>(a, row, n, lane, h, before, all);
        } else {
            r.template load<false>(a, row, n, lane);
            r.template map<false>(a, row, n, lane, h, before, all);
        }
        join(all, carry, q);
        if (!join.ok) continue;
        if (n == RUN) r.template out<true>(a, row, n, lane, before, q); else r.template out<false>(a, row, n, lane, before, q);
    }
    if (ranks > 1) cluster_sync();                                   // nobody leaves while another block may send to it; every block has read dh1, which may be dh0
    if (a.dh0 && w == 0 && rank == 0 && join.ok) lane.put_state(a.dh0 + b * a.cols, a.cols, carry);
}

// ---- host ----
ftp_status check_desc(const ftp_recurrence_desc* d, const char* who) {
    FTP_REQUIRE(d, FTP_EINVAL, "%s: null descriptor", who);
    FTP_REQUIRE(d->precision == FTP_FP32 || d->precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, d->precision);
    FTP_REQUIRE(d->act >= FTP_ACT_NONE && d->act <= FTP_ACT_SILU, FTP_EINVAL, "%s: unknown activation %d", who, d->act);
    FTP_REQUIRE(d->seqs >= 0 && d->len >= 0 && d->rows >= 0 && d->cols >= 1, FTP_EINVAL, "%s: seqs, len and rows must not be negative, cols must be positive", who);
    FTP_REQUIRE(d->seqs < (1ll << 31) && d->len < (1ll << 31) && d->rows < (1ll << 38) && d->cols < (1 << 30), FTP_ERANGE, "%s: tensor too large", who);
    const double steps = d->rows ? (double)d->rows : (double)d->seqs * (double)d->len;
    FTP_REQUIRE(steps * d->cols <= 274877906944.0 && (double)d->seqs * d->cols <= 274877906944.0, FTP_ERANGE, "%s: tensor too large", who);
    return check_pitches({d->ldf, d->ldv, d->ldo, d->ldy, d->lddf, d->lddv, d->lddo}, d->cols, who);
}
ftp_status check_offsets(const ftp_recurrence_desc* d, const int32_t* offsets, const char* who) {
    if (offsets) {
        FTP_REQUIRE(d->rows < (1ll << 31), FTP_ERANGE, "%s: offsets have 32 bits", who);
        return check_elements({offsets}, 4, who);
    }
    FTP_REQUIRE(d->rows == 0 || d->rows == d->seqs * d->len, FTP_EINVAL, "%s: rows must be seqs * len without offsets", who);
    return FTP_OK;
}
void fill(RecArgs& a, const ftp_recurrence_desc* d, const int32_t* offsets) {
    const auto ld = [&](int64_t v) { return v ? v : (int64_t)d->cols; };
    a.seqs = d->seqs; a.len = d->len; a.rows = offsets ? d->rows : d->seqs * d->len;
    a.cols = d->cols; a.act = d->act; a.coupled = d->coupled != 0;
    a.ldf = ld(d->ldf); a.ldv = ld(d->ldv); a.ldo = ld(d->ldo); a.ldy = ld(d->ldy);
    a.lddf = ld(d->lddf); a.lddv = ld(d->lddv); a.lddo = ld(d->lddo);
    a.offsets = offsets;
}
// two bf16 channels in one access: even pitches, addresses on four bytes
bool pairs(std::initializer_list<const void*> ps, std::initializer_list<int64_t> lds, int cols) {
    for (const void* p : ps) if (!on_bytes(p, 4)) return false;
    for (int64_t ld : lds) if (ld % 2) return false;
    return cols % 2 == 0;
}
// every row of it starts on 16 bytes, where the copy engine can fetch tiles
bool whole_rows(std::initializer_list<const void*> ps, std::initializer_list<int64_t> lds, size_t size, int64_t rows) {
    for (const void* p : ps) if (!on_bytes(p, 16)) return false;
    for (int64_t ld : lds) if (rows > 1 && ld * (int64_t)size % 16) return false;
    return rows < (1ll << 31) - 64;
}
template <typename T> bool tile_map(CUtensorMap* map, const void* p, int64_t ld, const RecArgs& a) {
    tc::EncodeTiledFn fn = tc::encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)a.cols, (cuuint64_t)a.rows}, strides[1] = {(cuuint64_t)((a.rows > 1 ? ld * (int64_t)sizeof(T) : (a.cols * (int64_t)sizeof(T) + 15) / 16 * 16))};
    const cuuint32_t box[2] = {(cuuint32_t)TILE<T>, RUN}, one[2] = {1, 1};
    return fn(map, sizeof(T) == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, one,
              CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Blocks of a cluster and runs of a block: the fewest turns of the resident blocks, a turn of a cluster a tenth longer for its barrier.
void shape(const RecArgs& a, int most, int per_sm, int* warps, int* ranks) {
    const int64_t runs = (a.len + RUN - 1) / RUN, units = a.seqs * a.tiles;
    *warps = 1;
    while (*warps < most && *warps < runs) *warps *= 2;
    double best = 0;
    *ranks = 0;
    for (int s = 1; s <= MOST_RANKS; s *= 2) {
        if (s > 1 && (int64_t)s * *warps / 2 >= runs) break;
        // the parts of eight blocks take the place of a third block, those of sixteen of a second one
        const int slots = SMS * (s > 8 ? 1 : s > 4 ? 2 : per_sm);
        const double turns = (double)((units * s + slots - 1) / slots), steps = (double)((runs + s * *warps - 1) / (s * *warps));
        const double cost = turns * steps * (s > 1 ? 1.1 : 1.0);
        if (!*ranks || cost < best) { best = cost; *ranks = s; }
    }
}

template <typename T, bool VEC, int FORM> ftp_status forward_as(const RecArgs& a, cudaStream_t st, const char* who) {
    const int64_t units = a.seqs * a.tiles;
    if (a.len <= RUN) {
        FTP_REQUIRE((units + 3) / 4 < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
        launch(recurrence_short_kernel<T, VEC, FORM>, dim3((unsigned)((units + 3) / 4)), dim3(128), 0, st, a);
        return FTP_OK;
    }
    int warps, ranks;
    shape(a, WARPS, 2, &warps, &ranks);
    FTP_REQUIRE(units * ranks < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    auto kern = recurrence_forward_kernel<T, VEC, FORM>;
    int* err = ffn::status_word();
    FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
    FTP_REQUIRE(ranks <= 8 || large_clusters(reinterpret_cast<const void*>(kern)), FTP_ECUDA, "%s: no clusters of %d blocks", who, ranks);
    const cudaError_t e = launch_cluster(kern, dim3((unsigned)(units * ranks)), 32 * warps, 0, ranks, st, a, err);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, bool VEC, int FORM> ftp_status backward_as(const RecArgs& a, cudaStream_t st, const char* who) {
    const int64_t units = a.seqs * a.tiles;
    int warps, ranks;
    shape(a, REG_WARPS<T>, sizeof(T) == 2 ? 3 : 2, &warps, &ranks);
    FTP_REQUIRE(units * ranks < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    auto kern = recurrence_backward_kernel<T, VEC, FORM>;
    const size_t smem = (size_t)(a.coupled ? 2 : 1) * RUN * 32 * warps * LANES<T> * 4;
    FTP_REQUIRE(more_shared(reinterpret_cast<const void*>(kern), 2 * RUN * 32 * WARPS * LANES<T> * 4), FTP_ECUDA, "%s: no shared memory", who);
    int* err = ffn::status_word();
    FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
    FTP_REQUIRE(ranks <= 8 || large_clusters(reinterpret_cast<const void*>(kern)), FTP_ECUDA, "%s: no clusters of %d blocks", who, ranks);
    const cudaError_t e = launch_cluster(kern, dim3((unsigned)(units * ranks)), 32 * warps, smem, ranks, st, a, err);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, int FORM> ftp_status forward_stream(const RecArgs& a, cudaStream_t st, const char* who) {
    const int64_t units = a.seqs * a.tiles;
    int warps, ranks;
    shape(a, WARPS, 2, &warps, &ranks);
    FTP_REQUIRE(units * ranks < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    Maps4 in{};
    CUtensorMap y;
    FTP_REQUIRE(tile_map<T>(&in.m[0], a.f, a.ldf, a) && tile_map<T>(&in.m[1], a.v, a.ldv, a) && (!FORM || tile_map<T>(&in.m[2], a.o, a.ldo, a)) && tile_map<T>(&y, a.y, a.ldy, a),
                FTP_ECUDA, "%s: cannot describe a tensor to the copy engine", who);
    int* err = ffn::status_word();
    FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
    auto kern = a.coupled ? recurrence_forward_stream_kernel<T, FORM, true> : recurrence_forward_stream_kernel<T, FORM, false>;
    const size_t maps = 2 * 32 * sizeof(Map<LANES<T>>), smem = 128 + warps * 6 * TILE_BYTES + maps * (warps + (ranks > 1 ? ranks : 0));
    FTP_REQUIRE(more_shared(reinterpret_cast<const void*>(kern), 128 + WARPS * 6 * TILE_BYTES + maps * (WARPS + MOST_RANKS)), FTP_ECUDA, "%s: no shared memory", who);
    FTP_REQUIRE(ranks <= 8 || large_clusters(reinterpret_cast<const void*>(kern)), FTP_ECUDA, "%s: no clusters of %d blocks", who, ranks);
    const cudaError_t e = launch_cluster(kern, dim3((unsigned)(units * ranks)), 32 * warps, smem, ranks, st, in, y, a, err);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, int FORM> ftp_status backward_stream(const RecArgs& a, cudaStream_t st, const char* who) {
    const int64_t units = a.seqs * a.tiles;
    int warps, ranks;
    shape(a, BACK_WARPS, 3, &warps, &ranks);
    FTP_REQUIRE(units * ranks < (1ll << 31), FTP_ERANGE, "%s: tensor too large", who);
    Maps4 in{}, out{};
    FTP_REQUIRE(tile_map<T>(&in.m[0], a.f, a.ldf, a) && tile_map<T>(&in.m[1], a.v, a.ldv, a) && (!FORM || tile_map<T>(&in.m[2], a.o, a.ldo, a)) && tile_map<T>(&in.m[3], a.dy, a.ldy, a) &&
                    tile_map<T>(&out.m[0], a.df, a.lddf, a) && tile_map<T>(&out.m[1], a.dv, a.lddv, a) && (!FORM || tile_map<T>(&out.m[2], a.dout, a.lddo, a)),
                FTP_ECUDA, "%s: cannot describe a tensor to the copy engine", who);
    int* err = ffn::status_word();
    FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
    auto kern = a.coupled ? recurrence_backward_stream_kernel<T, FORM, true> : recurrence_backward_stream_kernel<T, FORM, false>;
    const size_t maps = 2 * 32 * sizeof(Map<LANES<T>>), smem = 128 + warps * 8 * TILE_BYTES + maps * (warps + (ranks > 1 ? ranks : 0));
    FTP_REQUIRE(more_shared(reinterpret_cast<const void*>(kern), 128 + BACK_WARPS * 8 * TILE_BYTES + maps * (BACK_WARPS + MOST_RANKS)), FTP_ECUDA,
                "%s: no shared memory", who);
    FTP_REQUIRE(ranks <= 8 || large_clusters(reinterpret_cast<const void*>(kern)), FTP_ECUDA, "%s: no clusters of %d blocks", who, ranks);
    const cudaError_t e = launch_cluster(kern, dim3((unsigned)(units * ranks)), 32 * warps, smem, ranks, st, in, out, a, err);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}
template <typename T, bool VEC> ftp_status forward_of(const RecArgs& a, cudaStream_t st, const char* who) {
    if (a.len > RUN && whole_rows({a.f, a.v, a.o, a.y}, {a.ldf, a.ldv, a.o ? a.ldo : 0, a.ldy}, sizeof(T), a.rows))
        return !a.o ? forward_stream<T, 0>(a, st, who) : a.act == FTP_ACT_SILU ? forward_stream<T, 1>(a, st, who) : forward_stream<T, 2>(a, st, who);
    return !a.o ? forward_as<T, VEC, 0>(a, st, who) : a.act == FTP_ACT_SILU ? forward_as<T, VEC, 1>(a, st, who) : forward_as<T, VEC, 2>(a, st, who);
}
template <typename T, bool VEC> ftp_status backward_of(const RecArgs& a, cudaStream_t st, const char* who) {
    if (a.len > 0 && whole_rows({a.f, a.v, a.o, a.dy, a.df, a.dv, a.dout}, {a.ldf, a.ldv, a.o ? a.ldo : 0, a.ldy, a.lddf, a.lddv, a.o ? a.lddo : 0}, sizeof(T), a.rows))
        return !a.o ? backward_stream<T, 0>(a, st, who) : a.act == FTP_ACT_SILU ? backward_stream<T, 1>(a, st, who) : backward_stream<T, 2>(a, st, who);
    return !a.o ? backward_as<T, VEC, 0>(a, st, who) : a.act == FTP_ACT_SILU ? backward_as<T, VEC, 1>(a, st, who) : backward_as<T, VEC, 2>(a, st, who);
}

}  // namespace
}  // namespace token
}  // namespace ftp

using namespace ftp;
using namespace ftp::token;

extern "C" {

ftp_status ftp_recurrence_states(const ftp_recurrence_desc* d, int64_t* rows) {
    const char* who = "recurrence_states";
    if (ftp_status e = check_desc(d, who)) return e;
    FTP_REQUIRE(rows, FTP_EINVAL, "%s: null argument", who);
    *rows = (d->rows ? d->rows : d->seqs * d->len) / RUN + d->seqs;
    return FTP_OK;
}

ftp_status ftp_recurrence_forward(const ftp_recurrence_desc* d, const void* f, const void* v, const void* o, const float* h0, const int32_t* offsets, void* y,
                                  float* h1, float* states, void* stream) {
    const char* who = "recurrence_forward";
    if (ftp_status e = check_desc(d, who)) return e;
    if (ftp_status e = check_offsets(d, offsets, who)) return e;
    if (d->seqs == 0) return FTP_OK;
    RecArgs a{};
    fill(a, d, offsets);
    const bool empty = a.len == 0 || a.rows == 0;
    FTP_REQUIRE(empty || (f && v && y), FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(o || d->act == FTP_ACT_NONE, FTP_EINVAL, "%s: an activation without o", who);
    if (ftp_status e = check_elements({f, v, o, y}, d->precision == FTP_FP32 ? 4 : 2, who)) return e;
    if (ftp_status e = check_elements({h0, h1, states}, 4, who)) return e;
    if (ftp_status e = check_addresses({y, h1, states}, {f, v, o, offsets}, who)) return e;
    if (ftp_status e = check_addresses({y, states}, {h0}, who)) return e;
    a.f = f; a.v = v; a.o = o; a.h0 = h0; a.y = y; a.h1 = h1; a.states = states;
    if (empty) a.len = 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ftp_status e;
    if (d->precision == FTP_FP32) {
        a.tiles = (a.cols + TILE<float> - 1) / TILE<float>;
        e = forward_of<float, true>(a, st, who);
    } else {
        a.tiles = (a.cols + TILE<bf16> - 1) / TILE<bf16>;
        e = pairs({f, v, o, y}, {a.ldf, a.ldv, o ? a.ldo : 0, a.ldy}, a.cols) ? forward_of<bf16, true>(a, st, who) : forward_of<bf16, false>(a, st, who);
    }
    return e ? e : launched(who);
}

ftp_status ftp_recurrence_backward(const ftp_recurrence_desc* d, const void* f, const void* v, const void* o, const float* states, const int32_t* offsets,
                                   const void* dy, const float* dh1, void* df, void* dv, void* dout, float* dh0, void* stream) {
    const char* who = "recurrence_backward";
    if (ftp_status e = check_desc(d, who)) return e;
    if (ftp_status e = check_offsets(d, offsets, who)) return e;
    if (d->seqs == 0) return FTP_OK;
    RecArgs a{};
    fill(a, d, offsets);
    const bool empty = a.len == 0 || a.rows == 0;
    FTP_REQUIRE(empty || (f && v && states && dy && df && dv), FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE((o != nullptr) == (dout != nullptr), FTP_EINVAL, "%s: the gradient of o goes with o", who);
    FTP_REQUIRE(o || d->act == FTP_ACT_NONE, FTP_EINVAL, "%s: an activation without o", who);
    if (ftp_status e = check_elements({f, v, o, dy, df, dv, dout}, d->precision == FTP_FP32 ? 4 : 2, who)) return e;
    if (ftp_status e = check_elements({states, dh1, dh0}, 4, who)) return e;
    if (ftp_status e = check_addresses({df, dv, dout, dh0}, {f, v, o, states, offsets, dy}, who)) return e;
    if (ftp_status e = check_addresses({df, dv, dout}, {dh1}, who)) return e;
    a.f = f; a.v = v; a.o = o; a.dy = dy; a.dh1 = dh1; a.df = df; a.dv = dv; a.dout = dout; a.dh0 = dh0;
    a.states = const_cast<float*>(states);
    if (empty) a.len = 0;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    ftp_status e;
    if (d->precision == FTP_FP32) {
        a.tiles = (a.cols + TILE<float> - 1) / TILE<float>;
        e = backward_of<float, true>(a, st, who);
    } else {
        a.tiles = (a.cols + TILE<bf16> - 1) / TILE<bf16>;
        e = pairs({f, v, o, dy, df, dv, dout}, {a.ldf, a.ldv, o ? a.ldo : 0, a.ldy, a.lddf, a.lddv, o ? a.lddo : 0}, a.cols) ? backward_of<bf16, true>(a, st, who)
                                                                                                                             : backward_of<bf16, false>(a, st, who);
    }
    return e ? e : launched(who);
}

}  // extern "C"
