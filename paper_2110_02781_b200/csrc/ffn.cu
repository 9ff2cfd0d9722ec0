// Feed-forward operators: the kernels around the products (8-bit images, gradients through the activation, operand
// planes, bias gradients, the few-token products) and the C entry points.
#include <algorithm>
#include <atomic>
#include <initializer_list>
#include "ffn_math.cuh"
#include "kernels.h"
#include "launch.cuh"

namespace ftp {
namespace ffn {
namespace {

typedef __nv_bfloat16 bf16;
constexpr int SMS = 148;

template <typename... A>
void launch(A&&... args) {
    ++launches();
    ftp::launch(std::forward<A>(args)...);
}

__device__ int g_op_status;                  // set by a kernel whose bounded wait ran out; cleared by ftp_check_op_status
std::atomic<int*> g_status_addr[64] = {};

template <typename T> using Words8 = Words<T, 2 * (int)sizeof(T)>;
__device__ __forceinline__ void values8(const Words8<float>& r, int valid, float (&v)[8]) {
    unsigned u[8];
    r.end(valid, u);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(u[i]);
}
__device__ __forceinline__ void values8(const Words8<bf16>& r, int valid, float (&v)[8]) {
    unsigned u[4];
    r.end(valid, u);
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf_lo(u[i]); v[2 * i + 1] = bf_hi(u[i]); }
}

// One plane (bf16 rounding) or three (24 mantissa bits) of eight values; rows of a plane start on 16 bytes.
// A float is its nearest bf16, the nearest bf16 of the rest and the rest of that; both subtractions are exact.  A value
// that rounds beyond the largest bf16 is cut instead of rounded; an infinity or NaN goes to the first plane alone.
__device__ __forceinline__ void store_planes(bf16* p, long long plane, int planes, const float (&v)[8]) {
    unsigned o[4];
    if (planes == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = bf_pack(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<uint4*>(p) = make_uint4(o[0], o[1], o[2], o[3]);
        return;
    }
    float r[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = v[i];
#pragma unroll
    for (int s = 0; s < 3; ++s) {
        float h[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = __bfloat162float(__float2bfloat16(r[i]));
            if (s == 0) {
                const bool fin = (__float_as_uint(r[i]) & 0x7f800000u) != 0x7f800000u;
                if (fin && (__float_as_uint(h[i]) & 0x7fffffffu) == 0x7f800000u) h[i] = __uint_as_float(__float_as_uint(r[i]) & 0xffff0000u);
                r[i] = fin ? r[i] - h[i] : 0.f;
            } else
                r[i] -= h[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = bf_pack(h[2 * i], h[2 * i + 1]);
        *reinterpret_cast<uint4*>(p + s * plane) = make_uint4(o[0], o[1], o[2], o[3]);
    }
}

// Kernels that walk a matrix in groups of eight columns: EIGHT_U groups per thread and trip, their loads in flight together;
// group numbers have 32 bits (larger matrices are cut into launches of whole rows, see by_rows).
constexpr int EIGHT_U = 4;
struct Groups { unsigned total, per_row; };
template <typename F> __device__ __forceinline__ void group_at(const Groups& g, unsigned i, F&& f) {
    const unsigned r = i / g.per_row;
    f((long long)r, (int)(i - r * g.per_row) * 8);
}

// ---- operand planes: copies of bf16 rows at an aligned pitch, or the three planes of float rows ----
template <typename T>
__global__ void __launch_bounds__(256) planes_kernel(const T* __restrict__ x, const Groups g, int cols, long long ld, const Span all,
                                                     bf16* __restrict__ out, long long plane, int planes) {
    grid_dep_sync();
    const long long pitch = 8ll * g.per_row;
    for (unsigned i0 = blockIdx.x * 256 * EIGHT_U + threadIdx.x; i0 < g.total; i0 += gridDim.x * 256 * EIGHT_U) {
        Words8<T> raw[EIGHT_U];
#pragma unroll
        for (int u = 0; u < EIGHT_U; ++u)
            if (i0 + u * 256 < g.total) group_at(g, i0 + u * 256, [&](long long r, int c) { raw[u].begin(x + r * ld + c, cols - c, all); });
#pragma unroll
        for (int u = 0; u < EIGHT_U; ++u)
            if (i0 + u * 256 < g.total)
                group_at(g, i0 + u * 256, [&](long long r, int c) {
                    float v[8];
                    values8(raw[u], cols - c, v);
                    store_planes(out + r * pitch + c, plane, planes, v);
                });
    }
}

// ---- 8-bit images ----
// Sixteen values as they are in memory, zeros behind `valid`; VEC: rows on 16 bytes.
template <typename T> struct Raw16 { uint4 q[sizeof(T)]; };
template <typename T, bool VEC> struct Fetch16 {
    Words<T, 4 * (int)sizeof(T)> r;
    __device__ __forceinline__ void begin(const T* p, int valid, const Span& all) { r.begin(p, valid, all); }
    __device__ __forceinline__ Raw16<T> end(int valid) const {
        unsigned u[4 * sizeof(T)];
        r.end(valid, u);
        Raw16<T> o;
#pragma unroll
        for (int k = 0; k < (int)sizeof(T); ++k) o.q[k] = make_uint4(u[4 * k], u[4 * k + 1], u[4 * k + 2], u[4 * k + 3]);
        return o;
    }
};
template <typename T> struct Fetch16<T, true> {
    Raw16<T> r;
    __device__ __forceinline__ void begin(const T* p, int valid, const Span&) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T); ++k) r.q[k] = make_uint4(0u, 0u, 0u, 0u);
        if (valid >= 16) {
#pragma unroll
            for (int k = 0; k < (int)sizeof(T); ++k) r.q[k] = reinterpret_cast<const uint4*>(p)[k];
        } else {
            T* e = reinterpret_cast<T*>(r.q);
#pragma unroll
            for (int k = 0; k < 16; ++k) if (k < valid) e[k] = p[k];
        }
    }
    __device__ __forceinline__ Raw16<T> end(int) const { return r; }
};
__device__ __forceinline__ unsigned top16(const Raw16<float>& r) {   // bits of the largest magnitude, as a float's
    unsigned m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) m = max(max(max(r.q[k].x & 0x7fffffffu, r.q[k].y & 0x7fffffffu), max(r.q[k].z & 0x7fffffffu, r.q[k].w & 0x7fffffffu)), m);
    return m;
}
__device__ __forceinline__ unsigned top16(const Raw16<bf16>& r) {
    unsigned m = 0;                                                  // two at a time: magnitudes of bf16 compare as 16-bit integers
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        m = __vmaxu2(m, __vmaxu2(r.q[k].x & 0x7fff7fffu, r.q[k].y & 0x7fff7fffu));
        m = __vmaxu2(m, __vmaxu2(r.q[k].z & 0x7fff7fffu, r.q[k].w & 0x7fff7fffu));
    }
    return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ void values16(const Raw16<float>& r, float (&v)[16]) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        v[4 * k] = __uint_as_float(r.q[k].x); v[4 * k + 1] = __uint_as_float(r.q[k].y);
        v[4 * k + 2] = __uint_as_float(r.q[k].z); v[4 * k + 3] = __uint_as_float(r.q[k].w);
    }
}
__device__ __forceinline__ void values16(const Raw16<bf16>& r, float (&v)[16]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const unsigned u[4] = {r.q[k].x, r.q[k].y, r.q[k].z, r.q[k].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[8 * k + 2 * i] = bf_lo(u[i]); v[8 * k + 2 * i + 1] = bf_hi(u[i]); }
    }
}

// A thread holds 16 columns, two neighbouring threads a block of 32; U such pieces in flight: PACK_U, or one where that
// many would leave multiprocessors without a block.  Bound by instructions as much as by memory (8 columns, integer
// conversions and a piece at a time: 55 us for 16384 x 4096 bf16).
constexpr int PACK_U = 4;
template <typename T, int U, bool VEC>
__global__ void __launch_bounds__(256) pack_kernel(const T* __restrict__ x, const Groups g, int cols, long long ld, const Span all, const Image im) {
    grid_dep_sync();                                                 // g: groups of 16 columns here
    for (unsigned b0 = blockIdx.x * 256 * U; b0 < g.total; b0 += gridDim.x * 256 * U) {
        Fetch16<T, VEC> got[U];
        unsigned row[U], col[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned i = min(b0 + threadIdx.x + u * 256, g.total - 1);       // whole warps take part in the exchange below
            row[u] = i / g.per_row;
            col[u] = (i - row[u] * g.per_row) * 16;
            got[u].begin(x + (long long)row[u] * ld + col[u], max(0, cols - (int)col[u]), all);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const Raw16<T> raw = got[u].end(max(0, cols - (int)col[u]));
            unsigned top = top16(raw);
            top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
            const unsigned e = img_exp(top);
            const float inv = img_inv(e);
            float v[16];
            values16(raw, v);
            unsigned w[4];
            if (__uint_as_float(top) * inv < 127.5f) {               // no code is cut to 127
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    w[k] = pack_codes(__float_as_uint(fmaf(v[4 * k], inv, IMG_MAGIC)), __float_as_uint(fmaf(v[4 * k + 1], inv, IMG_MAGIC)),
                                      __float_as_uint(fmaf(v[4 * k + 2], inv, IMG_MAGIC)), __float_as_uint(fmaf(v[4 * k + 3], inv, IMG_MAGIC)));
            } else {
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = pack_codes(img_code(v[4 * k], inv), img_code(v[4 * k + 1], inv), img_code(v[4 * k + 2], inv), img_code(v[4 * k + 3], inv));
            }
            if (b0 + threadIdx.x + u * 256 < g.total) {
                *reinterpret_cast<uint4*>(im.q + row[u] * im.pitch + col[u]) = make_uint4(w[0], w[1], w[2], w[3]);
                if ((threadIdx.x & 1) == 0) im.e[row[u] * (im.pitch / IMG_BLOCK) + col[u] / IMG_BLOCK] = (uint8_t)e;
            }
        }
    }
}

struct Img8 { uint2 q; unsigned e; };
__device__ __forceinline__ Img8 img_fetch8(const Image& im, long long r, int c) {
    return Img8{*reinterpret_cast<const uint2*>(im.q + r * im.pitch + c), im.e[r * (im.pitch / IMG_BLOCK) + c / IMG_BLOCK]};
}
__device__ __forceinline__ void img_values8(const Img8& i, float (&v)[8]) {
    const float s = img_scale(i.e);
    float a[4], b[4];
    unpack_codes(i.q.x, s, a);
    unpack_codes(i.q.y, s, b);
#pragma unroll
    for (int k = 0; k < 4; ++k) { v[k] = a[k]; v[4 + k] = b[k]; }
}

__device__ __forceinline__ void store16(float* p, int valid, bool vec, const float (&v)[16]) {
    if (vec && valid >= 16) {
#pragma unroll
        for (int k = 0; k < 4; ++k) reinterpret_cast<float4*>(p)[k] = make_float4(v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) if (i < valid) p[i] = v[i];
}
__device__ __forceinline__ void store16(bf16* p, int valid, bool vec, const float (&v)[16]) {
    if (vec && valid >= 16) {
#pragma unroll
        for (int k = 0; k < 2; ++k)
            reinterpret_cast<uint4*>(p)[k] = make_uint4(bf_pack(v[8 * k], v[8 * k + 1]), bf_pack(v[8 * k + 2], v[8 * k + 3]), bf_pack(v[8 * k + 4], v[8 * k + 5]),
                                                        bf_pack(v[8 * k + 6], v[8 * k + 7]));
        return;
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) if (i < valid) p[i] = __float2bfloat16(v[i]);
}

// out: `ld` elements between rows; g: groups of 16 columns; block `block` of `blocks`
template <typename T, int U>
__device__ __forceinline__ void unpack_blocks(const Image& im, const Groups& g, int cols, T* __restrict__ out, long long ld, bool vec, unsigned block, unsigned blocks) {
    for (unsigned b0 = block * 256 * U; b0 < g.total; b0 += blocks * 256 * U) {
        uint4 q[U];
        unsigned e[U], row[U], col[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const unsigned i = min(b0 + threadIdx.x + u * 256, g.total - 1);
            row[u] = i / g.per_row;
            col[u] = (i - row[u] * g.per_row) * 16;
            q[u] = *reinterpret_cast<const uint4*>(im.q + row[u] * im.pitch + col[u]);
            e[u] = im.e[row[u] * (im.pitch / IMG_BLOCK) + col[u] / IMG_BLOCK];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (b0 + threadIdx.x + u * 256 >= g.total) break;
            const float s = img_scale(e[u]);
            const unsigned w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
            float v[16];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float f[4];
                unpack_codes(w[k], s, f);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[4 * k + i] = f[i];
            }
            store16(out + (long long)row[u] * ld + col[u], cols - (int)col[u], vec, v);
        }
    }
}
template <typename T, int U>
__global__ void __launch_bounds__(256) unpack_kernel(const Image im, const Groups g, int cols, T* __restrict__ out, long long ld, bool vec) {
    grid_dep_sync();
    unpack_blocks<T, U>(im, g, cols, out, ld, vec, blockIdx.x, gridDim.x);
}

// launch(first row, Groups, blocks) for pieces of at most 2^30 groups
template <typename F>
void by_rows(long long rows, long long per_row, F&& launch_piece) {
    const long long most = std::max<long long>(1, (1ll << 30) / per_row);
    for (long long r = 0; r < rows; r += most) {
        const long long n = std::min(most, rows - r), total = n * per_row;
        const long long blocks = (total + 256 * EIGHT_U - 1) / (256 * EIGHT_U);
        launch_piece(r, Groups{(unsigned)total, (unsigned)per_row}, dim3((unsigned)std::min<long long>(blocks, SMS * 64)));
    }
}
template <typename T>
void launch_planes(const T* x, long long rows, long long cols, long long ld, bf16* out, long long plane, int planes, cudaStream_t st) {
    const long long pitch = (cols + 7) / 8 * 8;
    by_rows(rows, pitch / 8, [&](long long r, Groups g, dim3 blocks) {
        launch(planes_kernel<T>, blocks, dim3(256), 0, st, x + r * ld, g, (int)cols, ld, span_of<T>(x, rows, cols, ld), out + r * pitch, plane, planes);
    });
}
inline Image image_from(const Image& im, long long r) { return Image{im.q + r * im.pitch, im.e + r * (im.pitch / IMG_BLOCK), im.pitch}; }
// one piece per thread where four leave multiprocessors idle
inline bool few_pieces(const Groups& g) { return g.total <= SMS * 256 * PACK_U; }
template <typename T>
void launch_pack(const T* x, long long rows, long long cols, long long ld, const Image& im, cudaStream_t st) {
    const bool vec = aligned(x, 16) && ld * (long long)sizeof(T) % 16 == 0;
    const Span all = span_of<T>(x, rows, cols, ld);
    by_rows(rows, im.pitch / 16, [&](long long r, Groups g, dim3 blocks) {
        const T* from = x + r * ld;
        const bool few = few_pieces(g);
        auto kern = few ? (vec ? pack_kernel<T, 1, true> : pack_kernel<T, 1, false>) : (vec ? pack_kernel<T, PACK_U, true> : pack_kernel<T, PACK_U, false>);
        launch(kern, few ? dim3((g.total + 255) / 256) : blocks, dim3(256), 0, st, from, g, (int)cols, ld, all, image_from(im, r));
    });
}
template <typename T>
void launch_unpack(const Image& im, long long rows, long long cols, T* out, long long ld, cudaStream_t st) {
    const bool vec = aligned(out, 16) && ld * (long long)sizeof(T) % 16 == 0;
    by_rows(rows, (cols + 15) / 16, [&](long long r, Groups g, dim3 blocks) {
        T* to = out + r * ld;
        if (few_pieces(g)) launch(unpack_kernel<T, 1>, dim3((g.total + 255) / 256), dim3(256), 0, st, image_from(im, r), g, (int)cols, to, ld, vec);
        else launch(unpack_kernel<T, PACK_U>, blocks, dim3(256), 0, st, image_from(im, r), g, (int)cols, to, ld, vec);
    });
}

// ---- operands of the products, made in one launch ----
// Up to three matrices that have to be copied, split into planes or unpacked before a product can read them; as blocks of
// their own in one kernel, or behind the blocks of the gradient kernel: a small call costs its launches.
enum { JOB_PLANES = 0, JOB_IMAGE = 1 };
struct Job {
    const void* src; Span all;               // JOB_PLANES
    Image im;                                // JOB_IMAGE
    long long ld;                            // elements between rows of src (JOB_IMAGE: of out)
    bf16* out; long long plane; int planes, cols, kind;
    Groups g;                                // groups of eight columns (JOB_IMAGE: sixteen)
    unsigned blocks;
};
struct Jobs { Job job[3]; int n; unsigned blocks; };

template <typename T>
__device__ __forceinline__ void run_jobs(const Jobs& all, unsigned block) {
    int j = 0;
    while (block >= all.job[j].blocks) block -= all.job[j++].blocks;
    const Job& p = all.job[j];
    if (p.kind == JOB_IMAGE) { unpack_blocks<bf16, PACK_U>(p.im, p.g, p.cols, p.out, p.ld, true, block, p.blocks); return; }
    const long long pitch = 8ll * p.g.per_row;
    for (unsigned i0 = block * 256 * EIGHT_U + threadIdx.x; i0 < p.g.total; i0 += p.blocks * 256 * EIGHT_U) {
        Words8<T> raw[EIGHT_U];
#pragma unroll
        for (int u = 0; u < EIGHT_U; ++u)
            if (i0 + u * 256 < p.g.total) group_at(p.g, i0 + u * 256, [&](long long r, int c) { raw[u].begin(static_cast<const T*>(p.src) + r * p.ld + c, p.cols - c, p.all); });
#pragma unroll
        for (int u = 0; u < EIGHT_U; ++u)
            if (i0 + u * 256 < p.g.total)
                group_at(p.g, i0 + u * 256, [&](long long r, int c) {
                    float v[8];
                    values8(raw[u], p.cols - c, v);
                    store_planes(p.out + r * pitch + c, p.plane, p.planes, v);
                });
    }
}
template <typename T>
__global__ void __launch_bounds__(256) jobs_kernel(const __grid_constant__ Jobs jobs) {
    grid_dep_sync();
    run_jobs<T>(jobs, blockIdx.x);
}
// false: too large for 32-bit group numbers
inline bool add_job(Jobs& all, Job j, long long rows, long long cols) {
    const int width = j.kind == JOB_IMAGE ? 16 : 8;
    const long long per_row = (cols + width - 1) / width, total = rows * per_row;
    if (total > 1 << 30 || all.n == 3) return false;
    j.cols = (int)cols;
    j.g = Groups{(unsigned)total, (unsigned)per_row};
    j.blocks = (unsigned)std::min<long long>((total + 256 * EIGHT_U - 1) / (256 * EIGHT_U), SMS * 16);
    all.job[all.n++] = j;
    all.blocks += j.blocks;
    return true;
}
template <typename T>
void run_now(Jobs& all, cudaStream_t st) {
    if (all.n) launch(jobs_kernel<T>, dim3(all.blocks), dim3(256), 0, st, all);
    all = Jobs{};
}

// ---- gradients through the activation ----
struct GradArgs {
    const void* dy; long long lddy;
    const void* pre[2];                      // STASH_FULL: `cols` elements between rows
    Image img[2];
    int act;
    long long rows; int cols;
    bf16* out[2]; long long plane; int planes;   // nullable; pitch = cols rounded up to 8
    float* sums;                             // nullable: [block rows][cols] column sums of a block row
    int rows_per_block;
    Span all_dy, all_pre[2];                 // where whole parts of rows off 16 bytes may be read
    unsigned blocks_x, blocks;               // of the gradient itself: along the columns, all; the blocks behind them run the jobs
};

// Eight values as they are in memory, every access fits
template <typename T> struct Raw8 { uint4 q[sizeof(T) / 2]; };
template <typename T, bool VEC> struct Fetch8 {
    Words8<T> r;
    __device__ __forceinline__ void begin(const T* p, int valid, const Span& all) { r.begin(p, valid, all); }
};
template <typename T> struct Fetch8<T, true> {
    Raw8<T> r;
    __device__ __forceinline__ void begin(const T* p, int, const Span&) {
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) r.q[k] = __ldcs(reinterpret_cast<const uint4*>(p) + k);
    }
};
__device__ __forceinline__ void values8(const Raw8<float>& r, int, float (&v)[8]) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        v[4 * k] = __uint_as_float(r.q[k].x); v[4 * k + 1] = __uint_as_float(r.q[k].y);
        v[4 * k + 2] = __uint_as_float(r.q[k].z); v[4 * k + 3] = __uint_as_float(r.q[k].w);
    }
}
__device__ __forceinline__ void values8(const Raw8<bf16>& r, int, float (&v)[8]) {
    const unsigned u[4] = {r.q[0].x, r.q[0].y, r.q[0].z, r.q[0].w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = bf_lo(u[i]); v[2 * i + 1] = bf_hi(u[i]); }
}

// act and its derivative at eight values, the choice outside the loop
template <bool FAST>
__device__ __forceinline__ void act_both8(const float (&z)[8], int act, float (&a)[8], float (&d)[8]) {
    switch (act) {
        case FTP_ACT_RELU:
#pragma unroll
            for (int k = 0; k < 8; ++k) act_both<FAST>(z[k], FTP_ACT_RELU, a[k], d[k]);
            break;
        case FTP_ACT_RELU6:
#pragma unroll
            for (int k = 0; k < 8; ++k) act_both<FAST>(z[k], FTP_ACT_RELU6, a[k], d[k]);
            break;
        case FTP_ACT_GELU:
#pragma unroll
            for (int k = 0; k < 8; ++k) act_both<FAST>(z[k], FTP_ACT_GELU, a[k], d[k]);
            break;
        case FTP_ACT_SILU:
#pragma unroll
            for (int k = 0; k < 8; ++k) act_both<FAST>(z[k], FTP_ACT_SILU, a[k], d[k]);
            break;
        default:
#pragma unroll
            for (int k = 0; k < 8; ++k) act_both<FAST>(z[k], FTP_ACT_NONE, a[k], d[k]);
    }
}

// linear: dz = dy act'(z).  gated: dg = dy u act'(g), du = dy act(g).  KIND: form of z or of g and u (STASH_NONE: the
// gradient passes unchanged).  A thread keeps eight columns and walks down rows_per_block / 8 rows, R of them in flight,
// so the column sums of dz cost registers only; they are added up in float over at most 64 values and then across warps and
// block rows in double, in a fixed order.  With one row in flight 2.3 TB/s at 8192 x 12288 bf16.
template <typename T, bool GATED, int KIND, bool VEC>
__global__ void __launch_bounds__(256) grad_kernel(const __grid_constant__ GradArgs p, const __grid_constant__ Jobs jobs) {
    grid_dep_sync();
    if (blockIdx.x >= p.blocks) { run_jobs<T>(jobs, blockIdx.x - p.blocks); return; }
    const int by = blockIdx.x / p.blocks_x, bx = blockIdx.x - by * p.blocks_x;
    constexpr bool FAST = sizeof(T) == 2;
    constexpr int R = VEC && sizeof(T) == 2 ? 4 : 2, P = GATED ? 2 : 1;
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = (bx * 32 + tx) * 8, valid = p.cols - c;
    const long long pitch = (p.cols + 7) / 8 * 8, r0 = (long long)by * p.rows_per_block, r1 = min(p.rows, r0 + p.rows_per_block);
    float sum[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (valid > 0) {
        for (long long rb = r0 + ty; rb < r1; rb += 8 * R) {
            Fetch8<T, VEC> dy[R], pre[P][R];
            Img8 img[P][R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const long long r = min(rb + 8 * i, r1 - 1);
                dy[i].begin(static_cast<const T*>(p.dy) + r * p.lddy + c, valid, p.all_dy);
#pragma unroll
                for (int q = 0; q < P; ++q) {
                    if (KIND == STASH_FULL) pre[q][i].begin(static_cast<const T*>(p.pre[q]) + r * p.cols + c, valid, p.all_pre[q]);
                    if (KIND == STASH_8BIT) img[q][i] = img_fetch8(p.img[q], r, c);
                }
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const long long r = rb + 8 * i;
                if (r >= r1) break;
                float d[8], z[8], a[8], da[8];
                values8(dy[i].r, valid, d);
                if (KIND == STASH_FULL) values8(pre[0][i].r, valid, z);
                if (KIND == STASH_8BIT) img_values8(img[0][i], z);
                if (KIND != STASH_NONE) act_both8<FAST>(z, p.act, a, da);
                if (GATED) {
                    float u[8], o[8];
                    if (KIND == STASH_FULL) values8(pre[P - 1][i].r, valid, u);
                    if (KIND == STASH_8BIT) img_values8(img[P - 1][i], u);
#pragma unroll
                    for (int k = 0; k < 8; ++k) { o[k] = d[k] * u[k] * da[k]; d[k] *= a[k]; }
                    if (!VEC)
#pragma unroll
                        for (int k = 0; k < 8; ++k) if (k >= valid) o[k] = d[k] = 0.f;
                    store_planes(p.out[0] + r * pitch + c, p.plane, p.planes, o);
                    store_planes(p.out[1] + r * pitch + c, p.plane, p.planes, d);
                } else {
                    if (KIND != STASH_NONE) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) d[k] *= da[k];
                    }
                    if (!VEC)
#pragma unroll
                        for (int k = 0; k < 8; ++k) if (k >= valid) d[k] = 0.f;
                    if (p.out[0]) store_planes(p.out[0] + r * pitch + c, p.plane, p.planes, d);
                    if (p.sums) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) sum[k] += d[k];
                    }
                }
            }
        }
    }
    if (!GATED && p.sums) {
        __shared__ float red[8][32 * 8 + 8];
#pragma unroll
        for (int k = 0; k < 8; ++k) red[ty][tx * 8 + k] = sum[k];
        __syncthreads();
        const int col = bx * 256 + threadIdx.x;
        if (col < p.cols) {
            double s = 0.0;
#pragma unroll
            for (int k = 0; k < 8; ++k) s += (double)red[k][threadIdx.x];
            p.sums[(long long)by * p.cols + col] = (float)s;
        }
    }
}
template <typename T, bool GATED, int KIND>
void launch_grad(GradArgs& g, bool vec, int chunks, Jobs& jobs, cudaStream_t st) {
    g.blocks_x = (unsigned)((g.cols + 255) / 256);
    g.blocks = g.blocks_x * chunks;
    launch(vec ? grad_kernel<T, GATED, KIND, true> : grad_kernel<T, GATED, KIND, false>, dim3(g.blocks + jobs.blocks), dim3(256), 0, st, g, jobs);
    jobs = Jobs{};
}

__global__ void __launch_bounds__(256) sums_kernel(const float* __restrict__ part, int chunks, int cols, float* __restrict__ out) {
    grid_dep_sync();
    __shared__ double red[8][33];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = blockIdx.x * 32 + tx;
    double s = 0.0;
    if (c < cols)
        for (int i = ty; i < chunks; i += 8) s += (double)part[(long long)i * cols + c];
    red[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && c < cols) {
#pragma unroll
        for (int k = 1; k < 8; ++k) s += red[k][tx];
        out[c] = (float)s;
    }
}

// ---- the workspace ----
struct Carve {
    char* base; size_t off = 0, size;
    bool dry() const { return base == nullptr; }
    void* take(size_t bytes) {
        void* p = base ? base + off : nullptr;
        off = (off + bytes + 255) / 256 * 256;
        return p;
    }
};

inline long long up8(long long n) { return (n + 7) / 8 * 8; }

// `rows` x `cols` of type T at `src` as an operand.  bf16 rows on 16 bytes are read in place, others copied; float rows
// become three planes.
template <typename T>
ftp_status make_operand(Operand* o, const void* src, long long rows, long long cols, long long ld, bool unaligned, Carve& ws, Jobs& jobs, cudaStream_t st, const char* who) {
    const bool f32 = sizeof(T) == 4;
    if (rows == 1) ld = up8(cols);                                   // never stepped over
    if (!f32 && !unaligned && ld % 8 == 0) {
        if (!ws.dry()) FTP_REQUIRE(aligned(src, 16), FTP_ERANGE, "%s: an operand does not start on a 16-byte boundary (set `unaligned`)", who);
        *o = Operand{static_cast<const bf16*>(src), rows, cols, ld, 0, 1};
        return FTP_OK;
    }
    const int planes = f32 ? 3 : 1;
    const long long pitch = up8(cols), plane = rows * pitch;
    bf16* p = static_cast<bf16*>(ws.take((size_t)plane * planes * 2));
    *o = Operand{p, rows, cols, pitch, plane, planes};
    if (ws.dry()) return FTP_OK;
    Job j{};
    j.kind = JOB_PLANES;
    j.all = span_of<T>(src, rows, cols, ld);
    j.src = src; j.ld = ld;
    j.out = p; j.plane = plane; j.planes = planes;
    if (!add_job(jobs, j, rows, cols)) launch_planes(static_cast<const T*>(src), rows, cols, ld, p, plane, planes, st);
    return FTP_OK;
}

// the values of an 8-bit image as an operand: one bf16 plane, exact
ftp_status image_operand(Operand* o, const void* image, long long rows, long long cols, Carve& ws, Jobs& jobs, cudaStream_t st) {
    const long long pitch = up8(cols);
    bf16* p = static_cast<bf16*>(ws.take((size_t)(rows * pitch) * 2));
    *o = Operand{p, rows, cols, pitch, rows * pitch, 1};
    if (ws.dry()) return FTP_OK;
    Job j{};
    j.kind = JOB_IMAGE;
    j.im = image_at(const_cast<void*>(image), rows, cols, 0);
    j.out = p; j.ld = pitch; j.planes = 1;
    if (!add_job(jobs, j, rows, cols)) launch_unpack(j.im, rows, cols, p, pitch, st);
    return FTP_OK;
}

ftp_status check_desc(const ftp_ffn_desc* d, const char* who) {
    FTP_REQUIRE(d, FTP_EINVAL, "%s: null descriptor", who);
    FTP_REQUIRE(d->precision == FTP_FP32 || d->precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, d->precision);
    FTP_REQUIRE(d->act >= FTP_ACT_NONE && d->act <= FTP_ACT_SILU, FTP_EINVAL, "%s: unknown activation %d", who, d->act);
    FTP_REQUIRE(d->stash >= STASH_NONE && d->stash <= STASH_8BIT, FTP_EINVAL, "%s: unknown form of kept values %d", who, d->stash);
    FTP_REQUIRE(d->rows >= 0 && d->cin >= 1 && d->cout >= 1, FTP_EINVAL, "%s: rows must not be negative, cin and cout must be positive", who);
    FTP_REQUIRE(d->rows < (1ll << 31) - 256 && d->cin < (1 << 30) && d->cout < (1 << 30), FTP_ERANGE, "%s: tensor too large", who);
    const long long mx = std::max<long long>(d->cin, d->cout), most = 1ll << 38;
    FTP_REQUIRE(d->rows * mx <= most && (long long)d->cin * d->cout <= most, FTP_ERANGE, "%s: tensor too large", who);
    FTP_REQUIRE((d->ldx == 0 || d->ldx >= d->cin) && (d->lddx == 0 || d->lddx >= d->cin) && (d->ldw == 0 || d->ldw >= d->cout) &&
                    (d->lddw == 0 || d->lddw >= d->cout) && (d->ldy == 0 || d->ldy >= d->cout), FTP_EINVAL, "%s: rows overlap (a pitch below the width)", who);
    FTP_REQUIRE(d->ldx < (1ll << 35) && d->lddx < (1ll << 35) && d->ldw < (1ll << 35) && d->lddw < (1ll << 35) && d->ldy < (1ll << 35) && d->ldr >= 0 &&
                    d->ldr < (1ll << 35), FTP_ERANGE, "%s: pitch too large", who);
    return FTP_OK;
}

template <typename T> int access_of(const void* p, long long ld) {
    if (aligned(p, 16) && ld * (long long)sizeof(T) % 16 == 0) return 2;
    return aligned(p, 4 * sizeof(T)) && ld % 4 == 0 ? 1 : 0;
}

template <typename T>
void set_out(Epi& e, void* y, long long ldy, const void* add, long long ldadd) {
    e.y = y; e.ldy = ldy; e.vec_y = access_of<T>(y, ldy);
    e.add = add; e.ldadd = ldadd; e.vec_add = add ? access_of<T>(add, ldadd) : 0;
}
template <typename T>
void set_stash(Epi& e, int kind, void* stash, long long rows, long long cols, int parts) {
    e.stash_kind = kind;
    for (int i = 0; i < parts; ++i) {
        if (kind == STASH_FULL) e.stash[i] = static_cast<T*>(stash) + (long long)i * rows * cols;
        if (kind == STASH_8BIT) e.img[i] = image_at(stash, rows, cols, i);
    }
    e.ldstash = cols;
    if (kind == STASH_FULL) e.vec_stash = std::min(access_of<T>(stash, cols), parts == 1 ? 2 : access_of<T>(e.stash[1], cols));
}

ftp_status check_stash(const ftp_ffn_desc* d, const void* stash, const char* who) {
    FTP_REQUIRE((d->stash != STASH_NONE) == (stash != nullptr), FTP_EINVAL, "%s: the descriptor and the pointer disagree on whether values are kept", who);
    FTP_REQUIRE(d->stash != STASH_8BIT || aligned(stash, 32), FTP_ERANGE, "%s: an image must start on a 32-byte boundary", who);
    return FTP_OK;
}
// Addresses: multiples of their elements' size, and no output where an input or another output starts (further overlaps
// cannot be told from columns of one matrix, which may be neighbours).
ftp_status check_addresses(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins, const char* who) {
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        if (!*o) continue;
        for (const void* i : ins) FTP_REQUIRE(*o != i, FTP_EINVAL, "%s: an output lies on an input", who);
        for (auto q = outs.begin(); q != o; ++q) FTP_REQUIRE(*o != *q, FTP_EINVAL, "%s: two outputs in one place", who);
    }
    return FTP_OK;
}
// An addend may be the result itself, element by element: with another pitch a row would be read after it was overwritten.
ftp_status check_in_place(const void* add, const void* out, int64_t ldadd, int64_t ldout, int64_t rows, int32_t cols, const char* who) {
    FTP_REQUIRE(!add || add != out || rows == 1 || (ldadd ? ldadd : cols) == (ldout ? ldout : cols), FTP_EINVAL, "%s: an addend in place of its result with another pitch", who);
    return FTP_OK;
}
ftp_status check_elements(std::initializer_list<const void*> all, size_t bytes, const char* who) {
    for (const void* p : all) FTP_REQUIRE(aligned(p, bytes), FTP_ERANGE, "%s: an address is not a multiple of its elements' size", who);
    return FTP_OK;
}
ftp_status check_ws(const Carve& need, const void* ws, size_t ws_bytes, const char* who) {
    FTP_REQUIRE(need.off == 0 || (ws && ws_bytes >= need.off), FTP_ENOMEM, "%s: workspace of %zu bytes, %zu needed", who, ws_bytes, need.off);
    FTP_REQUIRE(need.off == 0 || aligned(ws, 256), FTP_ERANGE, "%s: workspace must start on a 256-byte boundary", who);
    return FTP_OK;
}
ftp_status launched(const char* who) {
    const cudaError_t e = cudaGetLastError();
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}

// ---- forward of both operators (w[1]: the gated operator's second matrix) ----
template <typename T, bool GATED>
ftp_status forward(const ftp_ffn_desc* d, const void* x, const void* const* w, const float* bias, const void* residual, void* y, int stash_kind, void* stash,
                   Carve& ws, int* err, cudaStream_t st, const char* who, const Operand* given_x = nullptr, const Operand* given_w = nullptr) {
    Product p{};
    const long long ldx = d->ldx ? d->ldx : d->cin, ldw = d->ldw ? d->ldw : d->cout, ldy = d->ldy ? d->ldy : d->cout;
    p.e[0].bias = bias; p.e[0].act = d->act;
    p.e[0].vec_bias = bias && aligned(bias, 16);
    set_out<T>(p.e[0], y, ldy, residual, d->ldr ? d->ldr : d->cout);
    set_stash<T>(p.e[0], stash_kind, stash, d->rows, d->cout, GATED ? 2 : 1);
    if (!given_x && few_tokens(d->rows, d->cin, d->cout, sizeof(T) == 4, GATED ? 2 : 1)) {
        if (ws.dry()) return FTP_OK;
        if (!err) err = status_word();
        FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
        return run_few(x, ldx, w, ldw, GATED ? 2 : 1, (int)d->rows, d->cin, d->cout, sizeof(T) == 4, p.e[0], err, st, who);
    }
    Jobs jobs{};
    if (given_x) p.A[0] = *given_x;
    else if (ftp_status s = make_operand<T>(&p.A[0], x, d->rows, d->cin, ldx, d->unaligned, ws, jobs, st, who)) return s;
    for (int i = 0; i < (GATED ? 2 : 1); ++i) {
        if (given_w) p.B[i] = given_w[i];
        else if (ftp_status s = make_operand<T>(&p.B[i], w[i], d->cin, d->cout, ldw, d->unaligned, ws, jobs, st, who)) return s;
    }
    if (ws.dry()) return FTP_OK;
    if (!err) err = status_word();
    FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
    run_now<T>(jobs, st);
    p.parts = GATED ? 2 : 1;
    p.b_mn = 1;
    p.M = d->rows; p.N = d->cout; p.K = d->cin;
    p.epi = GATED ? EPI_GATED : EPI_LINEAR;
    p.out_f32 = sizeof(T) == 4;
    p.err = err;
    return run_product(p, st, who);
}

// Rows of a block row, an eighth of them to a thread: up to 1024 block rows of 64 rows, then longer ones, but never more than 64
// float additions in a sum (rounding errors of terms of one sign add up: 1.3e-5 of the result with 8192 rows a block row).
constexpr int GRAD_ROWS = 64, GRAD_CHUNKS = 1024, GRAD_MOST = 8 * 64;
// up to 256 rows in one block row, whose sums then are the bias gradient (a launch less; few columns then fill few SMs: 246 x 576
// x 1454 bf16 backward takes 40 us with a bias gradient, 19 without)
int grad_rows_per_block(long long rows) {
    if (rows <= 256) return 256;
    return (int)std::min<long long>(GRAD_MOST, std::max<long long>(GRAD_ROWS, (rows + GRAD_CHUNKS * 8 - 1) / (GRAD_CHUNKS * 8) * 8));
}
// without a bias gradient: enough blocks to fill the GPU four times over, 16 rows at least (246 x 576 x 1454 bf16 backward:
// 41 instead of 20 us with all rows in one block row)
int grad_rows_per_block(long long rows, long long cols) {
    const long long chunks = std::max<long long>(1, 4 * SMS / ((cols + 255) / 256)), want = ((rows + chunks - 1) / chunks + 7) / 8 * 8;
    return std::max<int>(rows > GRAD_ROWS * GRAD_CHUNKS ? grad_rows_per_block(rows) : 16, (int)std::min<long long>(want, GRAD_ROWS));
}

// ---- backward of both operators ----
template <typename T, bool GATED>
ftp_status backward(const ftp_ffn_desc* d, const void* x, const void* const* w, const void* stash, const void* dy, const void* addend, void* dx,
                    void* const* dw, float* dbias, Carve& ws, int* err, cudaStream_t st, const char* who) {
    const long long M = d->rows, ldx = d->ldx ? d->ldx : d->cin, ldw = d->ldw ? d->ldw : d->cout, ldy = d->ldy ? d->ldy : d->cout;
    const bool dry = ws.dry(), f32 = sizeof(T) == 4, want_dw = dry || dw[0], want_dx = dry || dx, recompute = GATED && d->stash == STASH_NONE;
    // a gradient that passes unchanged is read in place
    const bool direct = !GATED && !f32 && d->stash == STASH_NONE && !d->unaligned && (ldy % 8 == 0 || M == 1);
    Operand X{}, W[2] = {}, G[2] = {};
    Jobs jobs{};
    if (want_dw || recompute) {
        const ftp_status s = d->x_8bit ? image_operand(&X, x, M, d->cin, ws, jobs, st) : make_operand<T>(&X, x, M, d->cin, ldx, d->unaligned, ws, jobs, st, who);
        if (s) return s;
    }
    if (want_dx || recompute)
        for (int i = 0; i < (GATED ? 2 : 1); ++i)
            if (ftp_status s = make_operand<T>(&W[i], w[i], d->cin, d->cout, ldw, d->unaligned, ws, jobs, st, who)) return s;
    if (!dry) {
        if (direct) FTP_REQUIRE(aligned(dy, 16), FTP_ERANGE, "%s: an operand does not start on a 16-byte boundary (set `unaligned`)", who);
        if (!err) err = status_word();
        FTP_REQUIRE(err, FTP_ECUDA, "%s: no status word on this device", who);
    }
    int kind = d->stash;
    if (recompute) {
        stash = ws.take((size_t)(2 * M * d->cout) * sizeof(T));
        kind = STASH_FULL;
        if (!dry) run_now<T>(jobs, st);
        if (!dry)
            if (ftp_status s = forward<T, GATED>(d, nullptr, nullptr, nullptr, nullptr, nullptr, STASH_FULL, const_cast<void*>(stash), ws, err, st, who, &X, W)) return s;
    }
    // the gradient at the products' outputs
    GradArgs g{};
    const long long pitch = up8(d->cout);
    g.planes = f32 ? 3 : 1;
    g.plane = M * pitch;
    for (int i = 0; i < (GATED ? 2 : 1); ++i) {
        if (direct) G[i] = Operand{static_cast<const bf16*>(dy), M, d->cout, M == 1 ? pitch : ldy, 0, 1};
        else {
            g.out[i] = static_cast<bf16*>(ws.take((size_t)g.plane * g.planes * 2));
            G[i] = Operand{g.out[i], M, d->cout, pitch, g.plane, g.planes};
        }
    }
    g.rows_per_block = dry || dbias ? grad_rows_per_block(M) : grad_rows_per_block(M, d->cout);
    const int chunks = (int)((M + g.rows_per_block - 1) / g.rows_per_block);
    float* sums = GATED || chunks == 1 || !(dry || dbias) ? nullptr : static_cast<float*>(ws.take((size_t)chunks * d->cout * 4));
    if (dry) return FTP_OK;
    if (!direct || dbias) {
        g.dy = dy; g.lddy = ldy;
        g.act = d->act;
        g.rows = M; g.cols = d->cout;
        g.all_dy = span_of<T>(dy, M, d->cout, ldy);
        for (int i = 0; i < (GATED ? 2 : 1); ++i) {
            if (kind == STASH_FULL) {
                g.pre[i] = static_cast<const T*>(stash) + (long long)i * M * d->cout;
                g.all_pre[i] = span_of<T>(g.pre[i], M, d->cout, d->cout);
            }
            if (kind == STASH_8BIT) g.img[i] = image_at(const_cast<void*>(stash), M, d->cout, i);
        }
        const bool vec = d->cout % 8 == 0 && aligned(dy, 16) && ldy * (long long)sizeof(T) % 16 == 0 && aligned(g.pre[0], 16) && aligned(g.pre[1], 16);
        g.sums = dbias ? (chunks == 1 ? dbias : sums) : nullptr;
        if (kind == STASH_FULL) launch_grad<T, GATED, STASH_FULL>(g, vec, chunks, jobs, st);
        else if (kind == STASH_8BIT) launch_grad<T, GATED, STASH_8BIT>(g, vec, chunks, jobs, st);
        else if constexpr (!GATED) launch_grad<T, false, STASH_NONE>(g, vec, chunks, jobs, st);
        if (dbias && chunks > 1) launch(sums_kernel, dim3((d->cout + 31) / 32), dim3(256), 0, st, (const float*)sums, chunks, (int)d->cout, dbias);
    }
    run_now<T>(jobs, st);                                            // nothing left of them after the gradient kernel
    if (ftp_status s = launched(who)) return s;
    Product p{};
    p.err = err;
    p.epi = EPI_STORE;
    p.parts = GATED ? 2 : 1;
    if (dx) {
        p.cat_k = GATED;
        p.A[0] = G[0]; p.A[1] = G[1]; p.B[0] = W[0]; p.B[1] = W[1];
        p.M = M; p.N = d->cin; p.K = d->cout;
        p.out_f32 = f32;
        set_out<T>(p.e[0], dx, d->lddx ? d->lddx : d->cin, addend, d->ldr ? d->ldr : d->cin);
        if (ftp_status s = run_product(p, st, who)) return s;
    }
    if (dw[0]) {
        p.cat_k = 0;
        p.a_mn = p.b_mn = 1;
        p.A[0] = X; p.B[0] = G[0]; p.B[1] = G[1];
        p.M = d->cin; p.N = d->cout; p.K = M;
        p.out_f32 = f32 || d->dw_f32;
        const long long lddw = d->lddw ? d->lddw : d->cout;
        for (int i = 0; i < p.parts; ++i) {
            if (p.out_f32) set_out<float>(p.e[i], dw[i], lddw, nullptr, 0);
            else set_out<bf16>(p.e[i], dw[i], lddw, nullptr, 0);
        }
        if (ftp_status s = run_product(p, st, who)) return s;
    }
    return FTP_OK;
}

ftp_status zero_gradients(const ftp_ffn_desc* d, void* const* dw, int n, float* dbias, cudaStream_t st, const char* who) {
    const size_t e = d->precision == FTP_FP32 || d->dw_f32 ? 4 : 2, pitch = (size_t)(d->lddw ? d->lddw : d->cout) * e;
    for (int i = 0; i < n; ++i)
        if (dw[i]) FTP_REQUIRE(cudaMemset2DAsync(dw[i], pitch, 0, (size_t)d->cout * e, d->cin, st) == cudaSuccess, FTP_ECUDA, "%s: memset failed", who);
    if (dbias) FTP_REQUIRE(cudaMemsetAsync(dbias, 0, (size_t)d->cout * 4, st) == cudaSuccess, FTP_ECUDA, "%s: memset failed", who);
    return FTP_OK;
}

template <bool GATED>
ftp_status workspace_bytes(const ftp_ffn_desc* d, int32_t back, size_t* bytes, const char* who) {
    if (ftp_status s = check_desc(d, who)) return s;
    FTP_REQUIRE(bytes, FTP_EINVAL, "%s: null argument", who);
    Carve c{nullptr, 0, 0};
    const void* w[2] = {nullptr, nullptr};
    void* dw[2] = {nullptr, nullptr};
    if (d->rows > 0) {
        if (back) d->precision == FTP_FP32 ? backward<float, GATED>(d, nullptr, w, nullptr, nullptr, nullptr, nullptr, dw, nullptr, c, nullptr, nullptr, who)
                                           : backward<bf16, GATED>(d, nullptr, w, nullptr, nullptr, nullptr, nullptr, dw, nullptr, c, nullptr, nullptr, who);
        else d->precision == FTP_FP32 ? forward<float, GATED>(d, nullptr, w, nullptr, nullptr, nullptr, 0, nullptr, c, nullptr, nullptr, who)
                                      : forward<bf16, GATED>(d, nullptr, w, nullptr, nullptr, nullptr, 0, nullptr, c, nullptr, nullptr, who);
    }
    *bytes = c.off;
    return FTP_OK;
}

template <bool GATED>
ftp_status check_and_forward(const ftp_ffn_desc* d, const void* x, const void* w0, const void* w1, const float* bias, const void* residual, void* y, void* stash,
                             void* ws, size_t ws_bytes, int* err, cudaStream_t st, const char* who) {
    size_t need = 0;
    if (ftp_status s = workspace_bytes<GATED>(d, 0, &need, who)) return s;
    FTP_REQUIRE(d->ldr == 0 || !residual || d->ldr >= d->cout, FTP_EINVAL, "%s: rows overlap (a pitch below the width)", who);
    FTP_REQUIRE(!d->x_8bit, FTP_EUNSUPPORTED, "%s: the forward pass takes x in its own type", who);
    if (d->rows == 0) return FTP_OK;
    FTP_REQUIRE(x && w0 && (!GATED || w1) && (y || (GATED && stash)), FTP_EINVAL, "%s: null buffer", who);
    if (ftp_status s = check_stash(d, stash, who)) return s;
    const size_t e = d->precision == FTP_FP32 ? 4 : 2;
    if (ftp_status s = check_elements({x, w0, w1, residual, y, d->stash == STASH_FULL ? stash : nullptr}, e, who)) return s;
    if (ftp_status s = check_elements({bias}, 4, who)) return s;
    Carve c{nullptr, need, 0};
    if (ftp_status s = check_ws(c, ws, ws_bytes, who)) return s;
    if (ftp_status s = check_addresses({y, stash}, {x, w0, w1, bias}, who)) return s;
    if (ftp_status s = check_addresses({stash}, {residual}, who)) return s;
    if (ftp_status s = check_in_place(residual, y, d->ldr, d->ldy, d->rows, d->cout, who)) return s;
    Carve real{static_cast<char*>(ws) + (ws ? 0 : 256), 0, ws_bytes};
    const void* w[2] = {w0, w1};
    const ftp_status s = d->precision == FTP_FP32 ? forward<float, GATED>(d, x, w, bias, residual, y, d->stash, stash, real, err, st, who)
                                                  : forward<bf16, GATED>(d, x, w, bias, residual, y, d->stash, stash, real, err, st, who);
    return s ? s : launched(who);
}

template <bool GATED>
ftp_status check_and_backward(const ftp_ffn_desc* d, const void* x, const void* w0, const void* w1, const void* stash, const void* dy, const void* addend, void* dx,
                              void* dw0, void* dw1, float* dbias, void* ws, size_t ws_bytes, int* err, cudaStream_t st, const char* who) {
    size_t need = 0;
    if (ftp_status s = workspace_bytes<GATED>(d, 1, &need, who)) return s;
    FTP_REQUIRE(d->ldr == 0 || !addend || d->ldr >= d->cin, FTP_EINVAL, "%s: rows overlap (a pitch below the width)", who);
    FTP_REQUIRE(!GATED || (dw0 != nullptr) == (dw1 != nullptr), FTP_EINVAL, "%s: both weight gradients or neither", who);
    FTP_REQUIRE(!addend || dx, FTP_EINVAL, "%s: dx_addend without dx", who);
    void* dw[2] = {dw0, dw1};
    if (d->rows == 0) return zero_gradients(d, dw, GATED ? 2 : 1, dbias, st, who);
    const bool recompute = GATED && d->stash == STASH_NONE;
    FTP_REQUIRE(dy && ((!dw0 && !recompute) || x) && ((!dx && !recompute) || (w0 && (!GATED || w1))), FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(GATED || (d->act == FTP_ACT_NONE) == (d->stash == STASH_NONE), FTP_EINVAL, "%s: an activation's backward pass needs the kept values, and only that does", who);
    if (ftp_status s = check_stash(d, stash, who)) return s;
    FTP_REQUIRE(!d->x_8bit || !x || aligned(x, 32), FTP_ERANGE, "%s: an image must start on a 32-byte boundary", who);
    const size_t e = d->precision == FTP_FP32 ? 4 : 2;
    if (ftp_status s = check_elements({x, w0, w1, d->stash == STASH_FULL ? stash : nullptr, dy, addend, dx}, e, who)) return s;
    if (ftp_status s = check_elements({dw0, dw1}, d->dw_f32 ? 4 : e, who)) return s;
    if (ftp_status s = check_elements({dbias}, 4, who)) return s;
    Carve c{nullptr, need, 0};
    if (ftp_status s = check_ws(c, ws, ws_bytes, who)) return s;
    if (ftp_status s = check_addresses({dx, dw0, dw1, dbias}, {x, w0, w1, stash, dy}, who)) return s;
    if (ftp_status s = check_addresses({dw0, dw1, dbias}, {addend}, who)) return s;
    if (ftp_status s = check_in_place(addend, dx, d->ldr, d->lddx, d->rows, d->cin, who)) return s;
    Carve real{static_cast<char*>(ws) + (ws ? 0 : 256), 0, ws_bytes};
    const void* w[2] = {w0, w1};
    const ftp_status s = d->precision == FTP_FP32 ? backward<float, GATED>(d, x, w, stash, dy, addend, dx, dw, dbias, real, err, st, who)
                                                  : backward<bf16, GATED>(d, x, w, stash, dy, addend, dx, dw, dbias, real, err, st, who);
    return s ? s : launched(who);
}

}  // namespace

unsigned& launches() {
    static thread_local unsigned n = 0;
    return n;
}
ftp_status op_workspace(bool gated, const ftp_ffn_desc* d, bool backward, size_t* bytes, const char* who) {
    return gated ? workspace_bytes<true>(d, backward, bytes, who) : workspace_bytes<false>(d, backward, bytes, who);
}
ftp_status op_forward(bool gated, const ftp_ffn_desc* d, const void* x, const void* w0, const void* w1, const float* bias, const void* residual, void* y,
                      void* stash, void* ws, size_t ws_bytes, int* err, cudaStream_t st, const char* who) {
    return gated ? check_and_forward<true>(d, x, w0, w1, bias, residual, y, stash, ws, ws_bytes, err, st, who)
                 : check_and_forward<false>(d, x, w0, w1, bias, residual, y, stash, ws, ws_bytes, err, st, who);
}
ftp_status op_backward(bool gated, const ftp_ffn_desc* d, const void* x, const void* w0, const void* w1, const void* stash, const void* dy, const void* addend,
                       void* dx, void* dw0, void* dw1, float* dbias, void* ws, size_t ws_bytes, int* err, cudaStream_t st, const char* who) {
    return gated ? check_and_backward<true>(d, x, w0, w1, stash, dy, addend, dx, dw0, dw1, dbias, ws, ws_bytes, err, st, who)
                 : check_and_backward<false>(d, x, w0, w1, stash, dy, addend, dx, dw0, dw1, dbias, ws, ws_bytes, err, st, who);
}

// In host code the word's name is only a handle; the address a kernel may use has to be asked for, once per device.
int* status_word() {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    int* p = g_status_addr[dev].load(std::memory_order_acquire);
    if (!p) {
        void* a = nullptr;
        if (cudaGetSymbolAddress(&a, g_op_status) != cudaSuccess || !a) return nullptr;
        p = static_cast<int*>(a);
        g_status_addr[dev].store(p, std::memory_order_release);
    }
    return p;
}

}  // namespace ffn
}  // namespace ftp

using namespace ftp::ffn;

extern "C" {

ftp_status ftp_linear_workspace_bytes(const ftp_ffn_desc* d, int32_t backward, size_t* bytes) {
    return workspace_bytes<false>(d, backward, bytes, "linear_workspace_bytes");
}
ftp_status ftp_gated_workspace_bytes(const ftp_ffn_desc* d, int32_t backward, size_t* bytes) {
    return workspace_bytes<true>(d, backward, bytes, "gated_workspace_bytes");
}

ftp_status ftp_linear_forward(const ftp_ffn_desc* d, const void* x, const void* w, const float* bias, const void* residual, void* y, void* stash, void* ws,
                              size_t ws_bytes, void* stream) {
    return check_and_forward<false>(d, x, w, nullptr, bias, residual, y, stash, ws, ws_bytes, nullptr, static_cast<cudaStream_t>(stream), "linear_forward");
}
ftp_status ftp_gated_forward(const ftp_ffn_desc* d, const void* x, const void* w_gate, const void* w_up, void* h, void* stash, void* ws, size_t ws_bytes,
                             void* stream) {
    return check_and_forward<true>(d, x, w_gate, w_up, nullptr, nullptr, h, stash, ws, ws_bytes, nullptr, static_cast<cudaStream_t>(stream), "gated_forward");
}

ftp_status ftp_linear_backward(const ftp_ffn_desc* d, const void* x, const void* w, const void* stash, const void* dy, const void* dx_addend, void* dx, void* dw,
                               float* dbias, void* ws, size_t ws_bytes, void* stream) {
    return check_and_backward<false>(d, x, w, nullptr, stash, dy, dx_addend, dx, dw, nullptr, dbias, ws, ws_bytes, nullptr, static_cast<cudaStream_t>(stream),
                                     "linear_backward");
}
ftp_status ftp_gated_backward(const ftp_ffn_desc* d, const void* x, const void* w_gate, const void* w_up, const void* stash, const void* dh,
                              const void* dx_addend, void* dx, void* dw_gate, void* dw_up, void* ws, size_t ws_bytes, void* stream) {
    return check_and_backward<true>(d, x, w_gate, w_up, stash, dh, dx_addend, dx, dw_gate, dw_up, nullptr, ws, ws_bytes, nullptr, static_cast<cudaStream_t>(stream),
                                    "gated_backward");
}

ftp_status ftp_checkpoint_bytes(int64_t rows, int32_t cols, int32_t parts, size_t* bytes) {
    FTP_REQUIRE(bytes && rows >= 0 && cols >= 1 && parts >= 1, FTP_EINVAL, "checkpoint_bytes: bad argument");
    FTP_REQUIRE(rows * (long long)cols <= (1ll << 38) && rows < (1ll << 38) && parts <= 64 && cols < (1 << 30), FTP_ERANGE, "checkpoint_bytes: tensor too large");
    *bytes = (size_t)parts * image_part_bytes(rows, cols);
    return FTP_OK;
}

static ftp_status check_checkpoint(const void* x, const void* image, int64_t rows, int32_t cols, int64_t* ld, int32_t precision, int32_t part, const char* who) {
    FTP_REQUIRE(precision == FTP_FP32 || precision == FTP_BF16, FTP_EINVAL, "%s: unknown precision %d", who, precision);
    size_t bytes;
    FTP_REQUIRE(part >= 0 && part < 64, FTP_EINVAL, "%s: bad part %d", who, part);
    if (ftp_status s = ftp_checkpoint_bytes(rows, cols, 1, &bytes)) return s;
    if (*ld == 0) *ld = cols;
    FTP_REQUIRE(*ld >= cols && *ld < (1ll << 35), FTP_EINVAL, "%s: rows overlap (a pitch below the width)", who);
    FTP_REQUIRE(rows == 0 || (x && image), FTP_EINVAL, "%s: null buffer", who);
    FTP_REQUIRE(aligned(image, 32), FTP_ERANGE, "%s: an image must start on a 32-byte boundary", who);
    FTP_REQUIRE(rows == 0 || x != image, FTP_EINVAL, "%s: the image lies on its values", who);
    return check_elements({x}, precision == FTP_FP32 ? 4 : 2, who);
}

ftp_status ftp_checkpoint_pack(const void* x, int64_t rows, int32_t cols, int64_t ld, int32_t precision, void* image, int32_t part, void* stream) {
    if (ftp_status s = check_checkpoint(x, image, rows, cols, &ld, precision, part, "checkpoint_pack")) return s;
    if (rows == 0) return FTP_OK;
    const Image im = image_at(image, rows, cols, part);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (precision == FTP_FP32) launch_pack(static_cast<const float*>(x), rows, cols, ld, im, st);
    else launch_pack(static_cast<const bf16*>(x), rows, cols, ld, im, st);
    return launched("checkpoint_pack");
}

ftp_status ftp_checkpoint_unpack(const void* image, int32_t part, int64_t rows, int32_t cols, int32_t precision, void* x, int64_t ld, void* stream) {
    if (ftp_status s = check_checkpoint(x, image, rows, cols, &ld, precision, part, "checkpoint_unpack")) return s;
    if (rows == 0) return FTP_OK;
    const Image im = image_at(const_cast<void*>(image), rows, cols, part);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (precision == FTP_FP32) launch_unpack(im, rows, cols, static_cast<float*>(x), ld, st);
    else launch_unpack(im, rows, cols, static_cast<bf16*>(x), ld, st);
    return launched("checkpoint_unpack");
}

ftp_status ftp_check_op_status(void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    FTP_REQUIRE(cudaStreamIsCapturing(st, &cap) == cudaSuccess, FTP_ECUDA, "check_op_status: bad stream");
    FTP_REQUIRE(cap == cudaStreamCaptureStatusNone, FTP_ESTATE, "check_op_status: the stream is being captured");
    int* word = status_word();
    FTP_REQUIRE(word, FTP_ECUDA, "check_op_status: no status word on this device");
    int code = 0;
    cudaError_t e = cudaMemcpyAsync(&code, word, sizeof code, cudaMemcpyDeviceToHost, st);
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e == cudaSuccess && code) e = cudaMemsetAsync(word, 0, sizeof code, st);
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "check_op_status: %s", cudaGetErrorString(e));
    FTP_REQUIRE(code == 0, FTP_ETIMEOUT, "a bounded wait of a feed-forward kernel ran out (code %d)", code);
    return FTP_OK;
}

}  // extern "C"
