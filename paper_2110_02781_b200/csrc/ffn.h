// Feed-forward operators (linear, gated, 8-bit activation checkpoints): types shared by their translation units.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include "common.h"

namespace ftp {
namespace ffn {

// How the values before the activation are kept: not at all, in the tensors' type, or as an 8-bit image.
enum { STASH_NONE = 0, STASH_FULL = 1, STASH_8BIT = 2 };

// 8-bit image of `rows` x `cols` values: rows of `pitch` int8 codes (whole blocks of 32 columns), then one byte per
// block, the biased exponent of its power-of-two scale.  value = code * 2^(byte - 127); byte 255: the block held a NaN
// or an infinity and every value of it reads as NaN.
constexpr int IMG_BLOCK = 32;
struct Image {
    int8_t* q;
    uint8_t* e;
    long long pitch;                       // codes per row; blocks per row = pitch / 32
};
inline long long image_pitch(long long cols) { return (cols + IMG_BLOCK - 1) / IMG_BLOCK * IMG_BLOCK; }
inline size_t image_part_bytes(long long rows, long long cols) {
    const size_t p = (size_t)image_pitch(cols);
    return ((size_t)rows * (p + p / IMG_BLOCK) + 255) / 256 * 256;
}
inline Image image_at(void* base, long long rows, long long cols, int part) {
    char* b = static_cast<char*>(base) + (size_t)part * image_part_bytes(rows, cols);
    const long long p = image_pitch(cols);
    return Image{reinterpret_cast<int8_t*>(b), reinterpret_cast<uint8_t*>(b) + rows * p, p};
}

enum { EPI_STORE = 0, EPI_LINEAR = 1, EPI_GATED = 2 };

// What happens to a finished accumulator (a: the product; b: EPI_GATED's second product).
//   EPI_STORE   y = a + add
//   EPI_LINEAR  z = a + bias, kept in `stash`;  y = act(z) + add
//   EPI_GATED   a and b kept in `stash`;  y = act(a) * b
// Pitches in elements; vec_*: what the pointer and the pitch allow at columns that are multiples of an access: 2 = 16
// bytes, 1 = four elements, 0 = single elements.
struct Epi {
    void* y; long long ldy;
    const void* add; long long ldadd;
    const float* bias;
    void* stash[2]; long long ldstash;      // STASH_FULL: one plane per product
    Image img[2];                           // STASH_8BIT
    int stash_kind, act;
    int vec_y, vec_add, vec_stash, vec_bias;
};

// One operand of a product as the tensor cores read it: bf16 planes whose sum is the operand (1 for bf16 tensors and
// 8-bit images, 3 for float tensors), `rows` x `cols` each, `ld` elements between rows, `plane` elements between planes.
struct Operand {
    const __nv_bfloat16* p;
    long long rows, cols, ld, plane;
    int planes;
};

// D[M, N] = sum over parts of op(A_i) op(B_i).  a_mn / b_mn: the operand's rows run along the reduction (its contiguous
// axis is M or N); otherwise its contiguous axis is the reduction.  parts = 2 with cat_k: the reduction runs over A[0] B[0]
// and then over A[1] B[1].  parts = 2 without: two products A[0] B[0], A[0] B[1] of the same left operand, joined by
// EPI_GATED or stored to two outputs.
struct Product {
    Operand A[2], B[2];
    int parts, cat_k;
    int a_mn, b_mn;
    long long M;
    int N;
    long long K;
    int epi;
    Epi e[2];
    int out_f32;                            // type of y / add / stash: float, else bf16
    int* err;
};
ftp_status run_product(const Product& p, cudaStream_t st, const char* who);

// Products of a few tokens, read from the tensors as they are (ffn_few.cu).
constexpr int FEW_SMEM = 96 * 1024;          // of it for the tokens
bool few_tokens(long long rows, long long cin, long long cout, bool f32, int products);
ftp_status run_few(const void* x, long long ldx, const void* const* w, long long ldw, int products, int rows, int K, int N, bool f32, const Epi& e, int* err,
                   cudaStream_t st, const char* who);

int* status_word();                         // device word that a kernel whose bounded wait ran out writes a code to

// The entry points' work for callers inside the library: `err` is the status word that a timed-out wait writes to.
ftp_status op_workspace(bool gated, const ftp_ffn_desc* d, bool backward, size_t* bytes, const char* who);
ftp_status op_forward(bool gated, const ftp_ffn_desc* d, const void* x, const void* w0, const void* w1, const float* bias, const void* residual, void* y,
                      void* stash, void* ws, size_t ws_bytes, int* err, cudaStream_t st, const char* who);
ftp_status op_backward(bool gated, const ftp_ffn_desc* d, const void* x, const void* w0, const void* w1, const void* stash, const void* dy, const void* addend,
                       void* dx, void* dw0, void* dw1, float* dbias, void* ws, size_t ws_bytes, int* err, cudaStream_t st, const char* who);
unsigned& launches();                       // kernel launches of this thread so far

inline bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace ffn
}  // namespace ftp
