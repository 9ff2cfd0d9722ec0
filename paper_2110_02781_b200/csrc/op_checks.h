// Checks of arguments that the operators' entry points share.
#pragma once
#include <cuda_runtime.h>
#include <cstdint>
#include <initializer_list>
#include "common.h"

namespace ftp {

inline bool on_bytes(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Addresses: multiples of their elements' size, and no output where an input or another output starts (further overlaps
// cannot be told from columns of one matrix, which may be neighbours).
inline ftp_status check_addresses(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins, const char* who) {
    for (auto o = outs.begin(); o != outs.end(); ++o) {
        if (!*o) continue;
        for (const void* i : ins) FTP_REQUIRE(*o != i, FTP_EINVAL, "%s: an output lies on an input", who);
        for (auto q = outs.begin(); q != o; ++q) FTP_REQUIRE(*o != *q, FTP_EINVAL, "%s: two outputs in one place", who);
    }
    return FTP_OK;
}
// An addend may be the result itself, element by element: with another pitch a row would be read after it was overwritten.
inline ftp_status check_in_place(const void* add, const void* out, int64_t ldadd, int64_t ldout, int64_t rows, int32_t cols, const char* who) {
    FTP_REQUIRE(!add || add != out || rows == 1 || (ldadd ? ldadd : cols) == (ldout ? ldout : cols), FTP_EINVAL, "%s: an addend in place of its result with another pitch", who);
    return FTP_OK;
}
inline ftp_status check_elements(std::initializer_list<const void*> all, size_t bytes, const char* who) {
    for (const void* p : all) FTP_REQUIRE(on_bytes(p, bytes), FTP_ERANGE, "%s: an address is not a multiple of its elements' size", who);
    return FTP_OK;
}
inline ftp_status check_pitches(std::initializer_list<int64_t> all, int64_t cols, const char* who) {
    for (int64_t ld : all) {
        FTP_REQUIRE(ld == 0 || ld >= cols, FTP_EINVAL, "%s: rows overlap (a pitch below the width)", who);
        FTP_REQUIRE(ld < (1ll << 35), FTP_ERANGE, "%s: pitch too large", who);
    }
    return FTP_OK;
}
inline ftp_status launched(const char* who) {
    const cudaError_t e = cudaGetLastError();
    FTP_REQUIRE(e == cudaSuccess, FTP_ECUDA, "%s: launch failed: %s", who, cudaGetErrorString(e));
    return FTP_OK;
}

}  // namespace ftp
