// tbn_checks.h -- argument checks that the C entry points share (host code).
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <initializer_list>
#include <string>

#include "tbn.h"
#include "tbn_kernels.h"

namespace tbn {
namespace checks {

inline tbn_status fail(tbn_status s, const char* what) { return tbn::set_error(s, what); }

inline tbn_status done(hipError_t e, const char* where) {
    return e == hipSuccess ? TBN_OK : tbn::set_error(TBN_ERR_HIP, std::string(where) + ": " + hipGetErrorString(e));
}

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool known(tbn_dtype t) { return t == TBN_BF16 || t == TBN_F32; }
inline int64_t round256(int64_t v) { return (v + 255) / 256 * 256; }
inline int64_t size_of(tbn_dtype t) { return t == TBN_F32 ? 4 : 2; }

inline tbn_status check_ws(const void* ws, size_t bytes, int64_t need) {
    if (!ws || bytes < (size_t)need) return fail(TBN_ERR_WORKSPACE, "workspace too small");
    if (!aligned(ws, 16)) return fail(TBN_ERR_ALIGN, "workspace must be 16-byte aligned");
    return TBN_OK;
}

// Whether an output shares a byte with an input or with another output (operands that are not given are NULL).
struct Operand {
    const void* p;
    int64_t bytes;
};
inline bool meet(const void* p, int64_t bytes, const void* q, int64_t qbytes) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return a < b + (uintptr_t)qbytes && b < a + (uintptr_t)bytes;
}
inline bool overlap(std::initializer_list<Operand> outputs, std::initializer_list<Operand> inputs) {
    for (const Operand* o = outputs.begin(); o != outputs.end(); ++o) {
        if (!o->p) continue;
        for (const Operand& i : inputs)
            if (i.p && meet(o->p, o->bytes, i.p, i.bytes)) return true;
        for (const Operand* k = outputs.begin(); k != o; ++k)
            if (k->p && meet(o->p, o->bytes, k->p, k->bytes)) return true;
    }
    return false;
}

}  // namespace checks
}  // namespace tbn
