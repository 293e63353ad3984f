// What the translation units of the C ABI share: argument checks, workspace carve-up, event timing.
#pragma once
#include "../../include/atp.h"
#include "common.h"

#include <cstring>

namespace atp {

// Two events around the launches of one class while its timing is on (atp_profile_enable).
struct ProfScope {
    hipStream_t st;
    int cls;
    double flops, bytes;
    hipEvent_t a = nullptr, b = nullptr;   // null: off
    ProfScope(hipStream_t s, int cls, double flops, double bytes);
    ~ProfScope();
    ProfScope(const ProfScope&) = delete;
    ProfScope& operator=(const ProfScope&) = delete;
};

// Enum-typed arguments come from C callers and may hold any int: read the value without loading it as
// the enum type (which is undefined for values outside the enumerators), then range-check it.
template <class E>
inline int raw_enum(const E& e) {
    static_assert(sizeof(E) == sizeof(int), "C enums are int-sized in this ABI");
    int v;
    std::memcpy(&v, &e, sizeof v);
    return v;
}
inline bool bad_dtype(const atp_dtype& t) { const int v = raw_enum(t); return v != ATP_F32 && v != ATP_BF16; }

inline size_t align_up(size_t x) { return (x + 255) & ~(size_t)255; }
inline bool aligned16(const void* p) { return (((uintptr_t)p) & 15) == 0; }
inline size_t esize(atp_dtype t) { return t == ATP_BF16 ? 2 : 4; }

struct Carver {
    uint8_t* base;
    size_t off = 0;
    explicit Carver(void* p) : base(reinterpret_cast<uint8_t*>(p)) {}
    void* take(size_t bytes) {
        void* r = base ? base + off : nullptr;
        off += align_up(bytes);
        return r;
    }
};

constexpr int NUM_CU = 256;  // compute units of an MI355X

}  // namespace atp

#define ATP_HIP(expr)                               \
    do {                                            \
        hipError_t e__ = (expr);                    \
        if (e__ != hipSuccess) return ATP_ERR_DEVICE; \
    } while (0)
