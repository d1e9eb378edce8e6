// Element types of the encoder operators: loads, stores and conversions.
// Arithmetic is in float; a value is rounded (to nearest even) when stored.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace ndvm {
namespace ops {

typedef __bf16 bf16;
typedef _Float16 f16;

// Elements of a 16-byte access.
template <class T> constexpr int kVec = 16 / int(sizeof(T));

// Rows need no alignment beyond their elements': the hardware takes 16-byte
// accesses at any address that suits the element.
template <class T> struct Vec {
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};
template <class T> using vec = typename Vec<T>::type;

// Elements [0, count) of a vector at p; the others are 0.
template <class T> __device__ inline vec<T> load_vec(const T *p, int64_t count) {
    if (count >= kVec<T>) return *reinterpret_cast<const vec<T> *>(p);
    vec<T> r = 0;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
        if (i < count) r[i] = p[i];
    return r;
}
// PASSING: not to be kept in the caches.
template <bool PASSING = false, class T> __device__ inline void store_vec(T *p, vec<T> v, int64_t count) {
    if (count >= kVec<T>) {
        if (PASSING) __builtin_nontemporal_store(v, reinterpret_cast<vec<T> *>(p));
        else *reinterpret_cast<vec<T> *>(p) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i)
        if (i < count) p[i] = v[i];
}

// Calls f(T()) with the type that `dtype` names.
template <class F> hipError_t with_type(int dtype, F f) {
    switch (dtype) {
        case 0: return f(float());
        case 1: return f(bf16());
        default: return f(f16());
    }
}

}  // namespace ops
}  // namespace ndvm
