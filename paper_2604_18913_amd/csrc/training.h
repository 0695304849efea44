// What the calls around the reading share (embed.hip, policy.hip, clip.hip, packed.hip).
#pragma once

#include "reading.h"

namespace lkg {

// Sixteen bytes of a row.  Rows need no alignment but their elements' own: rows of odd sizes are read and written in whole
// chunks too, and only what is left behind the last one element by element.
template <class T> using Some = T __attribute__((ext_vector_type(16 / sizeof(T))));
template <class T> struct Loose { typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };

template <class T> __device__ __forceinline__ Some<T> load_some(const T *p, int count) {
    constexpr int V = 16 / sizeof(T);
    if (count >= V) return *(const typename Loose<T>::type *)p;
    Some<T> x = {};
#pragma unroll
    for (int e = 0; e < V - 1; e++)
        if (e < count) x[e] = p[e];
    return x;
}
template <class T> __device__ __forceinline__ void store_some(T *p, const Some<T> &x, int count) {
    constexpr int V = 16 / sizeof(T);
    if (count >= V) {
        *(typename Loose<T>::type *)p = x;
        return;
    }
#pragma unroll
    for (int e = 0; e < V - 1; e++)
        if (e < count) p[e] = x[e];
}

inline int size_of(int dtype) { return dtype == LOGOSKG_F32 ? 4 : 2; }
// Whether a place is one of whole elements: what the chunks above ask for, and the least that a caller's tensors have.
inline bool aligned_to(const void *p, int dtype) { return ((uintptr_t)p & (size_of(dtype) - 1)) == 0; }
inline const char *const kUnaligned = "an array is not aligned to its elements";

// A call works on the device that it is told; the caller's stays the current one behind it.
struct OnDevice {
    int before = -1;
    logoskg_status go(int device) {
        int now;
        LKG_HIP(hipGetDevice(&now));
        if (now == device) return LOGOSKG_OK;
        LKG_HIP(hipSetDevice(device));
        before = now;
        return LOGOSKG_OK;
    }
    ~OnDevice() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

}  // namespace lkg
