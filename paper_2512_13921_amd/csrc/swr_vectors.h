// swr_vectors.h -- rows of bf16 and float32 elements in 16-byte vectors, at any
// element's alignment, and sums over a wave: device code that several kernels
// of the library share.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace swr {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// 16 bytes of elements at any element's alignment: the hardware's wide loads
// and stores take unaligned addresses.
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) Loose {
    u32x4 v;
};

// (By value: bit casts of a vector's element itself read its first.)
__device__ inline float as_float(uint32_t u) { return __builtin_bit_cast(float, u); }

struct Bf16 {
    typedef uint16_t store;
    static constexpr int NE = 8;
    static __device__ float get(const u32x4& v, int i) {
        return as_float(i % 2 ? v[i / 2] & 0xffff0000u : v[i / 2] << 16);
    }
    static __device__ float one(store s) { return __builtin_bit_cast(float, (uint32_t)s << 16); }
    static __device__ store to(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }
    static __device__ u32x4 pack(const float* f) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (uint32_t)to(f[2 * i]) | (uint32_t)to(f[2 * i + 1]) << 16;
        return v;
    }
};
struct F32 {
    typedef float store;
    static constexpr int NE = 4;
    static __device__ float get(const u32x4& v, int i) { return as_float(v[i]); }
    static __device__ float one(store s) { return s; }
    static __device__ store to(float f) { return f; }
    static __device__ u32x4 pack(const float* f) {
        return u32x4{__builtin_bit_cast(uint32_t, f[0]), __builtin_bit_cast(uint32_t, f[1]),
                     __builtin_bit_cast(uint32_t, f[2]), __builtin_bit_cast(uint32_t, f[3])};
    }
};

// NE elements of a row from element e on, as they lie in memory, zeros past the
// row's width.  They become floats only when all of a row's loads are on their
// way: converted in the branch that loads them, each load is waited for there
// (forward, 16384 rows of 2048 bf16, 48.0 us, 43.4 so; 7710 of 4352, 62.9 and 44.8).
template <class E, int NE>
struct Slice {
    typedef typename E::store T;
    static constexpr int NV = NE / E::NE;
    u32x4 v[NV];
    __device__ void load(const T* row, int e, int width) {
        const int n = width - e;
        if (n >= NE) {
#pragma unroll
            for (int j = 0; j < NV; ++j) v[j] = ((const Loose<T>*)(row + e + j * E::NE))->v;
            return;
        }
        T t[NE] = {};
        if (n > 0) {   // (lanes past the row skip the elements' branches as a whole)
#pragma unroll
            for (int i = 0; i < NE - 1; ++i)
                if (i < n) t[i] = row[e + i];
        }
        __builtin_memcpy(v, t, sizeof v);
    }
    __device__ float operator[](int i) const { return E::get(v[i / E::NE], i % E::NE); }
};

// The same of a row of any width, as floats.
template <class E, int NE>
__device__ inline void load(const typename E::store* row, int e, int width, float* f) {
    if (e + NE <= width) {
        Slice<E, NE> s;
        s.load(row, e, width);
#pragma unroll
        for (int i = 0; i < NE; ++i) f[i] = s[i];
    } else {
#pragma unroll
        for (int i = 0; i < NE; ++i) f[i] = e + i < width ? E::one(row[e + i]) : 0.0f;
    }
}

template <class E, int NE>
__device__ inline void store(typename E::store* p, int n, const float* f) {
    if (n >= NE) {
#pragma unroll
        for (int j = 0; j < NE; j += E::NE) ((Loose<typename E::store>*)(p + j))->v = E::pack(f + j);
    } else if (n > 0) {
#pragma unroll
        for (int i = 0; i < NE - 1; ++i)
            if (i < n) p[i] = E::to(f[i]);
    }
}

__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ inline uint32_t wave_max(uint32_t v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, m));
    return v;
}

}  // namespace
}  // namespace swr
