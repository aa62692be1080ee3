// Loads, stores and conversions of the worker's operators: hidden states are
// fp32, bf16 or fp16 in memory and fp32 in registers.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace phub {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Storage types.  bf16 is kept as its 16 bits: conversion from it is a
// shift, to it rounds to nearest even (v_cvt_pk_bf16_f32 where the compiler
// has it for __bf16).
typedef __bf16 bf16;
typedef _Float16 fp16;

template <typename T>
constexpr int kPerLoad = 16 / int(sizeof(T));  // elements of a 16-byte access

// A 16-byte piece of a row.  Rows may start at any element, so the access
// is only as aligned as an element; gfx950 takes unaligned vector accesses.
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Piece {
    T e[kPerLoad<T>];
};

// n valid elements (a row's last piece may be short); the others are 0.
template <typename T>
__device__ __forceinline__ Piece<T> load_piece(const T* p, int n) {
    Piece<T> r;
    if (n >= kPerLoad<T>) {
        __builtin_memcpy(&r, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kPerLoad<T>; ++i) r.e[i] = i < n ? p[i] : T(0.0f);
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void store_piece(T* p, const float* v, int n) {
    Piece<T> r;
#pragma unroll
    for (int i = 0; i < kPerLoad<T>; ++i) r.e[i] = T(v[i]);
    if (n >= kPerLoad<T>) {
        __builtin_memcpy(p, &r, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kPerLoad<T>; ++i)
            if (i < n) p[i] = r.e[i];
    }
}

// Sum over the 64 lanes of a wave, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

}  // namespace
}  // namespace phub
