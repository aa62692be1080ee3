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

// Sum over the 64 lanes of a wave, in every lane (the same bits in each):
// within rows of 16 lanes by DPP, then across them by exchanges, none of which waits for
// LDS as a shuffle does.
template <int CONTROL>
__device__ __forceinline__ float add_dpp(float v) {
    const int moved = __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CONTROL, 0xf, 0xf, true);
    return v + __builtin_bit_cast(float, moved);
}

__device__ __forceinline__ float wave_sum(float v) {
    v = add_dpp<0xb1>(v);   // lane ^ 1
    v = add_dpp<0x4e>(v);   // lane ^ 2
    v = add_dpp<0x141>(v);  // the other half of 8 lanes
    v = add_dpp<0x140>(v);  // the other half of 16
    const uint32_t rows = __builtin_bit_cast(uint32_t, v);
    const auto near = __builtin_amdgcn_permlane16_swap(rows, rows, false, false);
    const uint32_t near0 = near[0], near1 = near[1];
    v = __builtin_bit_cast(float, near0) + __builtin_bit_cast(float, near1);
    const uint32_t halves = __builtin_bit_cast(uint32_t, v);
    const auto far = __builtin_amdgcn_permlane32_swap(halves, halves, false, false);
    const uint32_t far0 = far[0], far1 = far[1];
    return __builtin_bit_cast(float, far0) + __builtin_bit_cast(float, far1);
}

}  // namespace
}  // namespace phub
