// Pieces of 16 bytes of a row, at any alignment of its elements, and numbers of a type known at run time. Not part of the ABI.
#pragma once

#include "taser_internal.h"

template <typename T> constexpr int kTaserEach = 16 / sizeof(T);   // elements of a piece
template <typename T> struct TaserPiece { T x[kTaserEach<T>]; };

// Elements at .. at + EACH - 1 of a row of n; those past its end are `past`.
template <typename T> __device__ inline void taser_load_piece(const T* row, int64_t at, int64_t n, T past, TaserPiece<T>& p) {
    if (at + kTaserEach<T> <= n) {
        __builtin_memcpy(p.x, row + at, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kTaserEach<T>; ++i) p.x[i] = at + i < n ? row[at + i] : past;
    }
}
template <typename T> __device__ inline void taser_store_piece(T* row, int64_t at, int64_t n, const TaserPiece<T>& p) {
    if (at + kTaserEach<T> <= n) {
        __builtin_memcpy(row + at, p.x, 16);
    } else {
#pragma unroll
        for (int i = 0; i < kTaserEach<T>; ++i)
            if (at + i < n) row[at + i] = p.x[i];
    }
}

// N neighboring numbers of a type known at run time (the same for the whole wave), as floats; 0 past the end.
template <typename T, int N> __device__ inline void taser_load_as(const void* from, int64_t at, int64_t n, float (&to)[N]) {
    const T* p = (const T*)from + at;
    if (at + N <= n) {
        T x[N];
        __builtin_memcpy(x, p, sizeof(x));
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) to[i] = at + i < n ? (float)p[i] : 0.f;
    }
}
template <int N> __device__ inline void taser_load_floats(const void* from, int32_t type, int64_t at, int64_t n, float (&to)[N]) {
    if (type == TASER_F32) taser_load_as<float, N>(from, at, n, to);
    else if (type == TASER_F16) taser_load_as<_Float16, N>(from, at, n, to);
    else taser_load_as<__bf16, N>(from, at, n, to);
}
template <typename T, int N> __device__ inline void taser_store_as(void* to, int64_t at, int64_t n, const float (&from)[N]) {
    T* p = (T*)to + at;
    if (at + N <= n) {
        T x[N];
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = (T)from[i];
        __builtin_memcpy(p, x, sizeof(x));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (at + i < n) p[i] = (T)from[i];
    }
}
template <int N> __device__ inline void taser_store_floats(void* to, int32_t type, int64_t at, int64_t n, const float (&from)[N]) {
    if (type == TASER_F32) taser_store_as<float, N>(to, at, n, from);
    else if (type == TASER_F16) taser_store_as<_Float16, N>(to, at, n, from);
    else taser_store_as<__bf16, N>(to, at, n, from);
}
