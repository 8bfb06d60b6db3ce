// Rows of scores held in registers by NT threads, for the operators of
// include/tag_policy.h: four consecutive columns per thread and step, so a
// wavefront's loads cover whole cache lines, and reductions over the row's
// threads whose result every thread gets.
#pragma once

#include "tag_internal.hpp"

namespace tag {

// e^x for x <= 0 (or NaN), within a few ulp: x log2(e) in two parts, since the
// rounding of one would grow with |x|
__device__ __forceinline__ float exp_neg(float x) {
#pragma clang fp contract(off)
    const float t = x * 1.44269504f, lo = fmaf(x, 1.92596299e-8f, fmaf(x, 1.44269504f, -t)) * 0.693147181f;
    const float r = __builtin_amdgcn_exp2f(t);
    return x < -87.f ? 0.f : fmaf(r, lo, r);
}

template <typename T>
struct Quad;   // four elements as one load or store
template <>
struct Quad<float> {
    typedef float4 raw;
    static __device__ __forceinline__ void get(const raw &r, float (&v)[4]) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    static __device__ __forceinline__ raw put(const float (&v)[4]) { return raw{v[0], v[1], v[2], v[3]}; }
    static __device__ __forceinline__ float get1(float x) { return x; }
    static __device__ __forceinline__ float put1(float x) { return x; }
};
template <>
struct Quad<uint16_t> {
    typedef uint2 raw;
    static __device__ __forceinline__ void get(const raw &r, float (&v)[4]) {
        v[0] = __uint_as_float(r.x << 16); v[1] = __uint_as_float(r.x & 0xffff0000u);
        v[2] = __uint_as_float(r.y << 16); v[3] = __uint_as_float(r.y & 0xffff0000u);
    }
    static __device__ __forceinline__ raw put(const float (&v)[4]) { return raw{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3])}; }
    static __device__ __forceinline__ float get1(uint16_t x) { return bf2f(x); }
    static __device__ __forceinline__ uint16_t put1(float x) { return f2bf(x); }
};

// four columns from c of a row of n (past its end: fill)
template <typename T, bool VEC>
__device__ __forceinline__ void load4(const T *row, int64_t c, int64_t n, float fill, float (&v)[4]) {
    if (VEC && c + 4 <= n) {
        Quad<T>::get(*reinterpret_cast<const typename Quad<T>::raw *>(row + c), v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = c + i < n ? Quad<T>::get1(row[c + i]) : fill;
    }
}
template <typename T, bool VEC>
__device__ __forceinline__ void store4(T *row, int64_t c, int64_t n, const float (&v)[4]) {
    if (VEC && c + 4 <= n) {
        *reinterpret_cast<typename Quad<T>::raw *>(row + c) = Quad<T>::put(v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < n) row[c + i] = Quad<T>::put1(v[i]);
    }
}

// The threads of one row: NT of them, 256 / NT rows to a block of 256 threads
// (a row of 512 or more is a block of its own).
template <int NT>
struct RowTeam {
    static constexpr int kBlock = NT < 256 ? 256 : NT, kRows = kBlock / NT, kW = NT < 64 ? NT : 64, kWaves = (NT + 63) / 64;
    static __device__ __forceinline__ int tid() { return threadIdx.x % NT; }
    static __device__ __forceinline__ int row() { return threadIdx.x / NT; }
    // LDS written by the row's threads is read by others of them after this
    static __device__ __forceinline__ void sync() {
        if constexpr (NT > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    // op: commutative and associative up to rounding; the same tree in every call
    template <typename V, typename Op>
    static __device__ __forceinline__ V reduce(V v, Op op) {
#pragma unroll
        for (int o = kW / 2; o > 0; o >>= 1) v = op(v, V::shuffle(v, o, kW));
        if constexpr (kWaves > 1) {
            __shared__ V part[kWaves];
            __syncthreads();   // an earlier reduction's reads are done
            if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
            __syncthreads();
            v = part[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v = op(v, part[w]);
        }
        return v;
    }
};

// the maximum and its lowest column; nan: a NaN was among the values
struct RowMax {
    float m;
    int32_t at;
    int32_t nan;
    static __device__ __forceinline__ RowMax shuffle(const RowMax &v, int o, int w) {
        return RowMax{__shfl_xor(v.m, o, w), __shfl_xor(v.at, o, w), __shfl_xor(v.nan, o, w)};
    }
    static __device__ __forceinline__ RowMax join(const RowMax &a, const RowMax &b) {
        const bool second = b.m > a.m || (b.m == a.m && b.at < a.at);
        return RowMax{second ? b.m : a.m, second ? b.at : a.at, a.nan | b.nan};
    }
};
struct RowSum {
    float s;
    static __device__ __forceinline__ RowSum shuffle(const RowSum &v, int o, int w) { return RowSum{__shfl_xor(v.s, o, w)}; }
    static __device__ __forceinline__ RowSum join(const RowSum &a, const RowSum &b) { return RowSum{a.s + b.s}; }
};
struct RowSum2 {
    float s, t;
    static __device__ __forceinline__ RowSum2 shuffle(const RowSum2 &v, int o, int w) {
        return RowSum2{__shfl_xor(v.s, o, w), __shfl_xor(v.t, o, w)};
    }
    static __device__ __forceinline__ RowSum2 join(const RowSum2 &a, const RowSum2 &b) { return RowSum2{a.s + b.s, a.t + b.t}; }
};

}  // namespace tag
