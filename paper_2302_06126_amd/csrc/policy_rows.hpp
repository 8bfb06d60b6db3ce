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
// Results leave by non-temporal stores: rows written through the caches push out
// those that are still to be read (42,496 x 256 constrained bf16 scores 37 us
// without, 27 with; 64 x 262,140 79 | 74, balance gradients 38.3 | 37.8).  Rows that
// do not start at multiples of four columns are stored column by column (42,496 x
// 255: 45 us).
template <typename T, bool VEC>
__device__ __forceinline__ void store4(T *row, int64_t c, int64_t n, const float (&v)[4]) {
    if (VEC && c + 4 <= n) {
        typedef unsigned words __attribute__((ext_vector_type(sizeof(typename Quad<T>::raw) / 4)));
        __builtin_nontemporal_store(__builtin_bit_cast(words, Quad<T>::put(v)), reinterpret_cast<words *>(row + c));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < n) row[c + i] = Quad<T>::put1(v[i]);
    }
}

// One step of a reduction over 2^k lanes that ends with the result in each of
// them: within 16 lanes by register permutations (two of quads, two mirrors:
// lanes that agree already stand in for one another), beyond by swaps of halves.
// fmaxf-like ops only: commutative, both lanes of a pair get the same bits.
template <int STEP>
__device__ __forceinline__ int other_lane(int v) {
    constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;
    return __builtin_amdgcn_update_dpp(v, v, ctrl, 0xf, 0xf, true);
}
template <int LANES, typename Op>
__device__ __forceinline__ float lanes_reduce(float v, Op op) {
    v = op(v, __int_as_float(other_lane<0>(__float_as_int(v))));
    v = op(v, __int_as_float(other_lane<1>(__float_as_int(v))));
    v = op(v, __int_as_float(other_lane<2>(__float_as_int(v))));
    v = op(v, __int_as_float(other_lane<3>(__float_as_int(v))));
    if constexpr (LANES == 64) {
        auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
        auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = op(__uint_as_float(b[0]), __uint_as_float(b[1]));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ int lanes_min(int v) {
    v = min(v, other_lane<0>(v));
    v = min(v, other_lane<1>(v));
    v = min(v, other_lane<2>(v));
    v = min(v, other_lane<3>(v));
    if constexpr (LANES == 64) {
        auto a = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
        v = min((int)a[0], (int)a[1]);
        auto b = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
        v = min((int)b[0], (int)b[1]);
    }
    return v;
}

// A row's maximum (not NaN) and its lowest column; at: -2 if a NaN is among the
// values, INT32_MAX if every value is -inf.
struct RowMax {
    float m;
    int32_t at;
};
struct Two {
    float s, t;
};

// The threads of one row: NT of them (16, 64 or whole wavefronts), BLOCK / NT
// rows to a block.  The reductions' results reach every thread of the row, and
// are the same bits in every call.
template <int NT, int BLOCK = (NT < 256 ? 256 : NT)>
struct RowTeam {
    static_assert(NT == 16 || NT % 64 == 0, "teams of 16 lanes or of wavefronts");
    static constexpr int kBlock = BLOCK, kRows = BLOCK / NT, kL = NT < 64 ? NT : 64, kWaves = (NT + 63) / 64;
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
    // of each thread's own maximum and column
    static __device__ __forceinline__ RowMax max(RowMax v) {
        const float m = lanes_reduce<kL>(v.m, [](float a, float b) { return a > b ? a : b; });
        int at = lanes_min<kL>(v.at == -2 || v.m == m ? v.at : INT32_MAX);
        if constexpr (kWaves == 1) {
            return RowMax{m, at};
        } else {
            __shared__ RowMax part[kBlock / 64];
            const int w = threadIdx.x >> 6, w0 = w / kWaves * kWaves;
            __syncthreads();   // an earlier reduction's reads are done
            if ((threadIdx.x & 63) == 0) part[w] = RowMax{m, at};
            __syncthreads();
            RowMax r = part[w0];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) {
                const RowMax o = part[w0 + i];
                const bool nan = r.at == -2 || o.at == -2;
                const bool second = o.m > r.m || (o.m == r.m && o.at < r.at);
                r = second ? o : r;
                if (nan) r.at = -2;
            }
            return r;
        }
    }
    static __device__ __forceinline__ Two sum(Two v) {
        auto add = [](float a, float b) { return a + b; };
        v = Two{lanes_reduce<kL>(v.s, add), lanes_reduce<kL>(v.t, add)};
        if constexpr (kWaves > 1) {
            __shared__ Two part[kBlock / 64];
            const int w = threadIdx.x >> 6, w0 = w / kWaves * kWaves;
            __syncthreads();
            if ((threadIdx.x & 63) == 0) part[w] = v;
            __syncthreads();
            v = part[w0];
#pragma unroll
            for (int i = 1; i < kWaves; ++i) {
                v.s += part[w0 + i].s;
                v.t += part[w0 + i].t;
            }
        }
        return v;
    }
    static __device__ __forceinline__ float sum(float v) { return sum(Two{v, 0.f}).s; }
};

}  // namespace tag
