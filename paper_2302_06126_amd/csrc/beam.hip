// Beam search over the decision head's scores (include/tag_beam.h): one level's
// selection, and the reordering of the beams' states.
//
// Selection.  Continuations of one beam are ordered by their scores alone; those of
// two beams by the sums c = x + (total - log sum exp x), so that is what has to be
// exact: rows are summed in 64 bits, which the vector unit does at the rate of
// single fp32 operations, with exponentials of 18 instructions each: 288 to a
// wavefront's 1,024 scores, of 887 vector instructions (2,656 searches of 16 x 256) where
// a search fits a block, of 446 (64 rows of 262,140) where rows go in parts.  Vector
// issue and waits bound the large calls rather than memory.  Scores are read once.
//
// What is best is found without sorting.  Every thread (or group of columns) has a
// best candidate of its own; W of these at least reach the bar that bisection finds
// among them, so W candidates at least pass it, and hardly more: only those are
// listed, and ranked by counting.  That holds for any input: a list that overflows
// (equal scores, say) is cut back to its best W, in an order that ties do not leave
// open, as often as it fills.
#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/tag_beam.h"
#include "areas.hpp"
#include "policy_rows.hpp"

namespace tag {
namespace {

constexpr int kMaxWidth = 256;

struct BeamArgs {
    int32_t V, W, S;              // beams before and after, slices
    const void *x;
    int64_t xs;
    const float *total_in;
    const uint8_t *done;
    float *total;
    int32_t *parent, *slice;
    int32_t shift, fours;         // 2^shift threads of a row, of each of which `fours` times four columns are used
    // rows in parts
    int32_t segs, group, groups;  // parts of a row; 2^group columns of a group, and groups of a row
    float *seg_max, *group_max;   // [rows][segs], [rows][groups]
    double *seg_sum;              // [rows][segs]
};

// doubles (no NaN) as unsigned integers in the same order; both zeros are one
__device__ __forceinline__ uint64_t ordered(double d) {
    const uint64_t b = (uint64_t)__double_as_longlong(d + 0.0);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double unordered(uint64_t u) {
    return __longlong_as_double((long long)(u >> 63 ? u ^ 1ull << 63 : ~u));
}

// Step STEP of a reduction over 2, 4, 8, .. 64 lanes that ends in each of them: this
// lane's value and that of its partner, in the same order or the other (as in
// lanes_reduce, for commutative operations).
template <int STEP>
struct Pair {
    unsigned a, b;
    __device__ __forceinline__ explicit Pair(unsigned v) {
        if constexpr (STEP < 4) {
            a = v;
            b = (unsigned)other_lane<STEP>((int)v);
        } else if constexpr (STEP == 4) {
            const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
            a = p[0];
            b = p[1];
        } else {
            const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
            a = p[0];
            b = p[1];
        }
    }
};
template <int STEP, typename Op>
__device__ __forceinline__ unsigned join(unsigned v, Op op) {
    const Pair<STEP> p(v);
    return op(p.a, p.b);
}
template <int STEP, typename Op>
__device__ __forceinline__ float join(float v, Op op) {
    const Pair<STEP> p(__float_as_uint(v));
    return op(__uint_as_float(p.a), __uint_as_float(p.b));
}
template <int STEP, typename Op>
__device__ __forceinline__ double join(double v, Op op) {
    const uint64_t u = (uint64_t)__double_as_longlong(v);
    const Pair<STEP> lo((unsigned)u), hi((unsigned)(u >> 32));
    return op(__hiloint2double((int)hi.a, (int)lo.a), __hiloint2double((int)hi.b, (int)lo.b));
}
// over 2^n lanes, n the same for the wavefront
template <typename V, typename Op>
__device__ __forceinline__ V reduce_lanes(V v, int n, Op op) {
    if (n > 0) v = join<0>(v, op);
    if (n > 1) v = join<1>(v, op);
    if (n > 2) v = join<2>(v, op);
    if (n > 3) v = join<3>(v, op);
    if (n > 4) v = join<4>(v, op);
    if (n > 5) v = join<5>(v, op);
    return v;
}
// (no operand is a NaN; fmaxf would first quiet each)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max2(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
struct Larger {
    __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return max(a, b); }
    __device__ __forceinline__ float operator()(float a, float b) const { return max2(a, b); }
};
struct Smaller {
    __device__ __forceinline__ unsigned operator()(unsigned a, unsigned b) const { return min(a, b); }
};
struct Plus {
    template <typename V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

// The best W of a search's candidates (key, index), collected by a block of NT
// threads that call everything here together.  Candidates that pass the bar are
// appended to a list in LDS in any order; when it is full, its best W stay and the
// W-th becomes the bar.  The order is total (larger key, then lower index), so the
// result does not depend on the order in which they came.
template <int NT, int CAP>
struct Best {
    static_assert(NT == 64 || NT == 256 || NT == 1024, "1, 4 or 16 wavefronts");
    static_assert(CAP % NT == 0 && CAP >= NT + kMaxWidth, "room for a candidate of each thread beside the best W");
    static constexpr int kThreads = NT, kWaves = NT / 64, kOwn = CAP / NT, kRanked = CAP < 512 ? CAP : 512;
    struct Shared {
        double key[CAP];
        int32_t idx[CAP];
        unsigned count[2][kWaves];
        unsigned ends[2][kWaves];
        int32_t tail;
        __attribute__((aligned(16))) unsigned half[kRanked];
        int32_t same[kRanked];
    };
    // (a search of one wavefront shares its block with others)
    static __device__ __forceinline__ int tid() { return threadIdx.x % NT; }
    static __device__ __forceinline__ void sync() {
        if constexpr (NT > 64) {
            __syncthreads();
        } else {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        }
    }
    Shared &s;
    const int W;
    double bar = -INFINITY;      // a candidate passes above it, or at it up to the index
    int32_t bar_idx = -1;
    int n = 0, flip = 0;         // entries of the list
    uint64_t base = 0;           // keys less base, without `drop` bits, fit 32 bits
    int drop = 32;

    // (a barrier follows before the first candidate: raise's)
    __device__ Best(Shared &s_, int w) : s(s_), W(w) {
        if (tid() == 0) s.tail = 0;
    }
    __device__ bool passes(double key, int32_t idx) const { return key > bar || (key == bar && idx <= bar_idx); }
    static __device__ int lanes(bool b) { return __popcll(__ballot(b)); }
    // sum over the wavefronts of a number that each wavefront's lanes share
    __device__ int sum(int v) {
        if constexpr (kWaves == 1) return v;
        if ((tid() & 63) == 0) s.count[flip][tid() >> 6] = (unsigned)v;
        sync();
        const unsigned r = reduce_lanes(s.count[flip][tid() & (kWaves - 1)], kWaves == 16 ? 4 : 2, Plus());
        flip ^= 1;   // (written again only after the next barrier, which follows these reads)
        return __builtin_amdgcn_readfirstlane((int)r);
    }
    // Sets the bar from one candidate of each thread, the best that it has: as high
    // as W threads, or a few more, still pass (false: fewer have one).  Bisection of
    // the upper halves of the ordered keys between the block's ends, about five turns
    // of one barrier each.
    __device__ bool raise(double key) {
        const unsigned u = key > -INFINITY ? (unsigned)(ordered(key) >> 32) : 0u;
        unsigned hi = reduce_lanes(u, 6, Larger()), lo = reduce_lanes(u ? u : ~0u, 6, Smaller());
        int live = lanes(u != 0);
        if constexpr (kWaves > 1) {
            if ((tid() & 63) == 0) {
                s.ends[0][tid() >> 6] = hi;
                s.ends[1][tid() >> 6] = lo;
            }
        }
        live = sum(live);   // (and its barrier)
        if constexpr (kWaves > 1) {
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                hi = max(hi, s.ends[0][i]);
                lo = min(lo, s.ends[1][i]);
            }
        } else {
            sync();
        }
        if (live < W) return false;
        const unsigned best = hi;
        const int most = W + max(W / 4, 2);
        while (lo < hi) {   // W reach lo, fewer reach hi + 1; three probes between them to a turn
            const unsigned step = (hi - lo) / 4, t1 = lo + step + 1, t2 = t1 + step, t3 = min(t2 + step, hi);
            // (fewer than 1,024 each: some thread is at lo or below)
            const unsigned all = (unsigned)sum(lanes(u >= t1) | lanes(u >= t2) << 10 | lanes(u >= t3) << 20);
            const int c1 = all & 1023, c2 = all >> 10 & 1023, c3 = all >> 20;
            const unsigned t = c3 >= W ? t3 : c2 >= W ? t2 : c1 >= W ? t1 : lo;
            const int c = c3 >= W ? c3 : c2 >= W ? c2 : c1 >= W ? c1 : INT32_MAX;
            if (c3 < W) hi = (c2 >= W ? t3 : c1 >= W ? t2 : t1) - 1;
            lo = t;
            if (c <= most) break;
        }
        base = (uint64_t)lo << 32;
        drop = max(0, 32 - __clzll(((uint64_t)best << 32 | 0xffffffffull) - base));
        bar = unordered(base);
        bar_idx = INT32_MAX;
        return true;
    }
    // A score below which no score + off passes: the bar less off, by more than the roundings of either may be
    // (above -inf, which is no candidate).
    __device__ float least_score(double off) const {
        constexpr float lowest = -3.4028234664e38f;
        if (!(bar > -INFINITY)) return lowest;
        const double d = bar - off - 0x1p-50 * (fabs(bar) + fabs(off));
        const float f = (float)d;
        return fmaxf(f - fabsf(f) * 0x1p-22f - 0x1p-140f, lowest);
    }
    // Candidates that are likely to fit: of each thread `count`, which each(put) gives to
    // put(key, index).  A wavefront calls it together.  offered: all, whether they did.
    template <typename Each>
    __device__ void offer(int count, Each each) {
        int before = 0, all = 0;
        for (int b = 0;; ++b) {   // (over lanes, bit by bit: counts are small)
            if (__ballot(count >> b) == 0) break;
            const uint64_t m = __ballot(count >> b & 1);
            before += __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0)) << b;
            all += __popcll(m) << b;
        }
        if (all == 0) return;
        int at = 0;
        if ((tid() & 63) == 0) at = atomicAdd(&s.tail, all);
        at = __builtin_amdgcn_readfirstlane(at) + before;
        each([&](double key, int32_t idx) {
            if (at < CAP) {
                s.key[at] = key;
                s.idx[at] = idx;
            }
            ++at;
        });
    }
    __device__ bool offered() {
        sync();
        n = s.tail;
        return n <= CAP;
    }
    __device__ void clear() {
        sync();
        if (tid() == 0) s.tail = 0;
        n = 0;
        sync();
    }
    // one candidate of each thread (key -inf: none), however many pass
    __device__ void take(double key, int32_t idx) {
        int c = sum(lanes(passes(key, idx)));
        if (n + c > CAP) {
            keep_best();
            c = sum(lanes(passes(key, idx)));
        }
        append(passes(key, idx), key, idx);
        n += c;
    }
    __device__ void append(bool is, double key, int32_t idx) {
        const uint64_t m = __ballot(is);
        if (m == 0) return;
        int at = 0;
        if ((tid() & 63) == 0) at = atomicAdd(&s.tail, __popcll(m));
        at = __builtin_amdgcn_readfirstlane(at) +
             __builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
        if (is) {
            s.key[at] = key;
            s.idx[at] = idx;
        }
    }
    // leaves the best W of a list of more
    __device__ void keep_best() {
        sync();
        uint64_t u[kOwn];
        int32_t idx[kOwn];
#pragma unroll
        for (int r = 0; r < kOwn; ++r) {
            const int at = tid() + NT * r;
            u[r] = at < n ? ordered(s.key[at]) : 0ull;
            idx[r] = at < n ? s.idx[at] : 0;
        }
        // the largest K that W entries reach, bit by bit, or one that exactly W reach
        uint64_t K = 0;
        int reach = n;
        for (int b = 63; b >= 0 && reach != W; --b) {
            const uint64_t t = K | 1ull << b;
            int c = 0;
#pragma unroll
            for (int r = 0; r < kOwn; ++r) c += lanes(u[r] >= t);
            c = sum(c);
            if (c >= W) {
                K = t;
                reach = c;
            }
        }
        int32_t last = INT32_MAX;
        if (reach != W) {   // more at K than there is room for: those of the lowest indices
            int above = 0;
#pragma unroll
            for (int r = 0; r < kOwn; ++r) above += lanes(u[r] > K);
            const int need = W - sum(above);
            last = 0;
            for (int b = 30; b >= 0; --b) {
                const int32_t t = last + (int32_t)((1u << b) - 1u);
                int c = 0;
#pragma unroll
                for (int r = 0; r < kOwn; ++r) c += lanes(u[r] == K && idx[r] <= t);
                if (sum(c) < need) last += 1 << b;
            }
        }
        sync();   // (of one wavefront, sum has none)
        if (tid() == 0) s.tail = 0;
        sync();
#pragma unroll
        for (int r = 0; r < kOwn; ++r)
            append(u[r] > K || (u[r] == K && u[r] != 0 && idx[r] <= last), unordered(u[r]), idx[r]);
        n = W;
        bar = unordered(K);
        bar_idx = last;
    }
    // each(rank, key, index) of the best, at most W; returns how many.  An entry's rank is
    // the number of better ones, counted by 32 bits of the ordered keys (of the range
    // between the bar and the best), four at a time and shared by several threads;
    // where these are equal, the entries themselves decide.
    template <typename Each>
    __device__ int ranked(Each each) {
        if (n > kRanked) keep_best();
        sync();
        for (int i = tid(); i < (n + 3) / 4 * 4; i += NT) {
            const uint64_t u = i < n ? ordered(s.key[i]) : 0ull;
            s.half[i] = u > base ? (unsigned)((u - base) >> drop) : 0u;
        }
        for (int i = tid(); i < n; i += NT) s.same[i] = 0;
        sync();
        int share = 0;
        while (share < 4 && n << (share + 1) <= NT) ++share;
        const int p = tid() & ((1 << share) - 1);
        constexpr int kTurns = (kRanked + NT - 1) / NT;
        int rank[kTurns];
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int i = t * (NT >> share) + (tid() >> share);
            if (t * (NT >> share) >= n) break;
            const unsigned h = i < n ? s.half[i] : ~0u;
            unsigned r = 0;
            for (int j = 4 * p; j < n; j += 4 << share) {
                const uint4 o = *reinterpret_cast<const uint4 *>(s.half + j);
                r += (o.x > h) + (o.y > h) + (o.z > h) + (o.w > h);
            }
            rank[t] = (int)reduce_lanes(r, share, Plus());
            if (i < n && p == 0) atomicAdd(&s.same[rank[t]], 1);
        }
        sync();
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
            const int i = t * (NT >> share) + (tid() >> share);
            if (i >= n || p != 0) continue;
            int r = rank[t];
            const double k = s.key[i];
            const int32_t x = s.idx[i];
            if (s.same[r] > 1) {
                const unsigned h = s.half[i];
                for (int j = 0; j < n; j += 4) {
                    const uint4 o = *reinterpret_cast<const uint4 *>(s.half + j);
                    if (o.x != h && o.y != h && o.z != h && o.w != h) continue;
                    for (int q = j; q < min(j + 4, n); ++q)
                        if (s.half[q] == h) r += s.key[q] > k || (s.key[q] == k && s.idx[q] < x);
                }
            }
            if (r < W) each(r, k, x);
        }
        return min(n, W);
    }
};

template <typename T>
__device__ __forceinline__ float score(const BeamArgs &A, int64_t row, int64_t c) {
    return Quad<T>::get1(static_cast<const T *>(A.x)[row * A.xs + c]);
}

template <typename B>
__device__ __forceinline__ void write_beams(const BeamArgs &A, int64_t b, B &best, const uint8_t *done) {
    const int n = best.ranked([&](int r, double key, int32_t idx) {
        const int32_t v = idx / A.S;
        A.total[b * A.W + r] = (float)key;
        A.parent[b * A.W + r] = v;
        A.slice[b * A.W + r] = done[v] ? -1 : idx - v * A.S;
    });
    for (int r = n + B::tid(); r < A.W; r += B::kThreads) {
        A.total[b * A.W + r] = -INFINITY;
        A.parent[b * A.W + r] = A.slice[b * A.W + r] = -1;
    }
}

// four columns of a row of n from c, at any element (past its end: -inf)
template <typename T>
__device__ __forceinline__ void load_four(const T *row, int c, int n, float (&v)[4]) {
    typedef typename Quad<T>::raw raw;
    if (c + 4 <= n) {
        raw r;
        __builtin_memcpy(&r, row + c, sizeof(raw));
        Quad<T>::get(r, v);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = c + i < n ? Quad<T>::get1(row[c + i]) : -INFINITY;
    }
}
// Column of the k-th four of thread j of a row's 2^shift: the row's threads take four
// each at a time, or (RUNS) each wavefront 1,024 consecutive ones, 256 at a time.
template <bool RUNS>
__device__ __forceinline__ int column(int j, int shift, int k) {
    return RUNS && shift >= 6 ? (j >> 6) * 1024 + k * 256 + (j & 63) * 4 : 4 * (j + (k << shift));
}
// A thread's 16 columns of a row of n, or of its part from c0.
template <bool RUNS, typename T>
__device__ __forceinline__ void load_row(const T *row, int c0, int j, int shift, int n, float (&x)[16]) {
    if (c0 + (16 << shift) <= n) {   // (one address, and no ends to look at)
        typedef typename Quad<T>::raw raw;
        const T *p = row + c0 + column<RUNS>(j, shift, 0);
        const int step = RUNS && shift >= 6 ? 256 : 4 << shift;
        raw r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) __builtin_memcpy(&r[k], p + step * k, sizeof(raw));
#pragma unroll
        for (int k = 0; k < 4; ++k) Quad<T>::get(r[k], *reinterpret_cast<float(*)[4]>(x + 4 * k));
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            load_four(row, c0 + column<RUNS>(j, shift, k), n, *reinterpret_cast<float(*)[4]>(x + 4 * k));
    }
}

__device__ __forceinline__ float max4(const float *x) { return max2(max3(x[0], x[1], x[2]), x[3]); }
// maximum of a thread's scores, +inf if a NaN is among them; four[k]: of its k-th four
__device__ __forceinline__ float own_max(const float (&x)[16], float (&four)[4]) {
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 16; i += 2) nan = nan || __builtin_isunordered(x[i], x[i + 1]);
#pragma unroll
    for (int k = 0; k < 4; ++k) four[k] = max4(x + 4 * k);
    return nan ? INFINITY : max4(four);
}
// x[i], bit by bit of i (an index that is not known, and selects that stand for one, would
// put x in memory)
template <int E>
__device__ __forceinline__ float pick(const float (&x)[E], int i) {
    unsigned h[E];
#pragma unroll
    for (int k = 0; k < E; ++k) h[k] = __float_as_uint(x[k]);
#pragma unroll
    for (int n = E / 2; n > 0; n /= 2) {
        const unsigned m = 0u - (i & 1);
#pragma unroll
        for (int k = 0; k < E / 2; ++k)
            if (k < n) h[k] = (h[2 * k + 1] & m) | (h[2 * k] & ~m);
        i >>= 1;
    }
    return __uint_as_float(h[0]);
}
// Maximum and sum of a row's scores from 2^shift threads of 16 each, into all of them:
// several wavefronts of a row each relative to their own maximum, then joined.  The
// maximum is infinite, and the sum means nothing, where the row has no probabilities.
template <int NT>
struct RowSum {
    float max[NT / 64];
    double sum[NT / 64];
};
// e^x for x <= 0; below -700 that of -700 (a sum with a term of 1 in it does not see
// either).  2^(n + f) with |f| <= 1/2: n by adding 1.5 2^52, whose last bits it then is,
// 2^f = 1 + f q(f) by interpolation of q at eleven Chebyshev points (2e-17 off).  18
// instructions, of the fp32 rate: 42,496 x 256 scores 31 -> 26 us against the
// library's exp.  It is off by (1.4 + |x| / 7.8) 2^-53 of itself (3.2 million values
// against 128 bits: 3.7 at 20, 89 at 690), since log2 e is one number and its own
// rounding counts x times.  In a sum of S terms, the largest 1, that is ln S / 7.8
// roundings at most: with p = e^x / sum e^x, sum p |x| is the entropy of p less log
// sum e^x, and so at most ln S.
__device__ __forceinline__ double exp_below(double x) {
    constexpr double q[11] = {0.6931471805599453,    0.24022650695910097,   0.0555041086648216,    0.009618129107606888,
                              0.0013333558146416936, 0.0001540353044173605, 1.525273382983612e-05, 1.321544258792169e-06,
                              1.0178062445845774e-07, 7.072585949269223e-09, 4.4549605981865186e-10};
    constexpr double log2e = 1.4426950408889634, shift = 6755399441055744.0;
    x = x > -700.0 ? x : -700.0;
    const double t = fma(x, log2e, shift), f = fma(x, log2e, shift - t);
    double p = q[10];
#pragma unroll
    for (int i = 9; i >= 0; --i) p = fma(p, f, q[i]);
    p = fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}
// log x for x >= 1 (a sum with a term of 1 in it), within a few roundings of 64 bits: x =
// 2^e m with m in [0.7, 1.42), log m = 2 atanh f for f = (m - 1) / (m + 1), |f| < 0.172, by
// its series up to f^21 / 21.
__device__ __forceinline__ double log_from(double x) {
    int hi = __double2hiint(x), e = (hi >> 20) - 1023;
    hi = (hi & 0xfffff) | 0x3ff00000;
    if (hi >= 0x3ff6a09f) {   // (1.4142..)
        hi -= 1 << 20;
        ++e;
    }
    const double m = __hiloint2double(hi, __double2loint(x)), d = m - 1.0, b = m + 1.0;
    double r = __builtin_amdgcn_rcp(b);
    r = fma(r, fma(-b, r, 1.0), r);
    r = fma(r, fma(-b, r, 1.0), r);
    double f = d * r;
    f = fma(r, fma(-b, f, d), f);
    const double w = f * f;
    double p = 1.0 / 21.0;
#pragma unroll
    for (int k = 19; k >= 3; k -= 2) p = fma(p, w, 1.0 / k);
    return fma((double)e, 0.6931471805599453, fma(2.0 * f, w * p, 2.0 * f));
}
// sum of e^(x - m), m finite, in 64 bits, over the first `fours` times four
__device__ __forceinline__ double own_sum(const float (&x)[16], float m, int fours) {
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (k >= fours) break;
#pragma unroll
        for (int i = 0; i < 4; ++i) s += exp_below((double)x[4 * k + i] - (double)m);
    }
    return s;
}

template <int NT, bool ALL>   // ALL: every wavefront of the row takes the results, else its first
__device__ __forceinline__ double row_sum(const float (&x)[16], float &m, const int shift, const int fours,
                                          RowSum<NT> &part) {
    const int in_wave = min(shift, 6);
    m = reduce_lanes(m, in_wave, Larger());
    double sum = 0.0;
    if (m > -INFINITY && m < INFINITY) sum = own_sum(x, m, fours);
    sum = reduce_lanes(sum, in_wave, Plus());
    if constexpr (NT > 64) {
        if (shift > 6) {
            if ((threadIdx.x & 63) == 0) {
                part.max[threadIdx.x >> 6] = m;
                part.sum[threadIdx.x >> 6] = sum;
            }
            __syncthreads();
            if (!ALL && (threadIdx.x & ((1 << shift) - 1)) >= 64) return sum;
            // (a lane to each of the row's wavefronts)
            const int w = (threadIdx.x >> shift << (shift - 6)) + (threadIdx.x & ((1 << (shift - 6)) - 1));
            const float own = part.max[w];
            m = reduce_lanes(own, shift - 6, Larger());
            sum = 0.0;
            if (m > -INFINITY && m < INFINITY) sum = part.sum[w] * exp_below((double)own - (double)m);
            sum = reduce_lanes(sum, shift - 6, Plus());
        }
    }
    return sum;
}

// Searches whose scores fit one block's registers; those of one wavefront, four to a
// block.  One search of 64 x 256 9.1 us on its one CU: a chain of loads, sums, bar, list
// and ranks.  2,656 of 16 x 256 bf16 22.5 us: vector issue (9.4 million instructions of
// wavefronts, 3.1 of them exponentials, 17.5 us at four cycles and 2.1 GHz on all
// SIMDs) and waits.  Measured and not kept there: 64 scores to a thread (24 us), 32
// (21.6).  Searches of one row and one beam go the same way: 40,000 of 1 x 256 48 us,
// where memory would take 8.
constexpr int whole_block(int NT) { return NT > 64 ? NT : 256; }
template <typename T, int NT, int CAP>
__global__ void __launch_bounds__(whole_block(NT)) beam_whole(BeamArgs A, int32_t n) {
    using B = Best<NT, CAP>;
    constexpr int kSearches = whole_block(NT) / NT;
    __shared__ typename B::Shared shared_[kSearches];
    __shared__ RowSum<NT> part;
    __shared__ uint8_t finished_[kSearches][kMaxWidth];
    const int64_t b = (int64_t)blockIdx.x * kSearches + threadIdx.x / NT;
    if (b >= n) return;
    typename B::Shared &shared = shared_[threadIdx.x / NT];
    uint8_t *finished = finished_[threadIdx.x / NT];
    const int v = B::tid() >> A.shift, j = B::tid() & ((1 << A.shift) - 1);
    B best(shared, A.W);
    float total = -INFINITY, x[16];
    bool done = false;
    if (v < A.V) {   // (nothing waits for another load, though some beams' scores are not needed)
        total = A.total_in[b * A.V + v];
        done = A.done && A.done[b * A.V + v];
        const T *row = static_cast<const T *>(A.x) + (b * A.V + v) * A.xs;
        load_row<false>(row, 0, j, A.shift, A.S, x);
        if (j == 0) finished[v] = done;
    }
    const bool live = total - total == 0.f;
    if (!live || done) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = -INFINITY;
    }
    float four[4];
    const float own = own_max(x, four);
    float m = own;
    const double sum = row_sum<NT, true>(x, m, A.shift, A.fours, part);
    // what is added to the scores; a finished beam is its first slice alone
    double off = 0.0;
    float top = own;
    if (done && live) {
        off = total;
        if (j == 0) x[0] = top = 0.f;
    } else if (m > -INFINITY && m < INFINITY) {
        off = (double)total - ((double)m + log_from(sum));
    } else {
        top = -INFINITY;
    }
    best.raise((double)top + off);
    // what may pass, by a bound on the scores that is a little lower (a superset will do)
    const float least = top > -INFINITY ? best.least_score(off) : __builtin_nanf("");   // (nothing is at or above that)
    unsigned mask = 0;   // the first in bit 15
#pragma unroll
    for (int i = 0; i < 16; ++i) mask = mask + mask + (x[i] >= least);
    auto index = [&](int i) { return v * A.S + column<false>(j, A.shift, i / 4) + i % 4; };
    best.offer(__popc(mask), [&](auto put) {
        for (unsigned m = mask; m; m &= m - 1) {
            const int i = 16 - __ffs((int)m);
            put((double)pick(x, i) + off, index(i));
        }
    });
    if (!best.offered()) {
        best.clear();
#pragma unroll 1
        for (int i = 0; i < 4 * A.fours; ++i) best.take(top > -INFINITY ? (double)pick(x, i) + off : -INFINITY, index(i));
    }
    write_beams(A, b, best, finished);
}

// Rows in parts: a part's maximum and sum, and the maximum of every group of its
// columns, from one reading of the scores.  GROUP: 0, or that of rows of a block each
// (2^8 threads), whose reductions then are of fixed sizes (64 x 262,140 fp32 22.9 -> 21.1
// us).  67 MB in 17.9 us, 3.7 TB/s: vector issue, 446 instructions to a wavefront's 1,024
// scores, 288 of them exponentials (13.6 us at four cycles and 2.1 GHz on all SIMDs).
template <typename T, int GROUP>
__global__ void __launch_bounds__(256) beam_parts(BeamArgs A, int64_t rows) {
    __shared__ RowSum<256> part;
    const int shift = GROUP ? 8 : A.shift, group = GROUP ? GROUP : A.group;
    const int j = threadIdx.x & ((1 << shift) - 1);
    // (several rows to a block have one part each)
    const uint32_t item = (blockIdx.x << (8 - shift)) + (threadIdx.x >> shift);
    const uint32_t of = A.segs == 1 ? item : blockIdx.x / (uint32_t)A.segs;
    const int64_t row = of;
    const int32_t c0 = (int32_t)(item - of * A.segs) * 4096;
    float t = -INFINITY, x[16], four[4];
    bool done = false;
    if (row < rows) {   // (nothing waits for another load, though some beams' scores are not needed)
        t = A.total_in[row];
        done = A.done && A.done[row];
        load_row<true>(static_cast<const T *>(A.x) + row * A.xs, c0, j, shift, A.S, x);
    }
    const bool live = t - t == 0.f && !done;
    if (!live) {
        if (GROUP) return;   // (the block's one row)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = -INFINITY;
    }
    float m = own_max(x, four);
    if (live) {   // groups' maxima (not looked at where the row has no candidates)
        float *g = A.group_max + row * A.groups;
        if (group == 10) {
            const float w = reduce_lanes(m, 6, Larger());
            const int c = c0 + column<true>(j, shift, 0);
            if ((j & 63) == 0 && c < A.S) g[c >> 10] = w;
        } else {
            const int wide = group - 2;   // 2^wide lanes to a group
            const int c = c0 + column<true>(j, shift, 0);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float w = reduce_lanes(four[k], wide, Larger());
                const int ck = GROUP ? c + 256 * k : c0 + column<true>(j, shift, k);
                if ((j & ((1 << wide) - 1)) == 0 && ck < A.S) g[ck >> group] = w;
            }
        }
    }
    const double sum = row_sum<256, false>(x, m, shift, 4, part);
    if (live && j == 0) {
        A.seg_max[item] = m;
        A.seg_sum[item] = sum;
    }
}

// One block per search: what each beam adds to its scores, from its parts; the bar
// from the groups' maxima; then the candidates of the groups that reach it.  A chain
// of waits on one CU: 8 searches of 8 x 262,140 12.8 us, 5 of 200 x 4,099 26.4, 2 of 256
// x 31,000 63.  127 VGPRs (1,024 threads leave 128), 4 VGPRs and 41 SGPRs spilled (20
// bytes of scratch a lane).
// The bar is set from one candidate of each thread; where fewer than W threads have
// one, rows go one after the other instead.  A finished beam's stands in its first group
// of columns, and group i is thread i mod 1,024's, so where a row's groups are a
// multiple of 2^k all finished beams belong to 2^(10 - k) threads: 256 beams of 4,096
// slices (64 groups), 254 of them finished, take 536 us that way, of 8,192 (32 groups)
// 548, while those of 4,099 (65 groups) take 35.
constexpr int kListed = 2048;   // groups
template <typename T>
__global__ void __launch_bounds__(1024) beam_join(BeamArgs A) {
    using B = Best<1024, 2048>;
    __shared__ B::Shared shared;
    __shared__ double off[kMaxWidth];   // -inf: no candidates
    __shared__ uint8_t done[kMaxWidth];
    __shared__ int32_t list_column[kListed], n_listed;
    __shared__ uint8_t list_row[kListed];
    const int64_t b = blockIdx.x;
    B best(shared, A.W);
    if (threadIdx.x == 0) n_listed = 0;
    constexpr int kHeld = 16;   // groups' maxima in a thread's registers
    const int32_t total = A.V * A.groups;
    const float *maxima = A.group_max + b * total;
    float held[kHeld];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
        const int32_t i = threadIdx.x + 1024 * k;
        held[k] = i < total ? maxima[i] : -INFINITY;
    }
    // a row by as many threads as it has parts, at most a wavefront
    int share = 0;
    while (share < 6 && 1 << share < A.segs) ++share;
    const int wide = 1 << share;
    for (int v0 = 0; v0 < A.V; v0 += 1024 >> share) {
        const int v = v0 + (threadIdx.x >> share), i0 = threadIdx.x & (wide - 1);
        const int64_t row = b * A.V + v;
        float t = -INFINITY;
        bool fin = false;
        if (v < A.V) {
            t = A.total_in[row];
            fin = A.done && A.done[row];
        }
        const bool read = t - t == 0.f && !fin;
        const float *pm = A.seg_max + row * A.segs;
        const double *ps = A.seg_sum + row * A.segs;
        // (the first part of each thread's at once)
        float m0 = -INFINITY;
        double s0 = 0.0;
        if (v < A.V && i0 < A.segs) {   // (what stands there for a beam that does not read its scores is dropped)
            m0 = pm[i0];
            s0 = ps[i0];
        }
        if (!read) m0 = -INFINITY;
        float m = m0;
        if (read)
            for (int i = i0 + wide; i < A.segs; i += wide) m = fmaxf(m, pm[i]);
        m = reduce_lanes(m, share, Larger());
        const bool some = m > -INFINITY && m < INFINITY;
        double s = some && m0 > -INFINITY ? s0 * exp_below((double)m0 - (double)m) : 0.0;
        if (some)
            for (int i = i0 + wide; i < A.segs; i += wide)
                if (pm[i] > -INFINITY) s += ps[i] * exp_below((double)pm[i] - (double)m);
        s = reduce_lanes(s, share, Plus());
        if (v < A.V && i0 == 0) {
            off[v] = some ? (double)t - ((double)m + log_from(s)) : fin && t - t == 0.f ? (double)t : -INFINITY;
            done[v] = fin;
        }
    }
    // every group's best candidate: each(row, group of the row, key), the first kHeld of a thread from registers
    const int32_t up = 1024 / A.groups, rest = 1024 % A.groups;
    __syncthreads();   // (the rows' offsets)
    auto groups = [&](auto each) {
        int32_t v = threadIdx.x / A.groups, g = threadIdx.x - v * A.groups;
        for (int32_t i0 = threadIdx.x; i0 < total; i0 += 1024 * kHeld) {
            float m[kHeld];
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                const int32_t i = i0 + 1024 * k;
                m[k] = i0 < 1024 ? held[k] : i < total ? maxima[i] : -INFINITY;
            }
#pragma unroll
            for (int k = 0; k < kHeld; ++k) {
                if (i0 + 1024 * k >= total) break;
                const double o = off[v];   // (what stands there for rows without candidates is not looked at)
                double key = -INFINITY;
                if (o > -INFINITY) key = done[v] ? (g == 0 ? o : -INFINITY) : (double)m[k] + o;
                each(v, g, key);
                v += up;
                g += rest;
                if (g >= A.groups) {
                    g -= A.groups;
                    ++v;
                }
            }
        }
    };
    double top = -INFINITY;
    groups([&](int32_t, int32_t, double key) { top = key > top ? key : top; });
    if (best.raise(top)) {
        // the groups that reach the bar, then their candidates
        if (best.passes(top, -1)) {
            groups([&](int32_t v, int32_t g, double key) {
                if (key > -INFINITY && best.passes(key, -1)) {
                    const int at = atomicAdd(&n_listed, 1);
                    if (at < kListed) {
                        list_row[at] = (uint8_t)v;
                        list_column[at] = g << A.group;
                    }
                }
            });
        }
        __syncthreads();
        const int n = n_listed, places = min(n, kListed) << A.group;
        for (int32_t e0 = threadIdx.x; e0 - (int32_t)threadIdx.x < places; e0 += 8192) {
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int32_t e = e0 + 1024 * k;
                x[k] = -INFINITY;
                if (e < places) {
                    const int32_t v = list_row[e >> A.group], c = list_column[e >> A.group] + (e & ((1 << A.group) - 1));
                    if (done[v]) x[k] = c == 0 ? 0.f : -INFINITY;
                    else if (c < A.S) x[k] = score<T>(A, b * A.V + v, c);
                }
            }
            unsigned mask = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int32_t e = e0 + 1024 * k;
                if (x[k] > -INFINITY && best.passes((double)x[k] + off[list_row[e >> A.group]], -1)) mask |= 1u << k;
            }
            best.offer(__popc(mask), [&](auto put) {
                for (unsigned m = mask; m; m &= m - 1) {
                    const int k = __ffs((int)m) - 1;
                    const int32_t e = e0 + 1024 * k, v = list_row[e >> A.group];
                    put((double)pick(x, k) + off[v], v * A.S + list_column[e >> A.group] + (e & ((1 << A.group) - 1)));
                }
            });
        }
        if (best.offered() && n <= kListed) {
            write_beams(A, b, best, done);
            return;
        }
        best.clear();
    }
    // Too few groups to set a bar, or too many candidates at it: the rows that have candidates, one after the other,
    // four columns of each thread at a time.
    for (int32_t v = 0; v < A.V; ++v) {
        const double o = off[v];
        if (!(o > -INFINITY)) continue;
        const int32_t S = done[v] ? 1 : A.S;
        for (int32_t c0 = 0; c0 < S; c0 += 4096) {
            double key[4];
            int passing = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int32_t c = c0 + 1024 * k + threadIdx.x;
                key[k] = c >= S ? -INFINITY : done[v] ? o : (double)score<T>(A, b * A.V + v, c) + o;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) passing += B::lanes(best.passes(key[k], v * A.S + c0 + 1024 * k + threadIdx.x));
            if (best.sum(passing) == 0) continue;
            for (int k = 0; k < 4; ++k) {
                double q = key[0];
#pragma unroll
                for (int i = 1; i < 4; ++i) q = i == k ? key[i] : q;
                best.take(q, v * A.S + c0 + 1024 * k + (int32_t)threadIdx.x);
            }
        }
    }
    write_beams(A, b, best, done);
}

// -------------------------------------------------------------------- reorder
struct StateArgs {
    const char *in;
    char *out;
    int64_t in_search, in_beam, out_search, out_beam;
    int64_t first;                // first block
    int64_t wide;                 // 16-byte pieces of a row
    int32_t blocks, wide_blocks;  // blocks per search: of the wide pieces, then of the row's last bytes if there are any
    int32_t tail;                 // these bytes
};
constexpr int kStates = 16;       // arrays to a launch
struct ReorderArgs {
    int32_t V, W, n_states;
    int32_t cols, tail_cols;      // pieces (bytes at the end) of a row per block, powers of two
    const int32_t *parent;
    StateArgs s[kStates];
};

typedef unsigned piece __attribute__((ext_vector_type(4), aligned(1)));

// Columns [c0, c0 + cols) of every row of a search, all read before the first is
// written: out may be in.
template <int ITEMS, typename P>
__device__ __forceinline__ void reorder_columns(const ReorderArgs &A, const StateArgs &S, const int32_t *from, int64_t b,
                                                int64_t c0, int cols, int64_t end) {
    P v[ITEMS];
    const int shift = 31 - __clz(cols);
    const char *in = S.in + b * S.in_search;
    char *out = S.out + b * S.out_search;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int i = threadIdx.x + 256 * k, w = i >> shift;
        const int64_t c = c0 + (i & (cols - 1));
        if (w < A.W && c < end && from[w] >= 0)
            v[k] = *reinterpret_cast<const P *>(in + from[w] * S.in_beam + c * (int64_t)sizeof(P));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        const int i = threadIdx.x + 256 * k, w = i >> shift;
        const int64_t c = c0 + (i & (cols - 1));
        if (w < A.W && c < end && from[w] >= 0)
            *reinterpret_cast<P *>(out + w * S.out_beam + c * (int64_t)sizeof(P)) = v[k];
    }
}

// ITEMS: 16-byte pieces (or bytes of a row's end) per thread.  Memory bounds it: 128
// rows of 1.84 MB from one set of buffers to another 73 us, 360 MB at 4.9 TB/s; 64 rows
// of 222 KB in place 7.4 us by 4 to a thread, 8.8 by 16 (215 blocks).
template <int ITEMS>
__global__ void __launch_bounds__(256) beam_reorder(ReorderArgs A) {
    __shared__ int32_t from[kMaxWidth];
    int64_t bid = blockIdx.x;
    int at = 0;
#pragma unroll
    for (int i = 1; i < kStates; ++i)
        if (i < A.n_states && bid >= A.s[i].first) at = i;
    const StateArgs &S = A.s[at];
    bid -= S.first;
    const int64_t b = bid / S.blocks;
    const int32_t part = (int32_t)(bid - b * S.blocks);
    if ((int)threadIdx.x < A.W) {
        const int32_t p = A.parent[b * A.W + threadIdx.x];
        from[threadIdx.x] = p < A.V ? p : -1;
    }
    __syncthreads();
    if (part >= S.wide_blocks)
        reorder_columns<ITEMS, uint8_t>(A, S, from, b, S.wide * 16 + (part - S.wide_blocks) * A.tail_cols, A.tail_cols,
                                        S.wide * 16 + S.tail);
    else reorder_columns<ITEMS, piece>(A, S, from, b, (int64_t)part * A.cols, A.cols, S.wide);
}

// ---------------------------------------------------------------------- host
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

// The way that a level goes: one launch where each search's scores fit the registers
// of a block, else rows in parts and a launch that joins them.
struct Way {
    int32_t shift, fours, segs, group, groups;
    bool whole;
    int64_t blocks;   // of the parts
};
Way way(int32_t n, int32_t V, int32_t W, int32_t S) {
    Way w{};
    while (w.shift < 10 && 16 << w.shift < S) ++w.shift;
    w.whole = 16 << w.shift >= S && V << w.shift <= 1024;
    if (w.whole) {
        // More threads to a row than its scores need: as a wavefront has them anyway, or so that the threads' best set a
        // bar (317 searches of 37 x 12: 71 -> 9 us).
        while (4 << w.shift < S && V << (w.shift + 1) <= 1024 && (V << (w.shift + 1) <= 64 || V << w.shift < 2 * W)) ++w.shift;
        w.fours = std::min(4, (int32_t)((S + (4ll << w.shift) - 1) >> (w.shift + 2)));
        return w;
    }
    w.fours = 4;
    w.shift = std::min(w.shift, 8);
    w.segs = (int32_t)((S + 4095ll) / 4096);
    // Groups: of their V S / 2^g maxima each is looked at twice, of about W of them all 2^g scores are read again, at
    // about equal costs where 4^g is some 3 V S / W.
    const int32_t most = w.shift >= 6 ? 10 : w.shift + 2;
    for (w.group = 4; w.group + 2 <= most && ((int64_t)W << (2 * w.group + 2)) < (int64_t)3 * V * S;) w.group += 2;
    w.groups = (int32_t)((S + (1ll << w.group) - 1) >> w.group);
    const int64_t items = (int64_t)n * V * w.segs;
    w.blocks = (items + (256 >> w.shift) - 1) >> (8 - w.shift);
    return w;
}
size_t carve(int32_t n, int32_t V, const Way &w, void *base, BeamArgs *A) {
    if (w.whole) return 0;
    Carver c(base);
    const size_t rows = (size_t)n * V;
    A->seg_max = c.take<float>(rows * w.segs);
    A->seg_sum = c.take<double>(rows * w.segs);
    A->group_max = c.take<float>(rows * w.groups);
    return c.used;
}

template <typename T>
void launch_select(const BeamArgs &A, const Way &w, int32_t n, hipStream_t st) {
    if (w.whole) {
        const int threads = A.V << A.shift;
        const unsigned four = (unsigned)((n + 3) / 4);
        // (a wavefront ranks some 40 candidates by itself; a search of 1 x 256 slices, 64 beams after it: 14.4 us by
        // one, 10.0 by four)
        if (threads <= 64 && A.W <= 32) beam_whole<T, 64, 320><<<four, 256, 0, st>>>(A, n);
        else if (threads <= 256) beam_whole<T, 256, 512><<<n, 256, 0, st>>>(A, n);
        else beam_whole<T, 1024, 2048><<<n, 1024, 0, st>>>(A, n);
        return;
    }
    const int64_t rows = (int64_t)n * A.V;
    const unsigned blocks = (unsigned)w.blocks;
    if (w.shift < 8) beam_parts<T, 0><<<blocks, 256, 0, st>>>(A, rows);
    else if (w.group == 4) beam_parts<T, 4><<<blocks, 256, 0, st>>>(A, rows);
    else if (w.group == 6) beam_parts<T, 6><<<blocks, 256, 0, st>>>(A, rows);
    else if (w.group == 8) beam_parts<T, 8><<<blocks, 256, 0, st>>>(A, rows);
    else beam_parts<T, 10><<<blocks, 256, 0, st>>>(A, rows);
    beam_join<T><<<n, 1024, 0, st>>>(A);
}

tag_status check_beams(int32_t n, int32_t V, int32_t W) {
    if (n < 0 || V < 1 || W < 1) TAG_FAIL(TAG_EINVAL, "need n_search >= 0, width_in >= 1 and width >= 1");
    if (V > kMaxWidth || W > kMaxWidth) TAG_FAIL(TAG_ESHAPE, "at most 256 beams");
    return TAG_OK;
}
tag_status check_select(int32_t n, int32_t V, int32_t W, int32_t S) {
    const tag_status st = check_beams(n, V, W);
    if (st != TAG_OK) return st;
    if (S < 1) TAG_FAIL(TAG_EINVAL, "need n_slices >= 1");
    if ((int64_t)V * S > (1 << 30)) TAG_FAIL(TAG_ESHAPE, "at most 2^30 continuations of a search");
    // (a launch has fewer than 2^32 threads)
    if (n >= 1 << 22 || (n > 0 && way(n, V, W, S).blocks >= 1 << 24))
        TAG_FAIL(TAG_ESHAPE, "too many scores for a launch");
    return TAG_OK;
}

// rows of states
Area area(const void *p, int64_t n, int64_t rows, int64_t search, int64_t beam, int64_t row) {
    const int64_t span = (n - 1) * search + (rows - 1) * beam + row;
    const bool even = rows == 1 || n == 1 || (beam > 0 && search % beam == 0);   // (steps of 0 are no columns)
    const int64_t step = rows > 1 ? beam : n > 1 ? search : 0;
    return Area{(uintptr_t)p, (uintptr_t)p + span, even && step >= row ? step : 0, row};
}

}  // namespace
}  // namespace tag

using namespace tag;

extern "C" tag_status tag_beam_workspace(int32_t n_search, int32_t width_in, int32_t width, int32_t n_slices,
                                         size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    const tag_status st = check_select(n_search, width_in, width, n_slices);
    if (st != TAG_OK) return st;
    BeamArgs A{};
    *bytes = carve(n_search, width_in, way(n_search, width_in, width, n_slices), nullptr, &A);
    return TAG_OK;
}

extern "C" tag_status tag_beam_select(int32_t n_search, int32_t width_in, int32_t width, int32_t n_slices, int32_t dtype,
                                      const void *scores, int64_t score_stride, const float *total_in,
                                      const uint8_t *done, float *total, int32_t *parent, int32_t *slice,
                                      void *workspace, size_t ws_bytes, void *hip_stream) {
    clear_error();
    const tag_status st = check_select(n_search, width_in, width, n_slices);
    if (st != TAG_OK) return st;
    if (dtype != TAG_F32 && dtype != TAG_BF16) TAG_FAIL(TAG_EINVAL, "dtype must be TAG_F32 or TAG_BF16");
    if (n_search == 0) return TAG_OK;
    if (!scores || !total_in || !total || !parent || !slice)
        TAG_FAIL(TAG_EINVAL, "scores, total_in, total, parent and slice must be non-NULL");
    if (score_stride < n_slices) TAG_FAIL(TAG_EINVAL, "a row stride is below the number of slices");
    const size_t el = dtype == TAG_BF16 ? 2 : 4;
    if (!aligned(scores, el) || !aligned(total_in, 4) || !aligned(total, 4) || !aligned(parent, 4) || !aligned(slice, 4))
        TAG_FAIL(TAG_EINVAL, "an array is not aligned to its elements");
    const int64_t rows = (int64_t)n_search * width_in;
    if (rows > 1 && score_stride > ((int64_t)1 << 58) / rows)   // (products below, and the kernels', stay in 64 bits)
        TAG_FAIL(TAG_ESHAPE, "scores span at most 2^58 elements");
    const size_t wide = (size_t)n_search * width * 4;
    const Area in[3] = {flat_area(scores, ((rows - 1) * score_stride + n_slices) * el), flat_area(done, rows),
                        flat_area(total_in, rows * 4)};
    const Area out[3] = {flat_area(parent, wide), flat_area(slice, wide), flat_area(total, wide)};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i)
            if (out[o].meets(in[i]) && !(o == 2 && i == 2 && total == total_in && width == width_in))
                TAG_FAIL(TAG_EINVAL, "an output overlaps an input (total may be total_in where the widths are the same)");
        for (int p = 0; p < o; ++p)
            if (out[o].meets(out[p])) TAG_FAIL(TAG_EINVAL, "outputs overlap one another");
    }
    BeamArgs A{};
    const Way w = way(n_search, width_in, width, n_slices);
    const size_t need = carve(n_search, width_in, w, nullptr, &A);
    if (need > ws_bytes) TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_beam_workspace)");
    if (need && (!workspace || !aligned(workspace, 16)))
        TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    carve(n_search, width_in, w, workspace, &A);
    A.V = width_in; A.W = width; A.S = n_slices;
    A.x = scores; A.xs = score_stride;
    A.total_in = total_in; A.done = done;
    A.total = total; A.parent = parent; A.slice = slice;
    A.shift = w.shift; A.fours = w.fours; A.segs = w.segs; A.group = w.group; A.groups = w.groups;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dtype == TAG_BF16) launch_select<uint16_t>(A, w, n_search, stream);
    else launch_select<float>(A, w, n_search, stream);
    return launch_status("tag_beam_select");
}

extern "C" tag_status tag_beam_reorder(int32_t n_search, int32_t width_in, int32_t width, const int32_t *parent,
                                       const tag_beam_state *states, int32_t n_states, void *hip_stream) {
    clear_error();
    tag_status st = check_beams(n_search, width_in, width);
    if (st != TAG_OK) return st;
    if (n_states < 0 || n_states > 64) TAG_FAIL(TAG_EINVAL, "n_states must be in [0, 64]");
    if (n_search == 0 || n_states == 0) return TAG_OK;
    if (!parent || !states) TAG_FAIL(TAG_EINVAL, "parent and states must be non-NULL");
    if (!aligned(parent, 4)) TAG_FAIL(TAG_EINVAL, "parent is not aligned to its elements");
    const int64_t n = n_search;
    Area in[64], out[64];
    for (int32_t i = 0; i < n_states; ++i) {
        const tag_beam_state &s = states[i];
        if (s.row_bytes < 0) TAG_FAIL(TAG_EINVAL, "row_bytes must be >= 0");
        if (s.row_bytes > 0 && (!s.in || !s.out)) TAG_FAIL(TAG_EINVAL, "in and out must be non-NULL");
        if (s.in_search < 0 || s.in_beam < 0 || s.out_search < 0 || s.out_beam < 0)
            TAG_FAIL(TAG_EINVAL, "strides must be >= 0");
        const int64_t most = (int64_t)1 << 46;   // (products below stay in 64 bits)
        if (s.row_bytes > most || s.in_beam > most || s.out_beam > most || s.in_search > most || s.out_search > most)
            TAG_FAIL(TAG_ESHAPE, "rows and strides of at most 2^46 bytes");
        if (std::max(s.in_search, s.out_search) > ((int64_t)1 << 61) / n)
            TAG_FAIL(TAG_ESHAPE, "searches span at most 2^61 bytes");
        const int64_t span = (width - 1) * s.out_beam + s.row_bytes;
        if ((width > 1 && s.out_beam < s.row_bytes) || (n > 1 && s.out_search < span &&
            !(s.out_search >= s.row_bytes && (width == 1 || s.out_beam >= (n - 1) * s.out_search + s.row_bytes))))
            TAG_FAIL(TAG_EINVAL, "rows of out overlap");
        in[i] = s.row_bytes ? area(s.in, n, width_in, s.in_search, s.in_beam, s.row_bytes) : flat_area(nullptr, 0);
        out[i] = s.row_bytes ? area(s.out, n, width, s.out_search, s.out_beam, s.row_bytes) : flat_area(nullptr, 0);
        if (s.in == s.out && s.row_bytes > 0) {
            const int32_t rows = std::max(width, width_in);
            const bool strides = (rows == 1 || s.in_beam == s.out_beam) && (n == 1 || s.in_search == s.out_search);
            if (!strides || (n > 1 && width != width_in && s.out_search < (rows - 1) * s.out_beam + s.row_bytes))
                TAG_FAIL(TAG_EINVAL, "out may be in only with its strides, and searches that do not overlap");
        } else if (in[i].meets(out[i])) {
            TAG_FAIL(TAG_EINVAL, "out must be in, row by row, or not overlap it");
        }
    }
    const Area par = flat_area(parent, (size_t)n * width * 4);
    for (int32_t i = 0; i < n_states; ++i) {
        if (out[i].meets(par)) TAG_FAIL(TAG_EINVAL, "out overlaps parent");
        for (int32_t j = 0; j < n_states; ++j)
            if (i != j && (out[i].meets(in[j]) || (j < i && out[i].meets(out[j]))))
                TAG_FAIL(TAG_EINVAL, "out overlaps another array of states");
    }
    // As many pieces of a row to a block as leave room for every row: 4 to a thread, or 16 where that gives each CU
    // several blocks all the same (longer runs).
    int items = 16, cols = 0, tail_cols = 0;
    int64_t blocks[64], total = 0;
    for (;; items = 4) {
        for (cols = 256 * items; cols * width > 256 * items;) cols /= 2;
        tail_cols = std::min(cols, 16);
        total = 0;
        for (int32_t i = 0; i < n_states; ++i) {
            blocks[i] = (states[i].row_bytes / 16 + cols - 1) / cols + (states[i].row_bytes % 16 + tail_cols - 1) / tail_cols;
            total += std::min<int64_t>(blocks[i], 1 << 24) * n;
        }
        if (items == 4 || total >= 1024) break;
    }
    if (total >= 1 << 24) TAG_FAIL(TAG_ESHAPE, "too many or too large rows");   // (a launch has fewer than 2^32 threads)
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int32_t i0 = 0; i0 < n_states; i0 += kStates) {
        ReorderArgs A{};
        A.V = width_in; A.W = width; A.cols = cols; A.tail_cols = tail_cols; A.parent = parent;
        int64_t first = 0;
        for (int32_t i = i0; i < std::min(n_states, i0 + kStates); ++i) {
            const tag_beam_state &s = states[i];
            if (s.row_bytes == 0) continue;
            StateArgs &K = A.s[A.n_states++];
            K.in = static_cast<const char *>(s.in); K.out = static_cast<char *>(s.out);
            K.in_search = n > 1 ? s.in_search : 0; K.in_beam = width_in > 1 ? s.in_beam : 0;
            K.out_search = n > 1 ? s.out_search : 0; K.out_beam = width > 1 ? s.out_beam : 0;
            K.wide = s.row_bytes / 16; K.tail = (int32_t)(s.row_bytes % 16);
            K.wide_blocks = (int32_t)((K.wide + cols - 1) / cols);
            K.first = first; K.blocks = (int32_t)blocks[i];
            first += n * blocks[i];
        }
        if (first == 0) continue;
        if (items == 16) beam_reorder<16><<<(unsigned)first, 256, 0, stream>>>(A);
        else beam_reorder<4><<<(unsigned)first, 256, 0, stream>>>(A);
    }
    return launch_status("tag_beam_reorder");
}
