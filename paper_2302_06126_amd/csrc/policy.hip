// Operators on the decision head's scores (include/tag_policy.h): constrained
// priors and the balance loss with its gradient.  Both are a few operations
// per score, so memory bounds them: a row's scores are read once into
// registers, four consecutive columns per thread and step, and everything
// that the row needs (maximum, sum of exponentials, argmax) is reduced among
// its threads.
#include <algorithm>
#include <string>

#include "../../include/tag_policy.h"
#include "policy_rows.hpp"

namespace tag {
namespace {

// ------------------------------------------------------------------ constrain
struct ConArgs {
    int32_t Q, S;
    const void *x;
    int64_t xs;
    tag_constraints c;
    void *out;
    int64_t os;
    float *prior;
    int64_t ps;
    int32_t *argmax;
    float *best;
    float *rec;        // [Q][chunks][4]: max, sum, argmax, NaN flag of a part of a row
    int32_t chunks;
};

enum { kWhole = 0, kPart = 1, kFinish = 2 };

// a taken slice's score, each operation rounded
__device__ __forceinline__ float penalised(float y, int32_t taken, float rep, float pre, float frq) {
#pragma clang fp contract(off)
    y = y > 0.f ? y / rep : y * rep;
    return y - frq * (float)taken - pre;
}

// One row by NT threads, VPT columns each (kWhole), or one part of a row of
// NT * VPT columns: its maximum and sum (kPart), and in a second launch its
// outputs, from all of the row's records (kFinish).  Every load that does not
// wait for another is issued first.  The history's counts of the row's (part's)
// columns are LDS counters that its threads fill, so its length is not bounded;
// y is formed in the order that the header gives, each operation rounded.
// Memory bounds it: 42,496 x 256 bf16 with masks and biases per row, both results
// written, 143 MB in 27.8 us, 5.1 TB/s, the rate of a large copy.  In parts, 64 x
// 262,140: 31.3 us (134 MB) and 40.2 us (the same again, mostly from the last
// cache, and 67 MB written).
template <typename T, int NT, int VPT, bool VEC, int PASS>
__global__ void __launch_bounds__(RowTeam<NT>::kBlock) con_rows(ConArgs A) {
#pragma clang fp contract(off)   // (the same bits from the forms for aligned and for other rows)
    using Team = RowTeam<NT>;
    extern __shared__ __attribute__((aligned(16))) int32_t counts[];   // [kRows][NT * VPT] with a history
    constexpr int W = NT * VPT, NV = VPT / 4;
    const int tid = Team::tid();
    const int64_t item = (int64_t)blockIdx.x * Team::kRows + Team::row();
    const int64_t q0 = PASS == kWhole ? item : item / A.chunks;
    const int32_t part = PASS == kWhole ? 0 : (int32_t)(item % A.chunks);
    const bool live = q0 < A.Q;
    const int64_t q = live ? q0 : A.Q - 1;
    const int64_t c0 = (int64_t)part * W;
    const tag_constraints &C = A.c;
    int32_t *cnt = counts + Team::row() * W;
    const T *xr = static_cast<const T *>(A.x) + q * A.xs;
    float y[VPT], b[VPT];
    uint32_t ok[NV];
    // the first of the history, whatever its length: it is needed first
    constexpr int NH = 4;
    int32_t taken[NH], n_taken = 0;
    const int32_t *hist = nullptr;
    if (C.history) {
        hist = C.history + q * C.history_stride;
        n_taken = C.n_history;
        if (C.history_len) n_taken = min(n_taken, max(C.history_len[q], 0));
#pragma unroll
        for (int k = 0; k < NH; ++k) taken[k] = tid + NT * k < C.n_history ? hist[tid + NT * k] : -1;
    }
#pragma unroll
    for (int k = 0; k < NV; ++k)
        load4<T, VEC>(xr, c0 + 4 * (tid + NT * k), A.S, -INFINITY, *reinterpret_cast<float(*)[4]>(y + 4 * k));
    if (C.bias) {
        const float *br = C.bias + q * C.bias_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            load4<float, VEC>(br, c0 + 4 * (tid + NT * k), A.S, 0.f, *reinterpret_cast<float(*)[4]>(b + 4 * k));
    }
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int64_t c = c0 + 4 * (tid + NT * k);
        ok[k] = c < A.S ? (C.allow ? C.allow[q * C.allow_stride + (c >> 5)] >> (c & 31) : 15u) : 0u;
        if (c + 4 > A.S && c < A.S) ok[k] &= (1u << (A.S - c)) - 1u;   // (columns past the end)
    }
    if (C.history) {
        const float rep = C.repetition ? C.repetition[q] : 1.f, pre = C.presence ? C.presence[q] : 0.f,
                    frq = C.frequency ? C.frequency[q] : 0.f;
        const uint32_t span = (uint32_t)min((int64_t)W, A.S - c0);
#pragma unroll
        for (int k = 0; k < NV; ++k) *reinterpret_cast<int4 *>(cnt + 4 * (tid + NT * k)) = int4{0, 0, 0, 0};
        Team::sync();
        for (int32_t t = tid; t < n_taken; t += NH * NT) {
#pragma unroll
            for (int k = 0; k < NH; ++k) {
                const int64_t a = (int64_t)taken[k] - c0;
                if (t + NT * k < n_taken && a >= 0 && a < span) atomicAdd(cnt + a, 1);
            }
#pragma unroll
            for (int k = 0; k < NH; ++k) taken[k] = t + NT * (NH + k) < n_taken ? hist[t + NT * (NH + k)] : -1;
        }
        Team::sync();
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int4 n4 = *reinterpret_cast<const int4 *>(cnt + 4 * (tid + NT * k));
            const int32_t cn[4] = {n4.x, n4.y, n4.z, n4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (cn[i] > 0) y[4 * k + i] = penalised(y[4 * k + i], cn[i], rep, pre, frq);
            }
        }
    }
    if (C.bias) {
#pragma unroll
        for (int k = 0; k < VPT; ++k) y[k] += b[k];
    }
    RowMax mx{-INFINITY, INT32_MAX};
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        if (!((ok[k / 4] >> (k % 4)) & 1u)) y[k] = -INFINITY;
        if (PASS != kFinish && y[k] > mx.m) mx = RowMax{y[k], (int32_t)c0 + 4 * (tid + NT * (k / 4)) + k % 4};
    }
    float z = 0.f;
    if (PASS != kFinish) {
#pragma unroll
        for (int k = 0; k < VPT; ++k)
            if (y[k] != y[k]) mx.at = -2;
        mx = Team::max(mx);
    } else {
        // the row's records, joined in the same order by every part
        const float *rec = A.rec + q * A.chunks * 4;
        for (int32_t i = tid; i < A.chunks; i += NT) {
            const float4 r = *reinterpret_cast<const float4 *>(rec + 4 * (int64_t)i);
            const int32_t at = __float_as_int(r.z);
            const bool nan = mx.at == -2 || at == -2;
            if (r.x > mx.m) mx = RowMax{r.x, at};   // (a thread's records go up in columns)
            if (nan) mx.at = -2;
        }
        mx = Team::max(mx);
        for (int32_t i = tid; i < A.chunks; i += NT) {
            const float4 r = *reinterpret_cast<const float4 *>(rec + 4 * (int64_t)i);
            if (r.x > -INFINITY) z = fmaf(r.y, exp_neg(r.x - mx.m), z);
        }
    }
    const bool none = !(mx.m > -INFINITY), nan = mx.at == -2;
    if (PASS != kPart && A.out && live) {
        T *o = static_cast<T *>(A.out) + q * A.os;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            store4<T, VEC>(o, c0 + 4 * (tid + NT * k), A.S, *reinterpret_cast<float(*)[4]>(y + 4 * k));
    }
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        y[k] = none ? 0.f : exp_neg(y[k] - mx.m);
        if (PASS != kFinish) z += y[k];
    }
    z = Team::sum(z);
    if (!live) return;   // (after the last barrier)
    if (PASS == kPart) {
        if (tid == 0) *reinterpret_cast<float4 *>(A.rec + item * 4) = float4{mx.m, z, __int_as_float(mx.at), 0.f};
        return;
    }
    if (A.prior) {
        const float inv = nan ? __builtin_nanf("") : none ? 0.f : 1.f / z;
        float *p = A.prior + q * A.ps;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = y[4 * k + i] * inv;
            store4<float, VEC>(p, c0 + 4 * (tid + NT * k), A.S, v);
        }
    }
    if (part == 0 && tid == 0) {
        A.argmax[q] = nan || none ? -1 : mx.at;
        A.best[q] = nan ? __builtin_nanf("") : mx.m;
    }
}

// Longest row that one block keeps in registers; longer ones go by parts, in two
// launches that both read the scores.  Whole | by parts, us: 1 x 8,000 7.4 | 11.5,
// 2,000 x 8,000 27 | 46, 1 x 16,000 9.5 | 11.1, 500 x 16,000 19 | 28, 1,500 x 10,000
// 41 | 46.
constexpr int64_t kConWhole = 16384;
constexpr int kConPart = 4096;        // columns of a part of a longer one

template <typename T, int NT, int VPT, int PASS>
void launch_con_pass(const ConArgs &A, bool vec, int64_t items, hipStream_t st) {
    using Team = RowTeam<NT>;
    const unsigned grid = (unsigned)((items + Team::kRows - 1) / Team::kRows);
    const size_t lds = A.c.history ? sizeof(int32_t) * Team::kRows * NT * VPT : 0;
    if (vec) con_rows<T, NT, VPT, true, PASS><<<grid, Team::kBlock, lds, st>>>(A);
    else con_rows<T, NT, VPT, false, PASS><<<grid, Team::kBlock, lds, st>>>(A);
}

// Threads per row: 16 columns each (a wavefront takes four rows of up to 256, whose
// reductions cost it one), more threads only where those do not hold the row.
// 2,000 x 4,000 by 256 threads 14.5 us, by 1,024 34; 10,000 x 1,000 by 64 19, by 256 23;
// 42,496 x 256 by 16 36.9, by 64 36.2.
template <typename T>
void launch_constrain(const ConArgs &A, bool vec, hipStream_t st) {
    if (A.S <= 64) launch_con_pass<T, 16, 4, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 256) launch_con_pass<T, 16, 16, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 1024) launch_con_pass<T, 64, 16, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 4096) launch_con_pass<T, 256, 16, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 8192) launch_con_pass<T, 512, 16, kWhole>(A, vec, A.Q, st);
    else if (A.S <= kConWhole) launch_con_pass<T, 1024, 16, kWhole>(A, vec, A.Q, st);
    else {
        launch_con_pass<T, 256, kConPart / 256, kPart>(A, vec, (int64_t)A.Q * A.chunks, st);
        launch_con_pass<T, 256, kConPart / 256, kFinish>(A, vec, (int64_t)A.Q * A.chunks, st);
    }
}

int64_t con_chunks(int32_t S) { return S > kConWhole ? (S + (int64_t)kConPart - 1) / kConPart : 0; }

// bytes that rows of `n` elements at stride `stride` span
struct Span {
    uintptr_t b, e;
    Span(const void *p, int64_t rows, int64_t n, int64_t stride, size_t el)
        : b((uintptr_t)p), e((uintptr_t)p + (p && rows > 0 ? ((rows - 1) * stride + n) * el : 0)) {}
    bool meets(const Span &o) const { return b < e && o.b < o.e && b < o.e && o.b < e; }
};

inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

tag_status check_rows(int32_t Q, int32_t S, int32_t dtype) {
    if (Q < 0 || S < 1) TAG_FAIL(TAG_EINVAL, "need n_query >= 0 and n_slices >= 1");
    if (dtype != TAG_F32 && dtype != TAG_BF16) TAG_FAIL(TAG_EINVAL, "dtype must be TAG_F32 or TAG_BF16");
    return TAG_OK;
}

}  // namespace
}  // namespace tag

using namespace tag;

extern "C" tag_status tag_constrain_workspace(int32_t n_query, int32_t n_slices, size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    const tag_status st = check_rows(n_query, n_slices, TAG_F32);
    if (st != TAG_OK) return st;
    *bytes = (size_t)n_query * con_chunks(n_slices) * 4 * sizeof(float);
    return TAG_OK;
}

extern "C" tag_status tag_constrain(int32_t n_query, int32_t n_slices, int32_t dtype, const void *scores,
                                    int64_t score_stride, const tag_constraints *constraints, void *constrained,
                                    int64_t constrained_stride, float *prior, int64_t prior_stride, int32_t *argmax,
                                    float *best, void *workspace, size_t ws_bytes, void *hip_stream) {
    clear_error();
    tag_status st = check_rows(n_query, n_slices, dtype);
    if (st != TAG_OK) return st;
    if (!constraints) TAG_FAIL(TAG_EINVAL, "constraints must be non-NULL");
    if (n_query == 0) return TAG_OK;
    if (!scores || !argmax || !best) TAG_FAIL(TAG_EINVAL, "scores, argmax and best must be non-NULL");
    const int64_t S = n_slices, words = (S + 31) / 32;
    const size_t el = dtype == TAG_BF16 ? 2 : 4;
    const tag_constraints &c = *constraints;
    if (score_stride < S || (constrained && constrained_stride < S) || (prior && prior_stride < S))
        TAG_FAIL(TAG_EINVAL, "a row stride is below the number of slices");
    if ((c.allow && c.allow_stride != 0 && c.allow_stride < words) || (c.bias && c.bias_stride != 0 && c.bias_stride < S))
        TAG_FAIL(TAG_EINVAL, "allow_stride and bias_stride must be 0 or cover a row");
    if (c.n_history < 0 || (c.n_history > 0 && !c.history)) TAG_FAIL(TAG_EINVAL, "n_history needs a history");
    if (c.n_history > (1 << 30)) TAG_FAIL(TAG_ESHAPE, "at most 2^30 history entries");
    if (c.history && c.history_stride != 0 && c.history_stride < c.n_history)
        TAG_FAIL(TAG_EINVAL, "history_stride must be 0 or cover a row");
    if (!aligned(scores, el) || !aligned(constrained, el) || !aligned(prior, 4) || !aligned(c.bias, 4) ||
        !aligned(c.allow, 4) || !aligned(c.history, 4) || !aligned(c.history_len, 4) || !aligned(c.repetition, 4) ||
        !aligned(c.presence, 4) || !aligned(c.frequency, 4) || !aligned(argmax, 4) || !aligned(best, 4))
        TAG_FAIL(TAG_EINVAL, "an array is not aligned to its elements");
    if (constrained && constrained == scores ? constrained_stride != score_stride
                                             : Span(constrained, n_query, S, constrained_stride, el)
                                                   .meets(Span(scores, n_query, S, score_stride, el)))
        TAG_FAIL(TAG_EINVAL, "constrained must be the scores themselves, row by row, or not overlap them");
    if (Span(prior, n_query, S, prior_stride, 4).meets(Span(scores, n_query, S, score_stride, el)) ||
        Span(prior, n_query, S, prior_stride, 4).meets(Span(constrained, n_query, S, constrained_stride, el)))
        TAG_FAIL(TAG_EINVAL, "prior must not overlap scores or constrained");
    ConArgs A{};
    A.Q = n_query; A.S = n_slices;
    A.x = scores; A.xs = score_stride;
    A.c = c;
    if (c.n_history == 0) A.c.history = nullptr;
    A.out = constrained; A.os = constrained_stride;
    A.prior = prior; A.ps = prior_stride;
    A.argmax = argmax; A.best = best;
    A.chunks = (int32_t)std::max<int64_t>(1, con_chunks(n_slices));
    // (a launch has fewer than 2^32 threads: whole blocks of 256, or of a longer row's team)
    const int64_t team = S <= 256 ? 16 : S <= 1024 ? 64 : S <= 4096 || S > kConWhole ? 256 : S <= 8192 ? 512 : 1024;
    const int64_t block = std::max<int64_t>(team, 256), rows = block / team;
    if (((int64_t)n_query * A.chunks + rows - 1) / rows >= ((int64_t)1 << 32) / block)
        TAG_FAIL(TAG_ESHAPE, "too many rows of this length");
    size_t need = 0;
    tag_constrain_workspace(n_query, n_slices, &need);
    if (need > ws_bytes) TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_constrain_workspace)");
    if (need && (!workspace || !aligned(workspace, 16))) TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    A.rec = static_cast<float *>(workspace);
    // four columns as one load where every row of every array starts at a multiple of them
    const size_t q4 = 4 * el;
    const bool vec = aligned(scores, q4) && score_stride % 4 == 0 && aligned(constrained, q4) &&
                     (!constrained || constrained_stride % 4 == 0) && aligned(prior, 16) &&
                     (!prior || prior_stride % 4 == 0) && aligned(c.bias, 16) && (!c.bias || c.bias_stride % 4 == 0);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dtype == TAG_BF16) launch_constrain<uint16_t>(A, vec, stream);
    else launch_constrain<float>(A, vec, stream);
    return launch_status("tag_constrain");
}

namespace tag {
namespace {

// -------------------------------------------------------------------- balance
constexpr int kBalMaxS = 16384;
constexpr int kBalParts = 256;      // blocks that count decisions
constexpr int kBalGrad = 4096;      // blocks that walk the rows for their gradients, at most
constexpr int kBalSpan = 64;        // slices per merging block
constexpr int kBalInline = 256;     // slices whose h every gradient block forms itself

struct BalArgs {
    int32_t Q, S, M;
    const void *x;
    int64_t xs;
    const uint64_t *mask;
    const uint8_t *use;
    float coef;
    void *grad;
    int64_t gs;
    int32_t accumulate;
    float *loss;
    int32_t *count;
    float *load;
    // workspace
    int32_t *arg;        // [Q] argmax; -1: not used, -2: used with a NaN
    int32_t *hist;       // [parts][S] counts of one block's rows
    int32_t *used;       // [parts] its used rows
    double *part;        // [merging blocks][64] their slices' part of n load
    double *total;       // centre of h, n
    float *h;            // [S] less the centre
    double *lpart;       // [grad blocks] sums over rows of sum_a p_a h_a
    int32_t parts, lparts;
};

__device__ __forceinline__ uint64_t device_bits(int32_t M) { return M >= 64 ? ~0ull : (1ull << M) - 1ull; }

// The balance loss reads the scores twice: the counts of all rows' argmaxes are
// needed before the first gradient.  42,496 x 256 fp32 (44 MB): argmax 10.0 us (4.4
// TB/s), counts 6.6 (latency), gradients 18.1 (4.8 TB/s), loss 3.9 (a launch); the
// sums have launches of their own, since fences in blocks that have just written
// are dear (gradients 298 us so, in an earlier form with a fence and a count in
// every block for the last one through to add them up).

// Each used row's argmax (into arg), and how often the block's rows chose each
// slice: hist [S], then the used rows.
template <typename T, int NT, int VPT, bool VEC>
__device__ __forceinline__ void rows_argmax(const BalArgs &A, int32_t *hist) {
    using Team = RowTeam<NT, 1024>;
    for (int i = threadIdx.x; i <= A.S; i += 1024) hist[i] = 0;
    __syncthreads();
    const int tid = Team::tid();
    // (every thread of the block takes every turn: teams of several wavefronts meet in barriers)
    for (int64_t base = (int64_t)blockIdx.x * Team::kRows; base < A.Q; base += (int64_t)gridDim.x * Team::kRows) {
        const int64_t q0 = base + Team::row(), q = q0 < A.Q ? q0 : A.Q - 1;
        const bool use = !A.use || A.use[q] != 0;
        const T *xr = static_cast<const T *>(A.x) + q * A.xs;
        RowMax mx{-INFINITY, INT32_MAX};
        if (use) {
            float v[VPT];
            bool nan = false;
#pragma unroll
            for (int k = 0; k < VPT / 4; ++k)
                load4<T, VEC>(xr, 4 * (tid + NT * k), A.S, -INFINITY, *reinterpret_cast<float(*)[4]>(v + 4 * k));
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                if (v[k] > mx.m) mx = RowMax{v[k], 4 * (tid + NT * (k / 4)) + k % 4};
                nan = nan || v[k] != v[k];
            }
            if (nan) mx.at = -2;
        }
        mx = Team::max(mx);
        if (tid == 0 && q0 < A.Q) {
            const int32_t at = mx.at == INT32_MAX ? -1 : mx.at;
            A.arg[q] = at;
            if (at >= 0) atomicAdd(hist + at, 1);
            if (at != -1) atomicAdd(hist + A.S, 1);
        }
    }
    __syncthreads();
}

template <typename T, int NT, int VPT, bool VEC>
__global__ void __launch_bounds__(1024) bal_argmax(BalArgs A) {
    extern __shared__ int32_t hist[];
    rows_argmax<T, NT, VPT, VEC>(A, hist);
    for (int i = threadIdx.x; i < A.S; i += 1024) A.hist[(int64_t)blockIdx.x * A.S + i] = hist[i];
    if (threadIdx.x == 0) A.used[blockIdx.x] = hist[A.S];
}

// Counts of kBalSpan slices per block over the parts, and their part of the loads.
__global__ void __launch_bounds__(1024) bal_count(BalArgs A) {
    __shared__ int32_t sub[16][kBalSpan];
    __shared__ uint64_t mask[kBalSpan];
    __shared__ double each[kBalSpan], dev[16][64];   // what a slice gives each of its devices
    __shared__ int32_t used;
    const int t = threadIdx.x, c = t & 63, g = t >> 6, s = blockIdx.x * kBalSpan + c;
    uint64_t m = 0;
    if (g == 0 && s < A.S) m = A.mask[s] & device_bits(A.M);
    int32_t v[kBalParts / 16];
#pragma unroll
    for (int i = 0; i < kBalParts / 16; ++i) {
        const int p = g + 16 * i;
        v[i] = s < A.S && p < A.parts ? A.hist[(int64_t)p * A.S + s] : 0;
    }
    const int32_t mine = blockIdx.x == 0 && t < A.parts ? A.used[t] : 0;
    if (t == 0) used = 0;
    int32_t n = 0;
#pragma unroll
    for (int i = 0; i < kBalParts / 16; ++i) n += v[i];
    sub[g][c] = n;
    __syncthreads();
    if (mine) atomicAdd(&used, mine);
    if (g == 0) {
#pragma unroll
        for (int i = 1; i < 16; ++i) n += sub[i][c];
        if (s < A.S) A.count[s] = n;
        mask[c] = m;
        each[c] = m ? (double)n / (double)__popcll(m) : 0.0;
    }
    __syncthreads();
    double w = 0.0;   // device c, four slices per wavefront
#pragma unroll
    for (int i = 4 * g; i < 4 * g + 4; ++i) w += (mask[i] >> c) & 1ull ? each[i] : 0.0;
    dev[g][c] = w;
    __syncthreads();
    if (g == 0) {
#pragma unroll
        for (int i = 1; i < 16; ++i) w += dev[i][c];
        A.part[(int64_t)blockIdx.x * 64 + c] = w;
    }
    if (blockIdx.x == 0 && t == 0) A.total[1] = (double)used;
}

// Device t's load from the sum of its parts (threads t < 64, one wavefront), and
// the centre of h: its mean over slices that use every device equally, the mean
// load (the softmax's gradient does not see a shift of h, and what is left of h
// rounds less; its mean over the decisions taken, which stand far from the others
// where they are few, leaves gradients of 1 x 1,111 an error of 5.4e-7, this 1e-7).
__device__ __forceinline__ double device_load(const BalArgs &A, double s, double n, bool write, double *centre) {
    const int t = threadIdx.x;
    s = n > 0.0 ? s / n : 0.0;
    if (write && t < A.M) A.load[t] = (float)s;
    double c = s;
    for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
    *centre = c / A.M;
    return s;
}
// h of a slice less the centre
__device__ __forceinline__ float share_of(uint64_t mask, const double *load, double centre) {
    const double pop = (double)__popcll(mask);
    double w = 0.0;
    for (; mask; mask &= mask - 1) w += load[__ffsll((unsigned long long)mask) - 1];
    return (float)((pop > 0.0 ? w / pop : 0.0) - centre);
}

// Loads from the merging blocks' parts (in their order, by every block), then h of
// 1,024 slices per block.
__global__ void __launch_bounds__(1024) bal_shares(BalArgs A) {
    __shared__ double load[64], sub[16][64], centre;
    const int t = threadIdx.x, d = t & 63, g = t >> 6, nb = (A.S + kBalSpan - 1) / kBalSpan;
    const int32_t slice = blockIdx.x * 1024 + t;
    const uint64_t m = slice < A.S ? A.mask[slice] & device_bits(A.M) : 0;
    const double n = A.total[1];
    double p[kBalMaxS / kBalSpan / 16];
#pragma unroll
    for (int i = 0; i < kBalMaxS / kBalSpan / 16; ++i) {
        const int b = g + 16 * i;
        p[i] = b < nb ? A.part[(int64_t)b * 64 + d] : 0.0;
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kBalMaxS / kBalSpan / 16; ++i) s += p[i];
    sub[g][d] = s;
    __syncthreads();
    if (t < 64) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += sub[i][t];
        double c;
        load[t] = device_load(A, s, n, blockIdx.x == 0, &c);
        if (t == 0) centre = c;
        if (t == 0 && blockIdx.x == 0) A.total[0] = c;
    }
    __syncthreads();
    if (slice < A.S) A.h[slice] = share_of(m, load, centre);
}

// Gradient rows of the block's teams: each thread keeps h of its columns for
// every row.  Returns the sum of the team's rows' losses.
template <typename T, int NT, int VPT, bool VEC, int BLOCK>
__device__ __forceinline__ double rows_grad(const BalArgs &A, const float *hs, float scale) {
#pragma clang fp contract(off)   // (the same bits from the forms for aligned and for other rows)
    using Team = RowTeam<NT, BLOCK>;
    const int tid = Team::tid();
    float h[VPT];
#pragma unroll
    for (int k = 0; k < VPT / 4; ++k)
        load4<float, true>(hs, 4 * (tid + NT * k), A.S, 0.f, *reinterpret_cast<float(*)[4]>(h + 4 * k));
    double lsum = 0.0;
    for (int64_t base = (int64_t)blockIdx.x * Team::kRows; base < A.Q; base += (int64_t)gridDim.x * Team::kRows) {
        const int64_t q0 = base + Team::row(), q = q0 < A.Q ? q0 : A.Q - 1;
        const bool live = q0 < A.Q;
        const int32_t arg = A.arg[q];
        const T *xr = static_cast<const T *>(A.x) + q * A.xs;
        T *gr = static_cast<T *>(A.grad) + q * A.gs;
        float x[VPT];
        RowMax mx{-INFINITY, 0};
        if (arg != -1) {
#pragma unroll
            for (int k = 0; k < VPT / 4; ++k)
                load4<T, VEC>(xr, 4 * (tid + NT * k), A.S, -INFINITY, *reinterpret_cast<float(*)[4]>(x + 4 * k));
#pragma unroll
            for (int k = 0; k < VPT; ++k) mx.m = x[k] > mx.m ? x[k] : mx.m;
        }
        const float m = Team::max(mx).m;
        Two r{0.f, 0.f};
        if (arg != -1) {
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                x[k] = exp_neg(x[k] - m);
                r.s += x[k];
                r.t = fmaf(x[k], h[k], r.t);
            }
        }
        r = Team::sum(r);
        if (!live) continue;
        if (arg == -1) {
            if (!A.accumulate) {
                const float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = 0; k < VPT / 4; ++k) store4<T, VEC>(gr, 4 * (tid + NT * k), A.S, v);
            }
            continue;
        }
        const float inv = 1.f / r.s, mean = r.t * inv, f = scale * inv;
        lsum += (double)mean;
#pragma unroll
        for (int k = 0; k < VPT / 4; ++k) {
            float v[4];
            if (A.accumulate) load4<T, VEC>(gr, 4 * (tid + NT * k), A.S, 0.f, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float g = f * x[4 * k + i] * (h[4 * k + i] - mean);
                v[i] = A.accumulate ? v[i] + g : g;
            }
            store4<T, VEC>(gr, 4 * (tid + NT * k), A.S, v);
        }
    }
    return lsum;
}

__device__ __forceinline__ float row_scale(const BalArgs &A, double n) {
    return n > 0.0 ? (float)((double)A.coef * A.M / n) : 0.f;
}
__device__ __forceinline__ float total_loss(const BalArgs &A, double sum, double n, double centre) {
    return n > 0.0 ? (float)((double)A.coef * A.M * (sum / n + centre)) : 0.f;
}

// Gradient rows, and the block's sum of the rows' losses.
template <typename T, int NT, int VPT, bool VEC>
__global__ void __launch_bounds__(RowTeam<NT>::kBlock) bal_grad(BalArgs A) {
    using Team = RowTeam<NT>;
    __shared__ double lrow[Team::kRows], load[64], centre;
    __shared__ __attribute__((aligned(16))) float hs[kBalInline];
    const float *h = A.h;
    if (NT * VPT <= kBalInline) {   // few merging blocks: what bal_shares does, here, without its launch
        const int t = threadIdx.x, nb = (A.S + kBalSpan - 1) / kBalSpan;
        const uint64_t m = t < A.S ? A.mask[t] & device_bits(A.M) : 0;
        if (t < 64) {
            double p[kBalInline / kBalSpan], s = 0.0, c;
#pragma unroll
            for (int b = 0; b < kBalInline / kBalSpan; ++b) p[b] = b < nb ? A.part[(int64_t)b * 64 + t] : 0.0;
#pragma unroll
            for (int b = 0; b < kBalInline / kBalSpan; ++b) s += p[b];
            load[t] = device_load(A, s, A.total[1], blockIdx.x == 0, &c);
            if (t == 0) centre = c;
            if (t == 0 && blockIdx.x == 0) A.total[0] = c;
        }
        __syncthreads();
        hs[t] = share_of(m, load, centre);
        __syncthreads();
        h = hs;
    }
    const double lsum = rows_grad<T, NT, VPT, VEC, Team::kBlock>(A, h, row_scale(A, A.total[1]));
    if (Team::tid() == 0) lrow[Team::row()] = lsum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int r = 0; r < Team::kRows; ++r) s += lrow[r];
        A.lpart[blockIdx.x] = s;
    }
}

// Few rows: everything in one block, the scores' second reading from its cache.
// Its time grows with the turns that its teams take over the rows, that of the
// other way is four launches or five; this | those, us: 64 x 60 (a turn) 6.5 | 16.0,
// 256 x 60 (four) 10.8 | 16.5, 512 x 60 17.2 | 16.4; 64 x 256 (a turn) 10.1 | 17.0,
// 256 x 256 (four) 21.0 | 18.0; 16 x 1,000 (a turn) 14.8 | 21.9, 64 x 1,000 26.9 | 22.2.
constexpr int kBalSmallS = 1024;   // slices whose masks it keeps in LDS
constexpr int bal_small_turns(int vpt) { return vpt == 4 ? 6 : 2; }
template <typename T, int NT, int VPT, bool VEC>
__global__ void __launch_bounds__(1024) bal_small(BalArgs A) {
    using Team = RowTeam<NT, 1024>;
    __shared__ int32_t hist[kBalSmallS + 1];
    __shared__ uint64_t mask[kBalSmallS];
    __shared__ double each[kBalSmallS], load[64], sub[16][64], centre, lrow[Team::kRows];
    __shared__ __attribute__((aligned(16))) float h[kBalSmallS];
    const int t = threadIdx.x, d = t & 63, g = t >> 6;
    const uint64_t m = t < A.S ? A.mask[t] & device_bits(A.M) : 0;
    rows_argmax<T, NT, VPT, VEC>(A, hist);
    const int32_t used = hist[A.S];
    mask[t] = m;
    each[t] = m ? (double)hist[t] / (double)__popcll(m) : 0.0;   // (m = 0 past the slices)
    if (t < A.S) A.count[t] = hist[t];
    __syncthreads();
    double s = 0.0;
    for (int i = g; i < A.S; i += 16) s += (mask[i] >> d) & 1ull ? each[i] : 0.0;
    sub[g][d] = s;
    __syncthreads();
    if (t < 64) {
#pragma unroll
        for (int i = 1; i < 16; ++i) s += sub[i][t];
        double c;
        load[t] = device_load(A, s, (double)used, true, &c);
        if (t == 0) centre = c;
    }
    __syncthreads();
    h[t] = share_of(m, load, centre);
    __syncthreads();
    const double lsum = rows_grad<T, NT, VPT, VEC, 1024>(A, h, row_scale(A, (double)used));
    if (Team::tid() == 0) lrow[Team::row()] = lsum;
    __syncthreads();
    if (t < 64) {
        double l = t < Team::kRows ? lrow[t] : 0.0;
        for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o, 64);
        if (t == 0) A.loss[0] = total_loss(A, l, (double)used, centre);
    }
}

// the blocks' sums, in a fixed order
__global__ void __launch_bounds__(1024) bal_loss(BalArgs A) {
    __shared__ double red[16];
    const double n = A.total[1], centre = A.total[0];
    double v[kBalGrad / 1024];
#pragma unroll
    for (int i = 0; i < kBalGrad / 1024; ++i) {
        const int b = threadIdx.x + 1024 * i;
        v[i] = b < A.lparts ? A.lpart[b] : 0.0;
    }
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kBalGrad / 1024; ++i) s += v[i];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) s += red[w];
        A.loss[0] = total_loss(A, s, n, centre);
    }
}

template <typename T, int NT, int VPT>
void launch_bal(const BalArgs &A, bool vec, hipStream_t st) {
    if constexpr (NT <= 64) {
        if (A.Q <= bal_small_turns(VPT) * (1024 / NT)) {
            if (vec) bal_small<T, NT, VPT, true><<<1, 1024, 0, st>>>(A);
            else bal_small<T, NT, VPT, false><<<1, 1024, 0, st>>>(A);
            return;
        }
    }
    const size_t lds = sizeof(int32_t) * (A.S + 1);
    if (vec) bal_argmax<T, NT, VPT, true><<<A.parts, 1024, lds, st>>>(A);
    else bal_argmax<T, NT, VPT, false><<<A.parts, 1024, lds, st>>>(A);
    bal_count<<<(A.S + kBalSpan - 1) / kBalSpan, 1024, 0, st>>>(A);
    if (NT * VPT > kBalInline) bal_shares<<<(A.S + 1023) / 1024, 1024, 0, st>>>(A);
    if (vec) bal_grad<T, NT, VPT, true><<<A.lparts, RowTeam<NT>::kBlock, 0, st>>>(A);
    else bal_grad<T, NT, VPT, false><<<A.lparts, RowTeam<NT>::kBlock, 0, st>>>(A);
    bal_loss<<<1, 1024, 0, st>>>(A);
}

// threads per row
int bal_team(int32_t S) { return S <= 256 ? 16 : S <= 1024 ? 64 : S <= 4096 ? 256 : 1024; }

template <typename T>
void launch_balance(const BalArgs &A, bool vec, hipStream_t st) {
    if (A.S <= 64) launch_bal<T, 16, 4>(A, vec, st);
    else if (A.S <= 256) launch_bal<T, 16, 16>(A, vec, st);
    else if (A.S <= 1024) launch_bal<T, 64, 16>(A, vec, st);
    else if (A.S <= 4096) launch_bal<T, 256, 16>(A, vec, st);
    else launch_bal<T, 1024, 16>(A, vec, st);
}

size_t carve_bal(int32_t Q, int32_t S, void *base, BalArgs *A) {
    Carver c(base);
    const int64_t team = bal_team(S), rows = 1024 / team, grad_rows = team < 256 ? 256 / team : 1;
    A->parts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kBalParts, (Q + rows - 1) / rows));
    A->lparts = (int32_t)std::max<int64_t>(1, std::min<int64_t>(kBalGrad, (Q + grad_rows - 1) / grad_rows));
    A->total = c.take<double>(2);
    A->part = c.take<double>((size_t)((S + kBalSpan - 1) / kBalSpan) * 64);
    A->lpart = c.take<double>(A->lparts);
    A->h = c.take<float>(S);
    A->arg = c.take<int32_t>((size_t)std::max(Q, 1));
    A->used = c.take<int32_t>(A->parts);
    A->hist = c.take<int32_t>((size_t)A->parts * S);
    return c.used;
}

}  // namespace
}  // namespace tag

extern "C" tag_status tag_balance_workspace(int32_t n_query, int32_t n_slices, size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    const tag_status st = check_rows(n_query, n_slices, TAG_F32);
    if (st != TAG_OK) return st;
    if (n_slices > kBalMaxS) TAG_FAIL(TAG_ESHAPE, "at most 16384 slices");
    BalArgs A;
    *bytes = carve_bal(n_query, n_slices, nullptr, &A);
    return TAG_OK;
}

extern "C" tag_status tag_balance(int32_t n_query, int32_t n_slices, int32_t dtype, const void *scores,
                                  int64_t score_stride, const uint64_t *mask, int32_t n_dev, const uint8_t *use,
                                  float coef, void *grad, int64_t grad_stride, int32_t accumulate, float *loss,
                                  int32_t *count, float *load, void *workspace, size_t ws_bytes, void *hip_stream) {
    clear_error();
    tag_status st = check_rows(n_query, n_slices, dtype);
    if (st != TAG_OK) return st;
    if (n_slices > kBalMaxS) TAG_FAIL(TAG_ESHAPE, "at most 16384 slices");
    if (n_query < 1) TAG_FAIL(TAG_EINVAL, "need n_query >= 1");
    if (n_dev < 1 || n_dev > 64) TAG_FAIL(TAG_EINVAL, "n_dev must be in [1, 64]");
    if (!(coef >= 0.f) || coef == INFINITY) TAG_FAIL(TAG_EINVAL, "coef must be finite and >= 0");
    if (!scores || !mask || !grad || !loss || !count || !load || !workspace)
        TAG_FAIL(TAG_EINVAL, "scores, mask, grad, loss, count, load and workspace must be non-NULL");
    if (score_stride < n_slices || grad_stride < n_slices)
        TAG_FAIL(TAG_EINVAL, "a row stride is below the number of slices");
    if (accumulate && dtype != TAG_F32) TAG_FAIL(TAG_EINVAL, "accumulate needs TAG_F32");
    const size_t el = dtype == TAG_BF16 ? 2 : 4;
    if (!aligned(scores, el) || !aligned(grad, el) || !aligned(mask, 8) || !aligned(loss, 4) || !aligned(count, 4) ||
        !aligned(load, 4))
        TAG_FAIL(TAG_EINVAL, "an array is not aligned to its elements");
    if (Span(scores, n_query, n_slices, score_stride, el).meets(Span(grad, n_query, n_slices, grad_stride, el)))
        TAG_FAIL(TAG_EINVAL, "grad must not overlap scores");
    BalArgs A{};
    const size_t need = carve_bal(n_query, n_slices, nullptr, &A);
    if (need > ws_bytes) TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_balance_workspace)");
    if (!aligned(workspace, 16)) TAG_FAIL(TAG_EINVAL, "workspace must be 16-byte aligned");
    carve_bal(n_query, n_slices, workspace, &A);
    A.Q = n_query; A.S = n_slices; A.M = n_dev;
    A.x = scores; A.xs = score_stride;
    A.mask = mask; A.use = use; A.coef = coef;
    A.grad = grad; A.gs = grad_stride; A.accumulate = accumulate;
    A.loss = loss; A.count = count; A.load = load;
    const size_t q4 = 4 * el;
    const bool vec = aligned(scores, q4) && score_stride % 4 == 0 && aligned(grad, q4) && grad_stride % 4 == 0;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dtype == TAG_BF16) launch_balance<uint16_t>(A, vec, stream);
    else launch_balance<float>(A, vec, stream);
    return launch_status("tag_balance");
}
