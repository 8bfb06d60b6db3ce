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
// outputs, from all of the row's records (kFinish).  The history's counts of
// the row's (part's) columns are LDS counters that its threads fill, so its
// length is not bounded; y is formed in the order that the header gives, each
// operation rounded.
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
    float y[VPT];
#pragma unroll
    for (int k = 0; k < NV; ++k)
        load4<T, VEC>(xr, c0 + 4 * (tid + NT * k), A.S, -INFINITY, *reinterpret_cast<float(*)[4]>(y + 4 * k));
    if (C.history) {
#pragma unroll
        for (int k = 0; k < NV; ++k) *reinterpret_cast<int4 *>(cnt + 4 * (tid + NT * k)) = int4{0, 0, 0, 0};
        Team::sync();
        int32_t n = C.n_history;
        if (C.history_len) n = min(n, max(C.history_len[q], 0));
        const int32_t *h = C.history + q * C.history_stride;
        const uint32_t span = (uint32_t)min((int64_t)W, A.S - c0);
        for (int32_t t = tid; t < n; t += NT) {
            const int64_t a = (int64_t)h[t] - c0;
            if (a >= 0 && a < span) atomicAdd(cnt + a, 1);
        }
        Team::sync();
        const float rep = C.repetition ? C.repetition[q] : 1.f, pre = C.presence ? C.presence[q] : 0.f,
                    frq = C.frequency ? C.frequency[q] : 0.f;
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
        const float *br = C.bias + q * C.bias_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float b[4];
            load4<float, VEC>(br, c0 + 4 * (tid + NT * k), A.S, 0.f, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[4 * k + i] += b[i];
        }
    }
    if (C.allow) {
        const uint32_t *ar = C.allow + q * C.allow_stride;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t c = c0 + 4 * (tid + NT * k);
            const uint32_t bits = c < A.S ? ar[c >> 5] >> (c & 31) : 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (!((bits >> i) & 1u)) y[4 * k + i] = -INFINITY;
        }
    }
    RowMax mx{-INFINITY, INT32_MAX, 0};
    float z = 0.f;
    if (PASS != kFinish) {
#pragma unroll
        for (int k = 0; k < VPT; ++k) {
            const int32_t c = (int32_t)c0 + 4 * (tid + NT * (k / 4)) + k % 4;
            const bool in = c < A.S;   // (columns past the end hold -inf or a NaN of inf - inf)
            if (in && y[k] > mx.m) { mx.m = y[k]; mx.at = c; }
            if (in && y[k] != y[k]) mx.nan = 1;
        }
        mx = Team::reduce(mx, RowMax::join);
    } else {
        // the row's records, joined in the same order by every part
        float m = -INFINITY;
        const float *rec = A.rec + q * A.chunks * 4;
        for (int32_t i = tid; i < A.chunks; i += NT) {
            const float4 r = *reinterpret_cast<const float4 *>(rec + 4 * (int64_t)i);
            mx = RowMax::join(mx, RowMax{r.x, __float_as_int(r.z), __float_as_int(r.w)});
        }
        mx = Team::reduce(mx, RowMax::join);
        m = mx.m;
        for (int32_t i = tid; i < A.chunks; i += NT) {
            const float4 r = *reinterpret_cast<const float4 *>(rec + 4 * (int64_t)i);
            if (r.x > -INFINITY) z = fmaf(r.y, exp_neg(r.x - m), z);
        }
        z = Team::reduce(RowSum{z}, RowSum::join).s;
    }
    const bool none = !(mx.m > -INFINITY);
#pragma unroll
    for (int k = 0; k < VPT && PASS != kFinish; ++k) {
        const int32_t c = (int32_t)c0 + 4 * (tid + NT * (k / 4)) + k % 4;
        if (c < A.S && !none) z += exp_neg(y[k] - mx.m);
    }
    if (PASS != kFinish) z = Team::reduce(RowSum{z}, RowSum::join).s;
    if (!live) return;   // (after the last barrier)
    if (PASS == kPart) {
        if (tid == 0)
            *reinterpret_cast<float4 *>(A.rec + item * 4) = float4{mx.m, z, __int_as_float(mx.at), __int_as_float(mx.nan)};
        return;
    }
    if (A.out) {
        T *o = static_cast<T *>(A.out) + q * A.os;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            store4<T, VEC>(o, c0 + 4 * (tid + NT * k), A.S, *reinterpret_cast<float(*)[4]>(y + 4 * k));
    }
    if (A.prior) {
        const float inv = mx.nan ? __builtin_nanf("") : none ? 0.f : 1.f / z;
        float *p = A.prior + q * A.ps;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            float v[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = (none ? 1.f : exp_neg(y[4 * k + i] - mx.m)) * inv;
            store4<float, VEC>(p, c0 + 4 * (tid + NT * k), A.S, v);
        }
    }
    if (part == 0 && tid == 0) {
        A.argmax[q] = mx.nan || none ? -1 : mx.at;
        A.best[q] = mx.nan ? __builtin_nanf("") : mx.m;
    }
}

constexpr int64_t kConWhole = 8192;   // longest row that one block keeps in registers
constexpr int kConPart = 4096;        // columns of a part of a longer one

template <typename T, int NT, int VPT, int PASS>
void launch_con_pass(const ConArgs &A, bool vec, int64_t items, hipStream_t st) {
    using Team = RowTeam<NT>;
    const unsigned grid = (unsigned)((items + Team::kRows - 1) / Team::kRows);
    const size_t lds = A.c.history ? sizeof(int32_t) * Team::kRows * NT * VPT : 0;
    if (vec) con_rows<T, NT, VPT, true, PASS><<<grid, Team::kBlock, lds, st>>>(A);
    else con_rows<T, NT, VPT, false, PASS><<<grid, Team::kBlock, lds, st>>>(A);
}

template <typename T>
void launch_constrain(const ConArgs &A, bool vec, hipStream_t st) {
    if (A.S <= 64) launch_con_pass<T, 16, 4, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 256) launch_con_pass<T, 64, 4, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 1024) launch_con_pass<T, 64, 16, kWhole>(A, vec, A.Q, st);
    else if (A.S <= 4096) launch_con_pass<T, 256, 16, kWhole>(A, vec, A.Q, st);
    else if (A.S <= kConWhole) launch_con_pass<T, 512, 16, kWhole>(A, vec, A.Q, st);
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
    if (c.history && c.history_stride != 0 && c.history_stride < c.n_history)
        TAG_FAIL(TAG_EINVAL, "history_stride must be 0 or cover a row");
    if (!aligned(scores, el) || !aligned(constrained, el) || !aligned(prior, 4) || !aligned(c.bias, 4) ||
        !aligned(c.allow, 4) || !aligned(c.history, 4))
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
    if ((int64_t)n_query * A.chunks > INT32_MAX) TAG_FAIL(TAG_ESHAPE, "too many rows of this length");
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
constexpr int kBalBlocks = 2048;   // blocks that walk the rows
constexpr int kBalSpan = 256;      // slices per counting block

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
    double *part;        // [counting blocks][64] their slices' part of n load
    double *total;       // load [64], centre, n
    double *lpart;       // [kBalBlocks] sums over rows of sum_a p_a (h_a - centre)
    int32_t *done;       // [2] blocks that are through
};

__device__ __forceinline__ uint64_t device_bits(int32_t M) { return M >= 64 ? ~0ull : (1ull << M) - 1ull; }

// Each used row's argmax.
template <typename T, int NT, int VPT, bool VEC>
__global__ void __launch_bounds__(RowTeam<NT>::kBlock) bal_argmax(BalArgs A) {
    using Team = RowTeam<NT>;
    const int tid = Team::tid();
    if (blockIdx.x == 0 && threadIdx.x < 2) A.done[threadIdx.x] = 0;
    for (int64_t base = (int64_t)blockIdx.x * Team::kRows; base < A.Q; base += (int64_t)gridDim.x * Team::kRows) {
        const int64_t q0 = base + Team::row(), q = q0 < A.Q ? q0 : A.Q - 1;
        const bool use = !A.use || A.use[q] != 0;
        const T *xr = static_cast<const T *>(A.x) + q * A.xs;
        RowMax mx{-INFINITY, INT32_MAX, 0};
        if (use) {
#pragma unroll
            for (int k = 0; k < VPT / 4; ++k) {
                const int32_t c = 4 * (tid + NT * k);
                float v[4];
                load4<T, VEC>(xr, c, A.S, -INFINITY, v);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (v[i] > mx.m) { mx.m = v[i]; mx.at = c + i; }
                    if (v[i] != v[i]) mx.nan = 1;
                }
            }
        }
        mx = Team::reduce(mx, RowMax::join);
        if (tid == 0 && q0 < A.Q) A.arg[q] = mx.nan ? -2 : (mx.m > -INFINITY ? mx.at : -1);
    }
}

// the last block to get here (every thread of it): it sees what the others wrote before
__device__ __forceinline__ bool last_block(int32_t *done) {
    __shared__ int32_t mine;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) mine = atomicAdd(done, 1);
    __syncthreads();
    const bool last = mine == (int32_t)gridDim.x - 1;
    if (last) __threadfence();
    return last;
}

// Counts of kBalSpan slices per block over all rows' argmaxes (LDS counters; a
// wavefront first joins its lanes that agree with one of them, twice, since the
// decisions of a batch crowd on few slices), and their part of the loads; the
// last block through adds those up in block order.
__global__ void __launch_bounds__(1024) bal_count(BalArgs A) {
    __shared__ int32_t cnt[kBalSpan], used;
    const int t = threadIdx.x, lane = t & 63;
    const int32_t s0 = blockIdx.x * kBalSpan;
    if (t < kBalSpan) cnt[t] = 0;
    if (t == 0) used = 0;
    __syncthreads();
    int32_t n = 0;
    for (int64_t base = 0; base < A.Q; base += 1024) {
        int32_t a = base + t < A.Q ? A.arg[base + t] : -1;
        n += a != -1;
        a -= s0;
        bool want = a >= 0 && a < kBalSpan;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const uint64_t some = __ballot(want);
            if (!some) break;
            const int first = __ffsll((unsigned long long)some) - 1;
            const bool same = want && a == __shfl(a, first, 64);
            const uint64_t who = __ballot(same);
            if (lane == first) atomicAdd(cnt + a, __popcll(who));
            want = want && !same;
        }
        if (want) atomicAdd(cnt + a, 1);
    }
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    if (lane == 0) atomicAdd(&used, n);
    __syncthreads();
    if (t < kBalSpan && s0 + t < A.S) A.count[s0 + t] = cnt[t];
    // 16 threads per device
    const int d = t >> 4;
    const uint64_t valid = device_bits(A.M);
    double w = 0.0;
    for (int i = t & 15; i < kBalSpan && s0 + i < A.S; i += 16) {
        const uint64_t m = A.mask[s0 + i] & valid;
        if ((m >> d) & 1ull) w += (double)cnt[i] / (double)__popcll(m);
    }
    for (int o = 8; o > 0; o >>= 1) w += __shfl_xor(w, o, 16);
    if ((t & 15) == 0) A.part[(int64_t)blockIdx.x * 64 + d] = w;
    if (!last_block(A.done)) return;
    if (t < 64) {
        double s = 0.0;
        for (int b = 0; b < (int)gridDim.x; ++b)
            s += __hip_atomic_load(A.part + (int64_t)b * 64 + t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s = used > 0 ? s / (double)used : 0.0;
        if (t < A.M) A.load[t] = (float)s;
        A.total[t] = s;
        // centre of h: its mean over the decisions taken (softmax gradients do not see a shift of h, and
        // what is left of h rounds less)
        double c = s * s;
        for (int o = 32; o > 0; o >>= 1) c += __shfl_xor(c, o, 64);
        if (t == 0) { A.total[64] = c; A.total[65] = (double)used; }
    }
}

// Gradient rows and the loss: each thread keeps h of its columns for every row
// that its block walks.
template <typename T, int NT, int VPT, bool VEC>
__global__ void __launch_bounds__(RowTeam<NT>::kBlock) bal_grad(BalArgs A) {
#pragma clang fp contract(off)   // (the same bits from the forms for aligned and for other rows)
    using Team = RowTeam<NT>;
    __shared__ double load[66], lred[RowTeam<NT>::kBlock];
    const int tid = Team::tid();
    for (int i = threadIdx.x; i < 66; i += Team::kBlock) load[i] = A.total[i];
    __syncthreads();
    const double n = load[65], centre = load[64];
    const float scale = n > 0.0 ? (float)((double)A.coef * A.M / n) : 0.f;
    const uint64_t valid = device_bits(A.M);
    float h[VPT];
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
        const int32_t c = 4 * (tid + NT * (k / 4)) + k % 4;
        uint64_t m = c < A.S ? A.mask[c] & valid : 0;
        const double pop = (double)__popcll(m);
        double s = 0.0;
        while (m) {
            s += load[__ffsll((unsigned long long)m) - 1];
            m &= m - 1;
        }
        h[k] = (float)((pop > 0.0 ? s / pop : 0.0) - centre);
    }
    double lsum = 0.0;
    for (int64_t base = (int64_t)blockIdx.x * Team::kRows; base < A.Q; base += (int64_t)gridDim.x * Team::kRows) {
        const int64_t q0 = base + Team::row(), q = q0 < A.Q ? q0 : A.Q - 1;
        const bool live = q0 < A.Q;
        const int32_t arg = A.arg[q];
        const T *xr = static_cast<const T *>(A.x) + q * A.xs;
        T *gr = static_cast<T *>(A.grad) + q * A.gs;
        float x[VPT];
        float m = -INFINITY;
        if (arg != -1) {
#pragma unroll
            for (int k = 0; k < VPT / 4; ++k) {
                load4<T, VEC>(xr, 4 * (tid + NT * k), A.S, -INFINITY, *reinterpret_cast<float(*)[4]>(x + 4 * k));
#pragma unroll
                for (int i = 0; i < 4; ++i) m = x[4 * k + i] > m ? x[4 * k + i] : m;
            }
        }
        m = Team::reduce(RowMax{m, 0, 0}, RowMax::join).m;
        float z = 0.f, e = 0.f;
        if (arg != -1) {
#pragma unroll
            for (int k = 0; k < VPT; ++k) {
                x[k] = exp_neg(x[k] - m);
                z += x[k];
                e = fmaf(x[k], h[k], e);
            }
        }
        const RowSum2 r = Team::reduce(RowSum2{z, e}, RowSum2::join);
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
        if (tid == 0) lsum += (double)mean;
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
    // the block's sum, then (the last block) all of them, in a fixed order
    lred[threadIdx.x] = lsum;
    __syncthreads();
    if (threadIdx.x == 0) {
        double s = 0.0;
        for (int r = 0; r < Team::kRows; ++r) s += lred[r * NT];
        A.lpart[blockIdx.x] = s;
    }
    if (!last_block(A.done + 1)) return;
    double s = 0.0;
    for (int b = threadIdx.x; b < (int)gridDim.x; b += Team::kBlock)
        s += __hip_atomic_load(A.lpart + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    lred[threadIdx.x] = s;
    __syncthreads();
    for (int o = Team::kBlock / 2; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) lred[threadIdx.x] += lred[threadIdx.x + o];
        __syncthreads();
    }
    if (threadIdx.x == 0) A.loss[0] = n > 0.0 ? (float)((double)A.coef * A.M * (lred[0] / n + centre)) : 0.f;
}

template <typename T, int NT, int VPT>
void launch_bal(const BalArgs &A, bool vec, hipStream_t st) {
    using Team = RowTeam<NT>;
    const unsigned grid = (unsigned)std::min<int64_t>(kBalBlocks, (A.Q + Team::kRows - 1) / Team::kRows);
    const unsigned cgrid = (unsigned)((A.S + kBalSpan - 1) / kBalSpan);
    if (vec) bal_argmax<T, NT, VPT, true><<<grid, Team::kBlock, 0, st>>>(A);
    else bal_argmax<T, NT, VPT, false><<<grid, Team::kBlock, 0, st>>>(A);
    bal_count<<<cgrid, 1024, 0, st>>>(A);
    if (vec) bal_grad<T, NT, VPT, true><<<grid, Team::kBlock, 0, st>>>(A);
    else bal_grad<T, NT, VPT, false><<<grid, Team::kBlock, 0, st>>>(A);
}

template <typename T>
void launch_balance(const BalArgs &A, bool vec, hipStream_t st) {
    if (A.S <= 64) launch_bal<T, 16, 4>(A, vec, st);
    else if (A.S <= 256) launch_bal<T, 64, 4>(A, vec, st);
    else if (A.S <= 1024) launch_bal<T, 64, 16>(A, vec, st);
    else if (A.S <= 4096) launch_bal<T, 256, 16>(A, vec, st);
    else launch_bal<T, 1024, 16>(A, vec, st);
}

size_t carve_bal(int32_t Q, int32_t S, void *base, BalArgs *A) {
    Carver c(base);
    A->done = c.take<int32_t>(2);
    A->total = c.take<double>(66);
    A->part = c.take<double>((size_t)((S + kBalSpan - 1) / kBalSpan) * 64);
    A->lpart = c.take<double>(kBalBlocks);
    A->arg = c.take<int32_t>((size_t)std::max(Q, 1));
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
    if (!aligned(scores, el) || !aligned(grad, el) || !aligned(mask, 8))
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
