// Beam search over the decision head's scores (include/tag_beam.h): one level's
// selection, and the reordering of the beams' states.
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
};

// doubles (no NaN) as unsigned integers in the same order; both zeros are one
__device__ __forceinline__ uint64_t ordered(double d) {
    const uint64_t b = (uint64_t)__double_as_longlong(d + 0.0);
    return b >> 63 ? ~b : b | 1ull << 63;
}
__device__ __forceinline__ double unordered(uint64_t u) {
    return __longlong_as_double((long long)(u >> 63 ? u ^ 1ull << 63 : ~u));
}

// The best W of a search's candidates (key, index), collected by a block of NT
// threads that call everything here together.  Candidates that beat the bar are
// appended to a list in LDS in any order; when it is full, its best W stay and the
// W-th becomes the bar.  The order is total (larger key, then lower index), so the
// result does not depend on the order in which they came.
template <int NT, int CAP>
struct Best {
    static_assert(CAP % NT == 0 && CAP >= NT + kMaxWidth, "room for a candidate of each thread beside the best W");
    static constexpr int kWaves = NT / 64, kOwn = CAP / NT;
    struct Shared {
        double key[CAP];
        int32_t idx[CAP];
        int32_t count[2][kWaves];
        int32_t tail;
    };
    Shared &s;
    const int W;
    double bar = -INFINITY;      // a candidate passes above it, or at it up to the index
    int32_t bar_idx = -1;
    int n = 0, flip = 0;         // entries of the list

    __device__ Best(Shared &s_, int w) : s(s_), W(w) {
        if (threadIdx.x == 0) s.tail = 0;
        __syncthreads();
    }
    __device__ bool passes(double key, int32_t idx) const { return key > bar || (key == bar && idx <= bar_idx); }
    // sum over the wavefronts of a number that each wavefront's lanes share
    __device__ int sum(int v) {
        if ((threadIdx.x & 63) == 0) s.count[flip][threadIdx.x >> 6] = v;
        __syncthreads();
        int r = 0;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) r += s.count[flip][i];
        flip ^= 1;   // (written again only after the next barrier, which follows these reads)
        return r;
    }
    static __device__ int lanes(bool b) { return __popcll(__ballot(b)); }
    __device__ void append(bool is, double key, int32_t idx) {
        const uint64_t m = __ballot(is);
        if (m == 0) return;
        const int lane = threadIdx.x & 63;
        int at = 0;
        if (lane == 0) at = atomicAdd(&s.tail, __popcll(m));
        at = __shfl(at, 0, 64) + __popcll(m & ((1ull << lane) - 1ull));
        if (is) {
            s.key[at] = key;
            s.idx[at] = idx;
        }
    }
    // N candidates of each thread (key -inf: none)
    template <int N>
    __device__ void take(const double (&key)[N], const int32_t (&idx)[N]) {
        int c = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) c += lanes(passes(key[k], idx[k]));
        c = sum(c);
        if (n + c <= CAP) {
            if (c > 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) append(passes(key[k], idx[k]), key[k], idx[k]);
            }
            n += c;
            return;
        }
#pragma unroll 1
        for (int k = 0; k < N; ++k) {
            double kk = key[0];
            int32_t ii = idx[0];
#pragma unroll
            for (int q = 1; q < N; ++q) {
                kk = k == q ? key[q] : kk;
                ii = k == q ? idx[q] : ii;
            }
            c = sum(lanes(passes(kk, ii)));
            if (n + c > CAP) {
                keep_best();
                c = sum(lanes(passes(kk, ii)));
            }
            append(passes(kk, ii), kk, ii);
            n += c;
        }
    }
    // leaves the best W of a list of more
    __device__ void keep_best() {
        __syncthreads();
        uint64_t u[kOwn];
        int32_t idx[kOwn];
#pragma unroll
        for (int r = 0; r < kOwn; ++r) {
            const int at = threadIdx.x + NT * r;
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
        if (threadIdx.x == 0) s.tail = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kOwn; ++r)
            append(u[r] > K || (u[r] == K && u[r] != 0 && idx[r] <= last), unordered(u[r]), idx[r]);
        n = W;
        bar = unordered(K);
        bar_idx = last;
    }
    // each(rank, key, index) of the best, at most W; returns how many
    template <typename Each>
    __device__ int ranked(Each each) {
        if (n > W) keep_best();
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += NT) {
            const double k = s.key[i];
            const int32_t x = s.idx[i];
            int r = 0;
            for (int j = 0; j < n; ++j) r += s.key[j] > k || (s.key[j] == k && s.idx[j] < x);
            each(r, k, x);
        }
        return n;
    }
};

template <typename T>
__device__ __forceinline__ float score(const BeamArgs &A, int64_t row, int64_t c) {
    return Quad<T>::get1(static_cast<const T *>(A.x)[row * A.xs + c]);
}

template <typename B>
__device__ __forceinline__ void write_beams(const BeamArgs &A, int64_t b, B &best) {
    const int n = best.ranked([&](int r, double key, int32_t idx) {
        const int32_t v = idx / A.S;
        A.total[b * A.W + r] = (float)key;
        A.parent[b * A.W + r] = v;
        A.slice[b * A.W + r] = A.done && A.done[b * A.V + v] ? -1 : idx - v * A.S;
    });
    for (int r = n + threadIdx.x; r < A.W; r += blockDim.x) {
        A.total[b * A.W + r] = -INFINITY;
        A.parent[b * A.W + r] = A.slice[b * A.W + r] = -1;
    }
}

// One block per search: what each beam adds to its scores, a wavefront to a row,
// then all candidates.
template <typename T>
__global__ void __launch_bounds__(1024) beam_search(BeamArgs A) {
    using B = Best<1024, 2048>;
    __shared__ B::Shared shared;
    __shared__ double off[kMaxWidth];
    const int64_t b = blockIdx.x;
    const int lane = threadIdx.x & 63;
    for (int v = threadIdx.x >> 6; v < A.V; v += 16) {
        const float t = A.total_in[b * A.V + v];
        double o = -INFINITY;
        if (t - t == 0.f) {
            if (A.done && A.done[b * A.V + v]) {
                o = t;
            } else {
                float m = -INFINITY;
                bool bad = false;
                for (int64_t c = lane; c < A.S; c += 64) {
                    const float x = score<T>(A, b * A.V + v, c);
                    bad = bad || !(x < INFINITY);
                    m = fmaxf(m, x);
                }
                for (int i = 32; i > 0; i >>= 1) m = fmaxf(m, __shfl_xor(m, i, 64));
                if (__ballot(bad) == 0 && m > -INFINITY) {
                    double sum = 0.0;
                    for (int64_t c = lane; c < A.S; c += 64) sum += exp((double)score<T>(A, b * A.V + v, c) - (double)m);
                    for (int i = 32; i > 0; i >>= 1) sum += __shfl_xor(sum, i, 64);
                    o = (double)t - ((double)m + log(sum));
                }
            }
        }
        if (lane == 0) off[v] = o;
    }
    B best(shared, A.W);   // (a barrier)
    const int32_t total = A.V * A.S;
    for (int32_t base = 0; base < total; base += 1024) {
        double key[1] = {-INFINITY};
        const int32_t idx[1] = {base + (int32_t)threadIdx.x};
        if (idx[0] < total) {
            const int32_t v = idx[0] / A.S, a = idx[0] - v * A.S;
            const double o = off[v];
            if (o > -INFINITY) {
                if (A.done && A.done[b * A.V + v]) key[0] = a == 0 ? o : -INFINITY;
                else key[0] = (double)score<T>(A, b * A.V + v, a) + o;
            }
        }
        best.take(key, idx);
    }
    write_beams(A, b, best);
}

// -------------------------------------------------------------------- reorder
constexpr int kItems = 16;                    // 16-byte pieces (or bytes of a row's end) per thread
constexpr int kBlockItems = 256 * kItems;

struct StateArgs {
    const char *in;
    char *out;
    int64_t in_search, in_beam, out_search, out_beam;
    int64_t first;                // first block
    int64_t wide;                 // 16-byte pieces of a row
    int32_t blocks;               // blocks per search: of the wide pieces, then one of the row's last bytes if there are any
    int32_t tail;                 // these bytes
};
constexpr int kStates = 16;       // arrays to a launch
struct ReorderArgs {
    int32_t V, W, cols, n_states; // cols: pieces of a row per block, a power of two
    const int32_t *parent;
    StateArgs s[kStates];
};

typedef unsigned piece __attribute__((ext_vector_type(4), aligned(1)));

// Columns [c0, c0 + cols) of every row of a search, all read before the first is
// written: out may be in.
template <typename P>
__device__ __forceinline__ void reorder_columns(const ReorderArgs &A, const StateArgs &S, const int32_t *from, int64_t b,
                                                int64_t c0, int cols, int64_t end) {
    P v[kItems];
    const int shift = 31 - __clz(cols);
    const char *in = S.in + b * S.in_search;
    char *out = S.out + b * S.out_search;
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = threadIdx.x + 256 * k, w = i >> shift;
        const int64_t c = c0 + (i & (cols - 1));
        if (w < A.W && c < end && from[w] >= 0) v[k] = *reinterpret_cast<const P *>(in + from[w] * S.in_beam + c * (int64_t)sizeof(P));
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kItems; ++k) {
        const int i = threadIdx.x + 256 * k, w = i >> shift;
        const int64_t c = c0 + (i & (cols - 1));
        if (w < A.W && c < end && from[w] >= 0) *reinterpret_cast<P *>(out + w * S.out_beam + c * (int64_t)sizeof(P)) = v[k];
    }
}

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
    if (S.tail && part == S.blocks - 1) reorder_columns<uint8_t>(A, S, from, b, S.wide * 16, 16, S.wide * 16 + S.tail);
    else reorder_columns<piece>(A, S, from, b, (int64_t)part * A.cols, A.cols, S.wide);
}

// ---------------------------------------------------------------------- host
inline bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

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
    if (n >= 1 << 22) TAG_FAIL(TAG_ESHAPE, "fewer than 2^22 searches");   // (a launch has fewer than 2^32 threads)
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
    *bytes = 0;
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
    const size_t wide = (size_t)n_search * width * 4;
    const Area in[3] = {flat_area(scores, ((rows - 1) * score_stride + n_slices) * el), flat_area(done, rows), flat_area(total_in, rows * 4)};
    const Area out[3] = {flat_area(parent, wide), flat_area(slice, wide), flat_area(total, wide)};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 3; ++i)
            if (out[o].meets(in[i]) && !(o == 2 && i == 2 && total == total_in && width == width_in))
                TAG_FAIL(TAG_EINVAL, "an output overlaps an input (total may be total_in where the widths are the same)");
        for (int p = 0; p < o; ++p)
            if (out[o].meets(out[p])) TAG_FAIL(TAG_EINVAL, "outputs overlap one another");
    }
    (void)workspace;
    (void)ws_bytes;
    const BeamArgs A{width_in, width, n_slices, scores, score_stride, total_in, done, total, parent, slice};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (dtype == TAG_BF16) beam_search<uint16_t><<<n_search, 1024, 0, stream>>>(A);
    else beam_search<float><<<n_search, 1024, 0, stream>>>(A);
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
        if (std::max(s.in_search, s.out_search) > ((int64_t)1 << 61) / n) TAG_FAIL(TAG_ESHAPE, "searches span at most 2^61 bytes");
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
    // as many pieces of a row as leave room for every row
    int cols = kBlockItems;
    while (cols * width > kBlockItems) cols /= 2;
    int64_t blocks[64], total = 0;
    for (int32_t i = 0; i < n_states; ++i) {
        blocks[i] = (states[i].row_bytes / 16 + cols - 1) / cols + (states[i].row_bytes % 16 ? 1 : 0);
        if (blocks[i] < (1 << 24) / n + 1) total += n * blocks[i];
        else total = 1 << 24;
        if (total >= 1 << 24) TAG_FAIL(TAG_ESHAPE, "too many or too large rows");   // (a launch has fewer than 2^32 threads)
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int32_t i0 = 0; i0 < n_states; i0 += kStates) {
        ReorderArgs A{};
        A.V = width_in; A.W = width; A.cols = cols; A.parent = parent;
        int64_t first = 0;
        for (int32_t i = i0; i < std::min(n_states, i0 + kStates); ++i) {
            const tag_beam_state &s = states[i];
            if (s.row_bytes == 0) continue;
            StateArgs &K = A.s[A.n_states++];
            K.in = static_cast<const char *>(s.in); K.out = static_cast<char *>(s.out);
            K.in_search = n > 1 ? s.in_search : 0; K.in_beam = width_in > 1 ? s.in_beam : 0;
            K.out_search = n > 1 ? s.out_search : 0; K.out_beam = width > 1 ? s.out_beam : 0;
            K.wide = s.row_bytes / 16; K.tail = (int32_t)(s.row_bytes % 16);
            K.first = first; K.blocks = (int32_t)blocks[i];
            first += n * blocks[i];
        }
        if (first > 0) beam_reorder<<<(unsigned)first, 256, 0, stream>>>(A);
    }
    return launch_status("tag_beam_reorder");
}
