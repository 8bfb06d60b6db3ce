// Clipping of gradients by their global norm (include/tag_optim.h): one pass over
// everything for the sum of squares, and one that scales.
//
// A table in device memory, laid out once for a plan, cuts the arrays into chunks
// of 16 KiB, so that thousands of tensors of any size take two launches.  Sums are
// in 64 bits: squares of fp32 values stay in their range, and the vector unit
// does them at the rate of fp32.
#include <algorithm>
#include <cmath>
#include <exception>
#include <string>
#include <vector>

#include "../../include/tag_optim.h"
#include "areas.hpp"
#include "tag_internal.hpp"

namespace tag {
namespace {

constexpr int kChunkBytes = 16384, kVec = 16;   // bytes of a chunk, of a thread's access
constexpr int kPieces = kChunkBytes / (256 * kVec);
constexpr int kBlocks = 2048;                   // blocks of a launch, and sums in the workspace
constexpr int kAhead = 4;                       // single elements in flight per thread
constexpr int kNarrow = 256 * kAhead;           // of narrow rows, a chunk is what a block has in flight at once
constexpr int kWideRow = 1024;                  // from so many columns on a row is chunks of its own

// elements of one array: n consecutive ones, or rows of `cols` (0: consecutive)
struct Chunk {
    const char *g;
    char *out;
    int64_t gs, os;       // row strides in elements
    int32_t n, cols;
    int32_t bf16;
    uint32_t per_col;     // floor(2^32 / cols) + 1, for e / cols of e <= 1,024 and 1 < cols < 1,024 by one product
    int32_t pad[4];
    __device__ __forceinline__ int row(int e) const { return cols > 1 ? (int)__umulhi((unsigned)e, per_col) : e; }
};
static_assert(sizeof(Chunk) == 64, "an entry to a cache line's half");

struct ClipArgs {
    const Chunk *table;
    int64_t chunks;
    int32_t sums, writes;
    double *part;
    double max_norm;
    float *result;
};

typedef unsigned vec __attribute__((ext_vector_type(4)));
typedef unsigned any_vec __attribute__((ext_vector_type(4), aligned(2)));   // 16 bytes at any element

template <typename T>
struct Wide;   // elements of 16 bytes
template <>
struct Wide<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float get(const vec &r, int i) { return __uint_as_float(r[i]); }
    static __device__ __forceinline__ vec put(const float (&v)[4]) {
        return vec{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
    static __device__ __forceinline__ float get1(float v) { return v; }
    static __device__ __forceinline__ float put1(float v) { return v; }
};
template <>
struct Wide<uint16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const vec &r, int i) {
        return __uint_as_float(i % 2 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
    }
    static __device__ __forceinline__ vec put(const float (&v)[8]) {
        return vec{pack_bf2(v[0], v[1]), pack_bf2(v[2], v[3]), pack_bf2(v[4], v[5]), pack_bf2(v[6], v[7])};
    }
    static __device__ __forceinline__ float get1(uint16_t v) { return bf2f(v); }
    static __device__ __forceinline__ uint16_t put1(float v) { return f2bf(v); }
};

// A thread's pieces of a chunk of consecutive elements, as far as they are whole (0
// beyond); of either type, so that they can be on their way before anything else of
// the chunk is looked at.
struct Pieces {
    vec v[kPieces];
    __device__ __forceinline__ void load(const Chunk &C) {
        const int bytes = C.cols ? 0 : C.bf16 ? 2 * C.n : 4 * C.n;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int at = (threadIdx.x + 256 * k) * kVec;
            v[k] = vec{0, 0, 0, 0};
            if (at + kVec <= bytes) v[k] = *reinterpret_cast<const any_vec *>(C.g + at);
        }
    }
};
// the elements behind a chunk's whole pieces: first and number
template <typename T>
__device__ __forceinline__ int rest(const Chunk &C) { return C.n / Wide<T>::N * Wide<T>::N; }

// sum of a value over the block's 256 threads, in a fixed order
__device__ __forceinline__ double block_sum(double s) {
    __shared__ double red[4];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const Chunk &C, const Pieces &P) {
    using W = Wide<T>;
    const T *g = reinterpret_cast<const T *>(C.g);
    double s = 0.0;
    if (C.cols == 0) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
#pragma unroll
            for (int i = 0; i < W::N; ++i) {
                const double x = W::get(P.v[k], i);
                s += x * x;
            }
        const int e = rest<T>(C) + threadIdx.x;
        if (e < C.n) {
            const double x = W::get1(g[e]);
            s += x * x;
        }
    } else {
        float v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int e = threadIdx.x + 256 * k, r = C.row(e);
            v[k] = e < C.n ? W::get1(g[r * C.gs + (e - r * C.cols)]) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) s += (double)v[k] * (double)v[k];
    }
    return s;
}

// Reads bound it: 435 MB in 97 us, 4.5 TB/s (70 where the last call's results went past
// the caches and left a part of them there).  A chunk's pieces are on their way
// while the one before is summed, its entry of the table one turn earlier (114 us
// without).  1,200 tensors of 27 MB 7.6 us: two round trips to a block (10.2 with narrow
// rows in chunks of 16 KiB, several turns of single elements each).
__global__ void __launch_bounds__(256, 6) clip_norm(ClipArgs A) {
    double s = 0.0;
    const int64_t step = gridDim.x;
    int64_t c = blockIdx.x;   // (a block has one)
    Chunk C = A.table[c], N = A.table[c + step < A.chunks ? c + step : c];
    Pieces P;
    P.load(C);
    for (; c < A.chunks; c += step) {
        const Chunk after = A.table[c + 2 * step < A.chunks ? c + 2 * step : c];
        Pieces Q;
        if (c + step < A.chunks) Q.load(N);
        s += C.bf16 ? chunk_squares<uint16_t>(C, P) : chunk_squares<float>(C, P);
        C = N;
        N = after;
        P = Q;
    }
    s = block_sum(s);
    if (threadIdx.x == 0) A.part[blockIdx.x] = s;
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const Chunk &C, const Pieces &P, float scale) {
    using W = Wide<T>;
    const T *g = reinterpret_cast<const T *>(C.g);
    T *out = reinterpret_cast<T *>(C.out);
    const bool drop = scale == 0.f;   // (0 times an infinity is not 0)
    auto scaled = [&](float x) { return drop ? 0.f : x * scale; };
    if (C.cols == 0) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            const int at = (threadIdx.x + 256 * k) * kVec;
            float v[W::N];
#pragma unroll
            for (int i = 0; i < W::N; ++i) v[i] = scaled(W::get(P.v[k], i));
            if (at + kVec <= C.n * (int)sizeof(T)) __builtin_nontemporal_store((any_vec)W::put(v), reinterpret_cast<any_vec *>(C.out + at));
        }
        const int e = rest<T>(C) + threadIdx.x;
        if (e < C.n) out[e] = W::put1(scaled(W::get1(g[e])));
    } else {
        float v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int e = threadIdx.x + 256 * k, r = C.row(e);
            v[k] = e < C.n ? W::get1(g[r * C.gs + (e - r * C.cols)]) : 0.f;
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            const int e = threadIdx.x + 256 * k, r = C.row(e);
            if (e < C.n) out[r * C.os + (e - r * C.cols)] = W::put1(scaled(v[k]));
        }
    }
}

// Every block forms the norm from the sums, in the same order, with its first chunk
// on its way.  The chunks go backwards: the last ones that clip_norm has read are
// still in the caches (435 MB in and out 146 us, 6.0 TB/s), and results leave by
// non-temporal stores, so that more of them stay there.
__global__ void __launch_bounds__(256, 5) clip_apply(ClipArgs A) {
    const int64_t step = gridDim.x;
    int64_t c = A.writes ? A.chunks - 1 - blockIdx.x : -1;
    Chunk C{}, N{};
    Pieces P;
    if (c >= 0) {
        C = A.table[c];
        N = A.table[c >= step ? c - step : c];
        P.load(C);
    }
    double p[kBlocks / 256], s = 0.0;
#pragma unroll
    for (int i = 0; i < kBlocks / 256; ++i) {
        const int at = threadIdx.x + 256 * i;
        p[i] = at < A.sums ? A.part[at] : 0.0;
    }
#pragma unroll
    for (int i = 0; i < kBlocks / 256; ++i) s += p[i];
    const double norm = sqrt(block_sum(s));
    const float rounded = (float)norm;
    const float scale = !(rounded < INFINITY) ? 0.f : norm > A.max_norm ? (float)(A.max_norm / norm) : 1.f;
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        A.result[0] = rounded;
        A.result[1] = scale;
    }
    if (A.writes == 2 && scale == 1.f) return;
    for (; c >= 0; c -= step) {
        const Chunk after = A.table[c >= 2 * step ? c - 2 * step : c];
        Pieces Q;
        if (c >= step) Q.load(N);
        if (C.out && !(scale == 1.f && C.out == C.g)) {
            if (C.bf16) chunk_scale<uint16_t>(C, P, scale);
            else chunk_scale<float>(C, P, scale);
        }
        C = N;
        N = after;
        P = Q;
    }
}

// ---------------------------------------------------------------------- host
constexpr int64_t kMaxChunks = 1 << 26;

bool is_wide(const tag_clip_array &a) { return a.cols >= kWideRow; }
// rows one after the other, in g and out: one run of elements
bool is_flat(const tag_clip_array &a) {
    return a.rows == 1 || (a.g_stride == a.cols && (!a.out || a.out_stride == a.cols));
}
int64_t chunk_elements(const tag_clip_array &a) { return kChunkBytes / (a.dtype == TAG_BF16 ? 2 : 4); }

int64_t chunks_of(const tag_clip_array &a) {
    if (a.rows == 0 || a.cols == 0) return 0;
    const int64_t per = chunk_elements(a);
    if (is_flat(a)) return (a.rows * a.cols + per - 1) / per;
    if (is_wide(a)) return a.rows * ((a.cols + per - 1) / per);
    const int64_t rows = kNarrow / a.cols;
    return (a.rows + rows - 1) / rows;
}

tag_status check_clip(const tag_clip_array *a, int32_t n, int64_t *chunks) {
    if (n < 0 || (n > 0 && !a)) TAG_FAIL(TAG_EINVAL, "need n_arrays >= 0 and arrays");
    std::vector<Area> in, out;
    std::vector<int32_t> of;   // array of each out
    *chunks = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (a[i].rows < 0 || a[i].cols < 0) TAG_FAIL(TAG_EINVAL, "need rows >= 0 and cols >= 0");
        if (a[i].dtype != TAG_F32 && a[i].dtype != TAG_BF16) TAG_FAIL(TAG_EINVAL, "dtype must be TAG_F32 or TAG_BF16");
        in.push_back(flat_area(nullptr, 0));
        if (a[i].rows == 0 || a[i].cols == 0) continue;
        const size_t el = a[i].dtype == TAG_BF16 ? 2 : 4;
        if (!a[i].g) TAG_FAIL(TAG_EINVAL, "g must be non-NULL");
        if ((uintptr_t)a[i].g % el || (uintptr_t)a[i].out % el) TAG_FAIL(TAG_EINVAL, "an array is not aligned to its elements");
        if (a[i].rows > (int64_t)1 << 44 || a[i].cols > ((int64_t)1 << 44) / a[i].rows)
            TAG_FAIL(TAG_ESHAPE, "at most 2^44 elements of an array");
        if (a[i].rows > 1 && (a[i].g_stride < a[i].cols || (a[i].out && a[i].out_stride < a[i].cols)))
            TAG_FAIL(TAG_EINVAL, "a row stride is below the number of columns");
        if (a[i].rows > 1 && std::max(a[i].g_stride, a[i].out ? a[i].out_stride : 0) > ((int64_t)1 << 58) / a[i].rows)
            TAG_FAIL(TAG_ESHAPE, "strides span at most 2^58 elements");
        *chunks += chunks_of(a[i]);
        if (*chunks > kMaxChunks) TAG_FAIL(TAG_ESHAPE, "at most 2^26 chunks of 16 KiB");
        in[i] = rows_area(a[i].g, a[i].rows, a[i].g_stride * (int64_t)el, a[i].cols * (int64_t)el);
        if (!a[i].out) continue;
        if (a[i].out == a[i].g && a[i].rows > 1 && a[i].g_stride != a[i].out_stride)
            TAG_FAIL(TAG_EINVAL, "out may be g only with its stride");
        out.push_back(rows_area(a[i].out, a[i].rows, a[i].out_stride * (int64_t)el, a[i].cols * (int64_t)el));
        of.push_back(i);
    }
    // by their starts, so that only spans that meet are looked at
    struct Item {
        Area area;
        int32_t array;
        bool written;
    };
    std::vector<Item> items;
    for (int32_t i = 0; i < n; ++i) items.push_back(Item{in[i], i, false});
    for (size_t o = 0; o < out.size(); ++o) items.push_back(Item{out[o], of[o], true});
    std::sort(items.begin(), items.end(), [](const Item &x, const Item &y) { return x.area.b < y.area.b; });
    for (size_t i = 0; i < items.size(); ++i)
        for (size_t j = i + 1; j < items.size() && items[j].area.b < items[i].area.e; ++j) {
            const Item &x = items[i], &y = items[j];
            if (!(x.written || y.written) || !x.area.meets(y.area)) continue;
            if (x.array == y.array && a[x.array].out == a[x.array].g) continue;
            TAG_FAIL(TAG_EINVAL, "out must be g, or not overlap any array");
        }
    return TAG_OK;
}

std::vector<Chunk> lay_out(const tag_clip_array *arrays, int32_t n, int64_t chunks, int32_t *writes) {
    std::vector<Chunk> t;
    t.reserve(chunks);
    for (int32_t i = 0; i < n; ++i) {
        const tag_clip_array &a = arrays[i];
        if (a.rows == 0 || a.cols == 0) continue;
        if (a.out) *writes = *writes == 1 || a.out != a.g ? 1 : 2;
        const int64_t el = a.dtype == TAG_BF16 ? 2 : 4, per = chunk_elements(a);
        Chunk c{};
        c.bf16 = a.dtype == TAG_BF16;
        auto put = [&](int64_t row, int64_t col, int64_t count) {
            c.g = static_cast<const char *>(a.g) + (row * a.g_stride + col) * el;
            c.out = a.out ? static_cast<char *>(a.out) + (row * a.out_stride + col) * el : nullptr;
            c.n = (int32_t)count;
            t.push_back(c);
        };
        if (is_flat(a)) {
            const int64_t total = a.rows * a.cols;
            for (int64_t e = 0; e < total; e += per) put(0, e, std::min(per, total - e));
        } else if (is_wide(a)) {
            for (int64_t r = 0; r < a.rows; ++r)
                for (int64_t e = 0; e < a.cols; e += per) put(r, e, std::min(per, a.cols - e));
        } else {
            const int64_t rows = kNarrow / a.cols;
            c.cols = (int32_t)a.cols;
            c.gs = a.g_stride;
            c.os = a.out_stride;
            c.per_col = (uint32_t)((1ull << 32) / (uint64_t)a.cols + 1);
            for (int64_t r = 0; r < a.rows; r += rows) put(r, 0, std::min(rows, a.rows - r) * a.cols);
        }
    }
    return t;
}

}  // namespace
}  // namespace tag

using namespace tag;

extern "C" tag_status tag_clip_table_bytes(const tag_clip_array *arrays, int32_t n_arrays, size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    try {
        int64_t chunks;
        const tag_status st = check_clip(arrays, n_arrays, &chunks);
        if (st != TAG_OK) return st;
        *bytes = (size_t)chunks * sizeof(Chunk);
    } catch (const std::exception &) {
        TAG_FAIL(TAG_ENOSPACE, "not enough host memory for the plan");
    }
    return TAG_OK;
}

extern "C" tag_status tag_clip_prepare(const tag_clip_array *arrays, int32_t n_arrays, void *table, size_t table_bytes,
                                       void *hip_stream, tag_clip_plan *plan) {
    clear_error();
    if (!plan) TAG_FAIL(TAG_EINVAL, "plan must be non-NULL");
    try {
        int64_t chunks;
        const tag_status st = check_clip(arrays, n_arrays, &chunks);
        if (st != TAG_OK) return st;
        if ((size_t)chunks * sizeof(Chunk) > table_bytes)
            TAG_FAIL(TAG_ENOSPACE, "table too small (see tag_clip_table_bytes)");
        if (chunks && (!table || (uintptr_t)table % 16)) TAG_FAIL(TAG_EINVAL, "table must be non-NULL and 16-byte aligned");
        int32_t writes = 0;
        const std::vector<Chunk> t = lay_out(arrays, n_arrays, chunks, &writes);
        hipStream_t stream = static_cast<hipStream_t>(hip_stream);
        if (chunks) {
            TAG_HIP_CHECK(hipMemcpyAsync(table, t.data(), t.size() * sizeof(Chunk), hipMemcpyHostToDevice, stream));
            TAG_HIP_CHECK(hipStreamSynchronize(stream));
        }
        *plan = tag_clip_plan{table, chunks, writes};
    } catch (const std::exception &) {
        TAG_FAIL(TAG_ENOSPACE, "not enough host memory for the plan");
    }
    return TAG_OK;
}

extern "C" tag_status tag_clip_workspace(size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    *bytes = kBlocks * sizeof(double);
    return TAG_OK;
}

extern "C" tag_status tag_clip(const tag_clip_plan *plan, double max_norm, float *result, void *workspace,
                               size_t ws_bytes, void *hip_stream) {
    clear_error();
    if (!plan || !result) TAG_FAIL(TAG_EINVAL, "plan and result must be non-NULL");
    if (plan->chunks < 0 || plan->chunks > kMaxChunks || (plan->chunks && !plan->table) || plan->writes < 0 || plan->writes > 2)
        TAG_FAIL(TAG_EINVAL, "plan is not one of tag_clip_prepare");
    if (!(max_norm >= 0.0)) TAG_FAIL(TAG_EINVAL, "max_norm must be >= 0");
    if ((uintptr_t)result % 4) TAG_FAIL(TAG_EINVAL, "result is not aligned to its elements");
    if (ws_bytes < kBlocks * sizeof(double)) TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_clip_workspace)");
    if (!workspace || (uintptr_t)workspace % 16) TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    ClipArgs A{};
    A.table = static_cast<const Chunk *>(plan->table); A.chunks = plan->chunks;
    A.sums = (int32_t)std::min<int64_t>(plan->chunks, kBlocks); A.writes = plan->writes;
    A.part = static_cast<double *>(workspace);
    A.max_norm = max_norm; A.result = result;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (A.sums) clip_norm<<<A.sums, 256, 0, stream>>>(A);
    clip_apply<<<plan->writes ? std::max(A.sums, 1) : 1, 256, 0, stream>>>(A);
    return launch_status("tag_clip");
}
