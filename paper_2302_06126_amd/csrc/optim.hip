// Orthogonalised optimiser step (include/tag_optim.h): Newton-Schulz products on
// the matrix cores, around them the momentum and the update.
//
// A step of the iteration is three products of n x n by K: A = X X^T, A A and
// B X (n <= m; 2 n^2 m + 2 n^3 + 2 n^2 m flops, the first two symmetric, so
// half of their tiles are computed and written twice).  The 15 products of five
// steps depend on one another, so each is one launch over all matrices of all
// groups, and its epilogue forms the next operand: nothing but products runs in
// between.
//
// Operands.  Every matrix of the iteration has entries of magnitude <= 3.5 (X),
// 12.25 (A) or 15 (B) (checked on the host for the coefficients), so it is held
// as 2^12 times its value in two fp16 parts, hi = fp16(x) and lo = fp16(x - hi):
// each rounding leaves at most 2^-11 of what it rounds, so the pair holds x to
// 2^-22 of it (2^-24.7 root mean square; fp32's own rounding 2^-25.4).  A product
// is hi hi' + hi lo' + lo hi' (what is left out, lo lo', is below 2^-22 of it,
// 2^-24.8 root mean square): three fp16 matrix instructions instead of the six
// that exact bf16 splits need, or of fp32 ones at a sixteenth of the rate.
//
// bf16 matrices take the same products, and their result is rounded once.  With
// one part of the operands (2^-11 of them) the products of 4 of 1024 x 4096 take
// 670 us in place of 1,215, but the operands then cost about as much as that rounding,
// and where their roundings agree, as in a matrix of equal values, ten times as much.
//
// Layout.  The operands lie in the order in which a 32x32x16 instruction takes
// them ("fragments": 32 rows x 16 k, lane l holds 8 consecutive k of row l % 32,
// k / 8 % 2 = l / 32; 1 KiB), fragment (r, k) of a plane at (r kf + k) KiB, so a
// tile's k-step is a few contiguous runs, goes from memory into LDS by direct
// loads, and every LDS access is lane-linear (no bank conflicts).  Rows and
// columns are padded with zeros to multiples of 64.  X is kept in both orders
// (X for A, X^T for B X): a lane of the accumulators holds four consecutive rows
// of a column, which is the operand order of the transpose; the other order goes
// through LDS.
#include <algorithm>
#include <cmath>
#include <string>

#include "../../include/tag_optim.h"
#include "agg_common.hpp"

namespace tag {
namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef float f16v __attribute__((ext_vector_type(16)));

constexpr float kScale = 4096.f, kInvScale = 1.f / 4096.f;
constexpr int kFrag = 512;          // elements of a fragment
constexpr int kSumChunk = 4096;     // elements per sum-of-squares block
// Groups of one set of launches.  Their tables are kernel arguments, which a
// launch copies and every block reads from afar: small ones start sooner (15
// launches of 2.4 KB tables cost 25 us more than of 300 bytes).
constexpr int kSet = 8, kSetPlain = 16;

struct Arr {
    void *p;
    int64_t row, mat;
};

// a group on the host
struct Group {
    int32_t count, rows, cols;
    int32_t n, m, np, mp;        // n <= m, padded to multiples of 64
    bool trans, plain;           // rows > cols; no iteration
    int32_t chunks;              // sum-of-squares blocks per matrix
    Arr in, out, mom;            // in / out, or g / w and the momentum
    uint16_t *ops;               // operands of the group's matrices
    int64_t ops_stride;          // elements per matrix
    double *part;                // [count][chunks]
    float factor;                // of O(u) in the update
};

// what the kernels read of it; first: the group's first block (past the grid for groups that there are not)
struct NormGroup {
    Arr in, out, mom;
    double *part;
    int32_t rows, cols, chunks, first;
    int32_t plain, flat;         // flat: four consecutive elements of every array as one access
};
struct NormSet {
    NormGroup g[kSet + kSetPlain];
    int32_t n_groups;
    float lr, momentum, decay;
    int32_t nesterov;
};
struct PrepGroup {
    Arr in, mom;
    const double *part;
    uint16_t *ops;
    int64_t ops_stride;
    int32_t rows, cols, np, mp, chunks, first, flat;
};
struct PrepSet {
    PrepGroup g[kSet];
    float eps, momentum;
    int32_t nesterov;
};
struct ProductGroup {
    uint16_t *ops;
    int64_t ops_stride;
    int32_t np, mp, first;
};
struct ProductSet {
    ProductGroup g[kSet];
    float a, b, c;
    int32_t cur;                 // which of the two X buffers is read
};
struct EndGroup {
    Arr out;
    int32_t rows, cols;
    float factor;
};
struct SmallGroup {
    Arr in, out, mom;
    int32_t rows, cols, mp, first;
    float factor;
};
struct SmallSet {
    SmallGroup g[kSet];
    float a, b, c, eps;
    int32_t steps;
    float lr, momentum, decay;
    int32_t nesterov;
};
struct EndSet : ProductSet {     // of the last product
    EndGroup e[kSet];
    float lr, decay;
};

// operands of a matrix: X and X^T of both buffers (hi, lo planes), A, B
template <typename G>
__device__ __forceinline__ uint16_t *x_plane(const G &g, int mat, int buf, int t, int plane) {
    return g.ops + mat * g.ops_stride + (int64_t)(buf * 4 + t * 2 + plane) * g.np * g.mp;
}
template <typename G>
__device__ __forceinline__ uint16_t *s_plane(const G &g, int mat, int which, int plane) {
    return g.ops + mat * g.ops_stride + (int64_t)8 * g.np * g.mp + (int64_t)(which * 2 + plane) * g.np * g.np;
}

// group of a block (uniform selects among a few, all read at once)
template <int N, typename G>
__device__ __forceinline__ int find_group(const G (&g)[N], int n, int32_t &bid) {
    int at = 0, first = 0;
#pragma unroll
    for (int i = 1; i < N; ++i) {
        const bool in = i < n && bid >= g[i].first;
        at = in ? i : at;
        first = in ? g[i].first : first;
    }
    bid -= first;
    return at;
}

// two parts of 2^12 x
__device__ __forceinline__ void split2(float x0, float x1, unsigned &hi, unsigned &lo) {
    const h2 h = h2{(_Float16)x0, (_Float16)x1};
    const h2 l = h2{(_Float16)(x0 - (float)h.x), (_Float16)(x1 - (float)h.y)};
    hi = __builtin_bit_cast(unsigned, h);
    lo = __builtin_bit_cast(unsigned, l);
}
__device__ __forceinline__ float join2(unsigned hi, unsigned lo, int i) {
    const h2 h = __builtin_bit_cast(h2, hi), l = __builtin_bit_cast(h2, lo);
    return (float)h[i] + (float)l[i];
}

template <typename T>
__device__ __forceinline__ float get(const T *p);
template <>
__device__ __forceinline__ float get<float>(const float *p) { return *p; }
template <>
__device__ __forceinline__ float get<uint16_t>(const uint16_t *p) { return bf2f(*p); }

// ------------------------------------------------------- momentum and norms
// four consecutive elements
__device__ __forceinline__ float4 get4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 get4(const uint16_t *p) {
    const uint2 r = *reinterpret_cast<const uint2 *>(p);
    return float4{__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xffff0000u), __uint_as_float(r.y << 16),
                  __uint_as_float(r.y & 0xffff0000u)};
}

// Sums of squares of u per kSumChunk elements (in 64 bits: a gradient's squares
// leave the range of fp32), with the momentum update on the way; plain groups
// are finished here.  Memory bounds whole chunks: 2048 x 2048 fp32 5.7 us (2.9 TB/s,
// a launch and its tail).  The last chunk of a matrix or vector goes element by
// element, up to 16 turns of a thread with a memory round trip each: 1.7 M parameters
// of the 256-wide model, whose vectors and encoders end so, 12.2 us.
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) ns_norm(NormSet B) {
    __shared__ double red[4];
    int32_t bid = blockIdx.x;
    const NormGroup &G = B.g[find_group(B.g, B.n_groups, bid)];
    const int mat = bid / G.chunks, chunk = bid % G.chunks;
    const T *in = static_cast<const T *>(G.in.p) + mat * G.in.mat;
    float *mom = MUON ? static_cast<float *>(G.mom.p) + mat * G.mom.mat : nullptr;
    float *w = MUON && G.plain ? static_cast<float *>(G.out.p) + mat * G.out.mat : nullptr;
    const float keep = 1.f - B.lr * B.decay;
    // the momentum and u of one element, or the whole step of a plain one
    auto step = [&](float g, float &m, float &wt) {
        m = fmaf(B.momentum, m, g);
        const float u = B.nesterov ? fmaf(B.momentum, m, g) : m;
        wt = keep * wt - B.lr * u;
        return u;
    };
    double s = 0.0;
    const int64_t total = (int64_t)G.rows * G.cols, e0 = (int64_t)chunk * kSumChunk;
    constexpr int NV = kSumChunk / 1024;
    if (G.flat && e0 + kSumChunk <= total) {
        float4 g[NV], m[NV] = {}, v[NV] = {};
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t e = e0 + 4 * (threadIdx.x + 256 * k);
            g[k] = get4(in + e);
            if (MUON) m[k] = get4(mom + e);
            if (MUON && w) v[k] = get4(w + e);
        }
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t e = e0 + 4 * (threadIdx.x + 256 * k);
            if (MUON) {
                g[k].x = step(g[k].x, m[k].x, v[k].x); g[k].y = step(g[k].y, m[k].y, v[k].y);
                g[k].z = step(g[k].z, m[k].z, v[k].z); g[k].w = step(g[k].w, m[k].w, v[k].w);
                *reinterpret_cast<float4 *>(mom + e) = m[k];
                if (w) *reinterpret_cast<float4 *>(w + e) = v[k];
            }
            s += (double)g[k].x * g[k].x + (double)g[k].y * g[k].y + ((double)g[k].z * g[k].z + (double)g[k].w * g[k].w);
        }
    } else {
        const int64_t e1 = total < e0 + kSumChunk ? total : e0 + kSumChunk;
#pragma unroll 4
        for (int64_t e = e0 + threadIdx.x; e < e1; e += 256) {
            int64_t r = 0, c = e;
            if (G.rows > 1) {
                r = (uint32_t)e / (uint32_t)G.cols;   // (at most 2^31 elements)
                c = e - r * G.cols;
            }
            float u = get(in + r * G.in.row + c);
            if (MUON) {
                float *mp = mom + r * G.mom.row + c, m = *mp, wt = w ? w[r * G.out.row + c] : 0.f;
                u = step(u, m, wt);
                *mp = m;
                if (w) w[r * G.out.row + c] = wt;
            }
            s += (double)u * (double)u;
        }
    }
    if (MUON && w) return;
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) G.part[(int64_t)mat * G.chunks + chunk] = red[0] + red[1] + red[2] + red[3];
}

// X and X^T of the first buffer: one block per 64 x 64 tile of the padded
// matrix (as it is stored), through LDS.  Memory bounds it: 2048 x 2048 fp32 12.6
// us (17 MB read, 34 MB written).
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) ns_prepare(PrepSet B) {
    __shared__ float tile[64][65];
    __shared__ double red[4];
    int32_t bid = blockIdx.x;
    const PrepGroup &G = B.g[find_group(B.g, kSet, bid)];
    const bool trans = G.rows > G.cols;
    const int tr = (trans ? G.mp : G.np) / 64, tc = (trans ? G.np : G.mp) / 64;   // tiles down and along
    const int mat = bid / (tr * tc), t = bid % (tr * tc), r0 = t / tc * 64, c0 = t % tc * 64;
    const T *in = static_cast<const T *>(G.in.p) + mat * G.in.mat;
    const float *mom = MUON ? static_cast<const float *>(G.mom.p) + mat * G.mom.mat : nullptr;
    // 16 threads to a row of the tile, four columns each
    const int a = threadIdx.x >> 4, b = (threadIdx.x & 15) * 4;
    float u[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = r0 + a + 16 * k, c = c0 + b;
        const T *p = in + (int64_t)r * G.in.row + c;
        const float *q = MUON ? mom + (int64_t)r * G.mom.row + c : nullptr;
        float m[4] = {0.f, 0.f, 0.f, 0.f};
        if (G.flat && r < G.rows && c + 4 <= G.cols) {
            const float4 x = get4(p);
            u[k][0] = x.x; u[k][1] = x.y; u[k][2] = x.z; u[k][3] = x.w;
            if (MUON) {
                const float4 y = get4(q);
                m[0] = y.x; m[1] = y.y; m[2] = y.z; m[3] = y.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool is = r < G.rows && c + i < G.cols;
                u[k][i] = is ? get(p + i) : 0.f;
                if (MUON) m[i] = is ? q[i] : 0.f;
            }
        }
        if (MUON)
#pragma unroll
            for (int i = 0; i < 4; ++i) u[k][i] = B.nesterov ? fmaf(B.momentum, m[i], u[k][i]) : m[i];
    }
    double s = 0.0;
    for (int c = threadIdx.x; c < G.chunks; c += 256) s += G.part[(int64_t)mat * G.chunks + c];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    const double norm = sqrt(red[0] + red[1] + red[2] + red[3]);
    const double scale = (double)kScale / (norm + (double)B.eps);
    const bool bad = !(norm < INFINITY);
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            tile[a + 16 * k][b + i] = bad && r0 + a + 16 * k < G.rows && c0 + b + i < G.cols ? __builtin_nanf("")
                                                                                            : (float)((double)u[k][i] * scale);
    __syncthreads();
    // 16-byte pieces: 64 rows x 8 chunks of 8 k, for the stored order and its transpose
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int side = q >> 1, r = threadIdx.x & 63, ch = (threadIdx.x >> 6) + 4 * (q & 1);
        u4v hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = 8 * ch + 2 * e;
            unsigned h, l;
            if (side) split2(tile[k][r], tile[k + 1][r], h, l);
            else split2(tile[r][k], tile[r][k + 1], h, l);
            hi[e] = h;
            lo[e] = l;
        }
        const int row = (side ? c0 : r0) + r, k = (side ? r0 : c0) + 8 * ch;
        const bool xt = (side != 0) != trans;   // X has its n <= m rows
        const int kf = (xt ? G.np : G.mp) / 16;
        const int64_t at = ((int64_t)(row / 32) * kf + k / 16) * kFrag + (row % 32 + 32 * (k / 8 % 2)) * 8;
        *reinterpret_cast<u4v *>(x_plane(G, mat, 0, xt, 0) + at) = hi;
        *reinterpret_cast<u4v *>(x_plane(G, mat, 0, xt, 1) + at) = lo;
    }
}

// ------------------------------------------------------------------ products
enum { kGram = 0, kSquare = 1, kApply = 2, kFinal = 3, kUpdate = 4 };

// A barrier of the block at which each wavefront has waited for its own direct
// loads but the last N, and for its LDS reads: LDS that they have filled may be
// read, LDS that was read may be filled.  (The compiler's own barrier waits for
// every load in flight.)
template <int N>
__device__ __forceinline__ void wait_arrival() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// C = R S^T over one tile of T x T outputs per block, R and S operand planes of
// K/16 fragments per row, three part products a step.  Eight wavefronts: four
// cover the tile (T/2 x T/2 each) for the even fragments of k, four for the odd
// ones.  Stages of KF fragments of k go through a ring of NB LDS buffers by direct
// loads, up to NB stages ahead of the products (a stage's products take less time
// than a load from beyond the L2), and a stage's fragments are read from LDS while
// the last stage's are multiplied.
//
// 2048^3: B X 55 us (256 tiles, 940 TFLOP/s of fp16 products; a library's
// bf16 product of 2048^3 reaches 418, of 8192^3 1,164), of which 43 us of products
// at the 1.6 GHz that the chip then holds, 70% of their peak at it; X X^T and A A
// 44 to 45 us (136 tiles, half of the CUs, a higher clock).  Around the products a launch
// takes 2 us to the first load, 1 until it lands, 2 to join the halves of k, 4 to write
// 34 MB.  Four of 1024 x 4096: B X 124 us (830 TFLOP/s, blocks of 32 stages), X X^T 82
// (144 tiles).  Tried without gain: two stages of twice the length instead of four,
// stages' barriers by the compiler (which waits for every load), one wavefront per
// SIMD (the products wait for LDS: 60 us).
//
// The matrix cores round their sums towards minus infinity, a bias that grows
// with the number of steps where rounding errors grow with its root; the odd
// fragments are taken with one operand negated and subtracted at the end, so the
// two biases cancel.
template <int MODE>
struct SetOf { typedef ProductSet type; };
template <>
struct SetOf<kFinal> { typedef EndSet type; };
template <>
struct SetOf<kUpdate> { typedef EndSet type; };

template <int T, int MODE, typename OUT>
__global__ void __launch_bounds__(512, T == 64 ? 4 : 2) ns_product(typename SetOf<MODE>::type B) {
    constexpr int F = T / 32, W = F / 2, KF = 2, NB = 4;   // (the last stages: cases up to 4)
    constexpr int kStage = 4 * F * KF, L = kStage / 8;   // fragments of a stage, and each wavefront's share
    constexpr bool SYM = MODE == kGram || MODE == kSquare;
    __shared__ __attribute__((aligned(1024))) unsigned char sh[NB * kStage * 1024];
    int32_t bid = (int32_t)xcd_swizzle(blockIdx.x, gridDim.x);
    const int group = find_group(B.g, kSet, bid);
    ProductGroup G = B.g[0];
#pragma unroll
    for (int i = 1; i < kSet; ++i)
        if (group == i) G = B.g[i];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) & 7;
    const int kg = wave >> 2, wi = (wave >> 1) & 1, wj = wave & 1;
    const int nt = (G.np + T - 1) / T, mt = (G.mp + T - 1) / T, tiles = SYM ? nt * (nt + 1) / 2 : nt * mt;
    const int mat = bid / tiles, t = bid - mat * tiles;
    int I, J;
    if (SYM) {   // I <= J, in the order of J
        J = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        while (J * (J + 1) / 2 > t) --J;
        while ((J + 1) * (J + 2) / 2 <= t) ++J;
        I = t - J * (J + 1) / 2;
    } else {     // strips of eight rows of tiles
        const int strip = nt <= 8 ? 0 : t / (8 * mt), h = min(8, nt - 8 * strip), r = t - strip * 8 * mt;
        J = h == 8 ? r >> 3 : r / h;
        I = 8 * strip + r - J * h;
    }
    const int K = MODE == kGram ? G.mp : G.np, nk = K / 16;
    const int rfR = G.np / 32, rfS = (SYM ? G.np : G.mp) / 32;   // row fragments of R and S
    // the wavefront's fragments of a stage, as pointers to its lanes' 16 bytes
    const uint16_t *src[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        // (plain shifts of wave, and constants where its eight fragments are of one kind)
        const int side = i / (L / 2), f = wave + 8 * (i % (L / 2));
        const int plane = F * KF == 8 ? i % (L / 2) : f / (F * KF), rf = f % (F * KF) / KF, kf = f % KF;
        const uint16_t *p;
        if (MODE == kGram) p = x_plane(G, mat, B.cur, 0, plane);
        else if (MODE == kSquare) p = s_plane(G, mat, 0, plane);
        else p = side ? x_plane(G, mat, B.cur, 1, plane) : s_plane(G, mat, 1, plane);
        // (row fragments past the matrix: the last one again, its products unused)
        const int row = min((side ? J : I) * F + rf, (side ? rfS : rfR) - 1);
        src[i] = p + ((int64_t)row * nk + kf) * kFrag + lane * 8;
    }
    // (the tile as it leaves: below)
    constexpr int P = T + 4, NQ = T * T / 8 / 512, TK = T / 16;
    static_assert(T * P * 4 <= NB * kStage * 1024, "the ring holds the tile");
    const int prow = (threadIdx.x & 31), pk = 8 * (lane >> 5);   // of a piece, within its fragment
    auto load = [&](int buf) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            load_lds<16>(src[i], sh + (buf * kStage + wave + 8 * i) * 1024);
            src[i] += KF * kFrag;
        }
    };
    // (one block of accumulators per wavefront: a set for each part product, since consecutive products into one set
    // wait for one another)
    constexpr int NA = W == 2 ? 1 : 3, NK = KF / 2;
    f16v acc[W][W], more[NA];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
#pragma unroll
        for (int i = 0; i < W * W; ++i) acc[i / W][i % W][e] = 0.f;
#pragma unroll
        for (int i = 0; i < NA; ++i) more[i][e] = 0.f;
    }
    const unsigned neg = kg ? 0x80008000u : 0u;
    const int stages = nk / KF;
    struct Frags {
        h8 a[NK][W][2], b[NK][W][2];
    };
    auto fetch = [&](int s, Frags &f) {
        const u4v *fr = reinterpret_cast<const u4v *>(sh + (s % NB) * kStage * 1024);
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int p = 0; p < 2; ++p) {
                    const int kf = 2 * k + kg;
                    f.a[k][i][p] = __builtin_bit_cast(h8, fr[((p * F + wi * W + i) * KF + kf) * 64 + lane]);
                    f.b[k][i][p] = __builtin_bit_cast(h8, fr[(((2 + p) * F + wj * W + i) * KF + kf) * 64 + lane]);
                }
    };
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            h8 a[W][2];
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int p = 0; p < 2; ++p)
                    a[i][p] = __builtin_bit_cast(h8, __builtin_bit_cast(u4v, f.a[k][i][p]) ^ neg);
            auto product = [&](f16v &d, int i, int j, int pa, int pb) {
                d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][pa], f.b[k][j][pb], d, 0, 0, 0);
            };
            if constexpr (W == 1) {
                product(more[1], 0, 0, 1, 0);
                product(more[2], 0, 0, 0, 1);
                product(more[0], 0, 0, 0, 0);
            } else {
#pragma unroll
                for (int q = 0; q < 3; ++q)
#pragma unroll
                    for (int ij = 0; ij < 4; ++ij)
                        product(acc[ij / 2][ij % 2], ij / 2, ij % 2, q == 0, q == 1);
            }
        }
    };
#pragma unroll
    for (int s = 0; s < NB; ++s)
        if (s < stages) load(s);
    // While more stages are to be loaded than the ring holds: stage s + 1 has landed for every wavefront (later ones
    // stay in flight), and every wavefront's reads of stage s are done, so its buffer takes stage s + NB.
    auto turn_ring = [&](int s, const Frags &now, Frags &next) {
        wait_arrival<(NB - 2) * L>();
        fetch(s + 1, next);
        load(s % NB);
        multiply(now);
        // the reads go out first, the direct loads between the products
        constexpr int NM = (W == 2 ? 4 : 1) * NK * 3, M1 = NM / (L + 1);
        static_assert(L == 2 || L == 4, "two or four direct loads");
        __builtin_amdgcn_sched_group_barrier(0x100, 4 * NK * W, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, M1, 0);
        __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x8, M1, 0);
        __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
        if constexpr (L == 4) {
            __builtin_amdgcn_sched_group_barrier(0x8, M1, 0);
            __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, M1, 0);
            __builtin_amdgcn_sched_group_barrier(0x20, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, NM - L * M1, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    Frags f0, f1;
    int s = 0;
    if (stages > NB) {
        wait_arrival<(NB - 1) * L>();
        fetch(0, f0);
        for (int pairs = (stages - NB) / 2; pairs > 0; --pairs) {
            turn_ring(s, f0, f1);
            turn_ring(s + 1, f1, f0);
            s += 2;
        }
        if (s + NB < stages) {
            turn_ring(s, f0, f1);
            f0 = f1;
            ++s;
        }
        wait_arrival<0>();
    } else {
        wait_arrival<0>();
        fetch(0, f0);
    }
    // the last stages are all there
    switch (stages - s) {
        case 1: multiply(f0); break;
        case 2: fetch(s + 1, f1); multiply(f0); multiply(f1); break;
        case 3: fetch(s + 1, f1); multiply(f0); fetch(s + 2, f0); multiply(f1); multiply(f0); break;
        default: fetch(s + 1, f1); multiply(f0); fetch(s + 2, f0); multiply(f1); fetch(s + 3, f1); multiply(f0); multiply(f1);
    }
    if constexpr (W == 1) {
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[0][0][e] = more[0][e] + (more[1][e] + more[2][e]);
    }
    // What is left goes over the tile in LDS, by pieces of eight consecutive k of a row of the next operand: 64
    // threads to a fragment.  First in the order of S's rows (the transpose of the tile), with the term of the
    // iteration itself (c A A + b A, B X + a X), whose operand has that order too and is asked for now.
    float *tile = reinterpret_cast<float *>(sh);
    uint16_t *to[2][2];   // operand written in S's order, in R's; hi, lo
    const uint16_t *was[2] = {nullptr, nullptr};
#pragma unroll
    for (int pl = 0; pl < 2; ++pl) {
        if (SYM) to[0][pl] = to[1][pl] = s_plane(G, mat, MODE == kSquare, pl);
        else { to[0][pl] = x_plane(G, mat, 1 - B.cur, 1, pl); to[1][pl] = x_plane(G, mat, 1 - B.cur, 0, pl); }
        if (MODE != kGram) was[pl] = MODE == kSquare ? s_plane(G, mat, 0, pl) : x_plane(G, mat, B.cur, 1, pl);
    }
    auto piece = [&](int q, int &rf, int &kf) {                   // the fragment of a thread's piece
        const int f = wave + 8 * q;
        rf = f / TK;
        kf = f % TK;
    };
    u4v old[NQ][2];
    if (MODE != kGram) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            int rf, kf;
            piece(q, rf, kf);
            if (J * F + rf < rfS && I * TK + kf < G.np / 16) {
                const int64_t at = ((int64_t)(J * F + rf) * (G.np / 16) + I * TK + kf) * kFrag + lane * 8;
                old[q][0] = *reinterpret_cast<const u4v *>(was[0] + at);
                old[q][1] = *reinterpret_cast<const u4v *>(was[1] + at);
            }
        }
    }
    // the two halves of k meet in the tile: a wavefront puts down the blocks that its counterpart finishes (T = 64:
    // the odd ones put down theirs).  Lane l of a 32 x 32 block holds column l % 32, rows 8 (e / 4) + 4 (l / 32) + e % 4
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");   // the fragments' LDS is free
    auto cell = [&](int i, int j, int e) -> float & {
        return tile[((wi * W + i) * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * P + (wj * W + j) * 32 + (lane & 31)];
    };
    if (W == 2 || kg == 1) {
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) cell(W == 2 ? 1 - kg : 0, j, e) = W == 2 && !kg ? acc[W - 1][j][e] : acc[0][j][e];
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (W == 2 || kg == 0) {
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float &c = cell(W == 2 ? kg : 0, j, e);
                const float o = c, v = W == 2 && kg ? acc[W - 1][j][e] : acc[0][j][e];
                c = (kg ? o - v : v - o) * kInvScale;
            }
    }
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    constexpr bool LAST = MODE == kFinal || MODE == kUpdate;
    auto store = [&](uint16_t *const (&d)[2], int64_t at, const float (&v)[8]) {
        u4v hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            unsigned h, l;
            split2(v[2 * e], v[2 * e + 1], h, l);
            hi[e] = h;
            lo[e] = l;
        }
        *reinterpret_cast<u4v *>(d[0] + at) = hi;
        *reinterpret_cast<u4v *>(d[1] + at) = lo;
    };
    {
        const float cv = MODE == kSquare ? B.c : 1.f, ct = MODE == kSquare ? B.b : B.a;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            int rf, kf;
            piece(q, rf, kf);
            if (J * F + rf >= rfS || I * TK + kf >= G.np / 16) continue;
            float *c = tile + (kf * 16 + pk) * P + rf * 32 + prow, v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = c[e * P];
                if (MODE != kGram) {
                    v[e] = fmaf(ct, join2(old[q][0][e / 2], old[q][1][e / 2], e % 2), cv * v[e]);
                    c[e * P] = v[e];
                }
            }
            if (!LAST) store(to[0], ((int64_t)(J * F + rf) * (G.np / 16) + I * TK + kf) * kFrag + lane * 8, v);
        }
        if (MODE != kGram) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    }
    if (!LAST) {
        if (SYM && I == J) return;   // (its own transpose)
        const int nkR = (SYM ? G.np : G.mp) / 16;
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
            int rf, kf;
            piece(q, rf, kf);
            if (I * F + rf >= rfR || J * TK + kf >= nkR) continue;
            const float *c = tile + (rf * 32 + prow) * P + kf * 16 + pk;
            const float4 x = *reinterpret_cast<const float4 *>(c), y = *reinterpret_cast<const float4 *>(c + 4);
            const float v[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
            store(to[1], ((int64_t)(I * F + rf) * nkR + J * TK + kf) * kFrag + lane * 8, v);
        }
        return;
    }
    // rows of the result as it is stored: consecutive threads along them
    if constexpr (LAST) {
        const EndGroup &E = B.e[group];
        const bool trans = E.rows > E.cols;
        OUT *out = static_cast<OUT *>(E.out.p) + mat * E.out.mat;
        const int64_t r0 = (int64_t)(trans ? J : I) * T, c0 = (int64_t)(trans ? I : J) * T;
        const int sr = trans ? 1 : P, sc = trans ? P : 1;
        const float keep = 1.f - B.lr * B.decay, rate = B.lr * E.factor;
#pragma unroll 4
        for (int e = threadIdx.x; e < T * T; e += 512) {
            const int r = e / T, c = e % T;
            if (r0 + r >= E.rows || c0 + c >= E.cols) continue;
            OUT *p = out + (r0 + r) * E.out.row + c0 + c;
            const float o = tile[r * sr + c * sc] * kInvScale;
            if constexpr (MODE == kUpdate) *p = keep * *p - rate * o;
            else if constexpr (sizeof(OUT) == 2) *p = f2bf(o);
            else *p = o;
        }
    }
}

// ------------------------------------------------------------- small matrices
// A matrix of at most 64 by 64 MB: everything in one block, the operands in LDS,
// one launch instead of 17 (a 64 x 42 matrix: 68 -> 18 us).  Few products, many waits: 16x16x32 instructions
// (fragments of 16 rows x 32 k, lane l holds 8 consecutive k of row l % 16, k / 8
// % 4 = l / 16), so that eight wavefronts share the smallest matrix and a block
// has four values a lane.  What is read is held in registers until every
// wavefront is through with it, then written over.
struct Sums {   // of fragments of even and of odd k (one operand negated), of the main and the cross products
    f4 m[2], x[2];
    __device__ __forceinline__ Sums() { m[0] = m[1] = x[0] = x[1] = f4{0.f, 0.f, 0.f, 0.f}; }
    __device__ __forceinline__ void add(const h8 (&a)[2], const h8 (&b)[2], int odd) {
        x[odd] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[1], b[0], x[odd], 0, 0, 0);
        m[odd] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0], b[0], m[odd], 0, 0, 0);
        x[odd] = __builtin_amdgcn_mfma_f32_16x16x32_f16(a[0], b[1], x[odd], 0, 0, 0);
    }
    __device__ __forceinline__ f4 total() const { return ((m[0] - m[1]) + (x[0] - x[1])) * kInvScale; }
};

template <typename T, bool MUON, int MB>
__global__ void __launch_bounds__(512) ns_small(SmallSet B) {
    constexpr int kX = 64 * 64 * MB, kA = 64 * 64;   // elements of a plane
    __shared__ __attribute__((aligned(1024))) uint16_t X[2 * kX], XT[2 * kX], S[2 * kA];
    __shared__ double red[8];
    int32_t bid = blockIdx.x;
    const SmallGroup &G = B.g[find_group(B.g, kSet, bid)];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, quad = lane >> 4, col = lane & 15;
    const bool trans = G.rows > G.cols;
    const int n = trans ? G.cols : G.rows, m = trans ? G.rows : G.cols, kx = G.mp / 32;   // fragments along a row of X
    const T *in = static_cast<const T *>(G.in.p) + bid * G.in.mat;
    float *mom = MUON ? static_cast<float *>(G.mom.p) + bid * G.mom.mat : nullptr;
    // pieces of eight consecutive j of a row i, 64 threads to a fragment
    float u[MB][8];
    double s = 0.0;
#pragma unroll
    for (int q = 0; q < MB; ++q) {
        const int f = wave + 8 * q, i = f / kx * 16 + col, j0 = f % kx * 32 + 8 * quad;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = j0 + e;
            u[q][e] = 0.f;
            if (f < 4 * kx && i < n && j < m) {
                const int64_t r = trans ? j : i, c = trans ? i : j;
                float g = get(in + r * G.in.row + c);
                if (MUON) {
                    float *mp = mom + r * G.mom.row + c;
                    const float v = fmaf(B.momentum, *mp, g);
                    *mp = v;
                    g = B.nesterov ? fmaf(B.momentum, v, g) : v;
                }
                u[q][e] = g;
                s += (double)g * (double)g;
            }
        }
    }
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) red[wave] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int w = 0; w < 8; ++w) s += red[w];
    const double norm = sqrt(s), scale = (double)kScale / (norm + (double)B.eps);
    const bool bad = !(norm < INFINITY);
#pragma unroll
    for (int q = 0; q < MB; ++q) {
        const int f = wave + 8 * q;
        if (f >= 4 * kx) continue;
        u4v hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float x0 = (float)((double)u[q][2 * e] * scale), x1 = (float)((double)u[q][2 * e + 1] * scale);
            if (bad) x0 = x1 = __builtin_nanf("");   // (the padding too: nothing finite is left of such a matrix)
            unsigned h, l;
            split2(x0, x1, h, l);
            hi[e] = h;
            lo[e] = l;
        }
        *reinterpret_cast<u4v *>(X + f * kFrag + lane * 8) = hi;
        *reinterpret_cast<u4v *>(X + kX + f * kFrag + lane * 8) = lo;
    }
    __syncthreads();
    // X^T: pieces of eight consecutive i of a row j
#pragma unroll
    for (int q = 0; q < MB; ++q) {
        const int f = wave + 8 * q, j = f / 2 * 16 + col, i0 = f % 2 * 32 + 8 * quad;
        if (f >= 4 * kx) continue;
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            u4v v;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = i0 + e;
                const unsigned x = X[p * kX + (i / 16 * kx + j / 32) * kFrag + (i % 16 + 16 * (j / 8 % 4)) * 8 + j % 8];
                v[e / 2] = e % 2 ? v[e / 2] | x << 16 : x;
            }
            *reinterpret_cast<u4v *>(XT + p * kX + f * kFrag + lane * 8) = v;
        }
    }
    __syncthreads();
    // Lane l of a 16 x 16 block holds column l % 16, rows 4 (l / 16) + 0 .. 3: four consecutive k of a row of the
    // transpose, half of one of its pieces.  rf: that row's fragment, kb: the block's 16 k.
    auto at = [&](int rf, int kb, int nk) {
        const int k = kb * 16 + 4 * quad;
        return (rf * nk + k / 32) * kFrag + (col + 16 * (k / 8 % 4)) * 8 + k % 8;
    };
    auto put = [&](uint16_t *d, int plane, int o, f4 v) {
        uint2 h, l;
        split2(v[0], v[1], h.x, l.x);
        split2(v[2], v[3], h.y, l.y);
        *reinterpret_cast<uint2 *>(d + o) = h;
        *reinterpret_cast<uint2 *>(d + plane + o) = l;
    };
    auto here = [&](const uint16_t *d, int plane, int o) {   // what stands at a block's place
        const uint2 h = *reinterpret_cast<const uint2 *>(d + o), l = *reinterpret_cast<const uint2 *>(d + plane + o);
        return f4{join2(h.x, l.x, 0), join2(h.x, l.x, 1), join2(h.y, l.y, 0), join2(h.y, l.y, 1)};
    };
    auto frag = [&](const uint16_t *d, int plane, int f, h8 (&v)[2]) {
        v[0] = *reinterpret_cast<const h8 *>(d + f * kFrag + lane * 8);
        v[1] = *reinterpret_cast<const h8 *>(d + plane + f * kFrag + lane * 8);
    };
    auto negated = [&](h8 (&v)[2]) {
        v[0] = __builtin_bit_cast(h8, __builtin_bit_cast(u4v, v[0]) ^ 0x80008000u);
        v[1] = __builtin_bit_cast(h8, __builtin_bit_cast(u4v, v[1]) ^ 0x80008000u);
    };
    const int bi = wave >> 1, bj = wave & 1;   // rows of blocks, and the wavefront's blocks in it: bj, bj + 2, ..
    // C = R R^T of 64 x 64, R of nk fragments a row
    auto square = [&](const uint16_t *d, int plane, int nk, f4 (&v)[2]) {
        Sums c[2];
        for (int k = 0; k < nk; k += 2) {
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
                h8 a[2], b[2][2];
                frag(d, plane, bi * nk + k + odd, a);
                frag(d, plane, bj * nk + k + odd, b[0]);
                frag(d, plane, (bj + 2) * nk + k + odd, b[1]);
                if (odd) negated(a);
                c[0].add(a, b[0], odd);
                c[1].add(a, b[1], odd);
            }
        }
        v[0] = c[0].total();
        v[1] = c[1].total();
    };
    for (int step = 0; step < B.steps; ++step) {
        const bool last = step + 1 == B.steps;
        f4 v[2];
        square(X, kX, kx, v);   // A = X X^T, every block of it (the two orders of one off the diagonal are two blocks)
        put(S, kA, at(bj, bi, 2), v[0]);
        put(S, kA, at(bj + 2, bi, 2), v[1]);
        __syncthreads();
        square(S, kA, 2, v);    // B = c A A + b A
#pragma unroll
        for (int q = 0; q < 2; ++q) v[q] = B.c * v[q] + B.b * here(S, kA, at(bj + 2 * q, bi, 2));
        __syncthreads();
        put(S, kA, at(bj, bi, 2), v[0]);
        put(S, kA, at(bj + 2, bi, 2), v[1]);
        __syncthreads();
        // a X + B X in both orders: rows bi of X, columns bj, bj + 2, ..
        h8 r[2][2], rn[2];
        frag(S, kA, bi * 2, r[0]);
        frag(S, kA, bi * 2 + 1, r[1]);
        rn[0] = r[1][0];
        rn[1] = r[1][1];
        negated(rn);
        f4 vt[2 * MB], vx[2 * MB];
#pragma unroll
        for (int q = 0; q < 2 * MB; ++q) {
            const int j = bj + 2 * q;
            if (j >= 2 * kx) continue;
            h8 x[2][2];
            frag(XT, kX, j * 2, x[0]);
            frag(XT, kX, j * 2 + 1, x[1]);
            Sums t, o;
            t.add(r[0], x[0], 0);
            t.add(rn, x[1], 1);
            vt[q] = t.total() + B.a * here(XT, kX, at(j, bi, 2));
            if (last) continue;
            o.add(x[0], r[0], 0);
            o.add(x[1], rn, 1);
            vx[q] = o.total() + B.a * here(X, kX, at(bi, j, kx));
        }
        __syncthreads();
        if (!last) {
#pragma unroll
            for (int q = 0; q < 2 * MB; ++q) {
                const int j = bj + 2 * q;
                if (j >= 2 * kx) continue;
                put(XT, kX, at(j, bi, 2), vt[q]);
                put(X, kX, at(bi, j, kx), vx[q]);
            }
            __syncthreads();
            continue;
        }
        T *out = static_cast<T *>(G.out.p) + bid * G.out.mat;
        const float keep = 1.f - B.lr * B.decay, rate = B.lr * G.factor;
#pragma unroll
        for (int q = 0; q < 2 * MB; ++q) {
            const int gj = (bj + 2 * q) * 16 + col;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int gi = bi * 16 + 4 * quad + e;
                if (gi >= n || gj >= m) continue;
                T *p = out + (trans ? gj : gi) * G.out.row + (trans ? gi : gj);
                const float o = vt[q][e] * kInvScale;
                if constexpr (MUON) *p = keep * *p - rate * o;
                else if constexpr (sizeof(T) == 2) *p = f2bf(o);
                else *p = o;
            }
        }
    }
}

// ---------------------------------------------------------------------- host
int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

// workspace of one set of matrix groups, and the pointers into it
size_t carve_ns(Group *g, int32_t n, void *base) {
    Carver c(base);
    for (int i = 0; i < n; ++i) {
        Group &G = g[i];
        G.part = c.take<double>((size_t)G.count * G.chunks);
        G.ops_stride = 8ll * G.np * G.mp + 4ll * G.np * G.np;
        G.ops = c.take<uint16_t>((size_t)G.count * G.ops_stride);
    }
    return c.used;
}

Group shape_ns(int32_t count, int32_t rows, int32_t cols, bool plain) {
    Group G{};
    G.count = count; G.rows = rows; G.cols = cols; G.plain = plain;
    G.trans = rows > cols;
    G.n = std::min(rows, cols); G.m = std::max(rows, cols);
    if (!plain) { G.np = (int32_t)up64(G.n); G.mp = (int32_t)up64(G.m); }
    G.chunks = (int32_t)(((int64_t)rows * cols + kSumChunk - 1) / kSumChunk);
    return G;
}

constexpr int kMaxSide = 32768;   // rows or columns

tag_status check_shape(int32_t count, int32_t rows, int32_t cols, bool plain) {
    if (count < 1 || rows < 1 || cols < 1) TAG_FAIL(TAG_EINVAL, "need count, rows and cols >= 1");
    if (!plain && (rows > kMaxSide || cols > kMaxSide)) TAG_FAIL(TAG_ESHAPE, "at most 32768 rows or columns");
    // (a launch has fewer than 2^32 threads, over all groups of its set; plain groups have no tiles)
    const int64_t chunks = ((int64_t)rows * cols + kSumChunk - 1) / kSumChunk;
    const int64_t blocks = plain ? chunks : std::max((up64(rows) / 64) * (up64(cols) / 64), chunks);
    if (blocks > (1 << 19) / count) TAG_FAIL(TAG_ESHAPE, "too many or too large matrices in a group");
    return TAG_OK;
}

tag_status check_array(const tag_matrices &a, int32_t count, int32_t rows, int32_t cols, size_t el, bool written,
                       const char *what) {
    if (!a.base) TAG_FAIL(TAG_EINVAL, std::string(what) + " must be non-NULL");
    if ((uintptr_t)a.base % el) TAG_FAIL(TAG_EINVAL, std::string(what) + " must be aligned to its elements");
    if ((rows > 1 && a.row_stride < cols) || (count > 1 && a.matrix_stride < 0))
        TAG_FAIL(TAG_EINVAL, std::string(what) + ": a row stride is below the number of columns, or a stride negative");
    if (!written || count == 1) return TAG_OK;
    const int64_t span = (rows - 1) * (rows > 1 ? a.row_stride : 0) + cols;
    const bool apart = a.matrix_stride >= span;
    const bool woven = a.matrix_stride >= cols && (rows == 1 || a.row_stride >= (count - 1) * a.matrix_stride + cols);
    if (!apart && !woven) TAG_FAIL(TAG_EINVAL, std::string(what) + ": its matrices overlap");
    return TAG_OK;
}

// whether two arrays of one shape are the same one, element by element
bool same_place(const tag_matrices &a, const tag_matrices &b, int32_t count, int32_t rows) {
    return a.base == b.base && (rows == 1 || a.row_stride == b.row_stride) &&
           (count == 1 || a.matrix_stride == b.matrix_stride);
}

// Whether they share an element: exact where their strides are the same (parts of
// wider rows, say, which interleave); for others only whether both start at one.
bool overlap(const tag_matrices &a, const tag_matrices &b, int32_t count, int32_t rows, int32_t cols, size_t el) {
    if (a.base == b.base) return true;
    if ((rows > 1 && a.row_stride != b.row_stride) || (count > 1 && a.matrix_stride != b.matrix_stride)) return false;
    const int64_t bytes = (int64_t)((uintptr_t)b.base - (uintptr_t)a.base), row = rows > 1 ? a.row_stride : 0,
                  mat = count > 1 ? a.matrix_stride : 0;
    const int64_t d = bytes / (int64_t)el;   // (arrays are aligned to their elements)
    if (std::abs(d) >= (count - 1) * mat + (rows - 1) * row + cols) return false;
    // d = i mat + j row + k with |i| < count, |j| < rows, |k| < cols
    for (int64_t i = 1 - count; i < count; ++i) {
        const int64_t r = d - i * mat;
        const int64_t j = row > 0 ? std::min<int64_t>(std::max<int64_t>(r / row, 1 - rows), rows - 1) : 0;
        for (int64_t t = std::max<int64_t>(j - 1, 1 - rows); t <= std::min<int64_t>(j + 1, rows - 1); ++t)
            if (std::abs(r - t * row) < cols) return true;
    }
    return false;
}

// the largest |p| over [0, hi] of p(s) = s (a + b s^2 + c s^4), or with `poly` of
// b t + c t^2 over t in [0, hi^2]: at the ends and where the derivative is zero
double peak(double a, double b, double c, double hi, bool poly) {
    double best = 0.0;
    auto at = [&](double t) {
        if (!(t >= 0.0 && t <= hi * hi)) return;
        const double v = poly ? b * t + c * t * t : std::sqrt(t) * (a + b * t + c * t * t);
        best = std::max(best, std::fabs(v));
    };
    at(hi * hi);
    if (poly) {
        if (c != 0.0) at(-b / (2.0 * c));
    } else if (c != 0.0) {   // a + 3 b t + 5 c t^2 = 0
        const double d = 9.0 * b * b - 20.0 * a * c;
        if (d >= 0.0) {
            at((-3.0 * b + std::sqrt(d)) / (10.0 * c));
            at((-3.0 * b - std::sqrt(d)) / (10.0 * c));
        }
    } else if (b != 0.0) {
        at(-a / (3.0 * b));
    }
    return best;
}

tag_status check_ns(const tag_newton_schulz *ns) {
    if (!ns) TAG_FAIL(TAG_EINVAL, "the iteration must be non-NULL");
    if (ns->steps < 1 || ns->steps > 32) TAG_FAIL(TAG_EINVAL, "steps must be in [1, 32]");
    if (!(ns->eps > 0.f) || !std::isfinite(ns->eps)) TAG_FAIL(TAG_EINVAL, "eps must be positive and finite");
    if (!std::isfinite(ns->a) || !std::isfinite(ns->b) || !std::isfinite(ns->c))
        TAG_FAIL(TAG_EINVAL, "coefficients must be finite");
    double hi = 1.0;
    for (int i = 0; i < ns->steps; ++i) {
        if (peak(ns->a, ns->b, ns->c, hi, true) > 15.0)
            TAG_FAIL(TAG_EINVAL, "coefficients let an eigenvalue of B leave [-15, 15]");
        hi = peak(ns->a, ns->b, ns->c, hi, false);
        if (hi > 3.5) TAG_FAIL(TAG_EINVAL, "coefficients let a singular value leave [0, 3.5]");
    }
    return TAG_OK;
}

struct Options {
    tag_newton_schulz ns;
    tag_muon_options muon;
};

// block numbers of a kernel's groups: n of them, the rest past the grid
template <typename G, typename Blocks>
unsigned number_blocks(G *g, int32_t n, int32_t room, Blocks blocks) {
    int64_t first = 0;
    for (int i = 0; i < room; ++i) {
        g[i].first = i < n ? (int32_t)first : INT32_MAX;
        if (i < n) first += blocks(i);
    }
    return (unsigned)first;
}

bool quads(const Arr &a, size_t el, bool flat, int64_t cols) {   // rows of four-element pieces
    return (uintptr_t)a.p % (4 * el) == 0 && a.mat % 4 == 0 && (flat ? a.row == cols : a.row % 4 == 0);
}

int64_t product_tiles(const Group &G, int T, int mode) {
    const int64_t nt = (G.np + T - 1) / T, mt = (G.mp + T - 1) / T;
    return G.count * (mode == kGram || mode == kSquare ? nt * (nt + 1) / 2 : nt * mt);
}

template <int T, typename OUT>
void launch_product(const Group *g, int32_t n, EndSet &B, int mode, hipStream_t st) {
    const unsigned grid = number_blocks(B.g, n, kSet, [&](int i) { return product_tiles(g[i], T, mode); });
    const ProductSet &P = B;
    switch (mode) {
        case kGram: ns_product<T, kGram, float><<<grid, 512, 0, st>>>(P); break;
        case kSquare: ns_product<T, kSquare, float><<<grid, 512, 0, st>>>(P); break;
        case kApply: ns_product<T, kApply, float><<<grid, 512, 0, st>>>(P); break;
        case kFinal: ns_product<T, kFinal, OUT><<<grid, 512, 0, st>>>(B); break;
        default:
            if constexpr (sizeof(OUT) == 4) ns_product<T, kUpdate, float><<<grid, 512, 0, st>>>(B);
    }
}

// One set: at most kSet matrix groups (already carved) and kSetPlain plain ones.
template <typename T, bool MUON>
void run_set(const Group *mats, int32_t n, const Group *plain, int32_t n_plain, const Options &o, hipStream_t st) {
    NormSet N{};
    N.lr = o.muon.lr; N.momentum = o.muon.momentum; N.decay = o.muon.weight_decay; N.nesterov = o.muon.nesterov != 0;
    // matrices of at most 64 x 256 alone: one launch for all of them
    int32_t wide = 0;
    for (int i = 0; i < n; ++i) wide = std::max(wide, mats[i].np > 64 ? INT32_MAX : mats[i].mp);
    const bool small = n > 0 && wide <= 256;
    const int32_t norms = small ? 0 : n;   // groups that go the way of many launches
    N.n_groups = norms + n_plain;
    for (int i = 0; i < N.n_groups; ++i) {
        const Group &G = i < norms ? mats[i] : plain[i - norms];
        NormGroup &K = N.g[i];
        K.in = G.in; K.out = G.out; K.mom = G.mom; K.part = G.part;
        K.rows = G.rows; K.cols = G.cols; K.chunks = G.chunks; K.plain = G.plain;
        // (rows one after the other: the elements of a matrix are consecutive)
        auto flat = [&](const Arr &a, size_t el) { return quads(G.rows > 1 ? a : Arr{a.p, G.cols, a.mat}, el, true, G.cols); };
        K.flat = flat(G.in, sizeof(T)) && (!MUON || (flat(G.mom, 4) && (!G.plain || flat(G.out, 4))));
    }
    if (small) {
        SmallSet S{};
        S.a = o.ns.a; S.b = o.ns.b; S.c = o.ns.c; S.eps = o.ns.eps; S.steps = o.ns.steps;
        S.lr = N.lr; S.momentum = N.momentum; S.decay = N.decay; S.nesterov = N.nesterov;
        for (int i = 0; i < n; ++i) {
            const Group &G = mats[i];
            SmallGroup &K = S.g[i];
            K.in = G.in; K.out = G.out; K.mom = G.mom;
            K.rows = G.rows; K.cols = G.cols; K.mp = G.mp; K.factor = G.factor;
        }
        const unsigned blocks = number_blocks(S.g, n, kSet, [&](int i) { return (int64_t)mats[i].count; });
        if (wide <= 128) ns_small<T, MUON, 2><<<blocks, 512, 0, st>>>(S);
        else ns_small<T, MUON, 4><<<blocks, 512, 0, st>>>(S);
        if (n_plain == 0) return;
    }
    unsigned grid = number_blocks(N.g, N.n_groups, kSet + kSetPlain, [&](int i) {
        const Group &G = i < norms ? mats[i] : plain[i - norms];
        return (int64_t)G.count * G.chunks;
    });
    ns_norm<T, MUON><<<grid, 256, 0, st>>>(N);
    if (norms == 0) return;
    PrepSet P{};
    P.eps = o.ns.eps; P.momentum = N.momentum; P.nesterov = N.nesterov;
    EndSet E{};
    E.a = o.ns.a; E.b = o.ns.b; E.c = o.ns.c; E.lr = o.muon.lr; E.decay = o.muon.weight_decay;
    for (int i = 0; i < n; ++i) {
        const Group &G = mats[i];
        PrepGroup &K = P.g[i];
        K.in = G.in; K.mom = G.mom; K.part = G.part; K.ops = G.ops; K.ops_stride = G.ops_stride;
        K.rows = G.rows; K.cols = G.cols; K.np = G.np; K.mp = G.mp; K.chunks = G.chunks;
        K.flat = quads(G.in, sizeof(T), false, G.cols) && (!MUON || quads(G.mom, 4, false, G.cols));
        E.g[i].ops = G.ops; E.g[i].ops_stride = G.ops_stride; E.g[i].np = G.np; E.g[i].mp = G.mp;
        E.e[i].out = G.out; E.e[i].rows = G.rows; E.e[i].cols = G.cols; E.e[i].factor = G.factor;
    }
    grid = number_blocks(P.g, n, kSet, [&](int i) { return (int64_t)mats[i].count * (mats[i].np / 64) * (mats[i].mp / 64); });
    ns_prepare<T, MUON><<<grid, 256, 0, st>>>(P);
    // Tiles of 128 x 128 once more than half of the CUs get one, else of 64 x 64.  Always the smaller | from 64 of the
    // larger ones | above 128, us, fp32 (the larger take fewer bytes per product, the smaller spread further): 2 of
    // 1024 x 1024 281 | 372 | 281, 8 of 512 x 512 195 | 255 | 195, 40 of 256 x 256 178 | 207 | 175, 1500 x 1500 416 |
    // 488 | 412, 2048 x 2048 755 | 703 | 704.
    auto product = [&](int mode) {
        int64_t tiles = 0;
        for (int i = 0; i < n; ++i) tiles += product_tiles(mats[i], 128, mode);
        if (tiles > 128) launch_product<128, T>(mats, n, E, mode, st);
        else launch_product<64, T>(mats, n, E, mode, st);
    };
    for (int s = 0; s < o.ns.steps; ++s) {
        E.cur = s & 1;
        product(kGram);
        product(kSquare);
        product(s + 1 < o.ns.steps ? kApply : MUON ? kUpdate : kFinal);
    }
}

Arr arr(const tag_matrices &a, int32_t count) { return Arr{a.base, a.row_stride, count > 1 ? a.matrix_stride : 0}; }

Group group_of(const tag_ortho_group &g) {
    Group G = shape_ns(g.count, g.rows, g.cols, false);
    G.in = arr(g.in, g.count);
    G.out = arr(g.out, g.count);
    return G;
}

Group group_of(const tag_muon_group &g) {
    Group G = shape_ns(g.count, g.rows, g.cols, g.plain != 0);
    G.in = arr(g.g, g.count);
    G.out = arr(g.w, g.count);
    G.mom = arr(g.m, g.count);
    G.factor = (float)std::sqrt(std::max(1.0, (double)g.rows / g.cols));
    return G;
}

// Goes over the groups by sets, which run one after the other in the same
// workspace: each(matrix groups, plain groups).
template <typename G, typename Each>
void for_sets(const G *g, int32_t n, Each each) {
    int32_t im = 0, ip = 0;   // next group to be looked at for either
    while (im < n || ip < n) {
        Group mats[kSet], plain[kSetPlain];
        int32_t nm = 0, np = 0;
        for (; im < n && nm < kSet; ++im) {
            mats[nm] = group_of(g[im]);
            nm += !mats[nm].plain;
        }
        for (; ip < n && np < kSetPlain; ++ip) {
            plain[np] = group_of(g[ip]);
            np += plain[np].plain;
        }
        if (nm || np) each(mats, nm, plain, np);
    }
}

template <typename G>
size_t workspace_of(const G *g, int32_t n) {
    size_t most = 0;
    for_sets(g, n, [&](Group *mats, int32_t nm, const Group *, int32_t) { most = std::max(most, carve_ns(mats, nm, nullptr)); });
    return most;
}

template <typename T, bool MUON, typename G>
void run_groups(const G *g, int32_t n, const Options &o, void *workspace, hipStream_t st) {
    for_sets(g, n, [&](Group *mats, int32_t nm, const Group *plain, int32_t np) {
        carve_ns(mats, nm, workspace);
        run_set<T, MUON>(mats, nm, plain, np, o, st);
    });
}

tag_status check_ortho_groups(const tag_ortho_group *g, int32_t n, bool arrays, size_t el) {
    if (!g || n < 1) TAG_FAIL(TAG_EINVAL, "need at least one group");
    for (int32_t i = 0; i < n; ++i) {
        tag_status st = check_shape(g[i].count, g[i].rows, g[i].cols, false);
        if (st == TAG_OK && arrays) st = check_array(g[i].in, g[i].count, g[i].rows, g[i].cols, el, false, "in");
        if (st == TAG_OK && arrays) st = check_array(g[i].out, g[i].count, g[i].rows, g[i].cols, el, true, "out");
        if (st != TAG_OK) return st;
        if (arrays && !same_place(g[i].in, g[i].out, g[i].count, g[i].rows) &&
            overlap(g[i].in, g[i].out, g[i].count, g[i].rows, g[i].cols, el))
            TAG_FAIL(TAG_EINVAL, "out must be in, matrix by matrix and row by row, or not overlap it");
    }
    return TAG_OK;
}

tag_status check_muon_groups(const tag_muon_group *g, int32_t n, bool arrays) {
    if (!g || n < 1) TAG_FAIL(TAG_EINVAL, "need at least one group");
    for (int32_t i = 0; i < n; ++i) {
        tag_status st = check_shape(g[i].count, g[i].rows, g[i].cols, g[i].plain != 0);
        if (st == TAG_OK && arrays) st = check_array(g[i].g, g[i].count, g[i].rows, g[i].cols, 4, false, "g");
        if (st == TAG_OK && arrays) st = check_array(g[i].w, g[i].count, g[i].rows, g[i].cols, 4, true, "w");
        if (st == TAG_OK && arrays) st = check_array(g[i].m, g[i].count, g[i].rows, g[i].cols, 4, true, "m");
        if (st != TAG_OK) return st;
        auto meet = [&](const tag_matrices &a, const tag_matrices &b) {
            return overlap(a, b, g[i].count, g[i].rows, g[i].cols, 4);
        };
        if (arrays && (meet(g[i].w, g[i].g) || meet(g[i].w, g[i].m) || meet(g[i].g, g[i].m)))
            TAG_FAIL(TAG_EINVAL, "w, g and m must be different arrays");
    }
    return TAG_OK;
}

}  // namespace
}  // namespace tag

using namespace tag;

extern "C" tag_status tag_orthogonalise_workspace(const tag_ortho_group *groups, int32_t n_groups, size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    const tag_status st = check_ortho_groups(groups, n_groups, false, 4);
    if (st != TAG_OK) return st;
    *bytes = workspace_of(groups, n_groups);
    return TAG_OK;
}

extern "C" tag_status tag_orthogonalise(const tag_ortho_group *groups, int32_t n_groups, int32_t dtype,
                                        const tag_newton_schulz *ns, void *workspace, size_t ws_bytes,
                                        void *hip_stream) {
    clear_error();
    if (dtype != TAG_F32 && dtype != TAG_BF16) TAG_FAIL(TAG_EINVAL, "dtype must be TAG_F32 or TAG_BF16");
    tag_status st = check_ortho_groups(groups, n_groups, true, dtype == TAG_BF16 ? 2 : 4);
    if (st == TAG_OK) st = check_ns(ns);
    if (st != TAG_OK) return st;
    if (workspace_of(groups, n_groups) > ws_bytes)
        TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_orthogonalise_workspace)");
    if (!workspace || (uintptr_t)workspace % 16) TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const Options o{*ns, {}};
    if (dtype == TAG_BF16) run_groups<uint16_t, false>(groups, n_groups, o, workspace, stream);
    else run_groups<float, false>(groups, n_groups, o, workspace, stream);
    return launch_status("tag_orthogonalise");
}

extern "C" tag_status tag_muon_workspace(const tag_muon_group *groups, int32_t n_groups, size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    const tag_status st = check_muon_groups(groups, n_groups, false);
    if (st != TAG_OK) return st;
    *bytes = workspace_of(groups, n_groups);
    return TAG_OK;
}

extern "C" tag_status tag_muon_step(const tag_muon_group *groups, int32_t n_groups, const tag_newton_schulz *ns,
                                    const tag_muon_options *options, void *workspace, size_t ws_bytes,
                                    void *hip_stream) {
    clear_error();
    tag_status st = check_muon_groups(groups, n_groups, true);
    if (st == TAG_OK) st = check_ns(ns);
    if (st != TAG_OK) return st;
    if (!options) TAG_FAIL(TAG_EINVAL, "options must be non-NULL");
    if (!(options->lr >= 0.f) || !std::isfinite(options->lr)) TAG_FAIL(TAG_EINVAL, "lr must be finite and >= 0");
    if (!(options->momentum >= 0.f && options->momentum < 1.f)) TAG_FAIL(TAG_EINVAL, "momentum must be in [0, 1)");
    if (!(options->weight_decay >= 0.f) || !std::isfinite(options->weight_decay))
        TAG_FAIL(TAG_EINVAL, "weight_decay must be finite and >= 0");
    const size_t need = workspace_of(groups, n_groups);
    if (need > ws_bytes) TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_muon_workspace)");
    if (need && (!workspace || (uintptr_t)workspace % 16))
        TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    run_groups<float, true>(groups, n_groups, Options{*ns, *options}, workspace, static_cast<hipStream_t>(hip_stream));
    return launch_status("tag_muon_step");
}
