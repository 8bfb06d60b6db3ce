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
// that exact bf16 splits need, or of fp32 ones at a sixteenth of the rate.  bf16 matrices take hi hi' alone; X keeps both parts, since the
// a X term carries its error through every step.
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
constexpr int kMaxGroups = 16;      // groups of one set of launches
constexpr int kFrag = 512;          // elements of a fragment
constexpr int kSumChunk = 8192;     // elements per sum-of-squares block

struct Arr {
    void *p;
    int64_t row, mat;
};

struct NsGroup {
    int32_t count, rows, cols;
    int32_t n, m, np, mp;        // n <= m, padded to multiples of 64
    int32_t trans;               // rows > cols
    int32_t plain;
    int32_t chunks;              // sum-of-squares blocks per matrix
    Arr in, out, mom;            // in / out, or g / w and the momentum
    uint16_t *ops;               // operands of the group's matrices
    int64_t ops_stride;          // elements per matrix
    double *part;                // [count][chunks]
    float factor;                // of O(u) in the update
};

struct NsBatch {
    NsGroup g[kMaxGroups];
    int32_t first[kMaxGroups + 1];   // first block of each group
    int32_t n_groups;
    float a, b, c, eps;
    int32_t cur;                 // which of the two X buffers is read
    // update
    float lr, momentum, decay;
    int32_t nesterov;
};

// operands of a matrix: X and X^T of both buffers (hi, lo planes), A, B
__device__ __forceinline__ uint16_t *x_plane(const NsGroup &G, int mat, int buf, int t, int plane) {
    return G.ops + mat * G.ops_stride + (int64_t)(buf * 4 + t * 2 + plane) * G.np * G.mp;
}
__device__ __forceinline__ uint16_t *s_plane(const NsGroup &G, int mat, int which, int plane) {
    return G.ops + mat * G.ops_stride + (int64_t)8 * G.np * G.mp + (int64_t)(which * 2 + plane) * G.np * G.np;
}

// group of a block, and the block's number within it
__device__ __forceinline__ int find_group(const NsBatch &B, int32_t &bid) {
    int g = 0;
    while (g + 1 < B.n_groups && bid >= B.first[g + 1]) ++g;
    bid -= B.first[g];
    return g;
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
// Sums of squares of u per kSumChunk elements (in 64 bits: a gradient's squares
// leave the range of fp32), with the momentum update on the way; plain groups
// are finished here.
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) ns_norm(NsBatch B) {
    __shared__ double red[4];
    int32_t bid = blockIdx.x;
    const NsGroup &G = B.g[find_group(B, bid)];
    const int mat = bid / G.chunks, chunk = bid % G.chunks;
    const int64_t total = (int64_t)G.rows * G.cols, e0 = (int64_t)chunk * kSumChunk;
    const int64_t e1 = total < e0 + kSumChunk ? total : e0 + kSumChunk;
    const T *in = static_cast<const T *>(G.in.p) + mat * G.in.mat;
    float *mom = MUON ? static_cast<float *>(G.mom.p) + mat * G.mom.mat : nullptr;
    double s = 0.0;
#pragma unroll 4
    for (int64_t e = e0 + threadIdx.x; e < e1; e += 256) {
        const int64_t r = e / G.cols, c = e - r * G.cols;
        float u = get(in + r * G.in.row + c);
        if (MUON) {
            float *mp = mom + r * G.mom.row + c;
            const float m = B.momentum * *mp + u;
            *mp = m;
            u = B.nesterov ? fmaf(B.momentum, m, u) : m;
            if (G.plain) {
                float *w = static_cast<float *>(G.out.p) + mat * G.out.mat + r * G.out.row + c;
                *w = (1.f - B.lr * B.decay) * *w - B.lr * u;
            }
        }
        s += (double)u * (double)u;
    }
    if (MUON && G.plain) return;
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) G.part[(int64_t)mat * G.chunks + chunk] = red[0] + red[1] + red[2] + red[3];
}

// X and X^T of the first buffer: one block per 64 x 64 tile of the padded
// matrix, through LDS.
template <typename T, bool MUON>
__global__ void __launch_bounds__(256) ns_prepare(NsBatch B) {
    __shared__ float tile[64][65];   // [row of X][column]
    __shared__ double red[4];
    int32_t bid = blockIdx.x;
    const NsGroup &G = B.g[find_group(B, bid)];
    const int ti = G.np / 64, tj = G.mp / 64, mat = bid / (ti * tj), t = bid % (ti * tj), i0 = t / tj * 64, j0 = t % tj * 64;
    double s = 0.0;
    for (int c = threadIdx.x; c < G.chunks; c += 256) s += G.part[(int64_t)mat * G.chunks + c];
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    const double norm = sqrt(red[0] + red[1] + red[2] + red[3]);
    const double scale = (double)kScale / (norm + (double)B.eps);
    const bool bad = !(norm < INFINITY);
    const T *in = static_cast<const T *>(G.in.p) + mat * G.in.mat;
    const float *mom = MUON ? static_cast<const float *>(G.mom.p) + mat * G.mom.mat : nullptr;
    const int a = threadIdx.x & 63;
    for (int b = threadIdx.x >> 6; b < 64; b += 4) {
        // consecutive threads along the rows of the matrix as it is stored
        const int li = G.trans ? a : b, lj = G.trans ? b : a, i = i0 + li, j = j0 + lj;
        float x = 0.f;
        if (i < G.n && j < G.m) {
            const int64_t r = G.trans ? j : i, c = G.trans ? i : j;
            float u = get(in + r * G.in.row + c);
            if (MUON) {
                const float m = mom[r * G.mom.row + c];
                u = B.nesterov ? fmaf(B.momentum, m, u) : m;
            }
            x = bad ? __builtin_nanf("") : (float)((double)u * scale);
        }
        tile[li][lj] = x;
    }
    __syncthreads();
    // 16-byte pieces: 64 rows x 8 chunks of 8 k, for X then X^T
    for (int p = threadIdx.x; p < 1024; p += 256) {
        const int tr = p >> 9, r = p & 63, ch = (p >> 6) & 7;
        u4v hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int k = 8 * ch + 2 * e;
            unsigned h, l;
            if (tr) split2(tile[k][r], tile[k + 1][r], h, l);
            else split2(tile[r][k], tile[r][k + 1], h, l);
            hi[e] = h;
            lo[e] = l;
        }
        const int row = (tr ? j0 : i0) + r, k = (tr ? i0 : j0) + 8 * ch, kf = (tr ? G.np : G.mp) / 16;
        const int64_t at = ((int64_t)(row / 32) * kf + k / 16) * kFrag + (row % 32 + 32 * (k / 8 % 2)) * 8;
        *reinterpret_cast<u4v *>(x_plane(G, mat, 0, tr, 0) + at) = hi;
        *reinterpret_cast<u4v *>(x_plane(G, mat, 0, tr, 1) + at) = lo;
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
// K/16 fragments per row.  PARTS = 2: three part products a step, PARTS = 1: the
// hi planes alone.  Eight wavefronts: four cover the tile (T/2 x T/2 each) for
// the even fragments of k, four for the odd ones.  Stages of KF fragments of k go
// through a ring of NB LDS buffers by direct loads, up to NB stages ahead of the
// products (a stage's products take less time than a load from beyond the L2),
// and a stage's fragments are read from LDS while the last stage's are
// multiplied.
//
// The matrix cores round their sums towards minus infinity, a bias that grows
// with the number of steps where rounding errors grow with its root; the odd
// fragments are taken with one operand negated and subtracted at the end, so the
// two biases cancel.
template <int T, int PARTS, int MODE, typename OUT>
__global__ void __launch_bounds__(512) ns_product(NsBatch B) {
    constexpr int F = T / 32, W = F / 2, KF = PARTS == 2 ? 2 : 4, NB = 4;   // (the last stages: cases up to 4)
    constexpr int kStage = 2 * F * PARTS * KF, L = kStage / 8;   // fragments of a stage, and each wavefront's share
    constexpr bool SYM = MODE == kGram || MODE == kSquare;
    __shared__ __attribute__((aligned(1024))) unsigned char sh[NB * kStage * 1024];
    int32_t bid = (int32_t)xcd_swizzle(blockIdx.x, gridDim.x);
    const NsGroup &G = B.g[find_group(B, bid)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kg = wave >> 2, wi = (wave >> 1) & 1, wj = wave & 1;
    const int nt = (G.np + T - 1) / T, mt = (G.mp + T - 1) / T, tiles = SYM ? nt * (nt + 1) / 2 : nt * mt;
    const int mat = bid / tiles, t = bid % tiles;
    int I, J;
    if (SYM) {   // I <= J, in the order of J
        J = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
        while (J * (J + 1) / 2 > t) --J;
        while ((J + 1) * (J + 2) / 2 <= t) ++J;
        I = t - J * (J + 1) / 2;
    } else {     // strips of eight rows of tiles
        const int strip = t / (8 * mt), h = min(8, nt - 8 * strip), r = t - strip * 8 * mt;
        I = 8 * strip + r % h;
        J = r / h;
    }
    const int K = MODE == kGram ? G.mp : G.np, nk = K / 16;
    const int rfR = G.np / 32, rfS = (SYM ? G.np : G.mp) / 32;   // row fragments of R and S
    // the wavefront's fragments of a stage, as pointers to its lanes' 16 bytes
    const uint16_t *src[L];
#pragma unroll
    for (int i = 0; i < L; ++i) {
        const int f = wave + 8 * i, side = f / (F * PARTS * KF), plane = f / (F * KF) % PARTS, rf = f / KF % F, kf = f % KF;
        const uint16_t *p;
        if (MODE == kGram) p = x_plane(G, mat, B.cur, 0, plane);
        else if (MODE == kSquare) p = s_plane(G, mat, 0, plane);
        else p = side ? x_plane(G, mat, B.cur, 1, plane) : s_plane(G, mat, 1, plane);
        // (row fragments past the matrix: the last one again, its products unused)
        const int row = min((side ? J : I) * F + rf, (side ? rfS : rfR) - 1);
        src[i] = p + ((int64_t)row * nk + kf) * kFrag + lane * 8;
    }
    auto load = [&](int buf) {
#pragma unroll
        for (int i = 0; i < L; ++i) {
            load_lds<16>(src[i], sh + (buf * kStage + wave + 8 * i) * 1024);
            src[i] += KF * kFrag;
        }
    };
    // (one block of accumulators per wavefront: a set for each part product, or for each fragment of a stage, since
    // consecutive products into one set wait for one another)
    constexpr int NA = W == 2 ? 1 : PARTS == 2 ? 3 : 2, NK = KF / 2;
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
        h8 a[NK][W][PARTS], b[NK][W][PARTS];
    };
    auto fetch = [&](int s, Frags &f) {
        const u4v *fr = reinterpret_cast<const u4v *>(sh + (s % NB) * kStage * 1024);
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    const int kf = 2 * k + kg;
                    f.a[k][i][p] = __builtin_bit_cast(h8, fr[((p * F + wi * W + i) * KF + kf) * 64 + lane]);
                    f.b[k][i][p] = __builtin_bit_cast(h8, fr[(((PARTS + p) * F + wj * W + i) * KF + kf) * 64 + lane]);
                }
    };
    auto multiply = [&](const Frags &f) {
#pragma unroll
        for (int k = 0; k < NK; ++k) {
            h8 a[W][PARTS];
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
                    a[i][p] = __builtin_bit_cast(h8, __builtin_bit_cast(u4v, f.a[k][i][p]) ^ neg);
            auto product = [&](f16v &d, int i, int j, int pa, int pb) {
                d = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[i][pa], f.b[k][j][pb], d, 0, 0, 0);
            };
            if constexpr (W == 1) {
                if (PARTS == 2) {
                    product(more[1], 0, 0, PARTS - 1, 0);
                    product(more[NA - 1], 0, 0, 0, PARTS - 1);
                }
                product(PARTS == 2 ? more[0] : more[k % NA], 0, 0, 0, 0);
            } else {
#pragma unroll
                for (int q = PARTS == 2 ? 0 : 2; q < 3; ++q)
#pragma unroll
                    for (int ij = 0; ij < 4; ++ij)
                        product(acc[ij / 2][ij % 2], ij / 2, ij % 2, q == 0 ? PARTS - 1 : 0, q == 1 ? PARTS - 1 : 0);
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
        constexpr int NM = (W == 2 ? 4 : 1) * NK * (PARTS == 2 ? 3 : 1), M1 = NM / (L + 1);
        static_assert(L == 2 || L == 4, "two or four direct loads");
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * NK * W * PARTS, 0);
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
        for (int e = 0; e < 16; ++e) acc[0][0][e] = PARTS == 2 ? more[0][e] + (more[1][e] + more[NA - 1][e]) : more[0][e] + more[NA - 1][e];
    }
    // What is left goes over the tile in LDS, by pieces of eight consecutive k of a row of the next operand: 64
    // threads to a fragment.  First in the order of S's rows (the transpose of the tile), with the term of the
    // iteration itself (c A A + b A, B X + a X), whose operand has that order too and is asked for now.
    constexpr int P = T + 4, NQ = T * T / 8 / 512, TK = T / 16;
    static_assert(T * P * 4 <= NB * kStage * 1024, "the ring holds the tile");
    float *tile = reinterpret_cast<float *>(sh);
    uint16_t *to[2][2];   // operand written in S's order, in R's; hi, lo
    const uint16_t *was[2] = {nullptr, nullptr};
#pragma unroll
    for (int pl = 0; pl < 2; ++pl) {
        if (SYM) to[0][pl] = to[1][pl] = s_plane(G, mat, MODE == kSquare, pl);
        else { to[0][pl] = x_plane(G, mat, 1 - B.cur, 1, pl); to[1][pl] = x_plane(G, mat, 1 - B.cur, 0, pl); }
        if (MODE != kGram) was[pl] = MODE == kSquare ? s_plane(G, mat, 0, pl) : x_plane(G, mat, B.cur, 1, pl);
    }
    const int prow = (threadIdx.x & 31), pk = 8 * (lane >> 5);   // of a piece, within its fragment
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
    OUT *out = static_cast<OUT *>(G.out.p) + mat * G.out.mat;
    const int64_t r0 = (int64_t)(G.trans ? J : I) * T, c0 = (int64_t)(G.trans ? I : J) * T;
    const int sr = G.trans ? 1 : P, sc = G.trans ? P : 1;
    const float keep = 1.f - B.lr * B.decay, rate = B.lr * G.factor;
#pragma unroll 4
    for (int e = threadIdx.x; e < T * T; e += 512) {
        const int r = e / T, c = e % T;
        if (r0 + r >= G.rows || c0 + c >= G.cols) continue;
        OUT *p = out + (r0 + r) * G.out.row + c0 + c;
        const float o = tile[r * sr + c * sc] * kInvScale;
        if constexpr (MODE == kUpdate) *p = keep * *p - rate * o;
        else if constexpr (sizeof(OUT) == 2) *p = f2bf(o);
        else *p = o;
    }
}

// ---------------------------------------------------------------------- host
int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

// workspace of one set of groups, and the pointers into it
size_t carve_ns(NsGroup *g, int32_t n, void *base) {
    Carver c(base);
    for (int i = 0; i < n; ++i) {
        NsGroup &G = g[i];
        if (G.plain) continue;
        G.part = c.take<double>((size_t)G.count * G.chunks);
        G.ops_stride = 8ll * G.np * G.mp + 4ll * G.np * G.np;
        G.ops = c.take<uint16_t>((size_t)G.count * G.ops_stride);
    }
    return c.used;
}

void shape_ns(NsGroup *G, int32_t count, int32_t rows, int32_t cols, int32_t plain) {
    G->count = count; G->rows = rows; G->cols = cols; G->plain = plain;
    G->trans = rows > cols;
    G->n = std::min(rows, cols); G->m = std::max(rows, cols);
    G->np = (int32_t)up64(G->n); G->mp = (int32_t)up64(G->m);
    G->chunks = (int32_t)(((int64_t)rows * cols + kSumChunk - 1) / kSumChunk);
}

constexpr int kMaxSide = 32768;   // rows or columns

tag_status check_shape(int32_t count, int32_t rows, int32_t cols, bool plain) {
    if (count < 1 || rows < 1 || cols < 1) TAG_FAIL(TAG_EINVAL, "need count, rows and cols >= 1");
    if (!plain && (rows > kMaxSide || cols > kMaxSide)) TAG_FAIL(TAG_ESHAPE, "at most 32768 rows or columns");
    // (blocks are counted in 32 bits)
    const int64_t blocks = std::max((up64(rows) / 64) * (up64(cols) / 64), ((int64_t)rows * cols + kSumChunk - 1) / kSumChunk);
    if (blocks * count > (1 << 26)) TAG_FAIL(TAG_ESHAPE, "too many or too large matrices in a group");
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

template <typename Blocks>
unsigned set_blocks(NsBatch &B, Blocks blocks) {
    int64_t n = 0;
    for (int i = 0; i < B.n_groups; ++i) {
        B.first[i] = (int32_t)n;
        n += blocks(B.g[i]);
    }
    B.first[B.n_groups] = (int32_t)n;
    return (unsigned)n;
}

template <int T, int PARTS, typename OUT>
void launch_product(NsBatch &B, int mode, hipStream_t st) {
    const unsigned grid = set_blocks(B, [&](const NsGroup &G) -> int64_t {
        const int64_t nt = (G.np + T - 1) / T, mt = (G.mp + T - 1) / T;
        return G.count * (mode == kGram || mode == kSquare ? nt * (nt + 1) / 2 : nt * mt);
    });
    switch (mode) {
        case kGram: ns_product<T, PARTS, kGram, OUT><<<grid, 512, 0, st>>>(B); break;
        case kSquare: ns_product<T, PARTS, kSquare, OUT><<<grid, 512, 0, st>>>(B); break;
        case kApply: ns_product<T, PARTS, kApply, OUT><<<grid, 512, 0, st>>>(B); break;
        case kFinal: ns_product<T, PARTS, kFinal, OUT><<<grid, 512, 0, st>>>(B); break;
        default:
            if constexpr (sizeof(OUT) == 4) ns_product<T, PARTS, kUpdate, float><<<grid, 512, 0, st>>>(B);
    }
}

// Tiles of 128 x 128 once they fill the chip, else of 64 x 64.
template <int PARTS, typename OUT>
void launch_tiles(NsBatch &B, int mode, hipStream_t st) {
    int64_t n = 0;
    for (int i = 0; i < B.n_groups; ++i) {
        const NsGroup &G = B.g[i];
        const int64_t nt = (G.np + 127) / 128, mt = (G.mp + 127) / 128;
        n += G.count * (mode == kGram || mode == kSquare ? nt * (nt + 1) / 2 : nt * mt);
    }
    if (n >= 128) launch_product<128, PARTS, OUT>(B, mode, st);
    else launch_product<64, PARTS, OUT>(B, mode, st);
}

template <typename T, bool MUON, int PARTS>
void run_ns(NsBatch &all, int steps, hipStream_t st) {
    unsigned grid = set_blocks(all, [](const NsGroup &G) { return (int64_t)G.count * G.chunks; });
    ns_norm<T, MUON><<<grid, 256, 0, st>>>(all);
    NsBatch B = all;   // without the plain groups
    B.n_groups = 0;
    for (int i = 0; i < all.n_groups; ++i)
        if (!all.g[i].plain) B.g[B.n_groups++] = all.g[i];
    if (B.n_groups == 0) return;
    grid = set_blocks(B, [](const NsGroup &G) { return (int64_t)G.count * (G.np / 64) * (G.mp / 64); });
    ns_prepare<T, MUON><<<grid, 256, 0, st>>>(B);
    for (int s = 0; s < steps; ++s) {
        B.cur = s & 1;
        launch_tiles<PARTS, T>(B, kGram, st);
        launch_tiles<PARTS, T>(B, kSquare, st);
        launch_tiles<PARTS, T>(B, s + 1 < steps ? kApply : MUON ? kUpdate : kFinal, st);
    }
}

Arr arr(const tag_matrices &a) { return Arr{a.base, a.row_stride, a.matrix_stride}; }

void fill_ortho(NsBatch &B, const tag_ortho_group *g, int32_t n) {
    B.n_groups = n;
    for (int i = 0; i < n; ++i) {
        B.g[i] = NsGroup{};
        shape_ns(&B.g[i], g[i].count, g[i].rows, g[i].cols, 0);
        B.g[i].in = arr(g[i].in);
        B.g[i].out = arr(g[i].out);
    }
}

void fill_muon(NsBatch &B, const tag_muon_group *g, int32_t n) {
    B.n_groups = n;
    for (int i = 0; i < n; ++i) {
        B.g[i] = NsGroup{};
        shape_ns(&B.g[i], g[i].count, g[i].rows, g[i].cols, g[i].plain != 0);
        B.g[i].in = arr(g[i].g);
        B.g[i].out = arr(g[i].w);
        B.g[i].mom = arr(g[i].m);
        B.g[i].factor = (float)std::sqrt(std::max(1.0, (double)g[i].rows / g[i].cols));
    }
}

// sets of at most kMaxGroups groups run one after the other in the same workspace
template <typename Group, typename Fill>
size_t workspace_of(const Group *g, int32_t n, Fill fill) {
    size_t most = 0;
    for (int32_t i = 0; i < n; i += kMaxGroups) {
        NsBatch B{};
        const int32_t k = std::min(kMaxGroups, n - i);
        fill(B, g + i, k);
        most = std::max(most, carve_ns(B.g, k, nullptr));
    }
    return most;
}

tag_status check_ortho_groups(const tag_ortho_group *g, int32_t n, bool arrays, size_t el) {
    if (!g || n < 1) TAG_FAIL(TAG_EINVAL, "need at least one group");
    for (int32_t i = 0; i < n; ++i) {
        tag_status st = check_shape(g[i].count, g[i].rows, g[i].cols, false);
        if (st == TAG_OK && arrays) st = check_array(g[i].in, g[i].count, g[i].rows, g[i].cols, el, false, "in");
        if (st == TAG_OK && arrays) st = check_array(g[i].out, g[i].count, g[i].rows, g[i].cols, el, true, "out");
        if (st != TAG_OK) return st;
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
        if (arrays && (g[i].w.base == g[i].g.base || g[i].w.base == g[i].m.base || g[i].g.base == g[i].m.base))
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
    *bytes = workspace_of(groups, n_groups, fill_ortho);
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
    if (workspace_of(groups, n_groups, fill_ortho) > ws_bytes)
        TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_orthogonalise_workspace)");
    if (!workspace || (uintptr_t)workspace % 16) TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int32_t i = 0; i < n_groups; i += kMaxGroups) {
        NsBatch B{};
        fill_ortho(B, groups + i, std::min(kMaxGroups, n_groups - i));
        carve_ns(B.g, B.n_groups, workspace);
        B.a = ns->a; B.b = ns->b; B.c = ns->c; B.eps = ns->eps;
        if (dtype == TAG_BF16) run_ns<uint16_t, false, 1>(B, ns->steps, stream);
        else run_ns<float, false, 2>(B, ns->steps, stream);
    }
    return launch_status("tag_orthogonalise");
}

extern "C" tag_status tag_muon_workspace(const tag_muon_group *groups, int32_t n_groups, size_t *bytes) {
    clear_error();
    if (!bytes) TAG_FAIL(TAG_EINVAL, "bytes must be non-NULL");
    const tag_status st = check_muon_groups(groups, n_groups, false);
    if (st != TAG_OK) return st;
    *bytes = workspace_of(groups, n_groups, fill_muon);
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
    const size_t need = workspace_of(groups, n_groups, fill_muon);
    if (need > ws_bytes) TAG_FAIL(TAG_ENOSPACE, "workspace too small (see tag_muon_workspace)");
    if (need && (!workspace || (uintptr_t)workspace % 16))
        TAG_FAIL(TAG_EINVAL, "workspace must be non-NULL and 16-byte aligned");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    for (int32_t i = 0; i < n_groups; i += kMaxGroups) {
        NsBatch B{};
        fill_muon(B, groups + i, std::min(kMaxGroups, n_groups - i));
        carve_ns(B.g, B.n_groups, workspace);
        B.a = ns->a; B.b = ns->b; B.c = ns->c; B.eps = ns->eps;
        B.lr = options->lr; B.momentum = options->momentum; B.decay = options->weight_decay;
        B.nesterov = options->nesterov != 0;
        run_ns<float, true, 2>(B, ns->steps, stream);
    }
    return launch_status("tag_muon_step");
}
