// Orthogonalised updates: G / |G|, then steps of X <- a X + (b A + c A^2) X with A = X X' (of a tall matrix X <- a X + X (b A + c A^2), A = X' X: the
// shorter side's), as products of half precision (products.h) with 32-bit sums.
//
// What is rounded to 11 bits decides how far the result is off, since a step takes small singular values times `a` and a rounding's noise with them:
//   X     is kept in two parts (22 bits); only the products take its high part alone
//   A     = diag(d) + O with d in 32 bits, O rounded:  b A + c A^2 = diag(b d + c d^2) + b O + c ((d_i + d_j) O + O O)
//   b A + c A^2 likewise: its diagonal e is added to a, X <- (a + e) X + (what lies beside it) X
// In a simulation in 64 bits with these roundings the result is off by 1.4e-4 to 6.8e-4 of its norm over square, wide, and nearly rank deficient matrices;
// with diagonals rounded too 2.8e-3, with X rounded between steps up to 4.2e-2. A bfloat16 result's own rounding is 1.7e-3. Results in 32 bits and in
// half precision take both parts of every number (three products): 3e-7 to 4e-6, as much as sums of 32 bits cost.
//
// A and A^2 are symmetric: only tiles on and below the diagonal are computed, and stored twice.
#include <algorithm>
#include <cmath>

#include "products.h"
#include "step.h"

namespace iodf {

namespace {

constexpr int kNormBlocks = 1024;  // partial sums of squares of a matrix, at most

inline long long up(long long n, long long d) { return (n + d - 1) / d * d; }

// Where the matrices of a call come from and go to.
struct Source {
    const void* g[kMaxUpdates];
    float* m[kMaxUpdates];
    long long stride, batch;  // batch: elements from one matrix to the next, from g[0] on; 0: g and m have one for each
    float beta;
    int nesterov;
};
struct Target {
    void* w[kMaxUpdates];
    long long stride, batch;
    float keep, by;           // w <- keep w + by X, of updates
    int update;
};

struct Shape {
    int count, rows, cols, rp, cp, s, sp;  // rp, cp, sp: rounded up to 64; s the shorter side
};

// What goes into the norm and then into X, eight neighbours of a row: the gradient, or the momentum's view of it. `first`: the momentum is moved on.
template <typename TG, bool MUON, bool FIRST>
__device__ __forceinline__ void taken(const Source& src, int k, int r, int c, int cols, float (&v)[8]) {
    const int n = cols - c;
    const TG* const g = (MUON ? (const TG*)src.g[k] : (const TG*)src.g[0] + k * src.batch) + r * src.stride + c;
    load8(g, n, v);
    if (!MUON) return;
    float* const m = src.m[k] + (long long)r * cols + c;
    float was[8];
    load8(m, n, was);
    if (FIRST) {
#pragma unroll
        for (int j = 0; j < 8; ++j) was[j] = fmaf(src.beta, was[j], v[j]);
        store8(m, n, was);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = src.nesterov ? fmaf(src.beta, was[j], v[j]) : was[j];
}

// The sum over 256 threads, in each of them.
__device__ __forceinline__ double block_sum(double s, double* meet) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) s += __shfl_xor(s, i);
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = s;
    __syncthreads();
    return (meet[0] + meet[1]) + (meet[2] + meet[3]);
}

template <typename TG, bool MUON>
__global__ __launch_bounds__(256) void k_orth_norm(const Source src, const Shape z, double* sums) {
    __shared__ double meet[4];
    const int k = blockIdx.y, per = (z.cols + 7) / 8;
    double s = 0.0;
    for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < (unsigned)z.rows * per; i += gridDim.x * 256) {
        float v[8];
        taken<TG, MUON, true>(src, k, i / per, i % per * 8, z.cols, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j] * v[j];
    }
    s = block_sum(s, meet);
    if (threadIdx.x == 0) sums[k * gridDim.x + blockIdx.x] = s;
}

__device__ __forceinline__ void two_parts(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = fabsf(v) < 60000.f ? (_Float16)(v - (float)hi) : (_Float16)0.f;  // an infinity or NaN has no rest
}

// D / (norm + eps), times 2^x_exp, in two parts, with zeros around it.
template <typename TG, bool MUON>
__global__ __launch_bounds__(256) void k_orth_start(const Source src, const Shape z, const double* sums, int parts, float eps, float lift, _Float16* x,
                                                    long long plane) {
    __shared__ double meet[4];
    const int k = blockIdx.y, per = z.cp / 8;
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += sums[k * parts + i];
    const double by = (double)lift / (sqrt(block_sum(s, meet)) + (double)eps);
    x += k * (long long)z.rp * z.cp;
    for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < (unsigned)z.rp * per; i += gridDim.x * 256) {
        const int r = i / per, c = i % per * 8;
        float v[8] = {};
        if (r < z.rows && c < z.cols) taken<TG, MUON, false>(src, k, r, c, z.cols, v);
        _Float16 hi[8], lo[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) two_parts(c + j < z.cols ? (float)(v[j] * by) : 0.f, hi[j], lo[j]);
        u32x4 w;
        __builtin_memcpy(&w, hi, 16);
        *(u32x4*)(x + i * 8ll) = w;
        __builtin_memcpy(&w, lo, 16);
        *(u32x4*)(x + plane + i * 8ll) = w;
    }
}

struct SquareArgs {
    Side x;                 // X (first) or O (second), of matrix 0
    long long x_batch;
    int kts, tiles;         // tiles along the sum, tiles of a side
    int sp;
    float down;             // what a sum is multiplied with to be X X' or O O
    float lift, unlift;     // powers of two of what is stored; second: of O's inverse
    float b, c;
    float* d;               // diagonals [matrix][sp]: first writes A's, second reads them and writes e
    float* e;
    _Float16* out;          // [matrix][sp][sp], O or what lies beside the diagonal of b A + c A^2
    long long plane;
};

template <int PAIRS>
__device__ __forceinline__ void store4(_Float16* to, long long plane, const float (&v)[4]) {
    _Float16 hi[4], lo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) two_parts(v[j], hi[j], lo[j]);
    __builtin_memcpy(to, hi, 8);
    if (PAIRS > 1) __builtin_memcpy(to + plane, lo, 8);
}
template <int PAIRS>
__device__ __forceinline__ void load4(const _Float16* from, long long plane, float (&v)[4]) {
    _Float16 hi[4], lo[4];
    __builtin_memcpy(hi, from, 8);
    if (PAIRS > 1) __builtin_memcpy(lo, from + plane, 8);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (float)hi[j] + (PAIRS > 1 ? (float)lo[j] : 0.f);
}

// A tile on or below the diagonal of a symmetric product, and its mirror image.
template <int MW, int NW, int MT, int NT, bool SUMS, bool SECOND, int PAIRS>
__global__ __launch_bounds__(MW * NW * 64) void k_square(const SquareArgs a) {
    typedef Products<_Float16, MW, NW, MT, NT, SUMS, SUMS, PAIRS> P;
    static_assert(P::BM == P::BN, "tiles of a symmetric product are square");
    __shared__ __align__(16) uint16_t lds[P::LDS];
    const int k = blockIdx.y;
    int ti, tj;
    place_triangle(blockIdx.x, gridDim.x, a.tiles, ti, tj);
    Side x = a.x;
    x.p += k * a.x_batch;
    P p;
    p.run(x, x, ti * P::BM, tj * P::BN, 0, a.kts, lds);

    const long long square = (long long)a.sp * a.sp;
    _Float16* const out = a.out + k * square;
    const _Float16* const o = (const _Float16*)x.p;
    float* const d = a.d + (long long)k * a.sp;
    float* const e = a.e + (long long)k * a.sp;
    // four neighbours of row r, from sums in LDS
    struct Four {
        float sum[4], was[4], dr, dc[4];
        int r, c;
    };
    auto fetch = [&](Four& f, int r, int c, u32x4 w) {
        __builtin_memcpy(f.sum, &w, 16);
        f.r = r, f.c = c;
        if (SECOND && r < a.sp && c < a.sp) {
            load4<PAIRS>(o + (long long)r * a.sp + c, x.plane, f.was);
            f.dr = d[r];
            __builtin_memcpy(f.dc, d + c, 16);
        }
    };
    auto finish = [&](const Four& f) {
        if (f.r >= a.sp || f.c >= a.sp) return;
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float sum = f.sum[j] * a.down;
            const bool diagonal = f.r == f.c + j;
            if (!SECOND) {
                if (diagonal) d[f.r] = sum;
                v[j] = sum * a.lift;
            } else {
                const float ov = f.was[j] * a.unlift;
                if (diagonal) e[f.r] = fmaf(a.c, fmaf(f.dr, f.dr, sum), a.b * f.dr);
                v[j] = fmaf(a.c, fmaf(f.dr + f.dc[j], ov, sum), a.b * ov) * a.lift;
            }
            if (diagonal) v[j] = 0.f;
        }
        store4<PAIRS>(out + (long long)f.r * a.sp + f.c, a.plane, v);
    };
    typedef Staged<P, float, NW> Out;
    typedef StagedAcross<P, MW> Mirror;
    static_assert(Out::BYTES <= P::LDS * 2 && Mirror::BYTES <= P::LDS * 2, "outputs pass through the operands' LDS");
    constexpr int AT_ONCE = 4;
#pragma unroll
    for (int pass = 0; pass < NT / 2; ++pass) {
        if (pass) __syncthreads();
#pragma unroll
        for (int n = 2 * pass; n < 2 * pass + 2; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float v[4] = {p.acc[m][n][0], p.acc[m][n][1], p.acc[m][n][2], p.acc[m][n][3]};
                Out::put(lds, m, n, v);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Out::PER; i += AT_ONCE) {
            Four f[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                int row, col;
                Out::where(i + u, pass, row, col);
                fetch(f[u], tj * P::BN + row, ti * P::BM + col, Out::take(lds, i + u));
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) finish(f[u]);
        }
    }
    if (ti == tj) return;  // symmetric: all of it has been stored
#pragma unroll
    for (int pass = 0; pass < MT / 2; ++pass) {
        __syncthreads();
#pragma unroll
        for (int m = 2 * pass; m < 2 * pass + 2; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const float v[4] = {p.acc[m][n][0], p.acc[m][n][1], p.acc[m][n][2], p.acc[m][n][3]};
                Mirror::put(lds, m, n, v);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Mirror::PER; i += AT_ONCE) {
            Four f[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                int row, col;
                Mirror::where(i + u, pass, row, col);
                fetch(f[u], ti * P::BM + row, tj * P::BN + col, Mirror::take(lds, i + u));
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) finish(f[u]);
        }
    }
}

struct ApplyArgs {
    Side x, b;              // X and what lies beside the diagonal, of matrix 0
    long long x_batch;
    Shape z;
    int kts, tm, tn;
    float down, unlift;     // of a sum, of X's parts
    float a;                // the step's first coefficient
    const float* e;
    _Float16* to;           // the next X, times `lift`; NULL: the result goes to `target`
    long long plane;
    float lift;
};

template <typename TO>
__device__ __forceinline__ void deliver(const Target& t, int k, int r, int c, int n, float (&v)[4]) {
    TO* const to = (t.batch ? (TO*)t.w[0] + k * t.batch : (TO*)t.w[k]) + r * t.stride + c;
    if (t.update) {
        float was[4];
        get_quad(to, n, was);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(t.keep, was[j], t.by * v[j]);
    }
    put_quad(to, n, v);
}

// (a + e) X + B X: columns of X are the rows of the matrix instructions, so that a lane holds four neighbours of a row.
template <int MW, int NW, int MT, int NT, bool TALL, int PAIRS>
__global__ __launch_bounds__(MW * NW * 64) void k_apply(const ApplyArgs a, const Target target, const int type) {
    typedef Products<_Float16, MW, NW, MT, NT, !TALL, false, PAIRS> P;
    __shared__ __align__(16) uint16_t lds[P::LDS];
    const int k = blockIdx.y;
    int tm, tn;
    place_tile(blockIdx.x, gridDim.x, a.tm, a.tn, tm, tn);
    Side x = a.x, b = a.b;
    x.p += k * a.x_batch;
    b.p += (long long)k * a.z.sp * a.z.sp;
    P p;
    p.run(TALL ? b : x, TALL ? x : b, tm * P::BM, tn * P::BN, 0, a.kts, lds);

    const _Float16* const was = (const _Float16*)x.p;
    const float* const e = a.e + (long long)k * a.z.sp;
    const int rows = a.to ? a.z.rp : a.z.rows, cols = a.to ? a.z.cp : a.z.cols;
    _Float16* const to = a.to + k * a.x_batch;
    typedef Staged<P, float, NW> Out;
    static_assert(Out::BYTES <= P::LDS * 2, "outputs pass through the operands' LDS");
    constexpr int AT_ONCE = 4;
#pragma unroll
    for (int pass = 0; pass < NT / 2; ++pass) {
        if (pass) __syncthreads();
#pragma unroll
        for (int n = 2 * pass; n < 2 * pass + 2; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float v[4] = {p.acc[m][n][0], p.acc[m][n][1], p.acc[m][n][2], p.acc[m][n][3]};
                Out::put(lds, m, n, v);
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < Out::PER; i += AT_ONCE) {
            float x0[AT_ONCE][4], e0[AT_ONCE][4];
            int r[AT_ONCE], c[AT_ONCE];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                Out::where(i + u, pass, r[u], c[u]);
                r[u] += tn * P::BN, c[u] += tm * P::BM;
                if (r[u] >= rows || c[u] >= cols) continue;
                load4<2>(was + (long long)r[u] * a.z.cp + c[u], x.plane, x0[u]);
                if (TALL) __builtin_memcpy(e0[u], e + c[u], 16);
                else e0[u][0] = e0[u][1] = e0[u][2] = e0[u][3] = e[r[u]];
            }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u) {
                if (r[u] >= rows || c[u] >= cols) continue;
                float v[4];
                const u32x4 w = Out::take(lds, i + u);
                __builtin_memcpy(v, &w, 16);
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fmaf(a.a + e0[u][j], x0[u][j] * a.unlift, v[j] * a.down);
                if (a.to) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[j] *= a.lift;
                    store4<2>(to + (long long)r[u] * a.z.cp + c[u], a.plane, v);
                } else if (type == IODF_T_F32) {
                    deliver<float>(target, k, r[u], c[u], cols - c[u], v);
                } else if (type == IODF_T_BF16) {
                    deliver<__bf16>(target, k, r[u], c[u], cols - c[u], v);
                } else {
                    deliver<_Float16>(target, k, r[u], c[u], cols - c[u], v);
                }
            }
        }
    }
}

struct OrthPlan {
    Shape z;
    bool tall, parts;          // parts: three products
    int square_edge, apply_edge;
    int parts_of_norm;
    size_t sums, x0, x1, o, b, d, e, bytes;
};

OrthPlan orth_plan(long long count, int rows, int cols, int type) {
    OrthPlan p{};
    p.z = {(int)count, rows, cols, (int)up(rows, PK), (int)up(cols, PK), std::min(rows, cols), 0};
    p.z.sp = (int)up(p.z.s, PK);
    p.tall = rows > cols;
    p.parts = type != IODF_T_BF16;
    auto tiles = [&](long long n, int e) { return (n + e - 1) / e; };
    auto square = [&](int e) { return count * tiles(p.z.s, e) * (tiles(p.z.s, e) + 1) / 2; };
    auto apply = [&](int e) { return count * tiles(rows, e) * tiles(cols, e); };
    p.square_edge = square(256) >= 200 ? 256 : square(128) >= 200 ? 128 : 64;
    p.apply_edge = apply(256) >= 200 ? 256 : apply(128) >= 200 ? 128 : 64;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += up(bytes, 256);
        return was;
    };
    const size_t x = (size_t)count * p.z.rp * p.z.cp * 2 * 2, s = (size_t)count * p.z.sp * p.z.sp * 2 * (p.parts ? 2 : 1);
    p.parts_of_norm = (int)std::max<long long>(1, std::min<long long>({kNormBlocks, 2048 / std::max<long long>(1, count), ((long long)rows * ((cols + 7) / 8) + 255) / 256}));
    p.sums = take((size_t)count * p.parts_of_norm * 8);
    p.x0 = take(x), p.x1 = take(x), p.o = take(s), p.b = take(s);
    p.d = take((size_t)count * p.z.sp * 4), p.e = take((size_t)count * p.z.sp * 4);
    p.bytes = at;
    return p;
}

template <int MW, int NW, int MT, int NT, bool SUMS, bool SECOND, int PAIRS>
void square_with(SquareArgs a, int count, int s, hipStream_t st) {
    constexpr int E = MW * MT * 16;
    a.tiles = (s + E - 1) / E;
    k_square<MW, NW, MT, NT, SUMS, SECOND, PAIRS><<<dim3((unsigned)(a.tiles * (a.tiles + 1) / 2), count), MW * NW * 64, 0, st>>>(a);
}
template <bool SUMS, bool SECOND, int PAIRS>
void square(const SquareArgs& a, int edge, int count, int s, hipStream_t st) {
    if (edge == 256) square_with<2, 4, 8, 4, SUMS, SECOND, PAIRS>(a, count, s, st);
    else if (edge == 128) square_with<2, 2, 4, 4, SUMS, SECOND, PAIRS>(a, count, s, st);
    else square_with<2, 2, 2, 2, SUMS, SECOND, PAIRS>(a, count, s, st);
}

template <int MW, int NW, int MT, int NT, bool TALL, int PAIRS>
void apply_with(ApplyArgs a, const Target& t, int type, hipStream_t st) {
    constexpr int E = MW * MT * 16;
    a.tm = (a.z.cols + E - 1) / E, a.tn = (a.z.rows + E - 1) / E;
    k_apply<MW, NW, MT, NT, TALL, PAIRS><<<dim3((unsigned)a.tm * a.tn, a.z.count), MW * NW * 64, 0, st>>>(a, t, type);
}
template <bool TALL, int PAIRS>
void apply(const ApplyArgs& a, int edge, const Target& t, int type, hipStream_t st) {
    if (edge == 256) apply_with<2, 4, 8, 4, TALL, PAIRS>(a, t, type, st);
    else if (edge == 128) apply_with<2, 2, 4, 4, TALL, PAIRS>(a, t, type, st);
    else apply_with<2, 2, 2, 2, TALL, PAIRS>(a, t, type, st);
}

template <bool MUON>
void begin(const Source& src, int type, const OrthPlan& p, float eps, float lift, char* work, hipStream_t st) {
    double* const sums = (double*)(work + p.sums);
    _Float16* const x = (_Float16*)(work + p.x0);
    const long long n = (long long)p.z.rp * p.z.cp, plane = n * p.z.count;
    const dim3 sum_grid(p.parts_of_norm, p.z.count), grid((unsigned)std::min<long long>((n / 8 + 255) / 256, 2048), p.z.count);
    auto go = [&](auto t) {
        typedef decltype(t) TG;
        k_orth_norm<TG, MUON><<<sum_grid, 256, 0, st>>>(src, p.z, sums);
        k_orth_start<TG, MUON><<<grid, 256, 0, st>>>(src, p.z, sums, p.parts_of_norm, eps, lift, x, plane);
    };
    if (type == IODF_T_F32) go(0.f);
    else if (type == IODF_T_BF16) go((__bf16)0.f);
    else go((_Float16)0.f);
}

template <bool TALL, int PAIRS>
void polynomials(const OrthPlan& p, const OrthSteps& s, char* work, const Target& target, int type, hipStream_t st) {
    const long long xn = (long long)p.z.rp * p.z.cp, plane = xn * p.z.count, square_n = (long long)p.z.sp * p.z.sp;
    _Float16 *x = (_Float16*)(work + p.x0), *next = (_Float16*)(work + p.x1);
    _Float16 *const o = (_Float16*)(work + p.o), *const b = (_Float16*)(work + p.b);
    float *const d = (float*)(work + p.d), *const e = (float*)(work + p.e);
    for (int i = 0; i < s.n; ++i) {
        const float xl = ldexpf(1.f, s.x_exp[i]), ol = ldexpf(1.f, s.a_exp[i]), bl = ldexpf(1.f, s.b_exp[i]);
        SquareArgs q{};
        q.x = {(const uint16_t*)x, plane, p.z.cp, TALL ? p.z.cp : p.z.rp, TALL ? p.z.rp : p.z.cp};
        q.x_batch = xn, q.sp = p.z.sp, q.d = d, q.e = e, q.plane = square_n * p.z.count;
        q.kts = (TALL ? p.z.rp : p.z.cp) / PK;
        q.down = 1.f / (xl * xl), q.lift = ol, q.out = o;
        square<TALL, false, PAIRS>(q, p.square_edge, p.z.count, p.z.s, st);
        q.x = {(const uint16_t*)o, square_n * p.z.count, p.z.sp, p.z.sp, p.z.sp};
        q.x_batch = square_n, q.kts = p.z.sp / PK;
        q.down = 1.f / (ol * ol), q.unlift = 1.f / ol, q.lift = bl, q.b = s.b[i], q.c = s.c[i], q.out = b;
        square<false, true, PAIRS>(q, p.square_edge, p.z.count, p.z.s, st);
        ApplyArgs a{};
        a.x = {(const uint16_t*)x, plane, p.z.cp, TALL ? p.z.rp : p.z.cp, TALL ? p.z.cp : p.z.rp};
        a.b = {(const uint16_t*)b, square_n * p.z.count, p.z.sp, p.z.sp, p.z.sp};
        a.x_batch = xn, a.z = p.z, a.kts = p.z.sp / PK, a.down = 1.f / (xl * bl), a.unlift = 1.f / xl, a.a = s.a[i], a.e = e;
        a.plane = plane;
        if (i + 1 < s.n) a.to = next, a.lift = ldexpf(1.f, s.x_exp[i + 1]);
        apply<TALL, PAIRS>(a, p.apply_edge, target, type, st);
        std::swap(x, next);
    }
}

hipError_t run(const OrthPlan& p, const OrthSteps& s, char* work, const Target& t, int type, hipStream_t st) {
    if (p.tall) p.parts ? polynomials<true, 3>(p, s, work, t, type, st) : polynomials<true, 1>(p, s, work, t, type, st);
    else p.parts ? polynomials<false, 3>(p, s, work, t, type, st) : polynomials<false, 1>(p, s, work, t, type, st);
    return hipGetLastError();
}

}  // namespace

// How large singular values, and with them every entry of X, of A and of b A + c A^2, can get: 0..1 at first, then as the polynomials say, looked at in
// 4096 places, two percent added for what lies between them and for roundings.
bool orth_steps(int steps, const float* co, OrthSteps& s) {
    if (steps < 1 || steps > IODF_ORTH_MOST || !co) return false;
    s.n = steps;
    double most = 1.02;
    auto lift = [](double m) { return 14 - (int)std::ceil(std::log2(std::max(m, 1e-6))); };  // m times 2^that is at most 2^14
    for (int i = 0; i < steps; ++i) {
        const double a = co[3 * i], b = co[3 * i + 1], c = co[3 * i + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        double next = 0.0, beside = 0.0;
        for (int k = 0; k <= 4096; ++k) {
            const double v = most * k / 4096, v2 = v * v;
            next = std::max(next, std::fabs(v * (a + v2 * (b + v2 * c))));
            beside = std::max(beside, std::fabs(v2 * (b + v2 * c)));
        }
        s.a[i] = (float)a, s.b[i] = (float)b, s.c[i] = (float)c;
        s.x_exp[i] = lift(most), s.a_exp[i] = lift(most * most), s.b_exp[i] = lift(1.02 * beside);
        most = std::max(1.02 * next, 1e-3);
        if (!(most <= 64.0) || !(beside <= 4096.0)) return false;
    }
    s.x_exp[steps] = lift(most);
    return true;
}

size_t orth_workspace(const iodf_orth& a) { return orth_plan(a.count, a.rows, a.cols, a.out_type).bytes; }
size_t muon_workspace(const iodf_muon& a) { return orth_plan(a.count, a.rows, a.cols, a.weight_type).bytes; }

hipError_t launch_orthogonalise(const iodf_orth& a, const OrthSteps& s, void* work, hipStream_t st) {
    const OrthPlan p = orth_plan(a.count, a.rows, a.cols, a.out_type);
    Source src{};
    src.g[0] = a.in, src.stride = a.in_stride, src.batch = a.in_batch;
    Target t{};
    t.w[0] = a.out, t.stride = a.out_stride, t.batch = a.out_batch;
    begin<false>(src, a.in_type, p, a.eps, ldexpf(1.f, s.x_exp[0]), (char*)work, st);
    return run(p, s, (char*)work, t, a.out_type, st);
}

hipError_t launch_muon_step(const iodf_muon& a, const OrthSteps& s, void* work, hipStream_t st) {
    const OrthPlan p = orth_plan(a.count, a.rows, a.cols, a.weight_type);
    Source src{};
    Target t{};
    for (int k = 0; k < a.count; ++k) src.g[k] = a.grads[k], src.m[k] = a.momenta[k], t.w[k] = a.weights[k];
    src.stride = a.grad_stride, src.beta = a.beta, src.nesterov = a.nesterov;
    t.stride = a.weight_stride, t.update = 1;
    t.keep = (float)(1.0 - (double)a.rate * a.decay), t.by = (float)(-(double)a.rate * a.scale);
    begin<true>(src, a.grad_type, p, a.eps, ldexpf(1.f, s.x_exp[0]), (char*)work, st);
    return run(p, s, (char*)work, t, a.weight_type, st);
}

}  // namespace iodf
