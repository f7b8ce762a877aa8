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
#include <type_traits>

#include "orth_plan.h"
#include "products.h"
#include "step.h"

namespace iodf {

namespace {

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

// The sum of squares of every `all`-th eight neighbours, from the one that `at` counts.
template <typename TG, bool MUON>
__device__ __forceinline__ double squares(const Source& src, const Shape& z, int k, unsigned at, unsigned all) {
    const unsigned per = (z.cols + 7) / 8;
    double s = 0.0;
    for (unsigned i = at; i < z.rows * per; i += all) {
        float v[8];
        taken<TG, MUON, true>(src, k, i / per, i % per * 8, z.cols, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) s += (double)v[j] * v[j];
    }
    return s;
}

// Memory bounds it: 4096 x 8192 in bfloat16 with momenta 55 us (6.1 TB/s, the last-level cache helping), 4096 x 4096 of 32 bits 13.4.
template <typename TG, bool MUON>
__global__ __launch_bounds__(256) void k_orth_norm(const Source src, const Shape z, double* sums) {
    __shared__ double meet[4];
    const double s = block_sum(squares<TG, MUON>(src, z, blockIdx.y, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256), meet);
    if (threadIdx.x == 0) sums[blockIdx.y * gridDim.x + blockIdx.x] = s;
}

__device__ __forceinline__ void two_parts(float v, _Float16& hi, _Float16& lo) {
    hi = (_Float16)v;
    lo = fabsf(v) < 60000.f ? (_Float16)(v - (float)hi) : (_Float16)0.f;  // an infinity or NaN has no rest
}

// D times `by` in two parts, with zeros around it: every `all`-th eight neighbours.
template <typename TG, bool MUON>
__device__ __forceinline__ void start_x(const Source& src, const Shape& z, int k, double by, _Float16* x, long long plane, unsigned at, unsigned all) {
    const unsigned per = z.cp / 8;
    x += k * (long long)z.rp * z.cp;
    for (unsigned i = at; i < z.rp * per; i += all) {
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

// As k_orth_norm: 60 us and 26.
template <typename TG, bool MUON>
__global__ __launch_bounds__(256) void k_orth_start(const Source src, const Shape z, const double* sums, int parts, float eps, float lift, _Float16* x,
                                                    long long plane) {
    __shared__ double meet[4];
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += sums[blockIdx.y * parts + i];
    const double by = (double)lift / (sqrt(block_sum(s, meet)) + (double)eps);
    start_x<TG, MUON>(src, z, blockIdx.y, by, x, plane, blockIdx.x * 256 + threadIdx.x, gridDim.x * 256);
}

struct SquareArgs {
    Side x;                 // X (first) or O (second), of matrix 0
    long long x_batch;
    int kts, tiles;         // tiles along the sum, tiles of a side
    int pieces;             // 0: a workgroup has a tile's whole sum
    long long units;        // tiles along the sums of all tiles
    float* parts;
    int sp;
    float down;             // what a sum is multiplied with to be X X' or O O
    float lift, unlift;     // powers of two of what is stored; second: of O's inverse
    float b, c;
    float* d;               // diagonals [matrix][sp]: first writes A's, second reads them and writes e
    float* e;
    _Float16* out;          // [matrix][sp][sp], O or what lies beside the diagonal of b A + c A^2
    long long plane;
};

// Four numbers as they lie in memory: what a load that is not waited for yet holds.
template <int PARTS>
struct Raw4 {
    u32x2 w[PARTS];
    __device__ __forceinline__ void load(const _Float16* from, long long plane) {
        w[0] = *(const u32x2*)from;
        if (PARTS > 1) w[PARTS - 1] = *(const u32x2*)(from + plane);
    }
    __device__ __forceinline__ float get(int j) const {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < PARTS; ++k) v += (float)__builtin_bit_cast(_Float16, (uint16_t)(w[k][j / 2] >> j % 2 * 16));
        return v;
    }
};

// Sums of a block of X X' or O O from row m0 and column n0 on -> what is stored of it, and with `mirror` its mirror image (of a tile on the diagonal the
// block itself is that).
template <class P, int MW, int NW, bool SECOND, int PAIRS>
__device__ __forceinline__ void finish_square(const SquareArgs& a, P& p, int k, int m0, int n0, bool mirror, uint16_t* lds) {
    constexpr int MT = P::MT, NT = P::NT;
    constexpr int PARTS = PAIRS > 1 ? 2 : 1, AHEAD = MT % 4 == 0 ? 4 : MT % 3 == 0 ? 3 : MT;
    typedef Staged<P, uint16_t, NW, NT> Out;
    static_assert(Out::BYTES <= 2 * P::LDS, "outputs pass through the operands' LDS");
    const long long square = (long long)a.sp * a.sp;
    uint16_t* const out = (uint16_t*)a.out + k * square;
    const _Float16* const o = (const _Float16*)a.x.p + k * a.x_batch;  // second
    float* const d = a.d + (long long)k * a.sp;
    float* const e = a.e + (long long)k * a.sp;
    // rows and columns past sp stand in for the last ones where something is read
    const int r0 = m0 + P::wave_m() + P::row_of(), c0 = n0 + P::wave_n() + P::col_of();
    float dr[MT][4], dc[NT];
    if (SECOND) {
#pragma unroll
        for (int m = 0; m < MT; ++m) __builtin_memcpy(dr[m], d + min(r0 + m * 16, a.sp - 4), 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) dc[n] = d[min(c0 + n * 16, a.sp - 1)];
    }
    if (!mirror) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = r0 + m * 16 + j;
                    if (r != c0 + n * 16 || r >= a.sp) continue;
                    const float sum = p.acc[m][n][j] * a.down;
                    if (!SECOND) d[r] = sum;
                    else e[r] = fmaf(a.c, fmaf(dc[n], dc[n], sum), a.b * dc[n]);
                }
    }
    // Low parts in a pass of their own. What a lane holds is four rows of a column of sums: symmetric, so O is read as four neighbours of a row.
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        if (part) {
            lds_barrier();
            p.anew();
        }
        const Out staged;
        int r0 = m0 + P::wave_m() + P::row_of(), c0 = n0 + P::wave_n() + P::col_of();
        asm volatile("" : "+v"(r0), "+v"(c0));
        Raw4<PARTS> was[2][AHEAD];
        auto load = [&](int i) {  // of blocks i * AHEAD on, column by column
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int m = i * AHEAD % MT + u, n = i * AHEAD / MT;
                was[i & 1][u].load(o + (long long)min(c0 + n * 16, a.sp - 1) * a.sp + min(r0 + m * 16, a.sp - 4), a.x.plane);
            }
        };
        if (SECOND) load(0);
#pragma unroll
        for (int i = 0; i < MT * NT / AHEAD; ++i) {
            if (SECOND && i + 1 < MT * NT / AHEAD) load(i + 1);
            __builtin_amdgcn_sched_barrier(0);  // so far ahead and no further, which would not fit the registers
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                const int m = i * AHEAD % MT + u, n = i * AHEAD / MT;
                uint16_t v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    float w = p.acc[m][n][j] * a.down;
                    if (SECOND) {
                        const float ov = was[i & 1][u].get(j) * a.unlift;
                        w = fmaf(a.c, fmaf(dc[n] + dr[m][j], ov, w), a.b * ov);
                    }
                    _Float16 hi, lo;
                    two_parts(w * a.lift, hi, lo);
                    v[j] = __builtin_bit_cast(uint16_t, part ? lo : hi);
                }
                staged.put(lds, m, n, v);
            }
        }
        if (!mirror) {  // the diagonal is kept as d or e
            lds_barrier();
            const int r = max(m0, n0) + (int)threadIdx.x;
            if (r < min(m0 + P::BM, n0 + P::BN)) *(uint16_t*)((char*)lds + Out::place(r - n0, (r - m0) / 8) + (r - m0) % 8 * 2) = 0;
        }
        lds_barrier();
        uint16_t* const to = out + (part ? a.plane : 0);
#pragma unroll
        for (int i = 0; i < Out::PER; ++i) {
            if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
            int row, col;
            staged.where(i, 0, row, col);
            row += n0, col += m0;
            if (row < a.sp && col < a.sp) *(u32x4*)(to + (long long)row * a.sp + col) = staged.take(lds, i);
        }
        if (mirror) {
#pragma unroll
            for (int i = 0; i < Out::ACROSS; ++i) {
                if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                int row, col;
                staged.where_across(i, row, col);
                row += m0, col += n0;
                const s16x8 v = staged.take_across(lds, i);
                if (row < a.sp && col < a.sp) *(s16x8*)(to + (long long)row * a.sp + col) = v;
            }
        }
    }
}

// A tile on or below the diagonal of a symmetric product, all of its sum. 4096 x 4096 is 136 tiles of 256, one round of 92 us on half the compute units, or 253 of
// 192, one round of 71 on all of them (the second product 98 and 75). Of that a tile's way in and out is 15 us.
template <int MW, int NW, int MT, int NT, bool SUMS, bool SECOND, int PAIRS>
__global__ __launch_bounds__(MW * NW * 64) void k_square(const SquareArgs a) {
    typedef Products<_Float16, MW, NW, MT, NT, SUMS, SUMS, PAIRS> P;
    static_assert(P::BM == P::BN, "tiles of a symmetric product are square");
    __shared__ __align__(16) uint16_t lds[P::LDS];
    const int k = blockIdx.y;
    int ti, tj;
    place_triangle(by_die(blockIdx.x, gridDim.x), a.tiles, ti, tj);
    Side x = a.x;
    x.p += k * a.x_batch;
    P p;
    p.run(x, x, ti * P::BM, tj * P::BN, 0, a.kts, lds);
    finish_square<P, MW, NW, SECOND, PAIRS>(a, p, k, ti * P::BM, tj * P::BN, ti != tj, lds);
}

// The same where tiles are few or do not go round the compute units evenly: all tiles' steps along their sums are one line, of which every workgroup takes
// an equal piece, through the ends of tiles. A piece's part of a tile is kept as sums, in the order in which lanes hold them, in place piece + tile, and a
// second kernel adds a tile's parts up. The 4096 x 4096 above takes 75 and 29 us this way, more than tiles of 192; 1111 x 520 in
// 32 bits 10.9 and 10 where tiles of 64 take 16.4. It is for few tiles of long sums: 700 x 8200, 6 tiles of 256 with 128 steps.
__device__ __forceinline__ long long piece_begin(const SquareArgs& a, long long w) { return w * a.units / a.pieces; }
__device__ __forceinline__ long long piece_of(const SquareArgs& a, long long unit) { return ((unit + 1) * a.pieces - 1) / a.units; }

template <int MW, int NW, int MT, int NT, bool SUMS, int PAIRS>
__global__ __launch_bounds__(MW * NW * 64) void k_square_piece(const SquareArgs a) {
    typedef Products<_Float16, MW, NW, MT, NT, SUMS, SUMS, PAIRS> P;
    __shared__ __align__(16) uint16_t lds[P::LDS];
    const int w = by_die(blockIdx.x, gridDim.x);
    const long long begin = piece_begin(a, w);
    const int per = a.tiles * (a.tiles + 1) / 2;
    // the same in all lanes, which the compiler does not see behind a division
    int left = __builtin_amdgcn_readfirstlane((int)(piece_begin(a, w + 1) - begin)), tile = __builtin_amdgcn_readfirstlane((int)(begin / a.kts));
    int kt0 = __builtin_amdgcn_readfirstlane((int)(begin - (long long)tile * a.kts));
    for (; left > 0; ++tile, kt0 = 0) {
        const int kt1 = min(a.kts, kt0 + left), k = __builtin_amdgcn_readfirstlane(tile / per);
        int ti, tj;
        place_triangle(tile - k * per, a.tiles, ti, tj);
        ti = __builtin_amdgcn_readfirstlane(ti), tj = __builtin_amdgcn_readfirstlane(tj);
        Side x = a.x;
        x.p += k * a.x_batch;
        P p;
        p.run(x, x, ti * P::BM, tj * P::BN, kt0, kt1, lds);
        f32x4* const to = (f32x4*)a.parts + ((long long)(w + tile) * (MW * NW) + (threadIdx.x >> 6)) * (MT * NT * 64) + (threadIdx.x & 63);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) to[(m * NT + n) * 64] = p.acc[m][n];
        left -= kt1 - kt0;
    }
}

// A wave's part of a tile to a workgroup.
template <int MW, int NW, int MT, int NT, bool SECOND, int PAIRS>
__global__ __launch_bounds__(64) void k_square_join(const SquareArgs a) {
    typedef Products<_Float16, 1, 1, MT, NT, false, false, PAIRS> P;
    constexpr int WAVES = MW * NW;
    __shared__ __align__(16) uint16_t lds[Staged<P, uint16_t, 1, NT>::BYTES / 2];
    const int tile = blockIdx.x / WAVES, wave = blockIdx.x % WAVES, per = a.tiles * (a.tiles + 1) / 2, k = tile / per;
    int ti, tj;
    place_triangle(tile - k * per, a.tiles, ti, tj);
    P p;
    const int first = (int)piece_of(a, (long long)tile * a.kts), last = (int)piece_of(a, (tile + 1ll) * a.kts - 1);
    const f32x4* from = (const f32x4*)a.parts + ((long long)(first + tile) * WAVES + wave) * (MT * NT * 64) + threadIdx.x;
    constexpr int PART = WAVES * MT * NT * 64, AT_ONCE = 64 / (MT * NT);  // parts in flight, 256 registers
    p.clear();
    for (int w = first; w <= last; w += AT_ONCE, from += AT_ONCE * PART) {
        f32x4 v[AT_ONCE][MT * NT];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (w + u <= last) {
#pragma unroll
                for (int i = 0; i < MT * NT; ++i) v[u][i] = from[u * PART + i * 64];
            }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u)
            if (w + u <= last) {
#pragma unroll
                for (int i = 0; i < MT * NT; ++i) p.acc[i / NT][i % NT] += v[u][i];
            }
    }
    finish_square<P, 1, 1, SECOND, PAIRS>(a, p, k, ti * (MW * P::BM) + wave / NW * P::BM, tj * (NW * P::BN) + wave % NW * P::BN, ti != tj, lds);
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

// A pass of results, to the gradient's place or into the weights. Weights are read eight rows' chunks ahead.
template <typename TO, class Out>
__device__ __forceinline__ void deliver(const Target& t, int k, const Shape& z, int r0, int c0, int pass, const void* lds) {
    constexpr int AT_ONCE = 4;
    const Out staged;
    TO* const to = t.batch ? (TO*)t.w[0] + k * t.batch : (TO*)t.w[k];
#pragma unroll
    for (int i = 0; i < Out::PER; i += AT_ONCE) {
        float was[AT_ONCE][4];
        int r[AT_ONCE], c[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            staged.where(i + u, pass, r[u], c[u]);
            r[u] += r0, c[u] += c0;
            if (t.update && r[u] < z.rows && c[u] < z.cols) get_quad(to + r[u] * t.stride + c[u], z.cols - c[u], was[u]);
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; ++u) {
            if (r[u] >= z.rows || c[u] >= z.cols) continue;
            float v[4];
            const u32x4 w = staged.take(lds, i + u);
            __builtin_memcpy(v, &w, 16);
            if (t.update) {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = fmaf(t.keep, was[u][j], t.by * v[j]);
            }
            put_quad(to + r[u] * t.stride + c[u], z.cols - c[u], v);
        }
    }
}

template <typename TO>
__device__ __forceinline__ void deliver_quad(const Target& t, int k, int r, int c, int n, float (&v)[4]) {
    TO* const to = (t.batch ? (TO*)t.w[0] + k * t.batch : (TO*)t.w[k]) + r * t.stride + c;
    if (t.update) {
        float was[4];
        get_quad(to, n, was);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = fmaf(t.keep, was[j], t.by * v[j]);
    }
    put_quad(to, n, v);
}

// 4096 x 4096: 132 to 136 us (1010 to 1040 TFLOP/s) of which 97 are the products at the rate of long sums: every compute unit has one tile, so that nothing covers
// its first loads, and its 64 KB of X in two parts read and written.
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
    // in place: what the sums are to be. Columns and rows past the matrix stand in for the last ones where something is read.
    const int c0 = tm * P::BM, r0 = tn * P::BN, cl = c0 + P::wave_m() + P::row_of(), rl = r0 + P::wave_n() + P::col_of();
    float ec[MT][4];
    if (TALL) {
#pragma unroll
        for (int m = 0; m < MT; ++m) __builtin_memcpy(ec[m], e + min(cl + m * 16, a.z.cp - 4), 16);
    }
    constexpr int AHEAD = MT % 4 == 0 ? 4 : MT % 3 == 0 ? 3 : MT;
    Raw4<2> x0[2][AHEAD];
    auto load = [&](int i) {  // of blocks i * AHEAD on, column by column
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int m = i * AHEAD % MT + u, n = i * AHEAD / MT;
            x0[i & 1][u].load(was + (long long)min(rl + n * 16, a.z.rp - 1) * a.z.cp + min(cl + m * 16, a.z.cp - 4), x.plane);
        }
    };
    float er[NT];
    if (!TALL) {
#pragma unroll
        for (int n = 0; n < NT; ++n) er[n] = e[min(rl + n * 16, a.z.rp - 1)];
    }
    load(0);
#pragma unroll
    for (int i = 0; i < MT * NT / AHEAD; ++i) {
        if (i + 1 < MT * NT / AHEAD) load(i + 1);
        __builtin_amdgcn_sched_barrier(0);  // so far ahead and no further, which would not fit the registers
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int m = i * AHEAD % MT + u, n = i * AHEAD / MT;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                p.acc[m][n][j] = fmaf(a.a + (TALL ? ec[m][j] : er[n]), x0[i & 1][u].get(j) * a.unlift, p.acc[m][n][j] * a.down);
        }
    }
    if (a.to) {
        typedef Staged<P, uint16_t, NW, NT> Out;
        static_assert(Out::BYTES <= 2 * P::LDS, "outputs pass through the operands' LDS");
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            if (part) {
                lds_barrier();
                p.anew();
            }
            const Out staged;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    uint16_t v[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        _Float16 hi, lo;
                        two_parts(p.acc[m][n][j] * a.lift, hi, lo);
                        v[j] = __builtin_bit_cast(uint16_t, part ? lo : hi);
                    }
                    staged.put(lds, m, n, v);
                }
            lds_barrier();
            uint16_t* const to = (uint16_t*)a.to + k * a.x_batch + (part ? a.plane : 0);
#pragma unroll
            for (int i = 0; i < Out::PER; ++i) {
                if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                int row, col;
                staged.where(i, 0, row, col);
                row += r0, col += c0;
                if (row < a.z.rp && col < a.z.cp) *(u32x4*)(to + (long long)row * a.z.cp + col) = staged.take(lds, i);
            }
        }
        return;
    }
    typedef Staged<P, float, NW, 2> Out;
    static_assert(Out::BYTES <= 2 * P::LDS, "outputs pass through the operands' LDS");
#pragma unroll
    for (int pass = 0; pass < Out::PASSES; ++pass) {
        if (pass) lds_barrier();
        const Out staged;
#pragma unroll
        for (int n = 2 * pass; n < 2 * pass + 2; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float v[4] = {p.acc[m][n][0], p.acc[m][n][1], p.acc[m][n][2], p.acc[m][n][3]};
                staged.put(lds, m, n, v);
            }
        lds_barrier();
        if (type == IODF_T_F32) deliver<float, Out>(target, k, a.z, r0, c0, pass, lds);
        else if (type == IODF_T_BF16) deliver<__bf16, Out>(target, k, a.z, r0, c0, pass, lds);
        else deliver<_Float16, Out>(target, k, a.z, r0, c0, pass, lds);
    }
}

// ---- a short side of at most 64 ----

struct SlimArgs {
    _Float16* x;            // [matrix][rp][cp] in two parts; every workgroup changes its own blocks
    long long plane;
    Shape z;
    int groups, per;        // workgroups to a matrix, blocks of 64 along the longer side to a workgroup
    const float* from;      // [matrix][workgroup][64][64], parts of X X' times 2^(2 x_exp)
    float* to;
    OrthSteps steps;
};

// A workgroup adds up A's parts, has A^2 and b A + c A^2 in LDS, applies it to its own blocks of X, and adds what these give to the next A. That is a step
// with one launch (KIND STEP; FIRST: only the first A; LAST: the result goes to `target`), and where a workgroup has a whole matrix (ALL: at most 256 along
// the longer side) all steps with one, norm and start included. What bounds it is the launch and a dozen dependent trips to memory and LDS a step. As three
// launches a step 64 x 300 and 64 x 64 take 85 us, here 51 and 22.
enum { SLIM_FIRST, SLIM_STEP, SLIM_LAST, SLIM_ALL };

template <bool TALL, int PAIRS, int KIND, bool MUON>
__global__ __launch_bounds__(256) void k_slim(const SlimArgs a, const int step, const Source src, const int in_type, const float eps, const Target target,
                                              const int type) {
    constexpr int PARTS = PAIRS > 1 ? 2 : 1, S = 64;
    // X as its product reads it, and the next X as its own square does
    __shared__ __align__(16) uint16_t o[PARTS][S * S], m[PARTS][S * S], x[2][S * S], y[2][S * S];
    __shared__ __align__(16) float d[S], e[S];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, low = lane & 15, q = wave * 16 + lane / 16 * 4;
    const int k = blockIdx.y, g = blockIdx.x;
    auto in_rows = [](int r, int c) { return r * S + ((c / 8) ^ (r >> 1 & 7)) * 8 + c % 8; };
    auto in_sums = [](int r, int c) { return r * S + Lane<S, 64, true>::chunk(r, c / 8) * 8 + c % 8; };
    auto rows = [&](const uint16_t* t, int r0, int step) { return *(const s16x8*)(t + in_rows(r0 + low, step * 32 + lane / 16 * 8)); };
    auto sums = [&](const uint16_t* t, int c0, int step) {
        const int r = step * 32 + lane / 16 * 8 + (lane >> 2 & 3), c = c0 + (lane & 3) * 4;
        union { s16x4 h[2]; s16x8 v; } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + in_sums(r, c)));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + in_sums(r + 4, c)));
        return u.v;
    };
    // acc[n] += rows q .. q + 3 of one operand by columns 16 n + low of the other, fragments by plane, block and step; small products first
    auto multiply = [&](f32x4 (&acc)[4], auto left, auto right) {
#pragma unroll
        for (int p = PAIRS > 1 ? 0 : 2; p < 3; ++p)
#pragma unroll
            for (int step = 0; step < 2; ++step) {
                const s16x8 l = left(p == 1, step);
#pragma unroll
                for (int n = 0; n < 4; ++n) acc[n] = Mma<_Float16>::go(l, right(p == 0, n, step), acc[n]);
            }
    };
    auto put4 = [](uint16_t (*t)[S * S], int parts, int at, const float (&v)[4]) {
        _Float16 hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) two_parts(v[j], hi[j], lo[j]);
        __builtin_memcpy(&t[0][at], hi, 8);
        if (parts > 1) __builtin_memcpy(&t[parts - 1][at], lo, 8);
    };
    auto get = [](const uint16_t (*t)[S * S], int parts, int at, float (&v)[4]) {
        _Float16 hi[4], lo[4];
        __builtin_memcpy(hi, &t[0][at], 8);
        if (parts > 1) __builtin_memcpy(lo, &t[parts - 1][at], 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)hi[j] + (parts > 1 ? (float)lo[j] : 0.f);
    };

    // this workgroup's blocks of X, sixteen bytes at a time: asked for a block ahead
    const long long n = (long long)a.z.rp * a.z.cp;
    uint16_t* const xs = (uint16_t*)a.x + k * n;
    const int first = g * a.per, last = min((TALL ? a.z.rp : a.z.cp) / S, first + a.per);
    u32x4 raw[2][2];
    auto place = [&](int block, int i) {  // of chunk i of the thread's, in memory
        const int r = (i * 256 + tid) / 8, c = (i * 256 + tid) % 8 * 8;
        return TALL ? (long long)(block * S + r) * a.z.cp + c : (long long)r * a.z.cp + block * S + c;
    };
    auto ask = [&](int block) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
            for (int i = 0; i < 2; ++i) raw[p][i] = *(const u32x4*)(xs + p * a.plane + place(block, i));
    };
    if (KIND == SLIM_ALL) {
        __shared__ double meet[4];
        auto begin = [&](auto t) {
            typedef decltype(t) TG;
            const double by = (double)ldexpf(1.f, a.steps.x_exp[0]) / (sqrt(block_sum(squares<TG, MUON>(src, a.z, k, tid, 256), meet)) + (double)eps);
            start_x<TG, MUON>(src, a.z, k, by, a.x, a.plane, tid, 256);
        };
        if (in_type == IODF_T_F32) begin(0.f);
        else if (in_type == IODF_T_BF16) begin((__bf16)0.f);
        else begin((_Float16)0.f);
        __syncthreads();
    }
    ask(first);

    const bool stays = KIND == SLIM_ALL && a.per == 1;  // X never leaves LDS
    // four neighbours of A's row r
    auto put_a = [&](int r, int c, const f32x4& s, float square, float lift) {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = s[j] * square;
            if (r == c + j) d[r] = v[j];
            v[j] = r == c + j ? 0.f : v[j] * lift;
        }
        put4(o, PARTS, in_rows(r, c), v);
    };
    f32x4 next[4] = {};
    // step i; `begin`: only the first A
    auto pass = [&](int i, auto begin, auto end) {
        const float unlift = begin ? 0.f : ldexpf(1.f, -a.steps.x_exp[i]), lift = ldexpf(1.f, a.steps.x_exp[i + 1]);
        const float o_lift = begin ? 0.f : ldexpf(1.f, a.steps.a_exp[i]), b_lift = begin ? 1.f : ldexpf(1.f, a.steps.b_exp[i]);
        const float ca = begin ? 0.f : a.steps.a[i], cb = begin ? 0.f : a.steps.b[i], cc = begin ? 0.f : a.steps.c[i];
        if (!begin) {
            if (KIND == SLIM_ALL) {  // symmetric: four rows of a column are four neighbours of a row
#pragma unroll
                for (int b = 0; b < 4; ++b) put_a(b * 16 + low, q, next[b], unlift * unlift, o_lift);
            } else {
                f32x4 s[4] = {};
                const float* from = a.from + (long long)k * a.groups * S * S + tid * 4;
                for (int w = 0; w < a.groups; w += 8) {
                    f32x4 v[8][4];
#pragma unroll
                    for (int u = 0; u < 8; ++u)
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[u][j] = w + u < a.groups ? *(const f32x4*)(from + (w + u) * S * S + j * 1024) : f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int u = 0; u < 8; ++u)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[j] += v[u][j];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) put_a(j * 16 + tid / 16, tid % 16 * 4, s[j], unlift * unlift, o_lift);
            }
            lds_barrier();
            f32x4 acc[4] = {};
            multiply(acc, [&](int p, int step) { return rows(o[p * (PARTS - 1)], wave * 16, step); },
                     [&](int p, int b, int step) { return rows(o[p * (PARTS - 1)], b * 16, step); });
            const float down = 1.f / (o_lift * o_lift), un = 1.f / o_lift;
#pragma unroll
            for (int b = 0; b < 4; ++b) {  // symmetric again
                const int r = b * 16 + low;
                float was[4], v[4];
                get(o, PARTS, in_rows(r, q), was);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float sum = acc[b][j] * down, ov = was[j] * un;
                    if (r == q + j) e[r] = fmaf(cc, fmaf(d[r], d[r], sum), cb * d[r]);
                    v[j] = r == q + j ? 0.f : fmaf(cc, fmaf(d[r] + d[q + j], ov, sum), cb * ov) * b_lift;
                }
                put4(m, PARTS, in_rows(r, q), v);
            }
        }
#pragma unroll
        for (int b = 0; b < 4; ++b) next[b] = f32x4{0.f, 0.f, 0.f, 0.f};
        const float down = unlift / b_lift;
        for (int block = first; block < last; ++block) {
            lds_barrier();
            uint16_t (*const into)[S * S] = begin ? y : x;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int r = (i * 256 + tid) / 8, c = (i * 256 + tid) % 8 * 8;
                    u32x4 w = raw[p][i];
                    if (stays && !begin) w = *(const u32x4*)&y[p][TALL ? in_sums(r, c) : in_rows(r, c)];
                    *(u32x4*)&into[p][begin != TALL ? in_rows(r, c) : in_sums(r, c)] = w;
                }
            if (block + 1 < last) ask(block + 1);
            lds_barrier();
            if (!begin) {
                // outputs q .. q + 3 of a row of X's memory, 16 b + low
                f32x4 acc[4] = {};
                if (TALL)
                    multiply(acc, [&](int p, int step) { return rows(m[p * (PARTS - 1)], wave * 16, step); },
                             [&](int p, int b, int step) { return rows(x[p], b * 16, step); });
                else
                    multiply(acc, [&](int p, int step) { return sums(x[p], wave * 16, step); },
                             [&](int p, int b, int step) { return rows(m[p * (PARTS - 1)], b * 16, step); });
                float v[4][4];
#pragma unroll
                for (int b = 0; b < 4; ++b) {
                    const int r = b * 16 + low;
                    get(x, 2, TALL ? in_rows(r, q) : in_sums(r, q), v[b]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[b][j] = fmaf(ca + e[TALL ? q + j : r], v[b][j] * unlift, acc[b][j] * down) * (end ? 1.f : lift);
                    if (!end) put4(y, 2, TALL ? in_sums(r, q) : in_rows(r, q), v[b]);
                }
                if (end) {
                    float* const t = (float*)y;  // rows of 64 numbers, to be delivered as they lie
#pragma unroll
                    for (int b = 0; b < 4; ++b) __builtin_memcpy(t + (b * 16 + low) * S + (q ^ (low & 7) * 4), v[b], 16);
                    lds_barrier();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 16 + tid / 16, c = tid % 16 * 4, row = TALL ? block * S + r : r, col = TALL ? c : block * S + c;
                        if (row >= a.z.rows || col >= a.z.cols) continue;
                        float w[4];
                        __builtin_memcpy(w, t + r * S + (c ^ (r & 7) * 4), 16);
                        if (type == IODF_T_F32) deliver_quad<float>(target, k, row, col, a.z.cols - col, w);
                        else if (type == IODF_T_BF16) deliver_quad<__bf16>(target, k, row, col, a.z.cols - col, w);
                        else deliver_quad<_Float16>(target, k, row, col, a.z.cols - col, w);
                    }
                    continue;
                }
                lds_barrier();
#pragma unroll
                for (int p = 0; p < 2; ++p)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int r = (i * 256 + tid) / 8, c = (i * 256 + tid) % 8 * 8;
                        if (!stays) *(u32x4*)(xs + p * a.plane + place(block, i)) = *(const u32x4*)&y[p][TALL ? in_sums(r, c) : in_rows(r, c)];
                    }
            }
            if (TALL)
                multiply(next, [&](int p, int step) { return sums(y[p], wave * 16, step); }, [&](int p, int b, int step) { return sums(y[p], b * 16, step); });
            else
                multiply(next, [&](int p, int step) { return rows(y[p], wave * 16, step); }, [&](int p, int b, int step) { return rows(y[p], b * 16, step); });
        }
    };
    const std::true_type yes;
    const std::false_type no;
    if (KIND == SLIM_LAST) return pass(step, no, yes);
    if (KIND == SLIM_STEP) pass(step, no, no);
    else pass(-1, yes, no);
    if (KIND == SLIM_ALL) {
        for (int i = 0; i < a.steps.n; ++i) {
            if (!stays) {
                __syncthreads();  // X is in memory
                ask(first);
            }
            if (i + 1 < a.steps.n) pass(i, no, no);
            else pass(i, no, yes);
        }
        return;
    }
    float* const to = a.to + ((long long)k * a.groups + g) * S * S;
#pragma unroll
    for (int b = 0; b < 4; ++b) *(f32x4*)(to + (b * 16 + low) * S + q) = next[b];
}

// ---- one block of 128 x 128 ----

// A matrix of 65 to 128 rows and columns, all of it in a workgroup's LDS with zeros around it, X in two parts and A, then b A + c A^2, in the place of each other. Norm, start
// and all steps in one launch; tall ones go as the others do, which in a square of zeros is the same. A step reads a megabyte of fragments (three with both parts): LDS is busy
// for half of the time, the matrix units for an eighth, and the rest is the dependent ways between three products. 128 x 128 in bfloat16 51 us, as three launches a step 69.
template <int PAIRS, bool MUON>
__global__ __launch_bounds__(512) void k_block(const Shape z, const OrthSteps steps, const Source src, const int in_type, const float eps, const Target target,
                                               const int type) {
    constexpr int PARTS = PAIRS > 1 ? 2 : 1, S = 128;
    __shared__ __align__(16) uint16_t a[PARTS][S * S], x[2][S * S];
    __shared__ __align__(16) float d[S], e[S];
    __shared__ double meet[8];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, low = lane & 15, q = wave * 16 + lane / 16 * 4, k = blockIdx.x;
    auto at = [](int r, int c) { return r * S + ((c / 8) ^ (r >> 1 & 7)) * 8 + c % 8; };
    auto rows = [&](const uint16_t* t, int r0, int step) { return *(const s16x8*)(t + at(r0 + low, step * 32 + lane / 16 * 8)); };
    auto sums = [&](const uint16_t* t, int c0, int step) {
        const int r = step * 32 + lane / 16 * 8 + (lane >> 2 & 3), c = c0 + (lane & 3) * 4;
        union { s16x4 h[2]; s16x8 v; } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + at(r, c)));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(t + at(r + 4, c)));
        return u.v;
    };
    // four neighbours q .. q + 3 of row 16 b + low, small products first
    f32x4 acc[8];
    auto multiply = [&](auto left, auto right) {
#pragma unroll
        for (int b = 0; b < 8; ++b) acc[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = PAIRS > 1 ? 0 : 2; p < 3; ++p)
#pragma unroll
            for (int step = 0; step < S / 32; ++step) {
                const s16x8 l = left(p == 1, step);
#pragma unroll
                for (int b = 0; b < 8; ++b) acc[b] = Mma<_Float16>::go(l, right(p == 0, b, step), acc[b]);
            }
    };
    auto put4 = [](uint16_t (*t)[S * S], int parts, int to, const float (&v)[4]) {
        _Float16 hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) two_parts(v[j], hi[j], lo[j]);
        __builtin_memcpy(&t[0][to], hi, 8);
        if (parts > 1) __builtin_memcpy(&t[parts - 1][to], lo, 8);
    };
    auto get4 = [](const uint16_t (*t)[S * S], int parts, int from, float (&v)[4]) {
        _Float16 hi[4], lo[4];
        __builtin_memcpy(hi, &t[0][from], 8);
        if (parts > 1) __builtin_memcpy(lo, &t[parts - 1][from], 8);
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = (float)hi[j] + (parts > 1 ? (float)lo[j] : 0.f);
    };
    auto begin = [&](auto t) {
        typedef decltype(t) TG;
        double s = squares<TG, MUON>(src, z, k, tid, 512);
#pragma unroll
        for (int i = 1; i < 64; i *= 2) s += __shfl_xor(s, i);
        if (lane == 0) meet[wave] = s;
        __syncthreads();  // momenta are in memory, too
        s = 0.0;
        for (int w = 0; w < 8; ++w) s += meet[w];
        const double by = (double)ldexpf(1.f, steps.x_exp[0]) / (sqrt(s) + (double)eps);
#pragma unroll
        for (int i = 0; i < S * S / 8 / 512; ++i) {
            const int r = (i * 512 + tid) / (S / 8), c = (i * 512 + tid) % (S / 8) * 8;
            float v[8] = {};
            if (r < z.rows && c < z.cols) taken<TG, MUON, false>(src, k, r, c, z.cols, v);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                float w[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) w[j] = c + h * 4 + j < z.cols ? (float)(v[h * 4 + j] * by) : 0.f;
                put4(x, 2, at(r, c + h * 4), w);
            }
        }
        __syncthreads();
    };
    if (in_type == IODF_T_F32) begin(0.f);
    else if (in_type == IODF_T_BF16) begin((__bf16)0.f);
    else begin((_Float16)0.f);
    for (int i = 0; i < steps.n; ++i) {
        const bool end = i + 1 == steps.n;
        const float unlift = ldexpf(1.f, -steps.x_exp[i]), lift = end ? 1.f : ldexpf(1.f, steps.x_exp[i + 1]);
        const float o_lift = ldexpf(1.f, steps.a_exp[i]), b_lift = ldexpf(1.f, steps.b_exp[i]), ca = steps.a[i], cb = steps.b[i], cc = steps.c[i];
        multiply([&](int p, int step) { return rows(x[p], wave * 16, step); }, [&](int p, int b, int step) { return rows(x[p], b * 16, step); });
#pragma unroll
        for (int b = 0; b < 8; ++b) {  // symmetric: four rows of a column are four neighbours of a row
            const int r = b * 16 + low;
            float v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = acc[b][j] * (unlift * unlift);
                if (r == q + j) d[r] = v[j];
                v[j] = r == q + j ? 0.f : v[j] * o_lift;
            }
            put4(a, PARTS, at(r, q), v);
        }
        lds_barrier();
        multiply([&](int p, int step) { return rows(a[p * (PARTS - 1)], wave * 16, step); },
                 [&](int p, int b, int step) { return rows(a[p * (PARTS - 1)], b * 16, step); });
        const float down = 1.f / (o_lift * o_lift), un = 1.f / o_lift;
        float v[8][4];
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const int r = b * 16 + low;
            get4(a, PARTS, at(r, q), v[b]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float sum = acc[b][j] * down, ov = v[b][j] * un;
                if (r == q + j) e[r] = fmaf(cc, fmaf(d[r], d[r], sum), cb * d[r]);
                v[b][j] = r == q + j ? 0.f : fmaf(cc, fmaf(d[r] + d[q + j], ov, sum), cb * ov) * b_lift;
            }
        }
        lds_barrier();  // A has been read by all
#pragma unroll
        for (int b = 0; b < 8; ++b) put4(a, PARTS, at(b * 16 + low, q), v[b]);
        lds_barrier();
        multiply([&](int p, int step) { return sums(x[p], wave * 16, step); }, [&](int p, int b, int step) { return rows(a[p * (PARTS - 1)], b * 16, step); });
        const float back = unlift / b_lift;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const int r = b * 16 + low;
            get4(x, 2, at(r, q), v[b]);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[b][j] = fmaf(ca + e[r], v[b][j] * unlift, acc[b][j] * back) * lift;
        }
        lds_barrier();  // X has been read by all
        if (!end) {
#pragma unroll
            for (int b = 0; b < 8; ++b) put4(x, 2, at(b * 16 + low, q), v[b]);
            lds_barrier();
            continue;
        }
        float* const t = (float*)x;  // rows of 128 numbers, to be delivered as they lie
#pragma unroll
        for (int b = 0; b < 8; ++b) __builtin_memcpy(t + (b * 16 + low) * S + (q ^ (low & 7) * 4), v[b], 16);
        lds_barrier();
#pragma unroll
        for (int n = 0; n < S * S / 4 / 512; ++n) {
            const int r = n * 16 + tid / 32, c = tid % 32 * 4;
            if (r >= z.rows || c >= z.cols) continue;
            float w[4];
            __builtin_memcpy(w, t + r * S + (c ^ (r & 7) * 4), 16);
            if (type == IODF_T_F32) deliver_quad<float>(target, k, r, c, z.cols - c, w);
            else if (type == IODF_T_BF16) deliver_quad<__bf16>(target, k, r, c, z.cols - c, w);
            else deliver_quad<_Float16>(target, k, r, c, z.cols - c, w);
        }
    }
}

template <bool WHOLE, int MW, int NW, int MT, int NT, bool SUMS, bool SECOND, int PAIRS>
void square_with(SquareArgs a, const Cut& cut, int count, hipStream_t st) {
    const int per = cut.tiles * (cut.tiles + 1) / 2;
    a.tiles = cut.tiles, a.pieces = cut.pieces, a.units = (long long)count * per * a.kts;
    if constexpr (WHOLE) {
        k_square<MW, NW, MT, NT, SUMS, SECOND, PAIRS><<<dim3((unsigned)per, count), MW * NW * 64, 0, st>>>(a);
    } else {
        k_square_piece<MW, NW, MT, NT, SUMS, PAIRS><<<(unsigned)cut.pieces, MW * NW * 64, 0, st>>>(a);
        k_square_join<MW, NW, MT, NT, SECOND, PAIRS><<<(unsigned)(count * per * MW * NW), 64, 0, st>>>(a);
    }
}
template <bool SUMS, bool SECOND, int PAIRS>
void square(const SquareArgs& a, const Cut& cut, int count, hipStream_t st) {
    if (cut.pieces && cut.edge == 256) square_with<false, 2, 4, 8, 4, SUMS, SECOND, PAIRS>(a, cut, count, st);
    else if (cut.pieces) square_with<false, 2, 2, 4, 4, SUMS, SECOND, PAIRS>(a, cut, count, st);
    else if (cut.edge == 256) square_with<true, 2, 4, 8, 4, SUMS, SECOND, PAIRS>(a, cut, count, st);
    else if (cut.edge == 192) square_with<true, 2, 4, 6, 3, SUMS, SECOND, PAIRS>(a, cut, count, st);
    else square_with<true, 2, 2, 2, 2, SUMS, SECOND, PAIRS>(a, cut, count, st);
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
        q.down = 1.f / (xl * xl), q.lift = ol, q.out = o, q.parts = (float*)(work + p.pieces);
        square<TALL, false, PAIRS>(q, p.first, p.z.count, st);
        q.x = {(const uint16_t*)o, square_n * p.z.count, p.z.sp, p.z.sp, p.z.sp};
        q.x_batch = square_n, q.kts = p.z.sp / PK;
        q.down = 1.f / (ol * ol), q.unlift = 1.f / ol, q.lift = bl, q.b = s.b[i], q.c = s.c[i], q.out = b;
        square<false, true, PAIRS>(q, p.second, p.z.count, st);
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

template <bool TALL, int PAIRS>
void slim(const OrthPlan& p, const OrthSteps& s, char* work, const Target& target, int type, hipStream_t st) {
    SlimArgs a{};
    a.x = (_Float16*)(work + p.x0), a.plane = (long long)p.z.rp * p.z.cp * p.z.count, a.z = p.z, a.groups = p.groups, a.per = p.per, a.steps = s;
    float *parts = (float*)(work + p.pieces), *other = parts + (long long)p.z.count * p.groups * 64 * 64;
    const dim3 grid(p.groups, p.z.count);
    const Source none{};
    a.to = parts;
    k_slim<TALL, PAIRS, SLIM_FIRST, false><<<grid, 256, 0, st>>>(a, -1, none, 0, 0.f, target, type);
    for (int i = 0; i < s.n; ++i) {
        a.from = parts, a.to = other;
        if (i + 1 < s.n) k_slim<TALL, PAIRS, SLIM_STEP, false><<<grid, 256, 0, st>>>(a, i, none, 0, 0.f, target, type);
        else k_slim<TALL, PAIRS, SLIM_LAST, false><<<grid, 256, 0, st>>>(a, i, none, 0, 0.f, target, type);
        std::swap(parts, other);
    }
}

template <bool MUON>
hipError_t all_at_once(const Source& src, int in_type, const OrthPlan& p, const OrthSteps& s, float eps, char* work, const Target& target, int type, hipStream_t st) {
    if (p.block) {
        auto go = [&](auto kernel) { kernel<<<p.z.count, 512, 0, st>>>(p.z, s, src, in_type, eps, target, type); };
        p.parts ? go(k_block<3, MUON>) : go(k_block<1, MUON>);
        return hipGetLastError();
    }
    SlimArgs a{};
    a.x = (_Float16*)(work + p.x0), a.plane = (long long)p.z.rp * p.z.cp * p.z.count, a.z = p.z, a.groups = 1, a.per = p.per, a.steps = s;
    auto go = [&](auto kernel) { kernel<<<dim3(1, p.z.count), 256, 0, st>>>(a, 0, src, in_type, eps, target, type); };
    if (p.tall) p.parts ? go(k_slim<true, 3, SLIM_ALL, MUON>) : go(k_slim<true, 1, SLIM_ALL, MUON>);
    else p.parts ? go(k_slim<false, 3, SLIM_ALL, MUON>) : go(k_slim<false, 1, SLIM_ALL, MUON>);
    return hipGetLastError();
}

hipError_t run(const OrthPlan& p, const OrthSteps& s, char* work, const Target& t, int type, hipStream_t st) {
    if (p.groups) {
        if (p.tall) p.parts ? slim<true, 3>(p, s, work, t, type, st) : slim<true, 1>(p, s, work, t, type, st);
        else p.parts ? slim<false, 3>(p, s, work, t, type, st) : slim<false, 1>(p, s, work, t, type, st);
        return hipGetLastError();
    }
    if (p.tall) p.parts ? polynomials<true, 3>(p, s, work, t, type, st) : polynomials<true, 1>(p, s, work, t, type, st);
    else p.parts ? polynomials<false, 3>(p, s, work, t, type, st) : polynomials<false, 1>(p, s, work, t, type, st);
    return hipGetLastError();
}

}  // namespace

// How large singular values, and with them every entry of X, of A and of b A + c A^2, can get: 0..1 at first, then as the polynomials say, two percent
// added for roundings.
bool orth_steps(int steps, const float* co, OrthSteps& s) {
    if (steps < 1 || steps > IODF_ORTH_MOST || !co) return false;
    s.n = steps;
    double most = 1.02;
    auto lift = [](double m) { return 14 - (int)std::ceil(std::log2(std::max(m, 1e-6))); };  // m times 2^that is at most 2^14
    for (int i = 0; i < steps; ++i) {
        const double a = co[3 * i], b = co[3 * i + 1], c = co[3 * i + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c)) return false;
        // in x = v^2: the polynomial turns where a + 3 b x + 5 c x^2 = 0, b x + c x^2 at -b / 2 c
        const double end = most * most;
        double next = 0.0, beside = 0.0;
        auto look = [&](double x) {
            if (!(x >= 0.0 && x <= end)) return;
            next = std::max(next, std::fabs(std::sqrt(x) * (a + x * (b + x * c))));
            beside = std::max(beside, std::fabs(x * (b + x * c)));
        };
        look(end);
        if (c != 0.0) {
            const double root = std::sqrt(9.0 * b * b - 20.0 * a * c);  // NaN: it does not turn
            look((-3.0 * b + root) / (10.0 * c));
            look((-3.0 * b - root) / (10.0 * c));
            look(-b / (2.0 * c));
        } else if (b != 0.0) {
            look(-a / (3.0 * b));
        }
        s.a[i] = (float)a, s.b[i] = (float)b, s.c[i] = (float)c;
        s.x_exp[i] = lift(most), s.a_exp[i] = lift(most * most), s.b_exp[i] = lift(1.02 * beside);
        most = std::max(1.02 * next, 1e-3);
        if (!(most <= 64.0) || !(beside <= 4096.0)) return false;
    }
    s.x_exp[steps] = lift(most);
    return true;
}

static size_t workspace(long long count, int rows, int cols, int type) {
    const long long most = together(count, rows, cols);
    return std::max(orth_plan(most, rows, cols, type).bytes, count % most ? orth_plan(count % most, rows, cols, type).bytes : 0);
}

size_t orth_workspace(const iodf_orth& a) { return workspace(a.count, a.rows, a.cols, a.out_type); }
size_t muon_workspace(const iodf_muon& a) { return workspace(a.count, a.rows, a.cols, a.weight_type); }

hipError_t launch_orthogonalise(const iodf_orth& a, const OrthSteps& s, void* work, hipStream_t st) {
    const long long most = together(a.count, a.rows, a.cols);
    auto size_of = [](int type) { return type == IODF_T_F32 ? 4 : 2; };
    hipError_t rc = hipSuccess;
    for (long long at = 0; at < a.count && rc == hipSuccess; at += most) {
        const OrthPlan p = orth_plan(std::min(most, a.count - at), a.rows, a.cols, a.out_type);
        Source src{};
        src.g[0] = (const char*)a.in + at * a.in_batch * size_of(a.in_type), src.stride = a.in_stride, src.batch = a.in_batch;
        Target t{};
        t.w[0] = (char*)a.out + at * a.out_batch * size_of(a.out_type), t.stride = a.out_stride, t.batch = a.out_batch;
        if (p.block || p.groups == 1) {
            rc = all_at_once<false>(src, a.in_type, p, s, a.eps, (char*)work, t, a.out_type, st);
        } else {
            begin<false>(src, a.in_type, p, a.eps, ldexpf(1.f, s.x_exp[0]), (char*)work, st);
            rc = run(p, s, (char*)work, t, a.out_type, st);
        }
    }
    return rc;
}

hipError_t launch_muon_step(const iodf_muon& a, const OrthSteps& s, void* work, hipStream_t st) {
    const long long most = together(a.count, a.rows, a.cols);
    hipError_t rc = hipSuccess;
    for (long long at = 0; at < a.count && rc == hipSuccess; at += most) {
        const OrthPlan p = orth_plan(std::min(most, a.count - at), a.rows, a.cols, a.weight_type);
        Source src{};
        Target t{};
        for (int k = 0; k < p.z.count; ++k) src.g[k] = a.grads[at + k], src.m[k] = a.momenta[at + k], t.w[k] = a.weights[at + k];
        src.stride = a.grad_stride, src.beta = a.beta, src.nesterov = a.nesterov;
        t.stride = a.weight_stride, t.update = 1;
        t.keep = (float)(1.0 - (double)a.rate * a.decay), t.by = (float)(-(double)a.rate * a.scale);
        if (p.block || p.groups == 1) {
            rc = all_at_once<true>(src, a.grad_type, p, s, a.eps, (char*)work, t, a.weight_type, st);
        } else {
            begin<true>(src, a.grad_type, p, a.eps, ldexpf(1.f, s.x_exp[0]), (char*)work, st);
            rc = run(p, s, (char*)work, t, a.weight_type, st);
        }
    }
    return rc;
}

}  // namespace iodf
