// Softmax cross entropy of rows against a table of classes, and its gradient: products of 16-bit numbers (products.h) whose logits never reach
// memory as such.
//
// 32-bit operands: the gradients' sums go over rows and over classes, so that no power of two of a row, class or tensor would do for all that a sum has in it. A class that is
// hardly a target has probabilities alone for its gradient, 1e-9 and less of the largest number of g, and what updates weights by the size of their gradients goes by those
// too. So there numbers are three parts of bfloat16, whose range is theirs: six products. 4096 rows, 32768 classes of 1024 columns 4.7 ms; two parts of half precision and
// three products, which leave a number of 2^-27 of the largest 12 bits, took 2.2. A logit's sum is over columns, and logits of the forward pass are of two parts of half
// precision with a power of two for each row and each class, three products.
//
// Forward: a workgroup has the logits of a tile of classes and rows in registers and leaves, for each of its rows, their largest and
// the sum of exponentials relative to it; a second kernel joins the tiles of a row. Backward: the logits once more, from which g = (dloss + dlse) exp(s -
// lse) - dloss [target] goes to memory in 16 bits, piece by piece of the classes; du += g W and dw = g' u are two more products.
#include <algorithm>
#include <type_traits>

#include "loss_plan.h"
#include "products.h"
#include "step.h"

namespace iodf {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ---- getting operands ready ----

__device__ __forceinline__ float finite_max(float m, float v) {
    v = fabsf(v);
    return v < __builtin_inff() && v > m ? v : m;
}
__device__ __forceinline__ float block_max(float m, float* meet) {  // 256 threads
#pragma unroll
    for (int k = 1; k < 64; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
    if ((threadIdx.x & 63) == 0) meet[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(meet[0], meet[1]), fmaxf(meet[2], meet[3]));
    __syncthreads();
    return m;
}

// The largest number that g is made of, of each workgroup's share. 1000 rows 3 us, the launch.
__global__ __launch_bounds__(256) void k_maxima(long long rows, const uint8_t* live, const float* dloss, const float* dlse, float* maxima) {
    __shared__ float meet[4];
    float m = 0.f;
    for (long long t = (long long)blockIdx.x * 256 + threadIdx.x; t < rows; t += (long long)gridDim.x * 256) {
        if (live && !live[t]) continue;
        const float d = dloss ? dloss[t] : 0.f;
        m = finite_max(finite_max(m, d), dlse ? dlse[t] + d : d);
    }
    m = block_max(m, meet);
    if (threadIdx.x == 0) maxima[blockIdx.x] = m;
}

// The power of two that takes numbers up to m to just below 2^15.
__device__ __forceinline__ float lift(float m, float& inverse) {
    int e = 0;
    if (m > 0.f) {
        frexpf(m, &e);
        e = min(126, max(-112, 15 - e));
    }
    inverse = ldexpf(1.f, -e);
    return ldexpf(1.f, e);
}

struct ReadyArgs {
    const void* x[2];      // u and W
    uint16_t* y[2];        // NULL: stays where it is
    long long stride[2], rows[2];
    const uint8_t* live;   // of u's rows
    int cols, pitch;
    const float* maxima;   // NULL: no scales
    int parts;             // partial maxima
    Scales* scales;
};

// v in three parts of bfloat16, whose sum it is (but for parts below the smallest numbers there are), whatever its size. An infinity is the last part: that is multiplied with
// first parts alone, which are 0 where the other number is, while others may be 0 where it is not, and 0 times an infinity is none.
__device__ __forceinline__ void three_parts(float v, uint16_t (&part)[3]) {
    constexpr uint32_t MOST = 0x7f7f0000;  // the largest, where rounding would make an infinity
    const bool endless = fabsf(v) == __builtin_inff();
    float left = endless ? 0.f : v;
#pragma unroll
    for (int p = 0; p < 3; ++p) {
        float h = (float)(__bf16)left;
        if (p == 0 && fabsf(h) == __builtin_inff()) h = copysignf(__uint_as_float(MOST), v);
        part[p] = (uint16_t)(__float_as_uint(h) >> 16);
        left = fabsf(h) < __builtin_inff() ? left - h : 0.f;  // NaN has no rest
    }
    if (endless) part[2] = (uint16_t)(__float_as_uint(v) >> 16);
}

// Rows of `pitch` 16-bit numbers with zeros behind, and padded rows as zeros: as they are, or 32-bit numbers in three parts of bfloat16. And the scales of g. At most
// 1024 workgroups for a tensor, with two chunks in flight a thread.
template <typename TX, int PARTS>
__global__ __launch_bounds__(256) void k_ready(const ReadyArgs a) {
    __shared__ float meet[4];
    const int which = blockIdx.y;
    const unsigned per = a.pitch / 8;
    if (a.maxima && blockIdx.x + blockIdx.y == 0) {
        float m = 0.f;
        for (int i = threadIdx.x; i < a.parts; i += 256) m = fmaxf(m, a.maxima[i]);
        m = block_max(m, meet);
        Scales r;
        r.g = lift(2.f * m, r.ig);
        if (m > 0.f) {  // and to make the largest a power of two, see lift_of
            int e;
            const float rest = frexpf(m, &e);
            r.g /= rest, r.ig *= rest;
        }
        if (threadIdx.x == 0) *a.scales = r;
    }
    uint16_t* const y = a.y[which];
    if (!y) return;
    const long long rows = a.rows[which], stride = a.stride[which], plane = rows * a.pitch;
    const uint8_t* const live = which ? nullptr : a.live;
    const unsigned all = (unsigned)(rows * per);  // fits, as rows times cols is 2^34 at most
    const unsigned step = gridDim.x * 256;
    constexpr int AT_ONCE = 2;  // in flight
    for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < all; i += AT_ONCE * step) {
        Raw8<TX> raw[AT_ONCE];
        long long to[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const unsigned at = min(i + k * step, all - 1);
            const long long t = at / per;
            const int c = (int)(at % per) * 8;
            raw[k] = fetch8((const TX*)a.x[which] + t * stride + c, live && !live[t] ? 0 : a.cols - c, false);
            to[k] = t * a.pitch + c;
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (i + k * step >= all) break;
            if (PARTS == 1) {
                *(u32x4*)(y + to[k]) = u32x4{raw[k].w[0], raw[k].w[1], raw[k].w[2], raw[k].w[3]};
                continue;
            }
            float v[8];
            widen8(raw[k], v);
            uint16_t part[3][8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint16_t of[3];
                three_parts(v[j], of);
                part[0][j] = of[0], part[1][j] = of[1], part[2][j] = of[2];
            }
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                u32x4 w;
                __builtin_memcpy(&w, part[p], 16);
                *(u32x4*)(y + p * plane + to[k]) = w;
            }
        }
    }
}

constexpr int kShift = 12;  // low parts of the forward pass are held times 2^12

struct RowsArgs {
    const float* x[2];     // u and W
    uint16_t* y[2];
    int* e[2];             // [row] the power of two that its numbers are of
    long long stride[2], rows[2];
    unsigned first;        // workgroups of u, those of W behind them
    const uint8_t* live;   // of u's rows
    int cols, pitch;
};

// 32-bit rows in two parts of half precision, times the power of two that takes a row's largest number to just below 2^15. The low part of that may be 8, and is held
// times 2^12: so numbers keep 22 bits down to 2^-29 of the row's largest, and what is left below is 2^-51 of it. SPAN threads to a row, which keep 32 of its numbers each and read
// what is longer twice. 1023 and 10007 rows of 1111 numbers 16.2 us, 6.1 TB/s.
template <int SPAN>
__global__ __launch_bounds__(256) void k_rows(const RowsArgs a) {
    __shared__ float meet[4];
    constexpr int KEEP = 4;
    const int which = blockIdx.x >= a.first, lane = threadIdx.x % SPAN;
    const long long t = (long long)(blockIdx.x - (which ? a.first : 0)) * (256 / SPAN) + threadIdx.x / SPAN;
    if (SPAN < 256 && t >= a.rows[which]) return;
    const float* const x = a.x[which] + t * a.stride[which];
    const int n = !which && a.live && !a.live[t] ? 0 : a.cols;
    Raw8<float> keep[KEEP];
    float m = 0.f;
    auto look = [&](const Raw8<float>& raw) {
        float v[8];
        widen8(raw, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) m = finite_max(m, v[j]);
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k) keep[k] = fetch8(x + (k * SPAN + lane) * 8, n - (k * SPAN + lane) * 8, false);
#pragma unroll
    for (int k = 0; k < KEEP; ++k) look(keep[k]);
    for (int c = (KEEP * SPAN + lane) * 8; c < n; c += SPAN * 8) look(fetch8(x + c, n - c, false));
    if (SPAN < 256) {
#pragma unroll
        for (int k = 1; k < SPAN; k *= 2) m = fmaxf(m, __shfl_xor(m, k));
    } else {
        m = block_max(m, meet);
    }
    int e = 15;
    if (m > 0.f) frexpf(m, &e);
    e -= 15;
    if (lane == 0) a.e[which][t] = e;
    const long long plane = a.rows[which] * a.pitch;
    uint16_t* const y = a.y[which] + t * a.pitch;
    auto put = [&](const Raw8<float>& raw, int c) {
        float v[8];
        widen8(raw, v);
        _Float16 hi[8], lo[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float s = ldexpf(v[j], -e);
            const bool endless = fabsf(s) == __builtin_inff();  // all of it in the low part, as in three_parts
            hi[j] = endless ? (_Float16)0.f : (_Float16)s;
            lo[j] = (_Float16)((s - (float)hi[j]) * (1 << kShift));
        }
        u32x4 w;
        __builtin_memcpy(&w, hi, 16);
        *(u32x4*)(y + c) = w;
        __builtin_memcpy(&w, lo, 16);
        *(u32x4*)(y + plane + c) = w;
    };
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if ((k * SPAN + lane) * 8 < a.pitch) put(keep[k], (k * SPAN + lane) * 8);
    for (int c = (KEEP * SPAN + lane) * 8; c < a.pitch; c += SPAN * 8) put(fetch8(x + c, n - c, false), c);
}

// ---- logits ----

typedef float f32x2 __attribute__((ext_vector_type(2)));

struct LogitArgs {
    Side w, u;
    int kts;             // tiles along the columns
    int tm, tn;          // tiles of classes and rows
    int classes;         // of this piece
    long long first;     // the piece's first class
    long long all;       // classes of the table
    long long rows;
    const int* u_exp;    // [rows], [classes] powers of two that 32-bit operands are of, or NULL
    const int* w_exp;
    const Scales* scales;
    const int64_t* target;
    const uint8_t* live;
    f32x2* parts;        // forward: [tile of classes][rows] largest logit, and the sum of exponentials relative to it
    float* picked;       // [rows] the target's logit
    const float* lse;    // backward
    const float* dloss;
    const float* dlse;
    float* inverse;      // without scales: of what g is multiplied with
    uint16_t* g;         // [rows up to the tiles' end][ld]
    long long g_ld, g_plane;
    int per;             // tiles along the columns of a slice
    int slices;
    f32x4* sums;         // [slice][tile], in the order in which lanes hold them
};

template <typename T>
__device__ __forceinline__ uint16_t bits16(float v) {
    return __builtin_bit_cast(uint16_t, (T)v);
}

// (top, sum of exponentials relative to it) of two sets of logits, of either of which there may be none.
__device__ __forceinline__ f32x2 merged(f32x2 a, f32x2 b) {
    const float top = fmaxf(a[0], b[0]), base = top > -__builtin_inff() ? top : 0.f;
    return f32x2{top, a[1] * __builtin_amdgcn_exp2f((a[0] - base) * kLog2e) + b[1] * __builtin_amdgcn_exp2f((b[0] - base) * kLog2e)};
}

// ---- few rows ----

struct FewArgs {
    const void* w;       // where it lies: any stride and element
    const void* u;
    long long w_stride, u_stride;
    int classes, cols, rows, groups;  // groups: of 32 classes to a workgroup
    const int64_t* target;
    f32x2* parts;
    float* picked;
    float* g;            // gradients: [classes][rows up to a multiple of 16], the other two are not looked at then
    const uint8_t* live;
    const float* lse;
    const float* dloss;
    const float* dlse;
};

// Sixteen bytes along k of a row, of which n elements exist.
template <typename TX>
__device__ __forceinline__ u32x4 along(const TX* p, int n) {
    constexpr int E = 16 / (int)sizeof(TX);
    if (n >= E) return *(const u32x4_any*)p;
    TX t[E];
#pragma unroll
    for (int j = 0; j < E; ++j) t[j] = j < n ? p[j] : (TX)0.f;
    u32x4 w;
    __builtin_memcpy(&w, t, 16);
    return w;
}
template <typename TX>
__device__ __forceinline__ f32x4 product(u32x4 w, u32x4 u, f32x4 c) {
    return Mma<TX>::go(__builtin_bit_cast(s16x8, w), __builtin_bit_cast(s16x8, u), c);
}
template <>
__device__ __forceinline__ f32x4 product<float>(u32x4 w, u32x4 u, f32x4 c) {
#pragma unroll
    for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[j]), __uint_as_float(u[j]), c, 0, 0, 0);
    return c;
}

// Rows that do not fill a tile, of a table that would have to be copied for tiles: it is read once, as it lies, straight into registers, 32 classes to a workgroup whose four
// waves share out the columns. NB blocks of 16 rows. Which columns a lane holds is the same for both operands and otherwise of no matter: in 32 bits four neighbours are four
// products of the 32-bit matrix instruction.
template <typename TX, int NB, bool GRAD>
__global__ __launch_bounds__(256) void k_few(const FewArgs a) {
    constexpr int E = 16 / (int)sizeof(TX), STEP = 4 * E, AT_ONCE = NB <= 2 ? 4 : 2, SPAN = STEP * AT_ONCE;
    __shared__ f32x4 meet[4][2][NB][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, k = lane / 16 * E;
    f32x2 all[NB];
#pragma unroll
    for (int n = 0; n < NB; ++n) all[n] = f32x2{-__builtin_inff(), 0.f};
    for (int group = 0; group < a.groups; ++group) {
        const int c0 = (blockIdx.x * a.groups + group) * 32;
        if (c0 >= a.classes) break;
        const TX* w[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) w[b] = (const TX*)a.w + min(c0 + b * 16 + r, a.classes - 1) * a.w_stride + k;
        const TX* u[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n) u[n] = (const TX*)a.u + min(n * 16 + r, a.rows - 1) * a.u_stride + k;
        f32x4 acc[2][NB];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int n = 0; n < NB; ++n) acc[b][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        auto span = [&](int k0, auto inside) {
            u32x4 wf[2][AT_ONCE], uf[NB][AT_ONCE];
#pragma unroll
            for (int s = 0; s < AT_ONCE; ++s) {
                const int at = k0 + s * STEP, left = inside ? E : a.cols - at - k;
#pragma unroll
                for (int b = 0; b < 2; ++b) wf[b][s] = along(w[b] + at, left);
#pragma unroll
                for (int n = 0; n < NB; ++n) uf[n][s] = along(u[n] + at, left);
            }
#pragma unroll
            for (int s = 0; s < AT_ONCE; ++s)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int n = 0; n < NB; ++n) acc[b][n] = product<TX>(wf[b][s], uf[n][s], acc[b][n]);
        };
        int k0 = wave * SPAN;
        for (; k0 + SPAN <= a.cols; k0 += 4 * SPAN) span(k0, std::true_type());
        if (k0 < a.cols) span(k0, std::false_type());
        if (group) __syncthreads();
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int n = 0; n < NB; ++n) meet[wave][b][n][lane] = acc[b][n];
        __syncthreads();
#pragma unroll
        for (int n = wave; n < NB; n += 4) {  // the waves share out the blocks of rows
            const int t = n * 16 + r;
            const long long want = t < a.rows ? a.target[t] - c0 : -1;
            if (GRAD) {
                const bool there = t < a.rows && !(a.live && !a.live[t]);
                const float lse = there ? a.lse[t] : 0.f;
                float up = there && a.dloss ? a.dloss[t] : 0.f, both = up + (there && a.dlse ? a.dlse[t] : 0.f);
                if (there && (want < -c0 || want >= a.classes - c0)) up = both = __builtin_nanf("");
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const f32x4 s = (meet[0][b][n][lane] + meet[1][b][n][lane]) + (meet[2][b][n][lane] + meet[3][b][n][lane]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int c = b * 16 + lane / 16 * 4 + j;
                        if (c0 + c < a.classes) a.g[(c0 + c) * (NB * 16ll) + n * 16 + r] = there ? both * expf(s[j] - lse > 0.f ? 0.f : s[j] - lse) - (want == c ? up : 0.f) : 0.f;
                    }
                }
                continue;
            }
            float v[8], top = -__builtin_inff();
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const f32x4 s = (meet[0][b][n][lane] + meet[1][b][n][lane]) + (meet[2][b][n][lane] + meet[3][b][n][lane]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = b * 16 + lane / 16 * 4 + j;
                    v[b * 4 + j] = c0 + c < a.classes ? s[j] : -__builtin_inff();
                    if (want == c && c0 + c < a.classes) a.picked[t] = s[j];
                    top = fmaxf(top, v[b * 4 + j]);
                }
            }
            const float base = top > -__builtin_inff() ? top : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += __builtin_amdgcn_exp2f((v[j] - base) * kLog2e);
#pragma unroll
            for (int i = 0; i < NB; ++i)
                if (i == n) all[i] = merged(all[i], f32x2{top, sum});
        }
    }
    if (GRAD) return;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        if (n % 4 != wave) continue;
        f32x2 v = all[n];
        v = merged(v, f32x2{__shfl_xor(v[0], 16), __shfl_xor(v[1], 16)});
        v = merged(v, f32x2{__shfl_xor(v[0], 32), __shfl_xor(v[1], 32)});
        if (lane < 16 && n * 16 + r < a.rows) a.parts[(long long)blockIdx.x * a.rows + n * 16 + r] = v;
    }
}

// C neighbours of a row of which n exist, at any element's address.
template <typename Cols, int C>
__device__ __forceinline__ Cols get_cols(const float* from, int n) {
    typedef Cols Any __attribute__((aligned(4)));
    Cols v;
    if (n >= C) return *(const Any*)from;
#pragma unroll
    for (int j = 0; j < C; ++j) v[j] = j < n ? from[j] : 0.f;
    return v;
}
template <typename Cols, int C>
__device__ __forceinline__ void put_cols(float* to, int n, Cols v) {
    typedef Cols Any __attribute__((aligned(4)));
    if (n >= C) {
        *(Any*)to = v;
        return;
    }
#pragma unroll
    for (int j = 0; j < C - 1; ++j)
        if (j < n) to[j] = v[j];
}

struct FewGradArgs {
    const float* w;
    const float* u;
    long long w_stride, u_stride;
    int classes, cols, rows, per;  // per: classes to a wave
    const uint8_t* live;
    const float* g;
    float* du;                     // NULL: not asked for, as dw
    float* dw;
    long long du_stride, dw_stride;
    float* sums;                   // [workgroup along the classes][R][cols], rounded up to 256
    int slices, pitch;
};

// Gradients of up to 32 rows in 32 bits: a wave has 256 columns of u and of du in registers (128 of more than sixteen rows), goes through its classes, adds g W to du, and writes g' u to dw.
// Nothing is copied or scaled for it, and memory bounds it: with the logits before it W is read twice and dw written, 24000 classes of 6592 columns 427 us (4.4 TB/s).
template <int R>
__global__ __launch_bounds__(256) void k_few_grad(const FewGradArgs a) {
    constexpr int AT_ONCE = 4, C = R > 16 ? 2 : 4, OF = R > 16 ? R : 16;  // columns of a lane, numbers of a class in g
    typedef float Cols __attribute__((ext_vector_type(C)));
    __shared__ Cols meet[3][R][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = blockIdx.x * (64 * C) + lane * C, n = a.cols - c;
    Cols u[R], du[R] = {};
#pragma unroll
    for (int t = 0; t < R; ++t) u[t] = t < a.rows && n > 0 && !(a.live && !a.live[t]) ? get_cols<Cols, C>(a.u + t * a.u_stride + c, n) : Cols(0.f);
    const int v0 = ((int)blockIdx.y * 4 + wave) * a.per, v1 = min(a.classes, v0 + a.per);
    for (int v = v0; v < v1; v += AT_ONCE) {
        Cols w[AT_ONCE] = {};
        if (a.du && n > 0) {
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) w[k] = get_cols<Cols, C>(a.w + min(v + k, a.classes - 1) * a.w_stride + c, n);
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            if (v + k >= v1) break;
            const float* const g = a.g + (v + k) * (long long)OF;
            Cols out = {};
#pragma unroll
            for (int t = 0; t < R; ++t) {
                const float gt = g[t];
#pragma unroll
                for (int j = 0; j < C; ++j) du[t][j] = fmaf(gt, w[k][j], du[t][j]), out[j] = fmaf(gt, u[t][j], out[j]);
            }
            if (a.dw && n > 0) put_cols<Cols, C>(a.dw + (v + k) * a.dw_stride + c, n, out);
        }
    }
    if (!a.du) return;
#pragma unroll
    for (int t = 0; t < R; ++t)
        if (wave) meet[wave - 1][t][lane] = du[t];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int t = 0; t < R; ++t)
        *(Cols*)(a.sums + ((long long)blockIdx.y * R + t) * a.pitch + c) = (du[t] + meet[0][t][lane]) + (meet[1][t][lane] + meet[2][t][lane]);
}

// The workgroups' sums: 64 columns of a row to a workgroup, sixteen threads to four columns.
__global__ __launch_bounds__(256) void k_few_join(const FewGradArgs a, const int per_slice) {
    __shared__ f32x4 meet[256];
    const int c = blockIdx.x * 64 + threadIdx.x % 16 * 4, t = blockIdx.y;
    f32x4 s{0.f, 0.f, 0.f, 0.f};
    for (int k = threadIdx.x / 16; k < a.slices; k += 16) s += *(const f32x4*)(a.sums + ((long long)k * per_slice + t) * a.pitch + c);
    meet[threadIdx.x] = s;
    __syncthreads();
    if (threadIdx.x >= 16 || c >= a.cols) return;
    for (int k = 1; k < 16; ++k) s += meet[k * 16 + threadIdx.x];
    const bool there = !(a.live && !a.live[t]);
    const float v[4] = {there ? s[0] : 0.f, there ? s[1] : 0.f, there ? s[2] : 0.f, there ? s[3] : 0.f};
    put_quad(a.du + t * a.du_stride + c, a.cols - c, v);
}

// g is rounded to 16 bits, and in most programs dloss is the same number in every row: what the rounding does to it would be the same everywhere, and not
// average out. So g is multiplied with the number from 1/2 to 1 that makes a row's dloss (or, where that is 0, what its probabilities are multiplied
// with) a power of two: the first that is not 0 of 64 rows, four together, spread evenly over all, since those at the beginning may be padding. The same in all waves; a row's number
// is asked for first and used behind the products. 131072 rows of 256 classes 63 us; 256 rows in four loads 67.
__device__ __forceinline__ float lift_ask(const LogitArgs& a) {
    const int i = threadIdx.x & 63;
    const long long t = a.rows > 64 ? i / 4 * (a.rows / 16) + i % 4 : i;
    if (a.scales || t >= a.rows || (a.live && !a.live[t])) return 0.f;
    const float v = a.dloss ? fabsf(a.dloss[t]) : 0.f;
    return v == 0.f && a.dlse ? fabsf(a.dlse[t]) : v;
}
__device__ __forceinline__ float lift_of(float asked, float& inverse) {
    const unsigned long long some = __builtin_amdgcn_ballot_w64(asked > 0.f && asked < __builtin_inff());
    inverse = 1.f;
    if (some) {
        int e;
        inverse = 2.f * frexpf(__shfl(asked, __builtin_ctzll(some)), &e);
    }
    return 1.f / inverse;
}

// What bounds it is the products (see products.h) and, where columns are few, what goes to memory: g of 131072 rows and 256 classes of 512 columns 63 us, 3.2 TB/s.
// Classes are the rows of the matrix instructions, so that a lane holds 4 * MT classes of a row and reduces them in registers. Where tiles are few and
// columns many the columns are split: SLICE leaves a slice's sums, JOIN adds them up and goes on. 2 rows, 4131 classes of 7360 columns in bfloat16: 58 us whole,
// 21 split.
enum { WHOLE, SLICE, JOIN };

template <typename T, int MW, int NW, int MT, int NT, int PAIRS, int PARTS, int KIND>
__global__ __launch_bounds__(MW * NW * 64) void k_logits(const LogitArgs a) {
    typedef Products<T, MW, NW, MT, NT, false, false, PAIRS, PAIRS == 3 ? kShift : 0> P;
    __shared__ __align__(16) uint16_t lds[P::LDS];
    int tm, tn;
    place_tile(blockIdx.x, gridDim.x, a.tm, a.tn, tm, tn);
    const int m0 = tm * P::BM, n0 = tn * P::BN;
    const int wm = P::wave_m(), wn = P::wave_n();
    // what the rows' gradients need, asked for in front of the products
    float lse[NT], up[NT], both[NT], asked = 0.f;
    int want[NT];  // the target, counted from the wave's first class; -1: elsewhere, -2: no such row, or padding
    if (PARTS && KIND != SLICE) {
        if (PARTS < 3) asked = lift_ask(a);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const long long t = (long long)n0 + wn + n * 16 + P::col_of();
            const bool there = t < a.rows && !(a.live && !a.live[t]);
            lse[n] = up[n] = both[n] = 0.f, want[n] = -2;
            if (there) {
                want[n] = -1;
                lse[n] = a.lse[t];
                up[n] = a.dloss ? a.dloss[t] : 0.f;
                both[n] = up[n] + (a.dlse ? a.dlse[t] : 0.f);
                const long long target = a.target[t], from = a.first + m0 + wm;
                if (target < 0 || target >= a.all) up[n] = both[n] = __builtin_nanf("");
                if (target >= from && target < from + MT * 16) want[n] = (int)(target - from);
            }
        }
    }
    P p;
    f32x4* const sums = a.sums + ((long long)blockIdx.y * gridDim.x + blockIdx.x) * (P::BM * P::BN / 4) + (threadIdx.x >> 6) * (MT * NT * 64) + (threadIdx.x & 63);
    if (KIND == WHOLE) {
        p.run(a.w, a.u, m0, n0, 0, a.kts, lds);
    } else if (KIND == SLICE) {
        const int kt0 = blockIdx.y * a.per;
        p.run(a.w, a.u, m0, n0, kt0, min(a.kts, kt0 + a.per), lds);
#pragma unroll
        for (int i = 0; i < MT * NT; ++i) sums[i * 64] = p.acc[i / NT][i % NT];
        return;
    } else {
        constexpr int AT_ONCE = 32 / (MT * NT);
        const long long next = (long long)gridDim.x * (P::BM * P::BN / 4);
        p.clear();
        for (int k = 0; k < a.slices; k += AT_ONCE) {
            f32x4 v[AT_ONCE][MT * NT];
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (k + u < a.slices) {
#pragma unroll
                    for (int i = 0; i < MT * NT; ++i) v[u][i] = sums[(k + u) * next + i * 64];
                }
#pragma unroll
            for (int u = 0; u < AT_ONCE; ++u)
                if (k + u < a.slices) {
#pragma unroll
                    for (int i = 0; i < MT * NT; ++i) p.acc[i / NT][i % NT] += v[u][i];
                }
        }
    }

    if (PAIRS == 3) {  // the workspace goes on to the tiles' ends
        int eu[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) eu[n] = a.u_exp[n0 + wn + n * 16 + P::col_of()];
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            int ew[4];
            __builtin_memcpy(ew, a.w_exp + m0 + wm + m * 16 + P::row_of(), 16);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) p.acc[m][n][j] = ldexpf(p.acc[m][n][j], eu[n] + ew[j]);
        }
    }
    if constexpr (PARTS == 0) {
        float* const meet = (float*)lds;  // [MW][BN][2]
        const int left = a.classes - (m0 + wm);  // classes that exist from the wave's first on
        if (left < MT * 16) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (m * 16 + P::row_of() + j >= left) p.acc[m][n][j] = -__builtin_inff();
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int col = wn + n * 16 + P::col_of();
            const long long t = (long long)n0 + col;
            const long long want = t < a.rows ? a.target[t] - a.first - m0 - wm : -1;
            const int w = want >= 0 && want < min(left, MT * 16) ? (int)want : -1;
            if (__builtin_amdgcn_ballot_w64(w >= 0)) {
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (m * 16 + P::row_of() + j == w) a.picked[t] = p.acc[m][n][j];
            }
            float top = -__builtin_inff();
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) top = fmaxf(top, p.acc[m][n][j]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float base = top > -__builtin_inff() ? top : 0.f;
            float sum = 0.f;
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int j = 0; j < 4; ++j) sum += __builtin_amdgcn_exp2f((p.acc[m][n][j] - base) * kLog2e);  // the difference first: of huge logits the product's rounding is past 128
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if ((threadIdx.x & 63) < 16) {
                meet[((wm / (MT * 16)) * P::BN + col) * 2] = top;
                meet[((wm / (MT * 16)) * P::BN + col) * 2 + 1] = sum;
            }
        }
        __syncthreads();
        for (int col = threadIdx.x; col < P::BN; col += P::THREADS) {
            const long long t = (long long)n0 + col;
            if (t >= a.rows) break;
            float top = -__builtin_inff(), sum = 0.f;
#pragma unroll
            for (int k = 0; k < MW; ++k) top = fmaxf(top, meet[(k * P::BN + col) * 2]);
#pragma unroll
            for (int k = 0; k < MW; ++k) {
                const float mine = meet[(k * P::BN + col) * 2], s = meet[(k * P::BN + col) * 2 + 1];
                sum += mine > -__builtin_inff() ? s * __builtin_amdgcn_exp2f((mine - top) * kLog2e) : s;
            }
            a.parts[tm * a.rows + t] = f32x2{top, sum};
        }
    } else {
        typedef Staged<P, uint16_t, NW, (PARTS > 2 ? 1 : PARTS > 1 ? NT / 2 : NT)> Out;
        static_assert(PARTS * Out::BYTES <= P::LDS * 2, "g passes through the operands' LDS");
        float lift = 1.f;
        if (PARTS < 3) {
            float inverse;
            lift = lift_of(asked, inverse);
            if (a.scales) lift = a.scales->g;
            else if (blockIdx.x + threadIdx.x == 0) *a.inverse = inverse;
        }
#pragma unroll
        for (int pass = 0; pass < Out::PASSES; ++pass) {
            if (pass) lds_barrier();
            const Out staged;
#pragma unroll
            for (int n = pass * (NT / Out::PASSES); n < (pass + 1) * (NT / Out::PASSES); ++n) {
                const float gu = up[n] * lift, gb = both[n] * lift;
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    uint16_t part[PARTS][4];
                    const int v0 = m * 16 + P::row_of();
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        // no probability is past 1; of huge logits the two passes' roundings are, and 0 times their exponential is not 0
                        const float s = __builtin_elementwise_minimum(p.acc[m][n][j] - lse[n], 0.f);
                        const float e = PAIRS > 1 ? expf(s) : __builtin_amdgcn_exp2f(s * kLog2e);
                        float g = gb * e - (v0 + j == want[n] ? gu : 0.f);
                        g = want[n] != -2 && m0 + wm + v0 + j < a.classes ? g : 0.f;
                        if constexpr (PARTS > 2) {
                            uint16_t of[3];
                            three_parts(g, of);
                            part[0][j] = of[0], part[1][j] = of[1], part[2][j] = of[2];
                        } else {
                            part[0][j] = bits16<T>(g);
                            const float whole = (float)__builtin_bit_cast(T, part[0][j]);
                            if constexpr (PARTS > 1) part[1][j] = bits16<T>(fabsf(whole) < __builtin_inff() ? g - whole : 0.f);
                        }
                    }
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) staged.put((char*)lds + q * Out::BYTES, m, n, part[q]);
                }
            }
            lds_barrier();
            uint16_t* const g = a.g + n0 * a.g_ld + m0;
#pragma unroll
            for (int i = 0; i < Out::PER; ++i) {
                if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
                int row, col;
                staged.where(i, pass, row, col);
#pragma unroll
                for (int q = 0; q < PARTS; ++q) *(u32x4*)(g + row * a.g_ld + col + q * a.g_plane) = staged.take((char*)lds + q * Out::BYTES, i);
            }
        }
    }
}

// The tiles of a row: LANES threads to a row. 4 to 7 us, most of it the launch and two dependent trips to memory: with few rows many threads share a row's tiles (512 at
// one row), with many rows a thread has enough of them.
template <int LANES>
__global__ __launch_bounds__(256) void k_loss_join(long long rows, int tiles, int classes, const f32x2* parts, const float* picked, const int64_t* target,
                                                   const uint8_t* live, float* loss, float* lse) {
    __shared__ f32x2 meet[256];
    constexpr int ROWS = 256 / LANES, AT_ONCE = 8;
    const int at = threadIdx.x % ROWS, lane = threadIdx.x / ROWS;
    const long long t = (long long)blockIdx.x * ROWS + at;
    f32x2 all{-__builtin_inff(), 0.f};
    if (t < rows) {
        for (int k = lane; k < tiles; k += AT_ONCE * LANES) {
            f32x2 v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) v[i] = k + i * LANES < tiles ? parts[(k + i * LANES) * rows + t] : f32x2{-__builtin_inff(), 0.f};
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) all = merged(all, v[i]);
        }
    }
    meet[threadIdx.x] = all;
    __syncthreads();
    if (lane || t >= rows) return;
    for (int k = 1; k < LANES; ++k) all = merged(all, meet[k * ROWS + at]);
    const bool there = !(live && !live[t]);
    const float l = there ? all[0] + logf(all[1]) : 0.f;
    lse[t] = l;
    const int64_t w = there ? target[t] : 0;
    loss[t] = !there ? 0.f : w >= 0 && w < classes ? l - picked[t] : __builtin_nanf("");
}

// ---- gradients ----

struct GradArgs {
    Side a, b;           // the side of the outputs' columns, and of their rows
    int kts, per;        // tiles along the sum, and of a slice
    int tm, tn;
    long long rows;      // outputs
    int cols;
    void* out;
    long long ld;
    float* partial;      // not NULL: sums [slice][tile] in the order in which lanes hold them, added to where `add`
    int add;
    const float* down;   // factor of an output, or NULL
    const uint8_t* live; // of du's rows: a padded one's g is 0, which times an infinity in W would be NaN
};

// A tile of du = g W (sums of W, rows of g) or dw = g' u (sums of both). The outputs' columns are the matrix instructions' rows.
template <class P, typename TO, int NW>
__device__ __forceinline__ void grad_tile(const GradArgs& a, unsigned block, uint16_t* lds) {
    constexpr int MT = P::MT, NT = P::NT;
    typedef Staged<P, float, NW, 2> Out;
    static_assert(Out::BYTES <= P::LDS * 2, "outputs pass through the operands' LDS");
    const unsigned tiles = (unsigned)a.tm * a.tn, slice = block / tiles;
    int tm, tn;
    place_tile(block - slice * tiles, tiles, a.tm, a.tn, tm, tn);
    const int kt0 = slice * a.per, kt1 = min(a.kts, kt0 + a.per);
    P p;
    if (kt0 < kt1) {
        p.run(a.a, a.b, tm * P::BM, tn * P::BN, kt0, kt1, lds);
    } else {
        p.clear();
    }
    if (a.partial) {
        f32x4* const to = (f32x4*)a.partial + ((long long)slice * tiles + tm * a.tn + tn) * (P::BM * P::BN / 4) +
                          (threadIdx.x >> 6) * (MT * NT * 64) + (threadIdx.x & 63);
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                f32x4* const at = to + (m * NT + n) * 64;
                *at = a.add ? *at + p.acc[m][n] : p.acc[m][n];
            }
        return;
    }
    const float down = a.down ? *a.down : 1.f;
    const long long r0 = (long long)tn * P::BN;
    const int c0 = tm * P::BM;
    if (a.live) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const long long r = r0 + P::wave_n() + n * 16 + P::col_of();
            if (r < a.rows && a.live[r]) continue;
#pragma unroll
            for (int m = 0; m < MT; ++m) p.acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    }
#pragma unroll
    for (int pass = 0; pass < Out::PASSES; ++pass) {
        if (pass) lds_barrier();
        const Out staged;
#pragma unroll
        for (int n = 2 * pass; n < 2 * pass + 2; ++n)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const f32x4 s = p.acc[m][n];
                const float v[4] = {s[0] * down, s[1] * down, s[2] * down, s[3] * down};
                staged.put(lds, m, n, v);
            }
        lds_barrier();
#pragma unroll
        for (int i = 0; i < Out::PER; ++i) {
            if (i % 4 == 0) __builtin_amdgcn_sched_barrier(0);
            int row, col;
            staged.where(i, pass, row, col);
            if (r0 + row >= a.rows || c0 + col >= a.cols) continue;
            float v[4];
            const u32x4 w = staged.take(lds, i);
            __builtin_memcpy(v, &w, 16);
            put_quad((TO*)a.out + (r0 + row) * a.ld + c0 + col, a.cols - c0 - col, v);
        }
    }
}

// `first` workgroups for du's tiles and slices, the others for dw's: neither fills the chip by itself where rows and classes are few. 1000 rows, 5003 classes of
// 520 columns in half precision: 20.5 and 19.5 us one after the other and 5 to join, 29 and 4 in one launch, the whole call 72 us and 59. Large ones are bound by power and by the
// transposing reads: 8192 rows, 32768 classes of 4096 columns 1.60 ms for du and 1.71 to 1.78 for dw, 1370 and 1260 TFLOP/s.
template <typename T, typename TO, int MW, int NW, int MT, int NT, int PAIRS>
__global__ __launch_bounds__(MW * NW * 64) void k_loss_grad(const GradArgs du, const GradArgs dw, const unsigned first) {
    typedef Products<T, MW, NW, MT, NT, true, false, PAIRS> DU;
    typedef Products<T, MW, NW, MT, NT, true, true, PAIRS> DW;
    __shared__ __align__(16) uint16_t lds[DU::LDS];
    if (blockIdx.x < first) grad_tile<DU, TO, NW>(du, blockIdx.x, lds);
    else grad_tile<DW, TO, NW>(dw, blockIdx.x - first, lds);
}

// The slices' sums, one after the other, four neighbours of a row to a thread, of du, dw or both: which have slices.
template <typename TO, int MW, int NW, int MT, int NT>
__global__ __launch_bounds__(256) void k_grad_join(const GradArgs du, const GradArgs dw, int slices_du, int slices_dw) {
    const bool second = !slices_du || blockIdx.y;
    const GradArgs& a = second ? dw : du;
    const int slices = second ? slices_dw : slices_du;
    constexpr int BM = MW * MT * 16, BN = NW * NT * 16, PER = BM * BN / 4;
    const float down = a.down ? *a.down : 1.f;
    const long long n = (long long)a.tm * a.tn * PER;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const int tile = (int)(i / PER), in = (int)(i % PER), lane = in & 63, block = in / 64 % (MT * NT), wave = in / (MT * NT * 64);
        const long long r = (long long)(tile % a.tn) * BN + wave % NW * (NT * 16) + block % NT * 16 + (lane & 15);
        const int c = tile / a.tn * BM + wave / NW * (MT * 16) + block / NT * 16 + 4 * (lane >> 4);
        if (r >= a.rows || c >= a.cols) continue;
        const f32x4* const from = (const f32x4*)a.partial + i;
        f32x4 s = 0.f;
        int k = 0;
        for (; k + 8 <= slices; k += 8) {
            f32x4 v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = from[(k + u) * n];
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        for (; k < slices; ++k) s += from[k * n];
        if (a.live && !a.live[r]) s = 0.f;
        const float v[4] = {s[0] * down, s[1] * down, s[2] * down, s[3] * down};
        put_quad((TO*)a.out + r * a.ld + c, a.cols - c, v);
    }
}

template <typename TO>
__global__ __launch_bounds__(256) void k_zero_rows(TO* out, long long rows, int cols, long long ld) {
    const long long n = rows * cols;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long long)gridDim.x * 256) {
        const long long r = i / cols;
        out[r * ld + (i - r * cols)] = (TO)0.f;
    }
}

// ---- launches ----

unsigned blocks_for(long long threads) { return (unsigned)std::max<long long>(1, std::min<long long>((threads + 255) / 256, 1 << 16)); }

template <typename T, int PAIRS, int PARTS>
void logits(const LogitArgs& a, const Cut& cut, hipStream_t st) {
    LogitArgs r = a;
    r.slices = cut.slices, r.per = cut.per;
    r.tm = (a.classes + cut.edge - 1) / cut.edge, r.tn = (int)((a.rows + cut.edge - 1) / cut.edge);
    const unsigned tiles = (unsigned)r.tm * r.tn;
    auto go = [&](auto whole, auto slice, auto join) {
        if (cut.slices <= 1) {
            whole<<<tiles, 256, 0, st>>>(r);
        } else {
            slice<<<dim3(tiles, cut.slices), 256, 0, st>>>(r);
            join<<<tiles, 256, 0, st>>>(r);
        }
    };
    if constexpr (PAIRS > 1 || PARTS < 2) {
        if (cut.edge == 256) {
            k_logits<T, 2, 4, 8, 4, PAIRS, PARTS, WHOLE><<<tiles, 512, 0, st>>>(r);
            return;
        }
    }
    if (cut.edge == 128) go(k_logits<T, 2, 2, 4, 4, PAIRS, PARTS, WHOLE>, k_logits<T, 2, 2, 4, 4, PAIRS, 0, SLICE>, k_logits<T, 2, 2, 4, 4, PAIRS, PARTS, JOIN>);
    else go(k_logits<T, 2, 2, 2, 2, PAIRS, PARTS, WHOLE>, k_logits<T, 2, 2, 2, 2, PAIRS, 0, SLICE>, k_logits<T, 2, 2, 2, 2, PAIRS, PARTS, JOIN>);
}

// A piece's part of du, of dw or of both, whose tiles are alike then. Slices are joined where `joined` says of how many.
template <typename T, typename TO, int PAIRS>
void gradients(GradArgs du, GradArgs dw, const Cut* cut_du, const Cut* cut_dw, const int (&joined)[2], hipStream_t st) {
    unsigned blocks[2] = {}, most = 0;
    const int edge = (cut_du ? cut_du : cut_dw)->edge;
    auto place = [&](GradArgs& r, const Cut* c, int i) {
        if (!c) return;
        r.per = c->per;
        r.tm = (r.cols + edge - 1) / edge, r.tn = (int)((r.rows + edge - 1) / edge);
        blocks[i] = (unsigned)r.tm * r.tn * c->slices;
        if (joined[i]) most = std::max(most, blocks_for((long long)r.tm * r.tn * edge * edge / 4));
    };
    place(du, cut_du, 0), place(dw, cut_dw, 1);
    auto go = [&](auto kernel, auto join, int threads) {
        kernel<<<blocks[0] + blocks[1], threads, 0, st>>>(du, dw, blocks[0]);
        if (most) join<<<dim3(most, joined[0] && joined[1] ? 2 : 1), 256, 0, st>>>(du, dw, joined[0], joined[1]);
    };
    if constexpr (PAIRS != 2) {
        if (edge == 256) return go(k_loss_grad<T, TO, 2, 4, 8, 4, PAIRS>, k_grad_join<TO, 2, 4, 8, 4>, 512);
    }
    if (edge == 128) go(k_loss_grad<T, TO, 2, 2, 4, 4, PAIRS>, k_grad_join<TO, 2, 2, 4, 4>, 256);
    else go(k_loss_grad<T, TO, 2, 2, 2, 2, PAIRS>, k_grad_join<TO, 2, 2, 2, 2>, 256);
}

// Operands ready, scales; the rest of the arguments of the logits.
template <typename TX>
LogitArgs prepared(const iodf_class_loss& a, const LossPlan& p, char* work, bool backward, hipStream_t st) {
    LogitArgs l{};
    Scales* const s = p.scaled ? (Scales*)(work + p.scales) : nullptr;
    float* const maxima = s ? (float*)(work + p.maxima) : nullptr;
    if (s) k_maxima<<<p.maxima_parts, 256, 0, st>>>(a.rows, a.live, a.dloss, a.dlse, maxima);
    l.u = {(const uint16_t*)a.u, 0, a.u_stride, (int)a.rows, (int)a.rows};
    l.w = {(const uint16_t*)a.w, 0, a.w_stride, a.classes, a.classes};
    ReadyArgs r{};
    r.x[0] = a.u, r.x[1] = a.w, r.stride[0] = a.u_stride, r.stride[1] = a.w_stride, r.rows[0] = a.rows, r.rows[1] = a.classes;
    r.live = a.live, r.cols = a.cols, r.pitch = p.pitch, r.maxima = maxima, r.parts = p.maxima_parts, r.scales = s;
    if (p.u_ready) r.y[0] = (uint16_t*)(work + p.u), l.u.p = r.y[0], l.u.ld = p.pitch, l.u.plane = a.rows * p.pitch;
    if (p.w_ready) r.y[1] = (uint16_t*)(work + p.w), l.w.p = r.y[1], l.w.ld = p.pitch, l.w.plane = (long long)a.classes * p.pitch;
    const long long most = std::max<long long>(p.u_ready ? a.rows : 0, p.w_ready ? a.classes : 0) * (p.pitch / 8);
    const dim3 grid(std::min(blocks_for(most), 1024u), p.w_ready ? 2 : 1);
    if constexpr (sizeof(TX) == 2) {
        if (s || p.u_ready || p.w_ready) k_ready<TX, 1><<<grid, 256, 0, st>>>(r);
    } else if (backward) {
        k_ready<TX, 3><<<grid, 256, 0, st>>>(r);
    } else if (!p.few) {
        RowsArgs h{};
        int* const e[2] = {(int*)(work + p.u_exp), (int*)(work + p.w_exp)};
        for (int i = 0; i < 2; ++i) h.x[i] = (const float*)r.x[i], h.y[i] = r.y[i], h.e[i] = e[i], h.stride[i] = r.stride[i], h.rows[i] = r.rows[i];
        h.live = a.live, h.cols = a.cols, h.pitch = p.pitch, l.u_exp = e[0], l.w_exp = e[1];
        const int at_once = p.pitch <= 256 ? 32 : p.pitch <= 2048 ? 4 : 1;  // rows to a workgroup
        h.first = (unsigned)((a.rows + at_once - 1) / at_once);
        const unsigned blocks = h.first + (unsigned)((a.classes + at_once - 1) / at_once);
        at_once == 32 ? k_rows<8><<<blocks, 256, 0, st>>>(h) : at_once == 4 ? k_rows<64><<<blocks, 256, 0, st>>>(h) : k_rows<256><<<blocks, 256, 0, st>>>(h);
    }
    l.kts = p.kts, l.classes = a.classes, l.all = a.classes, l.rows = a.rows, l.scales = s, l.target = a.target, l.live = a.live;
    l.sums = (f32x4*)(work + p.sums);
    return l;
}

template <typename TX, typename T, int PAIRS>
hipError_t forward(const iodf_class_loss& a, char* work, hipStream_t st) {
    const LossPlan p = loss_plan(a, false);
    LogitArgs l = prepared<TX>(a, p, work, false, st);
    l.parts = (f32x2*)(work + p.parts), l.picked = (float*)(work + p.picked);
    if (p.few) {
        const FewArgs f{a.w, a.u, a.w_stride, a.u_stride, a.classes, a.cols, (int)a.rows, p.groups, a.target, l.parts, l.picked, nullptr, nullptr, nullptr, nullptr, nullptr};
        auto go = [&](auto kernel) { kernel<<<(unsigned)p.tiles, 256, 0, st>>>(f); };
        if (p.few == 1) go(k_few<TX, 1, false>);
        else if constexpr (sizeof(TX) == 4) p.few == 2 ? go(k_few<TX, 2, false>) : go(k_few<TX, 4, false>);
    } else {
        logits<T, PAIRS, 0>(l, p.logits, st);
    }
    auto join = [&](auto kernel, int rows) {
        kernel<<<(unsigned)((a.rows + rows - 1) / rows), 256, 0, st>>>(a.rows, p.tiles, a.classes, l.parts, l.picked, a.target, a.live, a.loss, a.lse);
    };
    if (a.rows < 2048) join(k_loss_join<64>, 4);
    else if (a.rows < 65536) join(k_loss_join<16>, 16);
    else join(k_loss_join<4>, 64);
    return hipGetLastError();
}

hipError_t few_backward(const iodf_class_loss& a, const LossPlan& p, char* work, hipStream_t st) {
    const FewArgs f{a.w, a.u, a.w_stride, a.u_stride, a.classes, a.cols, (int)a.rows, p.groups, a.target, nullptr, nullptr, (float*)(work + p.g), a.live, a.lse, a.dloss, a.dlse};
    if (p.few == 1) k_few<float, 1, true><<<(unsigned)p.tiles, 256, 0, st>>>(f);
    else k_few<float, 2, true><<<(unsigned)p.tiles, 256, 0, st>>>(f);
    const int span = p.few == 1 ? 256 : 128, across = (a.cols + span - 1) / span;
    const FewGradArgs g{(const float*)a.w, (const float*)a.u, a.w_stride, a.u_stride, a.classes, a.cols, (int)a.rows, p.few_per, a.live, f.g, (float*)a.du, (float*)a.dw, a.du_stride, a.dw_stride,
                        (float*)(work + p.du_sums), p.few_slices, across * span};
    auto go = [&](auto kernel) { kernel<<<dim3(across, p.few_slices), 256, 0, st>>>(g); };
    if (p.few_rows == 2) go(k_few_grad<2>);
    else if (p.few_rows == 4) go(k_few_grad<4>);
    else if (p.few_rows == 8) go(k_few_grad<8>);
    else if (p.few_rows == 16) go(k_few_grad<16>);
    else go(k_few_grad<32>);
    if (a.du) k_few_join<<<dim3((a.cols + 63) / 64, (unsigned)a.rows), 256, 0, st>>>(g, p.few_rows);
    return hipGetLastError();
}

template <typename TX, typename T, int PAIRS>
hipError_t backward(const iodf_class_loss& a, char* work, hipStream_t st) {
    if (a.rows == 0) {
        k_zero_rows<TX><<<blocks_for((long long)a.classes * a.cols), 256, 0, st>>>((TX*)a.dw, a.classes, a.cols, a.dw_stride);
        return hipGetLastError();
    }
    const LossPlan p = loss_plan(a, true);
    if constexpr (PAIRS > 1) {
        if (p.few) return few_backward(a, p, work, st);
    }
    LogitArgs l = prepared<TX>(a, p, work, true, st);
    const Scales* const s = l.scales;
    const Side w = l.w;
    l.lse = a.lse, l.dloss = a.dloss, l.dlse = a.dlse;
    l.inverse = (float*)(work + p.scales), l.g = (uint16_t*)(work + p.g), l.g_ld = p.piece, l.g_plane = p.rows_up * p.piece;
    float* const du_sums = a.du && (p.du.slices > 1 || p.piece < a.classes) ? (float*)(work + p.du_sums) : nullptr;
    float* const dw_sums = a.dw && p.dw.slices > 1 ? (float*)(work + p.dw_sums) : nullptr;
    for (long long v0 = 0; v0 < a.classes; v0 += p.piece) {
        const int n = (int)std::min<long long>(p.piece, a.classes - v0);
        l.first = v0, l.classes = n;
        l.w = w, l.w.p += v0 * w.ld, l.w.extent = l.w.depth = n;
        if constexpr (PAIRS > 1) logits<T, PAIRS, 3>(l, p.logits, st);
        else if (p.fine) logits<T, 1, 2>(l, p.logits, st);
        else logits<T, 1, 1>(l, p.logits, st);
        GradArgs du{}, dw{};
        const bool last = v0 + n == a.classes;
        du.a = {l.w.p, w.plane, w.ld, a.cols, n};
        du.b = {l.g, l.g_plane, l.g_ld, (int)p.rows_up, (int)p.rows_up};
        du.kts = (n + PK - 1) / PK, du.rows = a.rows, du.cols = a.cols, du.out = a.du, du.ld = a.du_stride;
        du.partial = du_sums, du.add = v0 > 0, du.live = a.live;
        du.down = p.wide ? nullptr : s ? &s->ig : l.inverse;
        dw.a = {l.u.p, l.u.plane, l.u.ld, a.cols, (int)a.rows};
        dw.b = {l.g, l.g_plane, l.g_ld, (int)p.piece, (int)p.rows_up};
        dw.kts = (int)((a.rows + PK - 1) / PK), dw.rows = n, dw.cols = a.cols, dw.out = (TX*)a.dw + v0 * a.dw_stride, dw.ld = a.dw_stride;
        dw.partial = dw_sums;
        dw.down = du.down;
        const int join_du = du_sums && last ? p.du.slices : 0, join_dw = dw_sums ? p.dw.slices : 0;
        auto go = [&](const Cut* cut_du, const Cut* cut_dw) {
            const int joined[2] = {cut_du ? join_du : 0, cut_dw ? join_dw : 0};
            // with g in two parts where the operand has one
            if constexpr (PAIRS > 1) gradients<T, TX, PAIRS>(du, dw, cut_du, cut_dw, joined, st);
            else if (p.fine) gradients<T, TX, 2>(du, dw, cut_du, cut_dw, joined, st);
            else gradients<T, TX, 1>(du, dw, cut_du, cut_dw, joined, st);
        };
        if (p.together) {
            go(&p.du, &p.dw);
        } else {
            if (a.du) go(&p.du, nullptr);
            if (a.dw) go(nullptr, &p.dw);
        }
    }
    return hipGetLastError();
}

}  // namespace

size_t class_loss_workspace(const iodf_class_loss& a, bool backward) { return loss_plan(a, backward).bytes; }

hipError_t launch_class_loss(const iodf_class_loss& a, void* work, hipStream_t st) {
    return a.type == IODF_T_F32    ? forward<float, _Float16, 3>(a, (char*)work, st)
           : a.type == IODF_T_BF16 ? forward<__bf16, __bf16, 1>(a, (char*)work, st)
                                   : forward<_Float16, _Float16, 1>(a, (char*)work, st);
}

hipError_t launch_class_loss_backward(const iodf_class_loss& a, void* work, hipStream_t st) {
    return a.type == IODF_T_F32    ? backward<float, __bf16, 6>(a, (char*)work, st)
           : a.type == IODF_T_BF16 ? backward<__bf16, __bf16, 1>(a, (char*)work, st)
                                   : backward<_Float16, _Float16, 1>(a, (char*)work, st);
}

}  // namespace iodf
