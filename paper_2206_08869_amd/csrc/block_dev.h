// Device helpers that the training operators share: vectors of eight columns in three types, the 8-bit checkpoint's rounding,
// sums over the lanes of a row.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block.h"

namespace iodf {

// Vectors at any element's address: rows of odd widths start anywhere, and this architecture loads and stores 16 bytes there too.
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// Eight elements as they lie in memory: what a load that is not waited for yet holds.
template <typename T>
struct Raw8 {
    uint32_t w[2 * sizeof(T)];
};

// From p on, of which the first n exist (n <= 0: none, and all are 0). `over`: eight elements from p on are memory of the tensor's, whatever they
// belong to; a row's last vector is then one load too, and cut8 takes what is not the row's out of it, when the load is waited for anyway.
template <typename T>
__device__ __forceinline__ Raw8<T> fetch8(const T* p, int n, bool over) {
    Raw8<T> r;
    if (n >= 8 || (over && n > 0)) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const u32x4_any a = *(const u32x4_any*)((const char*)p + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[4 * i + j] = a[j];
        }
    } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : (T)0.f;
        __builtin_memcpy(r.w, t, sizeof(t));
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void cut8(Raw8<T>& r, int n) {
    constexpr int PER = 4 / sizeof(T);  // elements of a word
    if (__builtin_amdgcn_ballot_w64(n > 0 && n < 8)) {
#pragma unroll
        for (int i = 0; i < 8 / PER; ++i) {
            const int left = n - i * PER;
            r.w[i] = left >= PER || n <= 0 ? r.w[i] : left > 0 ? r.w[i] & 0xffffu : 0u;
        }
    }
}

// The eight columns that a lane has of every row it takes, for the kernels that hold rows in registers. Lanes past the last column read the
// first ones, which costs no branch; their parameters are 0 and they store nothing.
struct Columns {
    int c0, n;       // first column, how many there are (0..8)
    int at;          // where the lane reads
    bool edge;       // whether some lane of the wave has 1..7
    template <typename T>
    __device__ __forceinline__ void cut(Raw8<T>& r) const {
        if (edge) cut8(r, n);
    }
};
__device__ __forceinline__ Columns columns_at(int c0, int cols) {
    const int left = cols - c0, n = left < 0 ? 0 : left > 8 ? 8 : left;
    return {c0, n, n ? c0 : 0, __builtin_amdgcn_ballot_w64(n > 0 && n < 8) != 0};
}
// To be cut in the lane that has some of the columns (cut8). `over`, the same for a wave's lanes or nearly: as of fetch8.
template <typename T>
__device__ __forceinline__ Raw8<T> fetch_row(const T* row, const Columns& c, bool over) {
    Raw8<T> r;
    const T* const p = row + c.at;
    if (!c.edge || __builtin_amdgcn_ballot_w64(!over) == 0) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) {
            const u32x4_any a = *(const u32x4_any*)((const char*)p + 16 * i);
#pragma unroll
            for (int j = 0; j < 4; ++j) r.w[4 * i + j] = a[j];
        }
        return r;
    }
    return fetch8(p, c.n, false);
}

// Rows of a [rows][cols] tensor from whose vectors (columns at a multiple of 8) eight elements lie before the tensor's end.
inline long long over_rows(long long rows, int cols, long long stride) {
    const long long past = (cols + 7) / 8 * 8 - cols;  // of the last vector, past its row
    return rows - (past + stride - 1) / stride;
}

__device__ __forceinline__ void widen8(const Raw8<float>& r, float v[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
}
__device__ __forceinline__ void widen8(const Raw8<__bf16>& r, float v[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(r.w[i] << 16);
        v[2 * i + 1] = __uint_as_float(r.w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen8(const Raw8<_Float16>& r, float v[8]) {
    _Float16 h[8];
    __builtin_memcpy(h, r.w, 16);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)h[i];
}

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float v[8]) {
    widen8(fetch8(p, n, false), v);
}

// Rounded to nearest, ties to even. Of a row's last vector the first n, in pieces of four, two and one.
template <typename T>
__device__ __forceinline__ void store8(T* p, int n, const float v[8]) {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)v[i];
    uint32_t w[2 * sizeof(T)];
    __builtin_memcpy(w, t, sizeof(t));
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) *(u32x4_any*)((char*)p + 16 * i) = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    } else if (n > 0) {
        typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
        typedef uint32_t u32_any __attribute__((aligned(2)));
        constexpr int HALF = sizeof(T);  // words of four elements
        if (n & 4) {
            if (HALF == 4) *(u32x4_any*)p = u32x4{w[0], w[1], w[2 % (2 * HALF)], w[3 % (2 * HALF)]};
            else *(u32x2_any*)p = u32x2{w[0], w[1]};
#pragma unroll
            for (int i = 0; i < HALF; ++i) w[i] = w[HALF + i];
            p += 4;
        }
        if (n & 2) {
            if (HALF == 4) *(u32x2_any*)p = u32x2{w[0], w[1]};
            else *(u32_any*)p = w[0];
#pragma unroll
            for (int i = 0; i < HALF / 2; ++i) w[i] = w[HALF / 2 + i];
            p += 2;
        }
        if (n & 1) {
            if (HALF == 4) *(u32_any*)p = w[0];
            else *(uint16_t*)p = (uint16_t)w[0];
        }
    }
}

// ---- lanes ----

template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_HALF_MIRROR = 0x141, DPP_MIRROR = 0x140, DPP_ROR4 = 0x124,
              DPP_ROR8 = 0x128;

// Sum over aligned runs of LPR lanes, the same in each of them.
template <int LPR>
__device__ __forceinline__ float lanes_sum(float v) {
    if (LPR >= 2) v += __uint_as_float(dpp<DPP_XOR1>(__float_as_uint(v)));
    if (LPR >= 4) v += __uint_as_float(dpp<DPP_XOR2>(__float_as_uint(v)));
    if (LPR >= 8) v += __uint_as_float(dpp<DPP_HALF_MIRROR>(__float_as_uint(v)));
    if (LPR >= 16) v += __uint_as_float(dpp<DPP_MIRROR>(__float_as_uint(v)));
    if (LPR >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if (LPR >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// Four sums at a time: lanes give away what their neighbour keeps, so that after two steps each holds one of the four, by its number mod 4.
__device__ __forceinline__ float fold4(const float v[4]) {
    const bool odd = threadIdx.x & 1, high = threadIdx.x & 2;
    const float a = (odd ? v[1] : v[0]) + __uint_as_float(dpp<DPP_XOR1>(__float_as_uint(odd ? v[0] : v[1])));
    const float b = (odd ? v[3] : v[2]) + __uint_as_float(dpp<DPP_XOR1>(__float_as_uint(odd ? v[2] : v[3])));
    return (high ? b : a) + __uint_as_float(dpp<DPP_XOR2>(__float_as_uint(high ? a : b)));
}
// The sum over lanes of an aligned run of LPR that have the same number mod 4.
template <int LPR>
__device__ __forceinline__ float lanes_sum_mod4(float v) {
    if (LPR == 8) return v + __uint_as_float(dpp<DPP_XOR1>(dpp<DPP_XOR2>(dpp<DPP_HALF_MIRROR>(__float_as_uint(v)))));  // lane ^ 4
    v += __uint_as_float(dpp<DPP_ROR4>(__float_as_uint(v)));
    v += __uint_as_float(dpp<DPP_ROR8>(__float_as_uint(v)));
    if (LPR >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    if (LPR >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    return v;
}

// One sum, or four, over the LPR threads of a row. Past a wave they meet in LDS, in two places by turns (`turn` counts the calls): with one
// barrier a call, nobody writes a place again before everybody has read it. Where all of a wave has the results, they are in scalar registers.
template <int LPR, int N>
struct RowSums {
    static constexpr int WAVES = LPR > 64 ? LPR / 64 : 1, W = WAVES <= 2 ? WAVES : WAVES <= 4 ? 4 : WAVES <= 8 ? 8 : 16;
    float at[2][N][W];
};
template <int LPR, int N>
__device__ __forceinline__ void row_sums(float v[N], RowSums<LPR, N>& meet, int& turn) {
    static_assert(N == 1 || N == 4, "");
    constexpr int L = LPR < 64 ? LPR : 64;
    const int lane = threadIdx.x & 63;
    float mine = N == 1 ? lanes_sum<L>(v[0]) : lanes_sum_mod4<L>(fold4(v));
    if (LPR > 64) {
        constexpr int W = RowSums<LPR, N>::W;
        float* const at = &meet.at[turn++ & 1][0][0];
        if (lane < N) at[lane * W + (threadIdx.x >> 6)] = mine;
        __syncthreads();
        mine = lanes_sum<W>(lane < N * W && lane % W < RowSums<LPR, N>::WAVES ? at[lane] : 0.f);  // W lanes to a sum
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), k * W));
    } else if (LPR == 64) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), k));
    } else if (N == 1) {
        v[0] = mine;
    } else {  // every quad of lanes holds the four
        v[0] = __uint_as_float(dpp<0x00>(__float_as_uint(mine)));
        v[1 % N] = __uint_as_float(dpp<0x55>(__float_as_uint(mine)));
        v[2 % N] = __uint_as_float(dpp<0xAA>(__float_as_uint(mine)));
        v[3 % N] = __uint_as_float(dpp<0xFF>(__float_as_uint(mine)));
    }
}

// ---- checkpoint ----
// A group of 32 columns is four neighbouring lanes. Its exponent byte e is the biased exponent of its largest magnitude, one more if
// that magnitude would round to 128 steps; the step is 2^(e - 133), so that the magnitude is 64 to 127 of them. A power of two
// costs up to one of the eight bits against amax / 127, but a value is then exact in bfloat16 (seven bits and a sign) and goes
// to the matrix cores unrounded. e stays within 16..254: below, steps and their inverses would leave the normal numbers. 255
// stands for a group that holds a NaN or an infinity: all of it reads as NaN.
__device__ __forceinline__ float code_step(uint32_t e) {
    return e == 255 ? __uint_as_float(0x7fc00000u) : __uint_as_float(((e > 6 ? e : 6) - 6) << 23);
}

// Codes of the eight values of this lane; the exponent byte is the same in the four lanes of the group.
__device__ __forceinline__ u32x2 encode8(const float v[8], uint32_t& e) {
    // the largest magnitude as a whole number, as which a NaN is the largest of all: of the positive values the largest signed number, of the
    // negative ones the largest unsigned one
    int pos = 0;
    uint32_t neg = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        pos = max(pos, (int)__float_as_uint(v[i]));
        neg = max(neg, __float_as_uint(v[i]));
    }
    uint32_t top = max((uint32_t)pos, neg & 0x7fffffffu);
    uint32_t o = dpp<DPP_XOR1>(top);
    top = o > top ? o : top;
    o = dpp<DPP_XOR2>(top);
    top = o > top ? o : top;
    e = (top + 0x10000u) >> 23;
    e = e < 16 ? 16 : e > 254 ? 254 : e;
    const float inv = __uint_as_float((260 - e) << 23);
    // v inv is exact; added to 3 * 2^22, whose neighbours are 1 apart, it is rounded to a whole number, whose lowest byte is the code
    uint32_t t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = __float_as_uint(fmaf(v[i], inv, 12582912.f));
    // the one exponent with which a code could pass 127, and what is not finite; asked for the whole wave, so that it is a branch
    if (__builtin_amdgcn_ballot_w64(top >= 0x7f7f0000u)) {
        if (top >= 0x7f7f0000u) {
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = (uint32_t)(int)fminf(fmaxf(rintf(v[i] * inv), -127.f), 127.f);
        }
        if (top >= 0x7f800000u) {
            e = 255;
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = 0;
        }
    }
    u32x2 w;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t low = __builtin_amdgcn_perm(t[4 * k + 1], t[4 * k], 0x0c0c0400u), high = __builtin_amdgcn_perm(t[4 * k + 3], t[4 * k + 2], 0x04000c0cu);
        w[k] = low | high;
    }
    return w;
}

__device__ __forceinline__ void numbers8(u32x2 q, float v[8]) {  // the codes without their step
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int)__builtin_amdgcn_sbfe((int)q[i >> 2], 8 * (i & 3), 8);
}
__device__ __forceinline__ void decode8(u32x2 q, float step, float v[8]) {
    numbers8(q, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] *= step;
}

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));

// Rounded to bfloat16, two to a register.
__device__ __forceinline__ bf8 narrow8(const float v[8]) {
    typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
    union { uint32_t w[4]; bf8 all; } u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf2 p = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
        u.w[i] = __builtin_bit_cast(uint32_t, p);
    }
    return u.all;
}

// One row's codes at columns c0.. (a multiple of 8) of a checkpoint with `pitch` columns.
__device__ __forceinline__ void store_codes(int8_t* q, uint8_t* e, long long row, int pitch, int c0, const float v[8]) {
    uint32_t ex;
    const u32x2 w = encode8(v, ex);  // every lane takes part: the group's maximum goes round its four lanes
    if (c0 < pitch) {
        *(u32x2*)(q + row * pitch + c0) = w;
        if ((c0 & 31) == 0) e[row * (pitch / 32) + c0 / 32] = (uint8_t)ex;
    }
}
// Eight codes and their exponent as they lie in memory (none past the pitch: zeros).
struct RawCodes {
    u32x2 q;
    uint32_t e;
};
__device__ __forceinline__ RawCodes fetch_codes(const int8_t* q, const uint8_t* e, long long row, int pitch, int c0) {
    RawCodes r = {u32x2{0, 0}, 16};
    if (c0 < pitch) {
        r.q = *(const u32x2*)(q + row * pitch + c0);
        r.e = e[row * (pitch / 32) + c0 / 32];
    }
    return r;
}
// Makes the compiler forget what it has widened from these, so that it is widened again where it is used next and not held in four times the
// registers until then.
template <typename T>
__device__ __forceinline__ void forget(Raw8<T>& r) {
#pragma unroll
    for (int i = 0; i < 2 * (int)sizeof(T); ++i) asm volatile("" : "+v"(r.w[i]));
}
__device__ __forceinline__ void forget(RawCodes& r) { asm volatile("" : "+v"(r.q), "+v"(r.e)); }

// ---- activations ----

// exp(x) within three units of its last bit or so. The product x log2(e), rounded, is off by as many units as it has whole bits, 60 at x = 80; what
// was rounded off and the constant's own rest come in again as a factor. Both ends are exact: infinity, 0 (the clamp only meets what is no
// number there).
__device__ __forceinline__ float exponential(float x) {
    const float p = x * 1.44269502f, rest = fmaf(x, 1.92596303e-8f, fmaf(x, 1.44269502f, -p));
    return __builtin_amdgcn_exp2f(p) * fmaf(__builtin_amdgcn_fmed3f(rest, -1.f, 1.f), 0.693147181f, 1.f);
}

// act(a), and its derivative. Relative errors in units of 2^-24: the logistic function some ten, with gelu another four times its argument, which
// is rounded as often. Below exp(-87), where its reciprocal leaves the normal numbers, it is 0.
template <int ACT>
__device__ __forceinline__ float activate(float a, float& slope) {
    if (ACT == IODF_ACT_RELU) {
        slope = a > 0.f ? 1.f : 0.f;
        return a < 0.f ? 0.f : a;  // a NaN stays one
    }
    const float k = 1.5957691216057308f;  // 2 sqrt(2 / pi)
    const float arg = ACT == IODF_ACT_SILU ? a : k * (a + 0.044715f * a * a * a);
    const float s = __builtin_amdgcn_rcpf(1.f + exponential(-arg));
    const float bend = s * (1.f - s);
    if (ACT == IODF_ACT_SILU) slope = s + a * bend;
    else slope = bend == 0.f ? s : s + a * bend * k * (1.f + 0.134145f * a * a);  // far out a * a may be infinite
    return a * s;
}

}  // namespace iodf
