// Gradient of a linear layer's weight from the 8-bit checkpoint of its input: dw[o][c] = scale[c] sum_t dy[t][o] X[t][c].
//
// The sum runs over rows, and both operands hold consecutive columns, so each matrix instruction's operand (eight rows of one column
// to a lane) is a transpose. Tiles of KT rows go to LDS as they lie in memory, codes widened to bfloat16 (exact: seven bits and a sign
// times a power of two) on the way, and the transposing LDS read takes them from there.
// dy of more than eight significant bits is the exact sum of two (half precision) or three (32 bits) bfloat16 parts, multiplied
// one after the other into the same sums.
#include "block_dev.h"

#include <algorithm>

namespace iodf {

namespace {

typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int KT = 32;  // rows of a tile: two matrix instructions deep

template <typename T> constexpr int parts_of() { return sizeof(T) == 4 ? 3 : 1; }
template <> constexpr int parts_of<_Float16>() { return 2; }

// Sixteen-byte chunk of column chunk c8 of row r of a tile W columns wide. The four rows that sixteen lanes read together would lie on
// the same banks; moved by 64 bytes a row they cover 256 bytes.
template <int W>
__device__ __forceinline__ int chunk_at(int r, int c8) {
    return r * (W / 8) + (W >= 128 ? c8 ^ ((r & 3) << 2) : c8 ^ ((r & 2) << 1));
}

template <int W>
__device__ __forceinline__ bf8 fragment(const __bf16* tile, int off, int step) {
    // rows step * 16 + 8 * (lane / 32) + 0..3 and + 4..7; `off` is the lane's own place
    union { s16x4 h[2]; bf8 v; } f;
    f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + off + step * 16 * W));
    f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + off + (step * 16 + 4) * W));
    return f.v;
}

template <typename TY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__((BM / WM) * (BN / WN) * 64) void k_wgrad(const iodf_wgrad a, int tiles_m, int tiles_n, int slice,
                                                                     float* partial) {
    constexpr int THREADS = (BM / WM) * (BN / WN) * 64, P = parts_of<TY>(), MT = WM / 32, NT = WN / 32;
    constexpr int AL = KT * BM / 8 / THREADS, BL = KT * BN / 8 / THREADS;
    __shared__ __bf16 at[2][P][KT * BM];
    __shared__ __bf16 bt[2][KT * BN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tile = blockIdx.x % (tiles_m * tiles_n), split = blockIdx.x / (tiles_m * tiles_n);
    const int m0 = tile / tiles_n * BM, n0 = tile % tiles_n * BN;
    const int pitch = (a.cols + 31) / 32 * 32;
    const long long t0 = (long long)split * slice, t1 = min((long long)a.rows, t0 + slice);
    const int wm = wave / (BN / WN) * WM, wn = wave % (BN / WN) * WN;

    int a_off[MT], b_off[NT];
    const int fr = (lane >> 5) * 8 + ((lane >> 2) & 3), fc = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int m = 0; m < MT; ++m) a_off[m] = chunk_at<BM>(fr, (wm + m * 32 + fc) / 8) * 8 + (fc & 7);
#pragma unroll
    for (int n = 0; n < NT; ++n) b_off[n] = chunk_at<BN>(fr, (wn + n * 32 + fc) / 8) * 8 + (fc & 7);

    float av[AL][8];
    u32x2 bq[BL];
    float bs[BL];
    auto fetch = [&](long long t) {
#pragma unroll
        for (int i = 0; i < AL; ++i) {
            const int k = threadIdx.x + i * THREADS, c = m0 + k % (BM / 8) * 8;
            const long long row = t + k / (BM / 8);
            const bool there = row < t1 && (!a.live || a.live[row]);
            load8((const TY*)a.dy + row * a.dy_stride + c, there ? a.out - c : 0, av[i]);
        }
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int k = threadIdx.x + i * THREADS, c = n0 + k % (BN / 8) * 8;
            const long long row = t + k / (BN / 8);
            bq[i] = u32x2{0, 0};
            bs[i] = 0.f;
            if (row < t1 && c < pitch && (!a.live || a.live[row])) {
                bq[i] = *(const u32x2*)(a.q + row * pitch + c);
                bs[i] = code_step(a.e[row * (pitch / 32) + c / 32]);
            }
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int i = 0; i < AL; ++i) {
            const int k = threadIdx.x + i * THREADS, at16 = chunk_at<BM>(k / (BM / 8), k % (BM / 8)) * 8;
            float rest[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) rest[j] = av[i][j];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                bf8 w;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    w[j] = (__bf16)rest[j];
                    const float got = (float)w[j];
                    rest[j] = fabsf(got) < __builtin_inff() ? rest[j] - got : 0.f;
                }
                *(bf8*)&at[buf][p][at16] = w;
            }
        }
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int k = threadIdx.x + i * THREADS, at16 = chunk_at<BN>(k / (BN / 8), k % (BN / 8)) * 8;
            float v[8];
            decode8(bq[i], bs[i], v);
            bf8 w;
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = (__bf16)v[j];
            *(bf8*)&bt[buf][at16] = w;
        }
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;

    if (t0 < t1) {
        fetch(t0);
        put(0);
    }
    __syncthreads();
    int buf = 0;
    for (long long t = t0; t < t1; t += KT) {
        const bool more = t + KT < t1;
        if (more) fetch(t + KT);
#pragma unroll
        for (int s = 0; s < KT / 16; ++s) {
            bf8 bf[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) bf[n] = fragment<BN>(bt[buf], b_off[n], s);
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    const bf8 af = fragment<BM>(at[buf][p], a_off[m], s);
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af, bf[n], acc[m][n], 0, 0, 0);
                }
        }
        if (more) put(buf ^ 1);
        __syncthreads();
        buf ^= 1;
    }

    // lane l holds column l % 32, rows 8 * (i / 4) + 4 * (l / 32) + i % 4 of each 32 x 32 block
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int c = n0 + wn + n * 32 + (lane & 31);
        if (c >= a.cols) continue;
        const float scale = !partial && a.col_scale ? a.col_scale[c] : 1.f;
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int o = m0 + wm + m * 32 + 8 * (i / 4) + 4 * (lane >> 5) + i % 4;
                if (o >= a.out) continue;
                if (partial) {
                    partial[((long long)split * a.out + o) * a.cols + c] = acc[m][n][i];
                } else {
                    float* const d = a.dw + o * a.dw_stride + c;
                    *d = (a.accumulate ? *d : 0.f) + scale * acc[m][n][i];
                }
            }
    }
}

// The slices' sums, in the order of the slices.
__global__ __launch_bounds__(256) void k_wgrad_join(const iodf_wgrad a, int splits, const float* partial) {
    const long long n = (long long)a.out * a.cols, i = blockIdx.x * 256ll + threadIdx.x;
    if (i >= n) return;
    float s = 0.f;
    for (int k = 0; k < splits; ++k) s += partial[k * n + i];
    const int o = (int)(i / a.cols), c = (int)(i - (long long)o * a.cols);
    float* const d = a.dw + o * a.dw_stride + c;
    *d = (a.accumulate ? *d : 0.f) + (a.col_scale ? a.col_scale[c] : 1.f) * s;
}

struct Plan {
    int tile, tiles_m, tiles_n, slice, splits;
};

Plan plan_of(const iodf_wgrad& a) {
    Plan p;
    auto tiles = [&](int b) { return (long long)((a.out + b - 1) / b) * ((a.cols + b - 1) / b); };
    p.tile = tiles(128) * ((a.rows + 255) / 256) >= 256 ? 128 : 64;
    if (a.dy_type == IODF_T_BF16 && a.out > 128 && a.cols > 128 && tiles(256) * ((a.rows + 1023) / 1024) >= 256) p.tile = 256;
    p.tiles_m = (a.out + p.tile - 1) / p.tile;
    p.tiles_n = (a.cols + p.tile - 1) / p.tile;
    const long long n = (long long)p.tiles_m * p.tiles_n;
    long long splits = std::max<long long>(1, 256 / n);
    splits = std::min<long long>(splits, std::max<long long>(1, a.rows / 128));
    p.slice = (int)(((a.rows + splits - 1) / splits + KT - 1) / KT * KT);
    p.splits = p.slice ? (int)((a.rows + p.slice - 1) / p.slice) : 1;
    return p;
}

template <typename TY>
hipError_t run(const iodf_wgrad& a, const Plan& p, float* partial, hipStream_t st) {
    const unsigned blocks = (unsigned)(p.tiles_m * p.tiles_n * p.splits);
    if (p.tile == 256) {
        if constexpr (parts_of<TY>() == 1) k_wgrad<TY, 256, 256, 128, 64><<<blocks, 512, 0, st>>>(a, p.tiles_m, p.tiles_n, p.slice, partial);
    } else if (p.tile == 128) {
        k_wgrad<TY, 128, 128, 64, 64><<<blocks, 256, 0, st>>>(a, p.tiles_m, p.tiles_n, p.slice, partial);
    } else {
        k_wgrad<TY, 64, 64, 32, 32><<<blocks, 256, 0, st>>>(a, p.tiles_m, p.tiles_n, p.slice, partial);
    }
    return hipGetLastError();
}

}  // namespace

size_t wgrad_workspace(const iodf_wgrad& a) {
    const Plan p = plan_of(a);
    return p.splits > 1 ? (size_t)p.splits * a.out * a.cols * 4 : 0;
}

hipError_t launch_weight_grad(const iodf_wgrad& a, void* work, hipStream_t st) {
    const Plan p = plan_of(a);
    float* const partial = p.splits > 1 ? (float*)work : nullptr;
    const hipError_t e = a.dy_type == IODF_T_F32    ? run<float>(a, p, partial, st)
                         : a.dy_type == IODF_T_BF16 ? run<__bf16>(a, p, partial, st)
                                                    : run<_Float16>(a, p, partial, st);
    if (e != hipSuccess || !partial) return e;
    const long long n = (long long)a.out * a.cols;
    k_wgrad_join<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(a, p.splits, partial);
    return hipGetLastError();
}

}  // namespace iodf
