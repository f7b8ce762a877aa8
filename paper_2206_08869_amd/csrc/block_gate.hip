// Checkpoints of single tensors, and the gated activation of a block's hidden layer with its gradients out of a checkpoint: passes
// over all elements, bound by memory. A thread takes VECS vectors of eight columns, a workgroup a run of neighbouring ones that
// goes on across row ends, so that narrow rows fill it too; a vector's four lanes are a group of the checkpoint.
#include "block_dev.h"

#include <algorithm>

namespace iodf {

namespace {

constexpr int TPB = 256, VECS = 2;

struct Grid {
    long long rows;
    int cols, pitch;
    unsigned vectors, magic;  // vectors of a row, and floor(2^32 / vectors) + 1
};

// Row and first column of this thread's vector k. Within a workgroup the vectors are counted from the row in which it starts, a
// number below vectors + TPB * VECS < 2^14, so the product with the reciprocal gives the exact quotient (vectors <= 2^13).
__device__ __forceinline__ void place(const Grid& g, long long row0, unsigned rem, int k, long long& row, int& c0, int& n) {
    const unsigned t = rem + k * TPB + threadIdx.x;
    const unsigned q = __umulhi(t, g.magic);
    row = row0 + q;
    c0 = (int)(t - q * g.vectors) * 8;
    n = row < g.rows ? g.cols - c0 : 0;
}

__device__ __forceinline__ void put_codes(const Grid& g, int8_t* q, uint8_t* e, long long row, int c0, const float v[8]) {
    store_codes(q, e, row, row < g.rows ? g.pitch : 0, c0, v);  // a pitch of 0 holds no column: nothing is stored past the last row
}

template <typename T>
__global__ __launch_bounds__(TPB) void k_pack(const Grid g, const T* x, long long stride, const uint8_t* live, int8_t* q, uint8_t* e) {
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    float v[VECS][8];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (live && n > 0 && !live[row]) n = 0;
        load8(x + row * stride + c0, n, v[k]);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        put_codes(g, q, e, row, c0, v[k]);
    }
}

template <typename T>
__global__ __launch_bounds__(TPB) void k_unpack(const Grid g, const int8_t* q, const uint8_t* e, T* y, long long stride) {
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    float v[VECS][8];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        load_codes(q, e, row, g.pitch, n > 0 ? c0 : g.pitch, v[k]);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        store8(y + row * stride + c0, n, v[k]);
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(TPB) void k_glu_forward(const Grid g, const iodf_glu a) {
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    float x[VECS][8], y[VECS][8];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (a.live && n > 0 && !a.live[row]) n = 0;
        load8((const T*)a.a + row * a.a_stride + c0, n, x[k]);
        load8((const T*)a.b + row * a.b_stride + c0, n, y[k]);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (a.aq) {
            put_codes(g, a.aq, a.ae, row, c0, x[k]);
            put_codes(g, a.bq, a.be, row, c0, y[k]);
        }
        float slope;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[k][i] *= activate<ACT>(x[k][i], slope);
        store8((T*)a.y + row * a.y_stride + c0, n, y[k]);
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(TPB) void k_glu_backward(const Grid g, const iodf_glu a) {
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    float x[VECS][8], b[VECS][8], d[VECS][8];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (a.live && n > 0 && !a.live[row]) n = 0;
        load8((const T*)a.dy + row * a.dy_stride + c0, n, d[k]);
        load_codes(a.aq, a.ae, row, g.pitch, n > 0 ? c0 : g.pitch, x[k]);
        load_codes(a.bq, a.be, row, g.pitch, n > 0 ? c0 : g.pitch, b[k]);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        float da[8], db[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float slope;
            const float act = activate<ACT>(x[k][i], slope);
            da[i] = d[k][i] * b[k][i] * slope;
            db[i] = d[k][i] * act;
            y[i] = act * b[k][i];
        }
        store8((T*)a.da + row * a.da_stride + c0, n, da);
        store8((T*)a.db + row * a.db_stride + c0, n, db);
        if (a.yq) put_codes(g, a.yq, a.ye, row, c0, y);
    }
}

Grid grid_of(long long rows, int cols, unsigned& blocks) {
    Grid g;
    g.rows = rows;
    g.cols = cols;
    g.pitch = code_pitch(cols);
    g.vectors = (unsigned)g.pitch / 8;
    g.magic = (unsigned)((1ull << 32) / g.vectors) + 1;
    blocks = (unsigned)((rows * g.vectors + TPB * VECS - 1) / (TPB * VECS));
    return g;
}

template <typename T>
hipError_t glu_forward_of(const iodf_glu& a, hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(a.rows, a.cols, blocks);
    if (a.act == IODF_ACT_RELU) k_glu_forward<T, IODF_ACT_RELU><<<blocks, TPB, 0, st>>>(g, a);
    else if (a.act == IODF_ACT_SILU) k_glu_forward<T, IODF_ACT_SILU><<<blocks, TPB, 0, st>>>(g, a);
    else k_glu_forward<T, IODF_ACT_GELU><<<blocks, TPB, 0, st>>>(g, a);
    return hipGetLastError();
}

template <typename T>
hipError_t glu_backward_of(const iodf_glu& a, hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(a.rows, a.cols, blocks);
    if (a.act == IODF_ACT_RELU) k_glu_backward<T, IODF_ACT_RELU><<<blocks, TPB, 0, st>>>(g, a);
    else if (a.act == IODF_ACT_SILU) k_glu_backward<T, IODF_ACT_SILU><<<blocks, TPB, 0, st>>>(g, a);
    else k_glu_backward<T, IODF_ACT_GELU><<<blocks, TPB, 0, st>>>(g, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(const void* x, int type, long long stride, long long rows, int cols, const uint8_t* live, int8_t* q,
                       uint8_t* e, hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(rows, cols, blocks);
    if (type == IODF_T_F32) k_pack<float><<<blocks, TPB, 0, st>>>(g, (const float*)x, stride, live, q, e);
    else if (type == IODF_T_BF16) k_pack<__bf16><<<blocks, TPB, 0, st>>>(g, (const __bf16*)x, stride, live, q, e);
    else k_pack<_Float16><<<blocks, TPB, 0, st>>>(g, (const _Float16*)x, stride, live, q, e);
    return hipGetLastError();
}

hipError_t launch_unpack(const int8_t* q, const uint8_t* e, long long rows, int cols, void* y, int type, long long stride,
                         hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(rows, cols, blocks);
    if (type == IODF_T_F32) k_unpack<float><<<blocks, TPB, 0, st>>>(g, q, e, (float*)y, stride);
    else k_unpack<__bf16><<<blocks, TPB, 0, st>>>(g, q, e, (__bf16*)y, stride);
    return hipGetLastError();
}

hipError_t launch_glu_forward(const iodf_glu& a, hipStream_t st) {
    return a.type == IODF_T_F32 ? glu_forward_of<float>(a, st) : a.type == IODF_T_BF16 ? glu_forward_of<__bf16>(a, st) : glu_forward_of<_Float16>(a, st);
}

hipError_t launch_glu_backward(const iodf_glu& a, hipStream_t st) {
    return a.type == IODF_T_F32 ? glu_backward_of<float>(a, st) : a.type == IODF_T_BF16 ? glu_backward_of<__bf16>(a, st) : glu_backward_of<_Float16>(a, st);
}

}  // namespace iodf
