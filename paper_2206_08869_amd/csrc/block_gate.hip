// Checkpoints of single tensors, and the gated activation of a block's hidden layer with its gradients out of a checkpoint: passes
// over all elements, bound by memory. A thread takes one or two vectors of eight columns, a workgroup a run of neighbouring ones that
// goes on across row ends, so that narrow rows fill it too; a vector's four lanes are a group of the checkpoint.
//
// Two vectors a thread where it loads little (a checkpoint, or 16 bits of one tensor), one elsewhere. Microseconds for 2^26 elements, silu,
// with one / two / four:          512 columns           1000 columns          floor (a copy's 5.1 TB/s)
//   pack      16 bits             38.4 / 36.0 / 40.4    41.6 / 41.0 / 43.0    39.7
//             32 bits             58.2 / 61.1 / 62.1    60.0 / 61.8 / 65.6    65.9
//   unpack    to 16 bits          33.3 / 32.7 / 33.5    36.5 / 33.9 / 34.3    39.7
//   glu       16 bits, saved      96.2 / 103 / 107      101 / 107 / 116       105
//             32 bits, saved      163 / 167 / 170       165 / 180 / 176       184
//   gradient  16 bits             113 / 119 / 120       115 / 122 / 131       119
//             32 bits             188 / 191 / 196       192 / 198 / 205       198
// Below the floor, since parts of tensors this size stay in the last-level cache from call to call. All are bound by memory; the arithmetic
// of an activation, its slope and two codes hides behind it.
#include "block_dev.h"

#include <algorithm>

namespace iodf {

namespace {

constexpr int TPB = 256;

template <typename T>
constexpr int pack_vecs() { return sizeof(T) == 2 ? 2 : 1; }
constexpr int UNPACK_VECS = 2, GLU_VECS = 1;

struct Grid {
    long long rows;
    int cols, pitch;
    unsigned vectors, magic;  // vectors of a row, and floor(2^32 / vectors) + 1
    long long over[2];        // rows of the inputs whose last vector may be read past its row
};

// Row and first column of this thread's vector k. Within a workgroup the vectors are counted from the row in which it starts, a
// number below vectors + TPB * VECS <= 2^13 + 2^9, so the product with the reciprocal gives the exact quotient (vectors <= 2^13).
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
    constexpr int VECS = pack_vecs<T>();
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    Raw8<T> r[VECS];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (live && n > 0 && !live[row]) n = 0;
        r[k] = fetch8(x + row * stride + c0, n, row < g.over[0]);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        cut8(r[k], n);
        float v[8];
        widen8(r[k], v);
        put_codes(g, q, e, row, c0, v);
    }
}

template <typename T>
__global__ __launch_bounds__(TPB) void k_unpack(const Grid g, const int8_t* q, const uint8_t* e, T* y, long long stride) {
    constexpr int VECS = UNPACK_VECS;
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    RawCodes r[VECS];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        r[k] = fetch_codes(q, e, row, g.pitch, n > 0 ? c0 : g.pitch);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        float v[8];
        decode8(r[k].q, code_step(r[k].e), v);
        store8(y + row * stride + c0, n, v);
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(TPB) void k_glu_forward(const Grid g, const iodf_glu a) {
    constexpr int VECS = GLU_VECS;
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    Raw8<T> ra[VECS], rb[VECS];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (a.live && n > 0 && !a.live[row]) n = 0;
        ra[k] = fetch8((const T*)a.a + row * a.a_stride + c0, n, row < g.over[0]);
        rb[k] = fetch8((const T*)a.b + row * a.b_stride + c0, n, row < g.over[1]);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        cut8(ra[k], n), cut8(rb[k], n);
        float x[8], y[8], slope;
        widen8(ra[k], x);
        widen8(rb[k], y);
        if (a.aq) {
            put_codes(g, a.aq, a.ae, row, c0, x);
            put_codes(g, a.bq, a.be, row, c0, y);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] *= activate<ACT>(x[i], slope);
        store8((T*)a.y + row * a.y_stride + c0, n, y);
    }
}

template <typename T, int ACT>
__global__ __launch_bounds__(TPB) void k_glu_backward(const Grid g, const iodf_glu a) {
    constexpr int VECS = GLU_VECS;
    const long long first = (long long)blockIdx.x * (TPB * VECS), row0 = first / g.vectors;
    const unsigned rem = (unsigned)(first - row0 * g.vectors);
    Raw8<T> rd[VECS];
    RawCodes ra[VECS], rb[VECS];
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        if (a.live && n > 0 && !a.live[row]) n = 0;
        rd[k] = fetch8((const T*)a.dy + row * a.dy_stride + c0, n, row < g.over[0]);
        ra[k] = fetch_codes(a.aq, a.ae, row, g.pitch, n > 0 ? c0 : g.pitch);
        rb[k] = fetch_codes(a.bq, a.be, row, g.pitch, n > 0 ? c0 : g.pitch);
    }
#pragma unroll
    for (int k = 0; k < VECS; ++k) {
        long long row;
        int c0, n;
        place(g, row0, rem, k, row, c0, n);
        cut8(rd[k], n);
        float d[8], x[8], b[8], da[8], db[8], y[8];
        widen8(rd[k], d);
        decode8(ra[k].q, code_step(ra[k].e), x);
        decode8(rb[k].q, code_step(rb[k].e), b);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float slope;
            const float act = activate<ACT>(x[i], slope);
            da[i] = d[i] * b[i] * slope;
            db[i] = d[i] * act;
            y[i] = act * b[i];
        }
        store8((T*)a.da + row * a.da_stride + c0, n, da);
        store8((T*)a.db + row * a.db_stride + c0, n, db);
        if (a.yq) put_codes(g, a.yq, a.ye, row, c0, y);
    }
}

Grid grid_of(long long rows, int cols, int vecs, unsigned& blocks, long long stride0 = 0, long long stride1 = 0) {
    Grid g;
    g.rows = rows;
    g.cols = cols;
    g.pitch = code_pitch(cols);
    g.vectors = (unsigned)g.pitch / 8;
    g.magic = (unsigned)((1ull << 32) / g.vectors) + 1;
    g.over[0] = stride0 ? over_rows(rows, cols, stride0) : 0;
    g.over[1] = stride1 ? over_rows(rows, cols, stride1) : 0;
    blocks = (unsigned)((rows * g.vectors + TPB * vecs - 1) / (TPB * vecs));
    return g;
}

template <typename T>
hipError_t glu_forward_of(const iodf_glu& a, hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(a.rows, a.cols, GLU_VECS, blocks, a.a_stride, a.b_stride);
    if (a.act == IODF_ACT_RELU) k_glu_forward<T, IODF_ACT_RELU><<<blocks, TPB, 0, st>>>(g, a);
    else if (a.act == IODF_ACT_SILU) k_glu_forward<T, IODF_ACT_SILU><<<blocks, TPB, 0, st>>>(g, a);
    else k_glu_forward<T, IODF_ACT_GELU><<<blocks, TPB, 0, st>>>(g, a);
    return hipGetLastError();
}

template <typename T>
hipError_t glu_backward_of(const iodf_glu& a, hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(a.rows, a.cols, GLU_VECS, blocks, a.dy_stride);
    if (a.act == IODF_ACT_RELU) k_glu_backward<T, IODF_ACT_RELU><<<blocks, TPB, 0, st>>>(g, a);
    else if (a.act == IODF_ACT_SILU) k_glu_backward<T, IODF_ACT_SILU><<<blocks, TPB, 0, st>>>(g, a);
    else k_glu_backward<T, IODF_ACT_GELU><<<blocks, TPB, 0, st>>>(g, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_pack(const void* x, int type, long long stride, long long rows, int cols, const uint8_t* live, int8_t* q,
                       uint8_t* e, hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(rows, cols, type == IODF_T_F32 ? pack_vecs<float>() : pack_vecs<__bf16>(), blocks, stride);
    if (type == IODF_T_F32) k_pack<float><<<blocks, TPB, 0, st>>>(g, (const float*)x, stride, live, q, e);
    else if (type == IODF_T_BF16) k_pack<__bf16><<<blocks, TPB, 0, st>>>(g, (const __bf16*)x, stride, live, q, e);
    else k_pack<_Float16><<<blocks, TPB, 0, st>>>(g, (const _Float16*)x, stride, live, q, e);
    return hipGetLastError();
}

hipError_t launch_unpack(const int8_t* q, const uint8_t* e, long long rows, int cols, void* y, int type, long long stride,
                         hipStream_t st) {
    unsigned blocks;
    const Grid g = grid_of(rows, cols, UNPACK_VECS, blocks);
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
