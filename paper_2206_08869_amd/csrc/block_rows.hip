// The join of two blocks of a residual network (norm behind, gate, residual scale, addition, norm before) and its gradients.
//
// A row is held in the registers of LPR threads, a vector or two of eight columns each, so that it is read once although its two norms are
// sums over it. All row types are widened to 32-bit floats on the way in and rounded once on the way out. Both passes are bound by memory.
#include "block_dev.h"

#include <algorithm>

namespace iodf {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Threads of a workgroup: several rows to a workgroup up to a wave a row, one row past that, whose sums meet in LDS.
template <int LPR>
constexpr int threads_of() { return LPR > 64 ? LPR : 256; }

// Which of a workgroup's rows a thread has a part in. Where a wave lies within one row, its number, and with it every address that hangs on
// it, is kept in scalar registers.
template <int LPR>
__device__ __forceinline__ int team_of() {
    return LPR > 64 ? 0 : LPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / LPR;
}

// 1 / sqrt(x) for x > 0. The instruction takes numbers below the normal ones, which a row of zeros and a tiny eps give, for 0.
__device__ __forceinline__ float inverse_root(float x) {
    const bool tiny = x < 0x1p-126f;
    return __builtin_amdgcn_rsqf(tiny ? x * 0x1p24f : x) * (tiny ? 0x1p12f : 1.f);
}

// coef[c] = alpha * gate[c] * w_post[c]
__device__ __forceinline__ void load_params(const float* p, int c0, int cols, float v[8], float absent) {
    if (p) {
        load8(p + c0, cols - c0, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = absent;
    }
}

// n = f / rms(f), h' = h + coef * n, x = h' / rms(h'), u = w_pre * x.
// As many workgroups as the chip holds, each with its columns' parameters in registers over all its rows; the next row is on its way while a row's
// two sums are taken. Where a wave has a whole row (up to 1024 columns, with two vectors a thread up from 512) no barrier is needed.
// With a checkpoint, 131072 x 512: 192 us for a stream in 32 bits, 137 us in 16 (both 4.9 TB/s; a large copy reaches 5.1); 4.9 to 5.4 TB/s for
// aligned widths from 512 to 16384, 5.3 at 128. Below 64 columns, with 8 threads a row, the time is the launch's and the rows' own (26 us).
template <typename TH, typename TF, int LPR, int NV>
__global__ __launch_bounds__(threads_of<LPR>()) void k_join_forward(const iodf_join a, const int over_h, const int over_f) {
    constexpr int TEAMS = threads_of<LPR>() / LPR;
    __shared__ RowSums<LPR, 1> meet;
    int turn = 0;
    const int team = team_of<LPR>(), tid = threadIdx.x % LPR;
    const int cols = a.cols, pitch = (cols + 31) / 32 * 32;
    const float inv_cols = 1.f / (float)cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    Columns c[NV];
    float coef[NV][8], wq[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        c[v] = columns_at((v * LPR + tid) * 8, cols);
        load_params(a.w_pre, c[v].c0, cols, wq[v], 0.f);
    }
    int group = -1;
    const int rows = (int)a.rows, gate_rows = a.gate && a.gate_rows < a.rows ? (int)a.gate_rows : 0;
    Raw8<TH> hr[NV];
    Raw8<TF> fr[NV];
    bool live = true;
    auto fetch = [&](int row) {
        if (a.live) live = a.live[row];
        const TH* const h = (const TH*)a.in_stream + (long long)row * a.in_stream_stride;
        const TF* const f = (const TF*)a.in_block + (long long)row * a.in_block_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            hr[v] = fetch_row(h, c[v], row < over_h);
            fr[v] = fetch_row(f, c[v], row < over_f);
        }
    };
    int row = blockIdx.x * TEAMS + team;
    if (row < rows) fetch(row);
    while (row < rows) {
        const int g = gate_rows ? row / gate_rows : 0;
        if (g != group) {
            group = g;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float wp[8];
                load_params(a.gate ? a.gate + (long long)g * cols : nullptr, c[v].c0, cols, coef[v], 1.f);
                load_params(a.w_post, c[v].c0, cols, wp, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) coef[v][i] = c[v].c0 + i < cols ? alpha * coef[v][i] * wp[i] : 0.f;
            }
        }
        float z[NV][8], n[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            c[v].cut(hr[v]), c[v].cut(fr[v]);
            widen8(hr[v], z[v]);
            widen8(fr[v], n[v]);
        }
        const bool now = live;
        const int next = row + gridDim.x * TEAMS;
        if (next < rows) fetch(next);  // on its way while this row's sums are taken
        if (!now)
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) n[v][i] = 0.f;
        float ip = 1.f;
        if (a.w_post) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) part += n[v][i] * n[v][i];
                s += c[v].n ? part : 0.f;
            }
            row_sums<LPR, 1>(&s, meet, turn);
            ip = inverse_root(s * inv_cols + a.eps);
        }
        const long long out = (long long)row * a.out_stream_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) n[v][i] *= ip;
            if (now)  // the gate of a padded row may be no number either
#pragma unroll
                for (int i = 0; i < 8; ++i) z[v][i] += coef[v][i] * n[v][i];
            store8((TH*)a.out_stream + out + c[v].c0, c[v].n, z[v]);
            if (a.nq) {
                if (!c[v].n)
#pragma unroll
                    for (int i = 0; i < 8; ++i) n[v][i] = 0.f;  // past the last column the checkpoint holds 0
                store_codes(a.nq, a.ne, row, pitch, c[v].c0, n[v]);
            }
        }
        if (a.inv_post && tid == 0) a.inv_post[row] = now ? ip : 0.f;
        if (a.w_pre) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float part = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) part += z[v][i] * z[v][i];
                s += c[v].n ? part : 0.f;
            }
            row_sums<LPR, 1>(&s, meet, turn);
            const float iq = inverse_root(s * inv_cols + a.eps);
            const long long uo = (long long)row * a.out_block_stride;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float o[8];
                if (!now || !c[v].n)
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[v][i] = 0.f;  // what stands in a padded row may be no number
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[v][i] *= iq;
                    o[i] = z[v][i] * wq[v][i];
                }
                if (!now)
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[v][i] = o[i] = 0.f;
                store8((TF*)a.out_block + uo + c[v].c0, c[v].n, o);
                if (a.xq) store_codes(a.xq, a.xe, row, pitch, c[v].c0, z[v]);
            }
            if (a.inv_pre && tid == 0) a.inv_pre[row] = now ? iq : 0.f;
        }
        row = next;
    }
}

// How the backward pass deals rows to workgroups: runs of `chunk` rows, each within one group of rows that share a gate, so that a
// run's sums belong to one row of dgate.
struct Runs {
    int per_group, chunk, groups, gate_rows;
};

// The gradients of a join, from dh', du and the codes of x and n:
// dx = du * w_pre, dz = dh' + inv_pre (dx - x mean(dx x)), dn = alpha gate w_post dz, df = inv_post (dn - n mean(dn n)); sums over the run's rows
// of du x and of dz n (where every row has a gate of its own: of gate dz n, and dgate is written at once).
// The second mean needs the first one, but it is linear in dz: with m = gate w_post n,
//   sum(m dz) = sum(m dh') + inv_pre (sum(m dx) - mean(dx x) sum(m x)),
// so that a row meets once, for four sums, and not twice. That sum is also the row's part of dalpha (and alpha may be 0).
// One vector to a thread, kept as it was loaded and widened again behind the meeting: held as 32-bit floats it would spill. Registers for four
// waves a SIMD where that spills little, three where rows are 32 bits or a wave's own.
// 32768 x 4096 in bfloat16: 249 to 272 us for 1.35 GB (5.0 to 5.4 TB/s). TB/s for 2^26 elements, stream and block in bfloat16 / in 32 bits: widths
// that fill their threads (1024, 1536, 2048, 4096) 4.4, 4.1, 4.2, 4.4 / 4.4, 4.3, 4.8, 4.9; that leave some of them idle (1112: 28 %, 2104: 49 %,
// 4104: 33 %) 4.0, 3.5, 3.5 / 3.7, 3.8, 4.8. Rows that start at any element, whose vectors straddle lines, cost another 4 to 10 %: 1111, 2100, 4095
// columns 3.6, 3.2, 4.0 / 3.5, 3.5, 4.7.
template <typename TH, typename TF, int LPR, bool OWN>
__global__ __launch_bounds__(threads_of<LPR>(), OWN ? 1 : sizeof(TF) == 4 || LPR <= 64 ? 3 : 4) void k_join_backward(
    const iodf_join a, const Runs runs, const int over_h, const int over_u, float* sum_pre, float* sum_post, double* sum_alpha) {
    constexpr int THREADS = threads_of<LPR>(), TEAMS = THREADS / LPR;
    __shared__ RowSums<LPR, 4> meet;
    int turn = 0;
    __shared__ float joined[TEAMS > 1 ? THREADS * 8 : 1];
    const int team = team_of<LPR>(), tid = threadIdx.x % LPR;
    const int cols = a.cols, pitch = (cols + 31) / 32 * 32, wide = (cols + 7) / 8 * 8;
    const float inv_cols = 1.f / (float)cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    const int group = OWN ? 0 : blockIdx.x / runs.per_group, part = OWN ? blockIdx.x : blockIdx.x % runs.per_group;
    const int rows = (int)a.rows;
    const int group_end = OWN ? rows : min((long long)rows, (long long)(group + 1) * runs.gate_rows);
    const int first = (OWN ? 0 : group * runs.gate_rows) + part * runs.chunk;
    const int last = min((long long)group_end, (long long)first + runs.chunk);
    float coef[8], wq[8], pre[8], post[8];
    float wp[8];
    const Columns c = columns_at(tid * 8, cols);
    load_params(a.w_pre, c.c0, cols, wq, 0.f);
    load_params(a.w_post, c.c0, cols, wp, 1.f);
    load_params(a.gate && !OWN ? a.gate + (long long)group * cols : nullptr, c.c0, cols, coef, 1.f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        coef[i] *= wp[i];
        pre[i] = post[i] = 0.f;
    }
    struct Row {
        Raw8<TH> h;
        Raw8<TF> u;
        RawCodes x, n;
        Raw8<float> gate;
        float iq, ip;
        bool live;
    };
    auto fetch = [&](int row) {
        Row r;
        r.live = true;
        if (a.live) r.live = a.live[row];
        const TH* const dh = (const TH*)a.in_stream + (long long)row * a.in_stream_stride;
        const TF* const du = (const TF*)a.in_block + (long long)row * a.in_block_stride;
        const long long q = (long long)row * pitch, e = (long long)row * (pitch / 32);
        r.h = fetch_row(dh, c, row < over_h);
        r.n = {*(const u32x2*)(a.nq + q + c.at), (a.ne + e)[c.at / 32]};
        if (a.w_pre) {
            r.u = fetch_row(du, c, row < over_u);
            r.x = {*(const u32x2*)(a.xq + q + c.at), (a.xe + e)[c.at / 32]};
        }
        if (OWN) r.gate = fetch_row(a.gate + (long long)row * cols, c, false);
        r.iq = a.w_pre ? a.inv_pre[row] : 0.f;
        r.ip = a.w_post ? a.inv_post[row] : 1.f;
        return r;
    };
    double to_alpha = 0;
    Row next;
    int row = first + team;
    if (row < last) next = fetch(row);
    for (; row < last; row += TEAMS) {
        Row r = next;
        if (row + TEAMS < last) next = fetch(row + TEAMS);  // on its way while this row's sums are taken
        TH* const dho = (TH*)a.out_stream + (long long)row * a.out_stream_stride;
        TF* const df = (TF*)a.out_block + (long long)row * a.out_block_stride;
        float* const dgate = OWN ? a.dgate + (long long)row * cols : nullptr;
        if (!r.live) {  // padding goes to dL/dh as it came, and nowhere else
            float dz[8];
            const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            widen8(r.h, dz);
            store8(dho + c.c0, c.n, dz);
            store8(df + c.c0, c.n, none);
            if (OWN) store8(dgate + c.c0, c.n, none);
            continue;
        }
        // a lane's eight columns have one step: the codes are used as numbers, and sums get their steps at the end
        float sum[4] = {0.f, 0.f, 0.f, 0.f};  // of dx x, m dh', m dx, m x
        const float sn = code_step(r.n.e), sx = a.w_pre ? code_step(r.x.e) : 0.f;
        {
            float dh[8], du[8], x[8], n[8], gate[8], part[4] = {0.f, 0.f, 0.f, 0.f};
            c.cut(r.h);
            if (a.w_pre) c.cut(r.u);
            widen8(r.h, dh);
            numbers8(r.n.q, n);
            if (OWN) widen8(r.gate, gate);
            if (a.w_pre) {
                widen8(r.u, du);
                numbers8(r.x.q, x);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float m = coef[i] * n[i];
                if (OWN) m *= gate[i];
                part[1] += m * dh[i];
                if (a.w_pre) {
                    const float dx = du[i] * wq[i];
                    pre[i] += du[i] * sx * x[i];
                    part[0] += dx * x[i];
                    part[2] += m * dx;
                    part[3] += m * x[i];
                }
            }
            sum[1] += c.n ? part[1] * sn : 0.f;
            if (a.w_pre) {
                sum[0] += c.n ? part[0] * sx : 0.f;
                sum[2] += c.n ? part[2] * sn : 0.f;
                sum[3] += c.n ? part[3] * sn * sx : 0.f;
            }
            forget(r.h), forget(r.n);
            if (a.w_pre) forget(r.u), forget(r.x);
        }
        row_sums<LPR, 4>(sum, meet, turn);
        const float mean_x = sum[0] * inv_cols, part_alpha = sum[1] + r.iq * (sum[2] - mean_x * sum[3]);
        const float mean_n = a.w_post ? alpha * part_alpha * inv_cols : 0.f, scale_n = alpha * r.ip;
        to_alpha += part_alpha;
        float dz[8], n[8], gate[8], share[8], dn[8];
        widen8(r.h, dz);
        numbers8(r.n.q, n);
        if (OWN) widen8(r.gate, gate);
        if (a.w_pre) {
            float du[8], x[8];
            widen8(r.u, du);
            numbers8(r.x.q, x);
            const float back = r.iq * mean_x * sx;
#pragma unroll
            for (int i = 0; i < 8; ++i) dz[i] = fmaf(r.iq, du[i] * wq[i], fmaf(-back, x[i], dz[i]));
        }
        const float back = r.ip * mean_n * sn;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            share[i] = dz[i] * sn * n[i];
            dn[i] = coef[i] * dz[i];
            if (OWN) {
                dn[i] *= gate[i];
                post[i] += gate[i] * share[i];
                share[i] *= alpha * coef[i];
            } else {
                post[i] += share[i];
            }
            dn[i] = fmaf(scale_n, dn[i], -back * n[i]);
        }
        store8(dho + c.c0, c.n, dz);
        store8(df + c.c0, c.n, dn);
        if (OWN) store8(dgate + c.c0, c.n, share);
    }
    // the teams' sums meet in the order of the teams
    if (TEAMS > 1) {
        __shared__ double alphas[TEAMS];
        if (tid == 0) alphas[team] = to_alpha;
        __syncthreads();
        to_alpha = 0;
        for (int m = 0; m < TEAMS; ++m) to_alpha += alphas[m];
    }
    if (threadIdx.x == 0) sum_alpha[blockIdx.x] = to_alpha;
    float* const to[2] = {sum_pre + (long long)blockIdx.x * wide, sum_post + (long long)blockIdx.x * wide};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = k ? post[i] : pre[i];
        if (TEAMS > 1) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) joined[i * THREADS + threadIdx.x] = t[i];
            __syncthreads();
            if (team == 0)
                for (int m = 1; m < TEAMS; ++m)
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[i] += joined[i * THREADS + m * LPR + tid];
        }
        if (team == 0 && c.c0 < wide) store8(to[k] + c.c0, 8, t);
    }
}

// The same for rows of more than 8192 columns, two vectors to each of 1024 threads: with 128 registers to a thread (64 KB of a row, its parameters
// and sums in 256 KB), nothing of a row is held. The vectors are taken one after the other, each fetched while the one before is worked on, once
// for the sums over the row and once more, out of L2, for the gradients; the columns' sums are in LDS and the parameters are read again.
// 4096 x 16384: 267 us in bfloat16, 314 us with a stream in 32 bits (2.5 and 3.0 TB/s); rows held in registers, which spilled: 575 and 785.
template <typename TH, typename TF, bool OWN>
__global__ __launch_bounds__(1024) void k_join_backward_far(const iodf_join a, const Runs runs, const int over_h, const int over_u, float* sum_pre,
                                                            float* sum_post, double* sum_alpha) {
    constexpr int THREADS = 1024, NV = kJoinMaxCols / (8 * THREADS);
    __shared__ RowSums<THREADS, 4> meet;
    __shared__ f32x4 sums[2][NV][2][THREADS];
    int turn = 0;
    const int tid = threadIdx.x, cols = a.cols, pitch = (cols + 31) / 32 * 32, wide = (cols + 7) / 8 * 8;
    const float inv_cols = 1.f / (float)cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    const int group = OWN ? 0 : blockIdx.x / runs.per_group, part = OWN ? blockIdx.x : blockIdx.x % runs.per_group;
    const int rows = (int)a.rows;
    const int group_end = OWN ? rows : min((long long)rows, (long long)(group + 1) * runs.gate_rows);
    const int first = (OWN ? 0 : group * runs.gate_rows) + part * runs.chunk;
    const int last = min((long long)group_end, (long long)first + runs.chunk);
    for (int v = 0; v < NV; ++v)
        for (int k = 0; k < 2; ++k) sums[k][v][0][tid] = sums[k][v][1][tid] = f32x4{0.f, 0.f, 0.f, 0.f};
    auto add = [&](int k, int v, const float (&s)[8]) {  // a thread's own place: no barrier
        sums[k][v][0][tid] += f32x4{s[0], s[1], s[2], s[3]};
        sums[k][v][1][tid] += f32x4{s[4], s[5], s[6], s[7]};
    };
    struct Vector {
        Raw8<TH> h;
        Raw8<TF> u;
        RawCodes x, n;
    };
    auto fetch = [&](int row, int v) {
        Vector r;
        const Columns c = columns_at((v * THREADS + tid) * 8, cols);
        r.h = fetch_row((const TH*)a.in_stream + (long long)row * a.in_stream_stride, c, row < over_h);
        r.n = {*(const u32x2*)(a.nq + (long long)row * pitch + c.at), (a.ne + (long long)row * (pitch / 32))[c.at / 32]};
        if (a.w_pre) {
            r.u = fetch_row((const TF*)a.in_block + (long long)row * a.in_block_stride, c, row < over_u);
            r.x = {*(const u32x2*)(a.xq + (long long)row * pitch + c.at), (a.xe + (long long)row * (pitch / 32))[c.at / 32]};
        }
        return r;
    };
    double to_alpha = 0;
    Vector next;
    if (first < last) next = fetch(first, 0);
    for (int row = first; row < last; ++row) {
        const bool live = !a.live || a.live[row];
        const float iq = a.w_pre ? a.inv_pre[row] : 0.f, ip = a.w_post ? a.inv_post[row] : 1.f;
        const float* const gate = a.gate ? a.gate + (long long)(OWN ? row : group) * cols : nullptr;
        float sum[4] = {0.f, 0.f, 0.f, 0.f};  // of dx x, m dh', m dx, m x
        if (live) {
#pragma unroll 1
            for (int v = 0; v < NV; ++v) {
                Vector r = next;
                next = fetch(row, v + 1 < NV ? v + 1 : 0);
                const Columns c = columns_at((v * THREADS + tid) * 8, cols);
                float dh[8], n[8], m[8], by[8], part[4] = {0.f, 0.f, 0.f, 0.f};
                load_params(a.w_post, c.c0, cols, m, 1.f);
                load_params(gate, c.c0, cols, by, 1.f);
                c.cut(r.h);
                widen8(r.h, dh);
                numbers8(r.n.q, n);
                const float sn = code_step(r.n.e);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    m[i] *= by[i] * n[i];
                    part[1] += m[i] * dh[i];
                }
                sum[1] += c.n ? part[1] * sn : 0.f;
                if (a.w_pre) {
                    float du[8], x[8], to_pre[8];
                    load_params(a.w_pre, c.c0, cols, by, 0.f);
                    c.cut(r.u);
                    widen8(r.u, du);
                    numbers8(r.x.q, x);
                    const float sx = code_step(r.x.e);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        to_pre[i] = du[i] * sx * x[i];
                        part[0] += du[i] * by[i] * x[i];
                        part[2] += m[i] * (du[i] * by[i]);
                        part[3] += m[i] * x[i];
                    }
                    add(0, v, to_pre);
                    sum[0] += c.n ? part[0] * sx : 0.f;
                    sum[2] += c.n ? part[2] * sn : 0.f;
                    sum[3] += c.n ? part[3] * sn * sx : 0.f;
                }
            }
            row_sums<THREADS, 4>(sum, meet, turn);
        }
        const float mean_x = sum[0] * inv_cols, part_alpha = sum[1] + iq * (sum[2] - mean_x * sum[3]);
        const float mean_n = a.w_post ? alpha * part_alpha * inv_cols : 0.f, scale_n = alpha * ip;
        if (live) to_alpha += part_alpha;
        TH* const dho = (TH*)a.out_stream + (long long)row * a.out_stream_stride;
        TF* const df = (TF*)a.out_block + (long long)row * a.out_block_stride;
        float* const dgate = OWN ? a.dgate + (long long)row * cols : nullptr;
#pragma unroll 1
        for (int v = 0; v < NV; ++v) {
            Vector r = next;
            if (v + 1 < NV) next = fetch(row, v + 1);
            else if (row + 1 < last) next = fetch(row + 1, 0);
            const Columns c = columns_at((v * THREADS + tid) * 8, cols);
            float dz[8], dn[8];
            if (!live) {  // padding goes to dL/dh as it came, and nowhere else
                widen8(r.h, dz);
#pragma unroll
                for (int i = 0; i < 8; ++i) dn[i] = 0.f;
                store8(dho + c.c0, c.n, dz);
                store8(df + c.c0, c.n, dn);
                if (OWN) store8(dgate + c.c0, c.n, dn);
                continue;
            }
            float n[8], coef[8], by[8];
            c.cut(r.h);
            widen8(r.h, dz);
            if (a.w_pre) {
                float du[8], x[8];
                load_params(a.w_pre, c.c0, cols, by, 0.f);
                c.cut(r.u);
                widen8(r.u, du);
                numbers8(r.x.q, x);
                const float back = iq * mean_x * code_step(r.x.e);
#pragma unroll
                for (int i = 0; i < 8; ++i) dz[i] = fmaf(iq, du[i] * by[i], fmaf(-back, x[i], dz[i]));
            }
            load_params(a.w_post, c.c0, cols, coef, 1.f);
            load_params(gate, c.c0, cols, by, 1.f);
            numbers8(r.n.q, n);
            const float sn = code_step(r.n.e), back = ip * mean_n * sn;
            float share[8], to_post[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                share[i] = dz[i] * sn * n[i];
                to_post[i] = OWN ? by[i] * share[i] : share[i];
                dn[i] = fmaf(scale_n, coef[i] * by[i] * dz[i], -back * n[i]);
                share[i] *= alpha * coef[i];
            }
            add(1, v, to_post);
            store8(dho + c.c0, c.n, dz);
            store8(df + c.c0, c.n, dn);
            if (OWN) store8(dgate + c.c0, c.n, share);
        }
    }
    if (tid == 0) sum_alpha[blockIdx.x] = to_alpha;
    for (int k = 0; k < 2; ++k)
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * THREADS + tid) * 8;
            float* const to = (k ? sum_post : sum_pre) + (long long)blockIdx.x * wide + c0;
            if (c0 < wide)
                for (int half = 0; half < 2; ++half) *(f32x4*)(to + 4 * half) = sums[k][v][half][tid];
        }
}

// The parameters' gradients from the runs' sums. A workgroup has FC columns and FR threads for each, which share the runs: in the first row of
// workgroups group by group for dgate = alpha w_post S and dw_post = alpha sum gate S, S a group's sum, in the second one over all runs for
// dw_pre; a workgroup of the third one adds the runs' parts of dalpha. Sixteen loads of a thread are in flight. 4096 columns, 512 runs: 10.5 us;
// 1111 columns, 7 gates: 5.4 us. A column's threads take the groups one after the other, FR at a time, so that many shared gates take long: the
// whole backward pass of 131072 x 512 in bfloat16 with 1, 1024, 16384 and 65536 gates takes 153, 179, 491 and 1760 us (a gate for each row: 254).
constexpr int FC = 16, FR = 64;  // a wave has four threads of each column

__device__ __forceinline__ float column_sum(const float* p, int n, int wide, int lane, int lanes) {
    float s[16] = {};
    for (int r = lane; r < n; r += 16 * lanes)
#pragma unroll
        for (int k = 0; k < 16; ++k) s[k] += r + k * lanes < n ? p[(long long)(r + k * lanes) * wide] : 0.f;
#pragma unroll
    for (int d = 8; d; d /= 2)
#pragma unroll
        for (int k = 0; k < d; ++k) s[k] += s[k + d];
    return s[0];
}

__global__ __launch_bounds__(FC* FR) void k_join_params(const iodf_join a, const Runs runs, int n_runs, const float* sum_pre,
                                                        const float* sum_post, const double* sum_alpha) {
    __shared__ double meet[FR / 4][FC];
    const int col = threadIdx.x % FC, lane = threadIdx.x / FC, c = blockIdx.x * FC + col;
    const int cols = a.cols, wide = (cols + 7) / 8 * 8;
    const bool there = c < cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    const float wp = there && a.w_post ? a.w_post[c] : 1.f;
    // the sum over `lanes` neighbouring lanes of a column, for the first of them: four are in a wave, then through LDS
    auto over_lanes = [&](double v, int lanes) {
        if (lanes >= 2) v += __shfl_xor(v, FC);
        if (lanes >= 4) v += __shfl_xor(v, 2 * FC);
        if (lanes > 4) {
            if (lane % 4 == 0) meet[lane / 4][col] = v;
            __syncthreads();
            if (lane % lanes == 0)
                for (int k = 1; k < lanes / 4; ++k) v += meet[lane / 4 + k][col];
            __syncthreads();
        }
        return v;
    };
    if (blockIdx.y == 2) {
        if (blockIdx.x) return;
        double s = 0;
        for (int k = threadIdx.x; k < n_runs; k += FC * FR) s += sum_alpha[k];
        for (int k = 1; k < FC; k *= 2) s += __shfl_xor(s, k);
        s = over_lanes(s, FR);
        if (threadIdx.x == 0) a.dalpha[0] = (float)s;
        return;
    }
    if (blockIdx.y) {
        if (!a.dw_pre) return;
        const double s = over_lanes(there ? column_sum(sum_pre + c, n_runs, wide, lane, FR) : 0.f, FR);
        if (lane == 0 && there) a.dw_pre[c] = (float)s;
        return;
    }
    // FR threads of a column are cut into `teams` for as many groups at a time
    const bool own_gate = runs.gate_rows == 1;
    const int per_group = own_gate ? n_runs : runs.per_group, groups = own_gate ? 1 : runs.groups;
    int lanes = 1;  // of a group: as many as leave every group a team of its own, where there are that many
    while (lanes < per_group && 2 * lanes * groups <= FR) lanes *= 2;
    const int teams = FR / lanes, team = lane / lanes, sub = lane % lanes;
    double weighted = 0;  // sum over this thread's groups of gate * S
    for (int g0 = 0; g0 < groups; g0 += teams) {
        const int g = g0 + team;
        const bool mine = there && g < groups;
        const double s = over_lanes(mine ? column_sum(sum_post + (long long)g * per_group * wide + c, per_group, wide, sub, lanes) : 0.f, lanes);
        if (mine && sub == 0) {
            if (own_gate || !a.gate) {
                weighted += s;  // the gates are in the sums already, or are 1
            } else {
                const long long at = (long long)g * cols + c;
                weighted += s == 0 ? 0 : a.gate[at] * s;  // the gate of padded rows alone may be no number
                a.dgate[at] = (float)(alpha * wp * s);
            }
        }
    }
    weighted = over_lanes(weighted, FR);
    if (lane == 0 && there && a.dw_post) a.dw_post[c] = (float)(alpha * weighted);
}

// Workgroups of a kernel that the chip holds at once.
template <typename K>
int resident(K kernel, int threads) {
    int per_cu = 0, cus = 0, device = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&per_cu, kernel, threads, 0) != hipSuccess || per_cu < 1) per_cu = 1;
    if (hipGetDevice(&device) != hipSuccess || hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, device) != hipSuccess || cus < 1) cus = 256;
    return per_cu * cus;
}

template <typename TH, typename TF, int LPR, int NV>
hipError_t forward_of(const iodf_join& a, hipStream_t st) {
    constexpr int TEAMS = threads_of<LPR>() / LPR;
    // as many workgroups as run at once: each keeps its columns' parameters in registers over all its rows
    static const int most = resident(k_join_forward<TH, TF, LPR, NV>, threads_of<LPR>());
    const long long blocks = std::min<long long>((a.rows + TEAMS - 1) / TEAMS, most);
    k_join_forward<TH, TF, LPR, NV><<<(unsigned)blocks, threads_of<LPR>(), 0, st>>>(a, (int)over_rows(a.rows, a.cols, a.in_stream_stride),
                                                                                     (int)over_rows(a.rows, a.cols, a.in_block_stride));
    return hipGetLastError();
}

// Threads to a row: the fewest that hold it, in powers of two up to a wave and in whole waves past that. Against powers of two alone, 192 and 768
// threads: 1100 columns 214 us against 222 (2^26 elements, 32-bit stream), 4200 columns 148 against 154 (16 bits), the same where these are full; 384
// against 512: 236 against 197 at 2100 columns, so there is none (two workgroups of 384 are twelve waves a unit, two of 512 sixteen).
// 513 to 1024 columns by one wave with two vectors a thread against two waves with one: 185 us against 190 at 1024, 212 against 224 at 700.
template <typename TH, typename TF>
hipError_t forward_types(const iodf_join& a, hipStream_t st) {
    if (a.cols <= 8 * 8) return forward_of<TH, TF, 8, 1>(a, st);
    if (a.cols <= 8 * 16) return forward_of<TH, TF, 16, 1>(a, st);
    if (a.cols <= 8 * 32) return forward_of<TH, TF, 32, 1>(a, st);
    if (a.cols <= 8 * 64) return forward_of<TH, TF, 64, 1>(a, st);
    if (a.cols <= 8 * 128) return forward_of<TH, TF, 64, 2>(a, st);
    if (a.cols <= 8 * 192) return forward_of<TH, TF, 192, 1>(a, st);
    if (a.cols <= 8 * 256) return forward_of<TH, TF, 256, 1>(a, st);
    if (a.cols <= 8 * 512) return forward_of<TH, TF, 512, 1>(a, st);
    if (a.cols <= 8 * 768) return forward_of<TH, TF, 768, 1>(a, st);
    if (a.cols <= 8 * 1024) return forward_of<TH, TF, 1024, 1>(a, st);
    return forward_of<TH, TF, 1024, 2>(a, st);
}

// Threads to a row of the backward pass, one vector to each, as above. 192 threads against 256: 304 us against 322 at 1100 columns, 768 against 1024:
// 253 against 290 at 4200 (32-bit stream); 384 against 512: within 3 % either way.
int backward_lanes(int cols) {
    for (int lanes : {8, 16, 32, 64, 128, 192, 256, 512, 768})
        if (cols <= 8 * lanes) return lanes;
    return 1024;
}
int backward_teams(int cols) { return backward_lanes(cols) > 64 ? 1 : 256 / backward_lanes(cols); }

// Runs of rows: as many workgroups as run at once, but at least four rows to a team while every unit has a workgroup: a run's sums cost as
// much as two rows of 16 bits.
Runs runs_of(long long rows, int cols, long long gate_rows) {
    Runs r;
    if (gate_rows > rows || gate_rows < 1) gate_rows = rows;
    const int teams = backward_teams(cols);
    const long long most = 256 * (backward_lanes(cols) > 64 ? 1024 / backward_lanes(cols) : 3), want = std::min(most, std::max(256ll, rows / (4 * teams)));
    r.gate_rows = (int)gate_rows;
    if (gate_rows == 1 && rows > 1) {
        r.groups = (int)rows;
        r.chunk = (int)std::max<long long>(2 * teams, (rows + want - 1) / want);
        r.per_group = 0;
    } else {
        r.groups = rows ? (int)((rows + gate_rows - 1) / gate_rows) : 1;
        const long long parts = std::max<long long>(1, want / r.groups);  // runs of a group
        r.chunk = (int)std::min(std::max(gate_rows, 1LL), std::max<long long>(2 * teams, (gate_rows + parts - 1) / parts));
        r.per_group = rows ? (int)((gate_rows + r.chunk - 1) / r.chunk) : 0;
        if (rows == 1) r.gate_rows = 2;  // one row is one group, not a gate for each row
    }
    return r;
}

long long n_runs(const Runs& r, long long rows) {
    return r.gate_rows == 1 ? (rows + r.chunk - 1) / r.chunk : (long long)r.groups * r.per_group;
}

size_t up16(size_t n) { return (n + 15) / 16 * 16; }

template <typename TH, typename TF, int LPR, bool FAR = false>
hipError_t backward_of(const iodf_join& a, void* work, hipStream_t st) {
    const Runs r = runs_of(a.rows, a.cols, a.gate ? a.gate_rows : a.rows);
    const long long n = n_runs(r, a.rows);
    const size_t wide = (a.cols + 7) / 8 * 8, tiles = (a.cols + FC - 1) / FC;
    double* const to_alpha = (double*)work;
    float* const pre = (float*)((char*)work + up16(n * 8));
    float* const post = pre + n * wide;
    const int over_h = (int)over_rows(a.rows, a.cols, a.in_stream_stride), over_u = a.w_pre ? (int)over_rows(a.rows, a.cols, a.in_block_stride) : 0;
    if (n) {
        const auto kernel = r.gate_rows == 1 ? (FAR ? k_join_backward_far<TH, TF, true> : k_join_backward<TH, TF, LPR, true>)
                                             : (FAR ? k_join_backward_far<TH, TF, false> : k_join_backward<TH, TF, LPR, false>);
        kernel<<<(unsigned)n, threads_of<LPR>(), 0, st>>>(a, r, over_h, over_u, pre, post, to_alpha);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.dalpha && !a.dgate && !a.dw_post && !a.dw_pre) return hipSuccess;
    k_join_params<<<dim3((unsigned)tiles, a.dalpha ? 3 : a.dw_pre ? 2 : 1), FC * FR, 0, st>>>(a, r, (int)n, pre, post, to_alpha);
    return hipGetLastError();
}

template <typename TH, typename TF>
hipError_t backward_types(const iodf_join& a, void* w, hipStream_t st) {
    if (a.cols > 8 * 1024) return backward_of<TH, TF, 1024, true>(a, w, st);
    switch (backward_lanes(a.cols)) {
        case 8: return backward_of<TH, TF, 8>(a, w, st);
        case 16: return backward_of<TH, TF, 16>(a, w, st);
        case 32: return backward_of<TH, TF, 32>(a, w, st);
        case 64: return backward_of<TH, TF, 64>(a, w, st);
        case 128: return backward_of<TH, TF, 128>(a, w, st);
        case 192: return backward_of<TH, TF, 192>(a, w, st);
        case 256: return backward_of<TH, TF, 256>(a, w, st);
        case 512: return backward_of<TH, TF, 512>(a, w, st);
        case 768: return backward_of<TH, TF, 768>(a, w, st);
        default: return backward_of<TH, TF, 1024>(a, w, st);
    }
}

}  // namespace

hipError_t launch_join_forward(const iodf_join& a, hipStream_t st) {
    if (a.block_type == IODF_T_F32) return forward_types<float, float>(a, st);
    if (a.block_type == IODF_T_BF16)
        return a.stream_type == IODF_T_F32 ? forward_types<float, __bf16>(a, st) : forward_types<__bf16, __bf16>(a, st);
    return a.stream_type == IODF_T_F32 ? forward_types<float, _Float16>(a, st) : forward_types<_Float16, _Float16>(a, st);
}

size_t join_workspace(long long rows, int cols, long long gate_rows) {
    const Runs r = runs_of(rows, cols, gate_rows);
    const size_t wide = (cols + 7) / 8 * 8, n = (size_t)n_runs(r, rows);
    return 16 + up16(n * 8) + 2 * n * wide * 4;
}

hipError_t launch_join_backward(const iodf_join& a, void* work, hipStream_t st) {
    if (a.block_type == IODF_T_F32) return backward_types<float, float>(a, work, st);
    if (a.block_type == IODF_T_BF16)
        return a.stream_type == IODF_T_F32 ? backward_types<float, __bf16>(a, work, st) : backward_types<__bf16, __bf16>(a, work, st);
    return a.stream_type == IODF_T_F32 ? backward_types<float, _Float16>(a, work, st) : backward_types<_Float16, _Float16>(a, work, st);
}

}  // namespace iodf
