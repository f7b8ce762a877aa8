// The join of two blocks of a residual network (norm behind, gate, residual scale, addition, norm before) and its gradients.
//
// A row is held in the registers of LPR threads, NV vectors of eight columns each, so that it is read once although its two norms are
// sums over it. All row types are widened to 32-bit floats on the way in and rounded once on the way out.
#include "block_dev.h"
#include "flow_kernels.h"

#include <algorithm>

namespace iodf {

namespace {

constexpr int TPB = 256;

template <int LPR>
constexpr int threads_of() { return LPR > TPB ? LPR : TPB; }

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
template <typename TH, typename TF, int LPR, int NV>
__global__ __launch_bounds__(threads_of<LPR>()) void k_join_forward(const iodf_join a) {
    constexpr int TEAMS = threads_of<LPR>() / LPR;
    __shared__ float sums[2][LPR > 64 ? LPR / 64 : 1];
    const int team = threadIdx.x / LPR, tid = threadIdx.x % LPR;
    const int cols = a.cols, pitch = (cols + 31) / 32 * 32;
    const float inv_cols = 1.f / (float)cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    float coef[NV][8], wq[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) load_params(a.w_pre, (v * LPR + tid) * 8, cols, wq[v], 0.f);
    int group = -1;
    const int rows = (int)a.rows, gate_rows = a.gate && a.gate_rows < a.rows ? (int)a.gate_rows : 0;
    for (int row = blockIdx.x * TEAMS + team; row < rows; row += gridDim.x * TEAMS) {
        const int g = gate_rows ? row / gate_rows : 0;
        if (g != group) {
            group = g;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c0 = (v * LPR + tid) * 8;
                float wp[8];
                load_params(a.gate ? a.gate + (long long)g * cols : nullptr, c0, cols, coef[v], 1.f);
                load_params(a.w_post, c0, cols, wp, 1.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) coef[v][i] = c0 + i < cols ? alpha * coef[v][i] * wp[i] : 0.f;
            }
        }
        const bool live = !a.live || a.live[row];
        const TH* const h = (const TH*)a.in_stream + (long long)row * a.in_stream_stride;
        const TF* const f = (const TF*)a.in_block + (long long)row * a.in_block_stride;
        float z[NV][8], n[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * LPR + tid) * 8;
            load8(h + c0, cols - c0, z[v]);
            load8(f + c0, live ? cols - c0 : 0, n[v]);
        }
        float ip = 1.f;
        if (a.w_post) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += n[v][i] * n[v][i];
            ip = 1.f / sqrtf(row_sum<LPR>(s, sums[0]) * inv_cols + a.eps);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[v][i] *= ip;
                z[v][i] += coef[v][i] * n[v][i];
            }
        TH* const ho = (TH*)a.out_stream + (long long)row * a.out_stream_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * LPR + tid) * 8;
            store8(ho + c0, cols - c0, z[v]);
            if (a.nq) store_codes(a.nq, a.ne, row, pitch, c0, n[v]);
        }
        if (a.inv_post && tid == 0) a.inv_post[row] = live ? ip : 0.f;
        if (a.w_pre) {
            float s = 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) s += z[v][i] * z[v][i];
            const float iq = 1.f / sqrtf(row_sum<LPR>(s, sums[1]) * inv_cols + a.eps);
            TF* const u = (TF*)a.out_block + (long long)row * a.out_block_stride;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c0 = (v * LPR + tid) * 8;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    z[v][i] = live ? z[v][i] * iq : 0.f;
                    o[i] = z[v][i] * wq[v][i];
                }
                store8(u + c0, cols - c0, o);
                if (a.xq) store_codes(a.xq, a.xe, row, pitch, c0, z[v]);
            }
            if (a.inv_pre && tid == 0) a.inv_pre[row] = live ? iq : 0.f;
        }
        if (LPR > 64) __syncthreads();  // a row with one norm would otherwise meet the next row's sums in the same slot
    }
}

// How the backward pass deals rows to workgroups: runs of `chunk` rows, each within one group of rows that share a gate, so that a
// run's sums belong to one row of dgate.
struct Runs {
    int per_group, chunk, groups, gate_rows;
};

// dx = du * w_pre, dz = dh' + inv_pre (dx - x mean(dx x)), dn = coef dz, df = inv_post (dn - n mean(dn n)); sums over the run's rows of
// du x and of dz n (where every row has a gate of its own: of gate dz n, and dgate is written at once).
template <typename TH, typename TF, int LPR, int NV>
__global__ __launch_bounds__(threads_of<LPR>()) void k_join_backward(const iodf_join a, const Runs runs, float* sum_pre, float* sum_post,
                                                                     unsigned* ticket) {
    constexpr int THREADS = threads_of<LPR>(), TEAMS = THREADS / LPR;
    __shared__ float sums[2][LPR > 64 ? LPR / 64 : 1];
    __shared__ float joined[TEAMS > 1 ? THREADS * 8 : 1];
    const int team = threadIdx.x / LPR, tid = threadIdx.x % LPR;
    const int cols = a.cols, pitch = (cols + 31) / 32 * 32, wide = (cols + 7) / 8 * 8;
    const float inv_cols = 1.f / (float)cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    const bool own_gate = runs.gate_rows == 1;
    if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
    const int group = own_gate ? 0 : blockIdx.x / runs.per_group, part = own_gate ? blockIdx.x : blockIdx.x % runs.per_group;
    const int rows = (int)a.rows;
    const int group_end = own_gate ? rows : min((long long)rows, (long long)(group + 1) * runs.gate_rows);
    const int first = (own_gate ? 0 : group * runs.gate_rows) + part * runs.chunk;
    const int last = min((long long)group_end, (long long)first + runs.chunk);
    float coef[NV][8], wq[NV][8], pre[NV][8], post[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c0 = (v * LPR + tid) * 8;
        float wp[8];
        load_params(a.w_pre, c0, cols, wq[v], 0.f);
        load_params(a.w_post, c0, cols, wp, 1.f);
        load_params(a.gate && !own_gate ? a.gate + (long long)group * cols : nullptr, c0, cols, coef[v], 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            coef[v][i] *= alpha * wp[i];
            pre[v][i] = post[v][i] = 0.f;
        }
    }
    for (int row = first + team; row < last; row += TEAMS) {
        const bool live = !a.live || a.live[row];
        const TH* const dh = (const TH*)a.in_stream + (long long)row * a.in_stream_stride;
        const TF* const du = (const TF*)a.in_block + (long long)row * a.in_block_stride;
        TH* const dho = (TH*)a.out_stream + (long long)row * a.out_stream_stride;
        TF* const df = (TF*)a.out_block + (long long)row * a.out_block_stride;
        float dz[NV][8], n[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * LPR + tid) * 8;
            load8(dh + c0, cols - c0, dz[v]);
            load_codes(a.nq, a.ne, row, pitch, live ? c0 : pitch, n[v]);
        }
        if (a.w_pre) {
            float x[NV][8], dx[NV][8], s = 0.f;
            const float iq = live ? a.inv_pre[row] : 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int c0 = (v * LPR + tid) * 8;
                load8(du + c0, live ? cols - c0 : 0, dx[v]);
                load_codes(a.xq, a.xe, row, pitch, live ? c0 : pitch, x[v]);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    pre[v][i] += dx[v][i] * x[v][i];
                    dx[v][i] *= wq[v][i];
                    s += dx[v][i] * x[v][i];
                }
            }
            s = row_sum<LPR>(s, sums[0]) * inv_cols;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) dz[v][i] += iq * (dx[v][i] - x[v][i] * s);
        }
        float s = 0.f;
        float dn[NV][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * LPR + tid) * 8;
            store8(dho + c0, cols - c0, dz[v]);
            float gate[8];
            if (own_gate) load8(a.gate + (long long)row * cols + c0, cols - c0, gate);
            float share[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = live ? dz[v][i] : 0.f;  // padding goes to dL/dh as it came, and nowhere else
                share[i] = d * n[v][i];
                dn[v][i] = coef[v][i] * d;
                if (own_gate) {
                    dn[v][i] *= gate[i];
                    post[v][i] += gate[i] * share[i];
                    share[i] *= coef[v][i];
                } else {
                    post[v][i] += share[i];
                }
                s += dn[v][i] * n[v][i];
            }
            if (own_gate) store8(a.dgate + (long long)row * cols + c0, cols - c0, share);
        }
        if (a.w_post) {
            s = row_sum<LPR>(s, sums[1]) * inv_cols;
            const float ip = live ? a.inv_post[row] : 0.f;
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int i = 0; i < 8; ++i) dn[v][i] = ip * (dn[v][i] - n[v][i] * s);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * LPR + tid) * 8;
            store8(df + c0, cols - c0, dn[v]);
        }
        if (LPR > 64) __syncthreads();
    }
    // the teams' sums meet in the order of the teams
    float* const to[2] = {sum_pre + (long long)blockIdx.x * wide, sum_post + (long long)blockIdx.x * wide};
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int c0 = (v * LPR + tid) * 8;
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = k ? post[v][i] : pre[v][i];
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
            if (team == 0 && c0 < wide) store8(to[k] + c0, 8, t);
        }
}

// The parameters' gradients from the runs' sums. A workgroup has FC columns and FR threads for each, which share the runs: dw_pre over
// all, and group by group dgate = alpha w_post S, dw_post = alpha sum gate S, S a group's sum. The workgroup that ends last
// adds the workgroups' parts of dalpha = sum gate w_post S, in their order.
constexpr int FC = 16, FR = 64;

__device__ __forceinline__ float column_sum(const float* p, int n, int wide, int lane, int lanes) {
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    int r = lane;
    for (; r + 3 * lanes < n; r += 4 * lanes)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] += p[(long long)(r + k * lanes) * wide];
    for (; r < n; r += lanes) s[0] += p[(long long)r * wide];
    return (s[0] + s[1]) + (s[2] + s[3]);
}

__global__ __launch_bounds__(FC* FR) void k_join_params(const iodf_join a, const Runs runs, int n_runs, const float* sum_pre,
                                                        const float* sum_post, double* parts, unsigned* ticket) {
    __shared__ float meet[FR][FC];
    __shared__ double total[FR][FC];
    const int col = threadIdx.x % FC, lane = threadIdx.x / FC, c = blockIdx.x * FC + col;
    const int cols = a.cols, wide = (cols + 7) / 8 * 8;
    const bool there = c < cols;
    const float alpha = a.alpha ? a.alpha[0] : 1.f;
    const float wp = there && a.w_post ? a.w_post[c] : 1.f;
    if (a.dw_pre) {
        meet[lane][col] = there ? column_sum(sum_pre + c, n_runs, wide, lane, FR) : 0.f;
        __syncthreads();
        if (lane == 0 && there) {
            double s = 0;
            for (int k = 0; k < FR; ++k) s += meet[k][col];
            a.dw_pre[c] = (float)s;
        }
        __syncthreads();
    }
    // FR threads of a column are cut into `teams` for as many groups at a time
    const bool own_gate = runs.gate_rows == 1;
    const int per_group = own_gate ? n_runs : runs.per_group, groups = own_gate ? 1 : runs.groups;
    int lanes = 1;
    while (lanes < per_group && lanes < FR) lanes *= 2;
    const int teams = FR / lanes, team = lane / lanes, sub = lane % lanes;
    double weighted = 0;  // sum over this thread's groups of gate * S
    for (int g0 = 0; g0 < groups; g0 += teams) {
        const int g = g0 + team;
        const bool mine = there && g < groups;
        meet[lane][col] = mine ? column_sum(sum_post + (long long)g * per_group * wide + c, per_group, wide, sub, lanes) : 0.f;
        if (lanes > 1) __syncthreads();
        if (mine && sub == 0) {
            double s = 0;
            for (int k = 0; k < lanes; ++k) s += meet[lane + k][col];
            if (own_gate || !a.gate) {
                weighted += s;  // the gates are in the sums already, or are 1
            } else {
                const long long at = (long long)g * cols + c;
                weighted += a.gate[at] * s;
                a.dgate[at] = (float)(alpha * wp * s);
            }
        }
        if (lanes > 1) __syncthreads();
    }
    total[lane][col] = weighted;
    __syncthreads();
    if (lane == 0) {
        double s = 0;
        for (int k = 0; k < FR; ++k) s += total[k][col];
        if (there && a.dw_post) a.dw_post[c] = (float)(alpha * s);
        total[0][col] = there ? wp * s : 0;
    }
    __syncthreads();
    if (a.dalpha && threadIdx.x == 0) {
        double s = 0;
        for (int k = 0; k < FC; ++k) s += total[0][k];
        __hip_atomic_store(&parts[blockIdx.x], s, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (__hip_atomic_fetch_add(ticket, 1u, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1) {
            s = 0;
            for (int k = 0; k < (int)gridDim.x; ++k) s += __hip_atomic_load(&parts[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            a.dalpha[0] = (float)s;
        }
    }
}

template <typename TH, typename TF, int LPR, int NV>
hipError_t forward_of(const iodf_join& a, hipStream_t st) {
    constexpr int TEAMS = threads_of<LPR>() / LPR;
    const long long blocks = (a.rows + TEAMS - 1) / TEAMS;
    // a workgroup keeps the parameters of its columns in registers over several rows
    k_join_forward<TH, TF, LPR, NV><<<(unsigned)std::min<long long>(blocks, 256 * 8), threads_of<LPR>(), 0, st>>>(a);
    return hipGetLastError();
}

template <typename TH, typename TF>
hipError_t forward_types(const iodf_join& a, hipStream_t st) {
    if (a.cols <= 64) return forward_of<TH, TF, 8, 1>(a, st);
    if (a.cols <= 128) return forward_of<TH, TF, 16, 1>(a, st);
    if (a.cols <= 256) return forward_of<TH, TF, 32, 1>(a, st);
    if (a.cols <= 512) return forward_of<TH, TF, 64, 1>(a, st);
    if (a.cols <= 1024) return forward_of<TH, TF, 64, 2>(a, st);
    if (a.cols <= 2048) return forward_of<TH, TF, 256, 1>(a, st);
    if (a.cols <= 4096) return forward_of<TH, TF, 256, 2>(a, st);
    if (a.cols <= 8192) return forward_of<TH, TF, 512, 2>(a, st);
    return forward_of<TH, TF, 1024, 2>(a, st);
}

int backward_teams(int cols) { return cols <= 64 ? 32 : cols <= 128 ? 16 : cols <= 256 ? 8 : cols <= 1024 ? 4 : 1; }

// Runs of rows: about four workgroups to a compute unit, each with at least two rows to a team.
Runs runs_of(long long rows, int cols, long long gate_rows) {
    Runs r;
    if (gate_rows > rows || gate_rows < 1) gate_rows = rows;
    const int teams = backward_teams(cols);
    const long long want = 1024;
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

template <typename TH, typename TF, int LPR, int NV>
hipError_t backward_of(const iodf_join& a, void* work, hipStream_t st) {
    const Runs r = runs_of(a.rows, a.cols, a.gate ? a.gate_rows : a.rows);
    const long long n = n_runs(r, a.rows);
    const size_t wide = (a.cols + 7) / 8 * 8, parts = (a.cols + FC - 1) / FC;
    unsigned* const ticket = (unsigned*)work;
    double* const part = (double*)((char*)work + 16);
    float* const pre = (float*)((char*)part + up16(parts * 8));
    float* const post = pre + n * wide;
    hipError_t e = hipSuccess;
    if (n) {
        k_join_backward<TH, TF, LPR, NV><<<(unsigned)n, threads_of<LPR>(), 0, st>>>(a, r, pre, post, ticket);
        e = hipGetLastError();
    } else {
        e = launch_fill_zero(ticket, 16, st);
    }
    if (e != hipSuccess) return e;
    k_join_params<<<(unsigned)parts, FC * FR, 0, st>>>(a, r, (int)n, pre, post, part, ticket);
    return hipGetLastError();
}

template <typename TH, typename TF>
hipError_t backward_types(const iodf_join& a, void* w, hipStream_t st) {
    if (a.cols <= 64) return backward_of<TH, TF, 8, 1>(a, w, st);
    if (a.cols <= 128) return backward_of<TH, TF, 16, 1>(a, w, st);
    if (a.cols <= 256) return backward_of<TH, TF, 32, 1>(a, w, st);
    if (a.cols <= 512) return backward_of<TH, TF, 64, 1>(a, w, st);
    if (a.cols <= 1024) return backward_of<TH, TF, 64, 2>(a, w, st);
    if (a.cols <= 2048) return backward_of<TH, TF, 256, 1>(a, w, st);
    if (a.cols <= 4096) return backward_of<TH, TF, 256, 2>(a, w, st);
    if (a.cols <= 8192) return backward_of<TH, TF, 512, 2>(a, w, st);
    return backward_of<TH, TF, 1024, 2>(a, w, st);
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
    const size_t wide = (cols + 7) / 8 * 8, parts = (cols + FC - 1) / FC;
    return 16 + up16(parts * 8) + 2 * (size_t)n_runs(r, rows) * wide * 4;
}

hipError_t launch_join_backward(const iodf_join& a, void* work, hipStream_t st) {
    if (a.block_type == IODF_T_F32) return backward_types<float, float>(a, work, st);
    if (a.block_type == IODF_T_BF16)
        return a.stream_type == IODF_T_F32 ? backward_types<float, __bf16>(a, work, st) : backward_types<__bf16, __bf16>(a, work, st);
    return a.stream_type == IODF_T_F32 ? backward_types<float, _Float16>(a, work, st) : backward_types<_Float16, _Float16>(a, work, st);
}

}  // namespace iodf
