// The join of two blocks of a residual network (norm behind, gate, residual scale, addition, norm before) and its gradients.
//
// A row is held in the registers of LPR threads, NV vectors of eight columns each, so that it is read once although its two norms are
// sums over it. All row types are widened to 32-bit floats on the way in and rounded once on the way out.
#include "block_dev.h"

#include <algorithm>

namespace iodf {

namespace {

// Threads of a workgroup: several rows to a workgroup up to a wave a row, one row past that, whose sums meet in LDS.
template <int LPR>
constexpr int threads_of() { return LPR > 64 ? LPR : 256; }

// Which of a workgroup's rows a thread has a part in. Where a wave lies within one row, its number, and with it every address that hangs on
// it, is kept in scalar registers.
template <int LPR>
__device__ __forceinline__ int team_of() {
    return LPR > 64 ? 0 : LPR == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / 64) : threadIdx.x / LPR;
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
            ip = __builtin_amdgcn_rsqf(s * inv_cols + a.eps);
        }
        const long long out = (long long)row * a.out_stream_stride;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                n[v][i] *= ip;
                z[v][i] += coef[v][i] * n[v][i];
            }
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
            const float iq = __builtin_amdgcn_rsqf(s * inv_cols + a.eps);
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

// dx = du * w_pre, dz = dh' + inv_pre (dx - x mean(dx x)), dn = alpha gate w_post dz, df = inv_post (dn - n mean(dn n)); sums over the run's rows
// of du x and of dz n (where every row has a gate of its own: of gate dz n, and dgate is written at once).
// The second mean needs the first one, but it is linear in dz: with m = gate w_post n,
//   sum(m dz) = sum(m dh') + inv_pre (sum(m dx) - mean(dx x) sum(m x)),
// so that a row meets once, for four sums, and not twice. That sum is also the row's part of dalpha (and alpha may be 0).
template <typename TH, typename TF, int LPR, int NV, bool OWN>
__global__ __launch_bounds__(threads_of<LPR>(), OWN ? 1 : sizeof(TF) == 4 || LPR <= 64 ? 3 : 4) void k_join_backward(const iodf_join a, const Runs runs, const int over_h, const int over_u,
                                                                     float* sum_pre, float* sum_post, double* sum_alpha) {
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
    float coef[NV][8], wq[NV][8], pre[NV][8], post[NV][8];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int c0 = (v * LPR + tid) * 8;
        float wp[8];
        load_params(a.w_pre, c0, cols, wq[v], 0.f);
        load_params(a.w_post, c0, cols, wp, 1.f);
        load_params(a.gate && !OWN ? a.gate + (long long)group * cols : nullptr, c0, cols, coef[v], 1.f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            coef[v][i] *= wp[i];
            pre[v][i] = post[v][i] = 0.f;
        }
    }
    Columns c[NV];
#pragma unroll
    for (int v = 0; v < NV; ++v) c[v] = columns_at((v * LPR + tid) * 8, cols);
    struct Row {
        Raw8<TH> h[NV];
        Raw8<TF> u[NV];
        RawCodes x[NV], n[NV];
        Raw8<float> gate[OWN ? NV : 1];
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
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            r.h[v] = fetch_row(dh, c[v], row < over_h);
            r.n[v] = {*(const u32x2*)(a.nq + q + c[v].at), (a.ne + e)[c[v].at / 32]};
            if (a.w_pre) {
                r.u[v] = fetch_row(du, c[v], row < over_u);
                r.x[v] = {*(const u32x2*)(a.xq + q + c[v].at), (a.xe + e)[c[v].at / 32]};
            }
            if (OWN) r.gate[v] = fetch_row(a.gate + (long long)row * cols, c[v], false);
        }
        r.iq = a.w_pre ? a.inv_pre[row] : 0.f;
        r.ip = a.w_post ? a.inv_post[row] : 1.f;
        return r;
    };
    double to_alpha = 0;
    constexpr bool AHEAD = NV == 1;  // two vectors to a thread leave no registers for another row
    Row next;
    int row = first + team;
    if (AHEAD && row < last) next = fetch(row);
    for (; row < last; row += TEAMS) {
        Row r = AHEAD ? next : fetch(row);
        if (AHEAD && row + TEAMS < last) next = fetch(row + TEAMS);  // on its way while this row's sums are taken
        TH* const dho = (TH*)a.out_stream + (long long)row * a.out_stream_stride;
        TF* const df = (TF*)a.out_block + (long long)row * a.out_block_stride;
        float* const dgate = OWN ? a.dgate + (long long)row * cols : nullptr;
        if (!r.live) {  // padding goes to dL/dh as it came, and nowhere else
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                float dz[8];
                const float none[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                widen8(r.h[v], dz);
                store8(dho + c[v].c0, c[v].n, dz);
                store8(df + c[v].c0, c[v].n, none);
                if (OWN) store8(dgate + c[v].c0, c[v].n, none);
            }
            continue;
        }
        // a lane's eight columns have one step: the codes are used as numbers, and sums get their steps at the end
        float sum[4] = {0.f, 0.f, 0.f, 0.f};  // of dx x, m dh', m dx, m x
        float sx[NV], sn[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float dh[8], du[8], x[8], n[8], gate[8], part[4] = {0.f, 0.f, 0.f, 0.f};
            c[v].cut(r.h[v]);
            if (a.w_pre) c[v].cut(r.u[v]);
            widen8(r.h[v], dh);
            numbers8(r.n[v].q, n);
            sn[v] = code_step(r.n[v].e);
            if (OWN) widen8(r.gate[v], gate);
            if (a.w_pre) {
                widen8(r.u[v], du);
                numbers8(r.x[v].q, x);
                sx[v] = code_step(r.x[v].e);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float m = coef[v][i] * n[i];
                if (OWN) m *= gate[i];
                part[1] += m * dh[i];
                if (a.w_pre) {
                    const float dx = du[i] * wq[v][i];
                    pre[v][i] += du[i] * sx[v] * x[i];
                    part[0] += dx * x[i];
                    part[2] += m * dx;
                    part[3] += m * x[i];
                }
            }
            sum[1] += c[v].n ? part[1] * sn[v] : 0.f;
            if (a.w_pre) {
                sum[0] += c[v].n ? part[0] * sx[v] : 0.f;
                sum[2] += c[v].n ? part[2] * sn[v] : 0.f;
                sum[3] += c[v].n ? part[3] * sn[v] * sx[v] : 0.f;
            }
            forget(r.h[v]), forget(r.n[v]);
            if (a.w_pre) forget(r.u[v]), forget(r.x[v]);
        }
        row_sums<LPR, 4>(sum, meet, turn);
        const float mean_x = sum[0] * inv_cols, part_alpha = sum[1] + r.iq * (sum[2] - mean_x * sum[3]);
        const float mean_n = a.w_post ? alpha * part_alpha * inv_cols : 0.f, scale_n = alpha * r.ip;
        to_alpha += part_alpha;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float dz[8], n[8], gate[8], share[8], dn[8];
            widen8(r.h[v], dz);
            numbers8(r.n[v].q, n);
            if (OWN) widen8(r.gate[v], gate);
            if (a.w_pre) {
                float du[8], x[8];
                widen8(r.u[v], du);
                numbers8(r.x[v].q, x);
                const float back = r.iq * mean_x * sx[v];
#pragma unroll
                for (int i = 0; i < 8; ++i) dz[i] = fmaf(r.iq, du[i] * wq[v][i], fmaf(-back, x[i], dz[i]));
            }
            const float back = r.ip * mean_n * sn[v];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                share[i] = dz[i] * sn[v] * n[i];
                dn[i] = coef[v][i] * dz[i];
                if (OWN) {
                    dn[i] *= gate[i];
                    post[v][i] += gate[i] * share[i];
                    share[i] *= alpha * coef[v][i];
                } else {
                    post[v][i] += share[i];
                }
                dn[i] = fmaf(scale_n, dn[i], -back * n[i]);
            }
            store8(dho + c[v].c0, c[v].n, dz);
            store8(df + c[v].c0, c[v].n, dn);
            if (OWN) store8(dgate + c[v].c0, c[v].n, share);
        }
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

// The parameters' gradients from the runs' sums. A workgroup has FC columns and FR threads for each, which share the runs: in the first row of
// workgroups group by group for dgate = alpha w_post S and dw_post = alpha sum gate S, S a group's sum, in the second one over all runs for
// dw_pre; a workgroup of the third one adds the runs' parts of dalpha.
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
                weighted += a.gate[at] * s;
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

template <typename TH, typename TF>
hipError_t forward_types(const iodf_join& a, hipStream_t st) {
    if (a.cols <= 8 * 8) return forward_of<TH, TF, 8, 1>(a, st);
    if (a.cols <= 8 * 16) return forward_of<TH, TF, 16, 1>(a, st);
    if (a.cols <= 8 * 32) return forward_of<TH, TF, 32, 1>(a, st);
    if (a.cols <= 8 * 64) return forward_of<TH, TF, 64, 1>(a, st);
    if (a.cols <= 8 * 128) return forward_of<TH, TF, 64, 2>(a, st);
    if (a.cols <= 8 * 192) return forward_of<TH, TF, 192, 1>(a, st);
    if (a.cols <= 8 * 256) return forward_of<TH, TF, 256, 1>(a, st);
    if (a.cols <= 8 * 384) return forward_of<TH, TF, 384, 1>(a, st);
    if (a.cols <= 8 * 512) return forward_of<TH, TF, 512, 1>(a, st);
    if (a.cols <= 8 * 768) return forward_of<TH, TF, 768, 1>(a, st);
    if (a.cols <= 8 * 1024) return forward_of<TH, TF, 1024, 1>(a, st);
    return forward_of<TH, TF, 1024, 2>(a, st);
}

// Threads to a row of the backward pass, one vector to each: a power of two up to a wave, then whole waves in steps of a half of the power below.
int backward_lanes(int cols) {
    for (int lanes : {8, 16, 32, 64, 128, 192, 256, 384, 512, 768})
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

template <typename TH, typename TF, int LPR, int NV>
hipError_t backward_of(const iodf_join& a, void* work, hipStream_t st) {
    const Runs r = runs_of(a.rows, a.cols, a.gate ? a.gate_rows : a.rows);
    const long long n = n_runs(r, a.rows);
    const size_t wide = (a.cols + 7) / 8 * 8, tiles = (a.cols + FC - 1) / FC;
    double* const to_alpha = (double*)work;
    float* const pre = (float*)((char*)work + up16(n * 8));
    float* const post = pre + n * wide;
    const int over_h = (int)over_rows(a.rows, a.cols, a.in_stream_stride), over_u = a.w_pre ? (int)over_rows(a.rows, a.cols, a.in_block_stride) : 0;
    if (n) {
        if (r.gate_rows == 1) k_join_backward<TH, TF, LPR, NV, true><<<(unsigned)n, threads_of<LPR>(), 0, st>>>(a, r, over_h, over_u, pre, post, to_alpha);
        else k_join_backward<TH, TF, LPR, NV, false><<<(unsigned)n, threads_of<LPR>(), 0, st>>>(a, r, over_h, over_u, pre, post, to_alpha);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (!a.dalpha && !a.dgate && !a.dw_post && !a.dw_pre) return hipSuccess;
    k_join_params<<<dim3((unsigned)tiles, a.dalpha ? 3 : a.dw_pre ? 2 : 1), FC * FR, 0, st>>>(a, r, (int)n, pre, post, to_alpha);
    return hipGetLastError();
}

template <typename TH, typename TF>
hipError_t backward_types(const iodf_join& a, void* w, hipStream_t st) {
    if (a.cols > 8 * 1024) return backward_of<TH, TF, 1024, 2>(a, w, st);
    switch (backward_lanes(a.cols)) {
        case 8: return backward_of<TH, TF, 8, 1>(a, w, st);
        case 16: return backward_of<TH, TF, 16, 1>(a, w, st);
        case 32: return backward_of<TH, TF, 32, 1>(a, w, st);
        case 64: return backward_of<TH, TF, 64, 1>(a, w, st);
        case 128: return backward_of<TH, TF, 128, 1>(a, w, st);
        case 192: return backward_of<TH, TF, 192, 1>(a, w, st);
        case 256: return backward_of<TH, TF, 256, 1>(a, w, st);
        case 384: return backward_of<TH, TF, 384, 1>(a, w, st);
        case 512: return backward_of<TH, TF, 512, 1>(a, w, st);
        case 768: return backward_of<TH, TF, 768, 1>(a, w, st);
        default: return backward_of<TH, TF, 1024, 1>(a, w, st);
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
