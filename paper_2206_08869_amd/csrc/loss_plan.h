// How the loss over a table of classes is cut into tiles, slices and pieces, and where what it needs lies in its workspace: rules on sizes, types and alignment, host code without HIP, which a
// test compiles by itself. Included by loss.hip alone.
#pragma once
#include <algorithm>
#include <cmath>

#include "../../include/iodf.h"
#include "plan.h"

namespace iodf {

namespace {

constexpr long long kPieceBytes = 512ll << 20;  // of g
constexpr int kMaxima = 1024;                   // partial maxima of a tensor, at most

// What g of half precision is multiplied with, and the inverse.
struct Scales {
    float g, ig;
};

// A product's tiles and the slices of its sum.
struct Cut {
    int edge, slices, per;
};

// Microseconds that workgroups of a kind take, all of them, on 256 compute units, each `per` tiles (64 along the sum) of `products`: those that fit LDS at a
// time go along together, then the next ones do. Times of a tile and (7, 5, 1.5) of the way to the first products and from the last ones are fitted to
// calls of two to a hundred thousand rows and classes, which they say within a fifth. Of six products tiles of 128 go over the sum once for each, as of one, and
// of tiles of 64 one fits LDS at a time.
float time_of(int edge, float workgroups, int per, int products) {
    const bool apart = products == 1 || products > 3;
    const float most = edge == 256 ? 1.f : edge == 128 ? (apart ? 2.f : 1.f) : products > 3 ? 1.f : products > 2 ? 2.f : products > 1 ? 3.f : 4.f;
    const float each = workgroups / 256.f, at_once = std::min(most, std::max(1.f, each));
    const float rounds = edge > 64 ? std::ceil(each / most) : std::max(1.f, each / most);
    const float step = edge == 256 ? 1.13f : edge == 128 ? (apart && (products > 1 || at_once > 1.f) ? 0.85f : 0.6f)
                       : products > 1 ? std::max(0.25f, 0.23f * at_once) : std::max(0.5f, 0.23f * at_once);
    return rounds * ((edge == 256 ? 7.f : edge == 128 ? 5.f : 1.5f) + per * products * step);
}

// What a gradient's product is: outputs m x n, tiles along its sum, and whether its sums go through memory anyway. m of 0: there is none.
struct Task {
    long long m, n;
    int kts;
    bool kept;
};

// The kind of tile and number of slices of least estimated time, of one product or of two in one launch. Large tiles read operands less often, small ones and
// slices fill the chip when outputs are few, slices at the price of their sums' way through memory and of a second launch.
float cut_of(const Task* tasks, int count, Cut* cuts, int products, int most) {
    float least = 0.f;
    const int planes = products > 3 ? 3 : products > 1 ? 2 : 1;
    for (const int edge : {256, 128, 64}) {
        if (edge > most) continue;
        struct { long long tiles; float read, outputs; } t[2] = {};
        for (int i = 0; i < count; ++i) {
            const Task& k = tasks[i];
            const long long tm = (k.m + edge - 1) / edge, tn = (k.n + edge - 1) / edge;
            const float once = (float)(k.m + k.n) / 5e6f, again = (float)(k.m * (tn - 1) + k.n * (tm - 1)) / 11e6f;
            t[i] = {tm * tn, (float)k.kts * PK * 2 * planes * (once + again), (float)(tm * tn) * edge * edge};
        }
        auto per_of = [&](int i, int slices) { return (tasks[i].kts + slices - 1) / slices; };
        auto may = [&](int i, int slices) { return slices == 1 || (slices <= 256 && tasks[i].kts / slices >= 2); };
        for (int s0 = 1; may(0, s0); s0 *= 2)
            for (int s1 = 1; count > 1 ? may(1, s1) : s1 == 1; s1 *= 2) {
                const int per = count > 1 ? std::max(per_of(0, s0), per_of(1, s1)) : per_of(0, s0);
                const float workgroups = (float)(t[0].tiles * s0 + (count > 1 ? t[1].tiles * s1 : 0));
                float time = std::max(t[0].read + t[1].read, time_of(edge, workgroups, per, products));
                bool join = false;
                for (int i = 0; i < count; ++i) {
                    const int slices = i ? s1 : s0;
                    if (slices > 1 || tasks[i].kept) join = true, time += t[i].outputs * 8.f * slices / 5e6f + 0.035f * slices;
                    else time += t[i].outputs * 4.f / 5e6f;
                }
                if (join) time += 5.f;
                if (least > 0.f && time >= least) continue;
                least = time;
                for (int i = 0; i < count; ++i) {
                    const int p = per_of(i, i ? s1 : s0);
                    cuts[i] = {edge, (tasks[i].kts + p - 1) / p, p};
                }
            }
    }
    return least;
}

// The kind of tile of the logits, classes x rows, and the slices of the columns.
Cut logits_cut(long long classes, long long rows, int kts, int products, int most) {
    Cut best{};
    float least = 0.f;
    for (const int edge : {256, 128, 64}) {
        if (edge > most) continue;
        const float tiles = (float)((classes + edge - 1) / edge) * (float)((rows + edge - 1) / edge);
        for (int slices = 1; slices == 1 || (edge < 256 && slices <= 64 && kts / slices >= 2); slices *= 2) {
            const int per = (kts + slices - 1) / slices;
            float t = time_of(edge, tiles * slices, per, products);
            if (slices > 1) t += 6.f + tiles * edge * edge * 8.f * slices / 5e6f;
            if (!best.edge || t < least) least = t, best = {edge, (kts + per - 1) / per, per};
        }
    }
    return best;
}

struct LossPlan {
    bool wide, u_ready, w_ready, scaled;  // 32-bit operands; whether u and W are copied; whether there are scales of g
    bool fine;                            // g in two parts though the operands have one
    int pitch, kts;
    int few, groups;                      // blocks of 16 rows of k_few (0: tiles), groups of classes to its workgroups
    int few_rows, few_per, few_slices;    // backward: R of k_few_grad, classes to a wave, workgroups along the classes
    Cut logits;
    int tiles;                            // of classes
    int maxima_parts;
    int planes;
    long long rows_up, piece;
    Cut du, dw;
    bool together;                        // du's and dw's products in one launch
    // byte offsets into the workspace
    size_t maxima, scales, u_exp, w_exp, u, w, sums, parts, picked, g, du_sums, dw_sums, bytes;
};

bool in_place(const void* p, long long stride, int cols, bool wide) { return !wide && cols % PK == 0 && stride % 8 == 0 && stride <= (1 << 22) && ((uintptr_t)p & 15) == 0; }

LossPlan loss_plan(const iodf_class_loss& a, bool backward) {
    LossPlan p{};
    p.wide = a.type == IODF_T_F32;
    p.planes = !p.wide ? 1 : backward ? 3 : 2;
    p.pitch = (int)up(a.cols, PK);
    p.kts = p.pitch / PK;
    p.u_ready = !in_place(a.u, a.u_stride, a.cols, p.wide) || (backward && a.live);
    p.w_ready = !in_place(a.w, a.w_stride, a.cols, p.wide);
    p.scaled = backward && a.type == IODF_T_F16;
    // Where a few numbers g make up a gradient, the rounding to 16 bits makes it up to twice as far off as its own last rounding does: of few rows (1 row, 79857
    // classes: 2.0 times), few classes (100000 rows, 14 classes: 1.4), few numbers altogether (14 rows, 7 classes: 1.6) or few columns, where products cost least
    // (23726 rows, 2091 classes of 11 columns: 1.5); 200 rows, 300 classes of 8000 columns 1.26 times, 21 rows, 40000 classes of 3000 1.17. A second part costs a
    // second product: 256 rows, 4000 classes of 512 columns 28 us for 22, 32000 classes of 4096 columns 607 for 339.
    p.fine = backward && !p.wide && (a.rows <= 16 || a.classes <= 32 || a.cols <= 128 || a.rows * a.classes <= 65536);
    // g of few classes is not made wider than a tile of them
    const int most = backward && a.classes <= 64 ? 64 : backward && (p.fine || a.classes <= 128) ? 128 : 256;
    p.logits = logits_cut(a.classes, a.rows, p.kts, !p.wide ? 1 : backward ? 6 : 3, most);
    p.tiles = (a.classes + p.logits.edge - 1) / p.logits.edge;
    p.rows_up = up(a.rows, p.logits.edge);
    // us by k_few and by a copy and tiles, 32000 classes of 1111 columns: in 32 bits 32 and 77 for a row, 49 and 76 for 32, 78 and 76 for 64; in bfloat16 29 and
    // 42 for a row, 37 and 43 for 16, 57 and 43 for 32.
    if (!backward && p.w_ready && a.rows <= (p.wide ? 64 : 16)) {
        const int blocks = (int)((a.rows + 15) / 16), groups = (a.classes + 31) / 32;
        p.few = blocks <= 1 ? 1 : blocks <= 2 ? 2 : 4;
        p.groups = (groups + 2047) / 2048;
        p.tiles = (groups + p.groups - 1) / p.groups;
        p.u_ready = p.w_ready = false;
    }
    // us by k_few and k_few_grad and by tiles, in 32 bits: 24000 classes of 6592 columns 427 and 1088 for a row, 538 and 1088 for 16, 887 and 1088 for 17; 32000 of 1111 188 and 273 for 32;
    // 300 of 96 17 and 19 for 17. With more than 16 rows not where a few classes have long rows, whose sums k_few does not split as well: 100 of 5000 41 and 26 for 24. In bfloat16,
    // where tiles read W as it lies, 363 and 405, 115 and 113, 20 and 21 for a row: not by these.
    if (backward && p.wide && a.rows && (a.rows <= 16 || (a.rows <= 32 && a.cols <= 4ll * a.classes))) {
        p.few = a.rows <= 16 ? 1 : 2;
        const int groups = (a.classes + 31) / 32, span = p.few == 1 ? 256 : 128, across = (a.cols + span - 1) / span, waves = std::max(1, 512 / across) * 4;
        p.groups = (groups + 2047) / 2048;
        p.tiles = (groups + p.groups - 1) / p.groups;
        p.few_rows = a.rows <= 2 ? 2 : a.rows <= 4 ? 4 : a.rows <= 8 ? 8 : a.rows <= 16 ? 16 : 32;
        p.few_per = std::max(4, (a.classes + waves - 1) / waves);
        p.few_slices = (a.classes + 4 * p.few_per - 1) / (4 * p.few_per);
        const size_t g = (size_t)up((long long)a.classes * p.few * 16 * 4, 256);
        p.g = 0, p.du_sums = g;
        p.bytes = g + (a.du ? (size_t)p.few_slices * p.few_rows * across * span * 4 : 0);
        return p;
    }
    p.maxima_parts = (int)std::max<long long>(1, std::min<long long>(kMaxima, (a.rows + 511) / 512));
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += up(bytes, 256);
        return was;
    };
    if (p.scaled) p.maxima = take((size_t)p.maxima_parts * 4);
    if (backward) p.scales = take(sizeof(Scales));
    if (p.wide && !backward && !p.few) p.u_exp = take((size_t)p.rows_up * 4), p.w_exp = take((size_t)p.tiles * p.logits.edge * 4);
    if (p.u_ready) p.u = take((size_t)p.planes * a.rows * p.pitch * 2);
    if (p.w_ready) p.w = take((size_t)p.planes * a.classes * p.pitch * 2);
    if (!p.few && p.logits.slices > 1) p.sums = take((size_t)p.logits.slices * p.tiles * up(a.rows, p.logits.edge) * p.logits.edge * 4);
    if (!backward) {
        p.parts = take((size_t)p.tiles * a.rows * 8), p.picked = take((size_t)a.rows * 4);
    } else if (a.rows) {
        const int g_planes = p.wide ? 3 : p.fine ? 2 : 1;
        const long long edge = p.logits.edge;  // whole tiles: products read up to a multiple of 64 along their sums
        p.piece = std::max(edge, kPieceBytes / (p.rows_up * 2 * g_planes) / edge * edge);
        p.piece = std::min(p.piece, up(a.classes, edge));
        p.g = take((size_t)g_planes * p.rows_up * p.piece * 2);
        const long long here = std::min<long long>(p.piece, a.classes);
        const int products = p.wide ? 6 : p.fine ? 2 : 1;
        const Task tasks[2] = {{a.cols, a.rows, (int)((here + PK - 1) / PK), here < a.classes}, {a.cols, here, (int)((a.rows + PK - 1) / PK), false}};
        const int most = p.fine ? 128 : 256;
        // As for both, whichever are asked for: a gradient has the same bits with the other and without.
        Cut cuts[2];
        const float alone = cut_of(tasks, 1, &p.du, products, most) + cut_of(tasks + 1, 1, &p.dw, products, most);
        if (cut_of(tasks, 2, cuts, products, most) < alone) p.together = a.du && a.dw, p.du = cuts[0], p.dw = cuts[1];
        auto sums = [&](const Cut& c, long long rows) { return (size_t)c.slices * up(rows, c.edge) * up(a.cols, c.edge) * 4; };
        if (a.du && (p.du.slices > 1 || p.piece < a.classes)) p.du_sums = take(sums(p.du, a.rows));
        if (a.dw && p.dw.slices > 1) p.dw_sums = take(sums(p.dw, here));
    }
    p.bytes = at;
    return p;
}

}  // namespace

}  // namespace iodf
