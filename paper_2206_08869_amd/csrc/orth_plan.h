// How an orthogonalising is cut into tiles and pieces, and where what it needs lies in its workspace: rules on sizes and types, host code without HIP, which a test compiles by
// itself. Included by orth.hip alone.
#pragma once
#include <algorithm>
#include <cmath>

#include "../../include/iodf.h"
#include "plan.h"

namespace iodf {

namespace {

constexpr int kNormBlocks = 1024;  // partial sums of squares of a matrix, at most

struct Shape {
    int count, rows, cols, rp, cp, s, sp;  // rp, cp, sp: rounded up to 64; s the shorter side
};

// A square product's tiles, and how many workgroups go through them piece by piece (0: one to a tile).
struct Cut {
    int edge, tiles, pieces;
};

// Estimated times in us, from these measurements (4096 x 4096, 8192 x 2048, 2048 x 512 eight times, 1111 x 520, 777 x 333 three times): a step along a tile's sum and
// product takes 1.13 with tiles of 256, 0.7 of 192, 0.23 to 0.25 a tile of 64 and compute unit; a piece's 1.5 to 1.9 and 0.3 to 0.75, and joining goes by the sums moved. Of
// three products 2048 x 512 eight times takes 131 us with tiles of 256, 94 of 192, 34.5 of 64, 28 + 14 in pieces of 128.
Cut cut_of(long long count, int s, int kts, int products, bool sums) {
    Cut best{};
    float least = 0.f;
    auto take = [&](float t, const Cut& c) {
        if (!best.edge || t < least) least = t, best = c;
    };
    const float steps = (float)kts * products;
    for (const int edge : {256, 192, 64}) {  // whole tiles
        const int n = (s + edge - 1) / edge;
        const float tiles = (float)count * n * (n + 1) / 2;
        if (edge == 64) take(3.f + steps * std::max(products > 1 ? 0.24f : 0.5f, (products > 1 ? 0.25f : 0.23f) * tiles / 256.f), {edge, n, 0});
        else take(15.f + (edge == 256 ? 1.13f : 0.7f) * steps * std::ceil(tiles / 256.f), {edge, n, 0});
    }
    for (const int edge : {256, 128}) {  // pieces
        const int n = (s + edge - 1) / edge, most = edge == 256 || products > 1 ? 256 : 512;
        const long long tiles = count * n * (n + 1) / 2, units = tiles * kts;
        for (int pieces = most; pieces >= 8; pieces /= 2) {
            if (pieces > units || pieces < tiles / 2) continue;
            const float step = edge == 256 ? (sums ? 1.9f : 1.5f) : (sums ? 0.75f : 0.45f) * (products > 1 ? 0.67f : 1.f) * (pieces > 256 ? 2.f : pieces > 128 ? 1.3f : 1.f);
            const float parts = (float)pieces / tiles + 1.f, moved = (float)(pieces + tiles) * edge * edge * 8e-6f;
            take(step * products * std::ceil((float)units / pieces) + 10.f + 0.4f * parts * edge / 128 + 0.15f * moved, {edge, n, pieces});
        }
    }
    return best;
}

struct OrthPlan {
    Shape z;
    bool tall, parts;          // parts: three products
    bool block;                // by k_block
    int groups, per;           // of k_slim, 0: not by it
    Cut first, second;
    int apply_edge;
    int parts_of_norm;
    size_t sums, x0, x1, o, b, d, e, pieces, bytes;
};

OrthPlan orth_plan(long long count, int rows, int cols, int type) {
    OrthPlan p{};
    p.z = {(int)count, rows, cols, (int)up(rows, PK), (int)up(cols, PK), std::min(rows, cols), 0};
    p.z.sp = (int)up(p.z.s, PK);
    p.tall = rows > cols;
    p.parts = type != IODF_T_BF16;
    auto tiles = [&](long long n, int e) { return (n + e - 1) / e; };
    auto apply = [&](int e) { return count * tiles(rows, e) * tiles(cols, e); };
    if (p.z.s <= 64) {
        const int blocks = std::max(p.z.rp, p.z.cp) / 64;
        p.per = blocks <= 4 ? blocks : blocks <= 32 ? (blocks + 15) / 16 : (blocks + 31) / 32;
        p.groups = (blocks + p.per - 1) / p.per;
    }
    p.first = cut_of(count, p.z.s, (p.tall ? p.z.rp : p.z.cp) / PK, p.parts ? 3 : 1, p.tall);
    p.second = cut_of(count, p.z.s, p.z.sp / PK, p.parts ? 3 : 1, false);
    // Tiles of 256 where they half fill the chip, else of 64. us with 256, 128 and 64, a product: 4096 x 4096 133, 167, 213; 8192 x 2048 86, 99, 125; 2048 x 512 eight
    // times 41, 26, 28; 1024 x 4096 48, 25, 22. Three: 4096 x 4096 339, 467, 514; 3000 x 1500 twice 120, 139, 122; 2048 x 512 eight times 62, 52, 49; 2048 x 2048 143,
    // 70, 75; 277 x 1329 eight times 48, 36, 20; 1111 x 520 57, 24, 11.
    p.apply_edge = apply(256) >= 130 ? 256 : 64;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t was = at;
        at += up(bytes, 256);
        return was;
    };
    const size_t x = (size_t)count * p.z.rp * p.z.cp * 2 * 2, s = (size_t)count * p.z.sp * p.z.sp * 2 * (p.parts ? 2 : 1);
    p.parts_of_norm = (int)std::max<long long>(1, std::min<long long>({kNormBlocks, 2048 / std::max<long long>(1, count), ((long long)rows * ((cols + 7) / 8) + 255) / 256}));
    p.sums = take((size_t)count * p.parts_of_norm * 8);
    p.block = p.z.s > 64 && std::max(rows, cols) <= 128;
    if (p.block) {
        p.bytes = at;
        return p;
    }
    p.x0 = take(x);
    if (p.groups) {
        p.pieces = take((size_t)2 * count * p.groups * 64 * 64 * 4);
        p.bytes = at;
        return p;
    }
    p.x1 = take(x), p.o = take(s), p.b = take(s);
    p.d = take((size_t)count * p.z.sp * 4), p.e = take((size_t)count * p.z.sp * 4);
    size_t most = 0;
    for (const Cut& c : {p.first, p.second})
        if (c.pieces) most = std::max(most, (size_t)(count * c.tiles * (c.tiles + 1) / 2 + c.pieces) * c.edge * c.edge * 4);
    p.pieces = take(most);
    p.bytes = at;
    return p;
}

// How many matrices go together: those whose scratch, 16 bytes an element and less, stays within a gigabyte or so, one at least. Fewer would not fill the chip, more do not make it
// fuller: 2^26 elements are 1024 tiles of 256.
long long together(long long count, int rows, int cols) {
    return std::max<long long>(1, std::min<long long>(count, (1ll << 26) / (up(rows, PK) * up(cols, PK))));
}

}  // namespace

}  // namespace iodf
