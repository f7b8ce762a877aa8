// Gradient of a linear layer's weight from the 8-bit checkpoint of its input: dw[o][c] = scale[c] sum_t dy[t][o] X[t][c].
//
// The sum runs over rows, and both operands hold consecutive columns, so each matrix instruction's operand (eight rows of one column
// to a lane) is a transpose. Tiles of KT rows go to LDS as they lie in memory, codes widened to bfloat16 (exact: seven bits and a sign
// times a power of two) on the way, and the transposing LDS read takes them from there.
// dy of more than eight significant bits is the exact sum of two (half precision) or three (32 bits) bfloat16 parts, multiplied
// one after the other into the same sums. A part is what fits of the rest, cut off and not rounded: rounded, the largest 32-bit numbers would be
// infinite.
#include "block_dev.h"

#include <algorithm>
#include <type_traits>

namespace iodf {

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr int KT = 32;  // rows of a tile: two matrix instructions deep
constexpr int kLiveRows = 1 << 17;  // of a slice, whose padding is kept as bits in LDS, a word for a tile

template <typename T> constexpr int parts_of() { return sizeof(T) == 4 ? 3 : 1; }
template <> constexpr int parts_of<_Float16>() { return 2; }

// Where column chunk c8 (sixteen bytes) of row r of a tile W columns wide lies. The four rows that sixteen lanes read together would be on
// the same banks; moved by 64 bytes a row they cover 256 bytes. Every other eight chunks change places in pairs, for the lanes that
// write two chunks each and so every second one at a time.
template <int W>
__device__ __forceinline__ int chunk_at(int r, int c8) {
    return r * (W / 8) + (W >= 128 ? c8 ^ ((r & 3) << 2) ^ (c8 >> 3 & 1) : c8 ^ ((r & 2) << 1));
}

template <int W>
__device__ __forceinline__ bf8 fragment(const __bf16* tile, int off, int step) {
    // rows step * 16 + 8 * (lane / 32) + 0..3 and + 4..7; `off` is the lane's own place
    union { s16x4 h[2]; bf8 v; } f;
    f.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + off + step * 16 * W));
    f.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + off + (step * 16 + 4) * W));
    return f.v;
}

struct Tiles {
    int m, n, splits, slice;  // tiles of outputs, slices of the rows and rows of a slice
};

// Which tile and slice a workgroup takes. Workgroups go round the eight dies (each with an L2 of its own) in turn; a die gets neighbours: the
// tiles of one slice, in blocks four tiles high, so that a panel of either operand is fetched into as few L2s as may be.
__device__ __forceinline__ void place(const Tiles& t, int& m, int& n, int& split) {
    const unsigned all = gridDim.x, share = all / 8, b = blockIdx.x;
    const unsigned l = b < share * 8 ? b % 8 * share + b / 8 : b, tiles = t.m * t.n;
    split = (int)(l / tiles);
    const unsigned k = l - split * tiles, band = k / (4 * t.n), in = k - band * 4 * t.n;
    const unsigned high = min(4u, t.m - band * 4);
    m = (int)(band * 4 + in % high);
    n = (int)(in / high);
}

// A wave's MT x NT blocks of 32 x 32 outputs from row o0 and column c0 on: lane l holds column l % 32, rows 8 * (i / 4) + 4 * (l / 32) + i % 4 of
// each. Row addresses are scalar, a lane adds its own offset.
template <int MT, int NT>
__device__ __forceinline__ void store_outputs(const f32x16 (&acc)[MT][NT], const iodf_wgrad& a, int o0, int c0, int split, float* partial) {
    const int lane = threadIdx.x & 63, high = 4 * (lane >> 5), low = lane & 31;
    o0 = __builtin_amdgcn_readfirstlane(o0), c0 = __builtin_amdgcn_readfirstlane(c0);
    const long long ld = partial ? a.cols : a.dw_stride;
    float* const base = (partial ? partial + (long long)split * a.out * a.cols : a.dw) + o0 * ld + c0;
    const bool add = !partial && a.accumulate, inside = o0 + MT * 32 <= a.out && c0 + NT * 32 <= a.cols;
    float scale[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) scale[n] = !partial && a.col_scale && c0 + n * 32 + low < a.cols ? a.col_scale[c0 + n * 32 + low] : 1.f;
    const long long off = high * ld + low;
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int r = m * 32 + 8 * (i / 4) + i % 4;
            float* const row = base + r * ld;
            if (inside && !add) {
#pragma unroll
                for (int n = 0; n < NT; ++n) row[off + n * 32] = scale[n] * acc[m][n][i];
            } else if (o0 + r + high < a.out) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    if (c0 + n * 32 + low < a.cols) row[off + n * 32] = (add ? row[off + n * 32] : 0.f) + scale[n] * acc[m][n][i];
            }
        }
}

// BM x BN outputs to a workgroup of four waves, a quarter to each. Operands come through registers, two tiles ahead: for every type of dy, for
// layers too small for tiles of 256, and for narrow ones, which are bound by memory. 100000 rows, 1000 x 37 weights: 40 us, 5.1 TB/s;
// 4096 rows, 1024 x 1024: 36 us with the slices' sums; 16384 rows, 4096 x 4096, dy in 32 bits: 1650 us, 1000 TFLOP/s of the three
// parts' products, in half precision 1222 us, 900 TFLOP/s of two. Tiles of 64 rows instead of 32, half as many barriers: the same within 1 %, 8 % behind for the smallest.
// Padding (LIVE) is bits in LDS and costs 4 to 9 %: 40.5 us instead of 38.4 at 4096 rows, 1024 x 1024; a byte loaded beside each chunk of dy and of
// codes cost up to 140 % (20000 rows, 1030 x 1100, 32 bits: 247 us against 566, 229 without padding).
template <typename TY, int BM, int BN, bool LIVE>
__global__ __launch_bounds__(256) void k_wgrad(const iodf_wgrad a, const Tiles tiles, float* partial) {
    constexpr int THREADS = 256, P = parts_of<TY>(), WM = BM / 2, WN = BN / 2, MT = WM / 32, NT = WN / 32;
    constexpr int AL = KT * BM / 8 / THREADS, BL = KT * BN / 8 / THREADS;  // chunks of eight of dy and of codes that a thread loads
    __shared__ __bf16 at[2][P][KT * BM];
    __shared__ __bf16 bt[2][KT * BN];
    __shared__ uint32_t alive[LIVE ? kLiveRows / KT : 1];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int m0, n0, split;
    place(tiles, m0, n0, split);
    m0 *= BM, n0 *= BN;
    const int pitch = (a.cols + 31) / 32 * 32, epitch = pitch / 32;
    const long long t0 = (long long)split * tiles.slice, t1 = min((long long)a.rows, t0 + tiles.slice);
    const int wm = wave / 2 * WM, wn = wave % 2 * WN;
    if (LIVE) {  // bit r of word k: row t0 + 32 k + r is no padding
        for (int k = wave * 64; k < (int)(t1 - t0); k += THREADS) {
            const unsigned long long bits = __builtin_amdgcn_ballot_w64(t0 + k + lane < t1 && a.live[t0 + k + lane]);
            if (lane < 2) alive[k / 32 + lane] = (uint32_t)(bits >> 32 * lane);
        }
        __syncthreads();
    }

    int a_off[MT], b_off[NT];
    const int fr = (lane >> 5) * 8 + ((lane >> 2) & 3), fc = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int m = 0; m < MT; ++m) a_off[m] = chunk_at<BM>(fr, (wm + m * 32 + fc) / 8) * 8 + (fc & 7);
#pragma unroll
    for (int n = 0; n < NT; ++n) b_off[n] = chunk_at<BN>(fr, (wn + n * 32 + fc) / 8) * 8 + (fc & 7);

    // Chunks past the last column repeat the first, and one that sticks out of its row reads on: both only reach outputs that are not stored.
    // Rows past the slice's end repeat its last one. Only in the eight rows before dy's end, where reading on could leave it, is a chunk that sticks
    // out taken element by element.
    const int ar = tid / (BM / 8), ac = tid % (BM / 8) * 8, br = tid / (BN / 8), bc = tid % (BN / 8) * 8;
    const int acol = m0 + ac < a.out ? m0 + ac : 0, bcol = n0 + bc < pitch ? n0 + bc : 0;
    const TY* const dy = (const TY*)a.dy + ar * a.dy_stride + acol;
    const long long a_step = THREADS * 8 / BM * a.dy_stride;
    const int b_off0 = br * pitch + bcol, e_off0 = br * epitch + bcol / 32, b_step = THREADS * 8 / BN * pitch, e_step = THREADS * 8 / BN * epitch;
    struct Stage {
        Raw8<TY> a[AL];
        RawCodes b[BL];
    };
    auto fetch = [&](Stage& s, long long t, auto guarded) {
        if (!guarded) {
#pragma unroll
            for (int i = 0; i < AL; ++i) s.a[i] = fetch8(dy + t * a.dy_stride + i * a_step, 8, true);
#pragma unroll
            for (int i = 0; i < BL; ++i) s.b[i] = {*(const u32x2*)(a.q + t * pitch + (b_off0 + i * b_step)), (a.e + t * epitch)[e_off0 + i * e_step]};
        } else {
            const bool apart = t1 + 8 > a.rows && a.out % 8 != 0;
#pragma unroll
            for (int i = 0; i < AL; ++i) {
                const long long row = t + ar + i * (THREADS * 8 / BM), at = row < t1 ? row : t1 - 1;
                const TY* const p = (const TY*)a.dy + at * a.dy_stride + acol;
                s.a[i] = apart ? fetch8(p, a.out - acol, false) : fetch8(p, 8, true);
            }
#pragma unroll
            for (int i = 0; i < BL; ++i) {
                const long long row = t + br + i * (THREADS * 8 / BN), at = row < t1 ? row : t1 - 1;
                s.b[i] = {*(const u32x2*)(a.q + at * pitch + bcol), a.e[at * epitch + bcol / 32]};
            }
        }
    };
    // bit r: row r of the tile at t adds something; asked for with rows of the slice in it only
    auto rows_of = [&](long long t, auto guarded) {
        uint32_t rows = LIVE ? alive[(int)(t - t0) / KT] : ~0u;
        if (guarded && t1 - t < KT) rows &= (1u << (int)(t1 - t)) - 1;
        return rows;
    };
    // What adds nothing goes in as zeros of dy and as codes of an exponent with which they are finite (they may stand for NaN, which would outlast
    // the zeros).
    auto put = [&](const Stage& s, int buf, uint32_t rows, auto guarded) {
        const bool some = LIVE || guarded;
#pragma unroll
        for (int i = 0; i < AL; ++i) {
            const int r = ar + i * (THREADS * 8 / BM), to = chunk_at<BM>(r, ac / 8) * 8;
            const bool there = !some || rows >> r & 1;
            if (P == 1) {
                bf8 w;
                __builtin_memcpy(&w, s.a[i].w, 16);
                *(bf8*)&at[buf][0][to] = there ? w : bf8{};
            } else {
                float rest[8];
                widen8(s.a[i], rest);
#pragma unroll
                for (int j = 0; j < 8; ++j) rest[j] = there ? rest[j] : 0.f;
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    u32x4 w;  // the upper halves, two to a word
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = __builtin_amdgcn_perm(__float_as_uint(rest[2 * j + 1]), __float_as_uint(rest[2 * j]), 0x07060302u);
                    *(u32x4*)&at[buf][p][to] = w;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {  // a NaN stays one, an infinity has no rest
                        const float got = __uint_as_float(__float_as_uint(rest[j]) & 0xffff0000u);
                        rest[j] = p || fabsf(rest[j]) != __builtin_inff() ? rest[j] - got : 0.f;
                    }
                }
            }
        }
#pragma unroll
        for (int i = 0; i < BL; ++i) {
            const int r = br + i * (THREADS * 8 / BN);
            float v[8];
            decode8(s.b[i].q, code_step(!some || rows >> r & 1 ? s.b[i].e : 16), v);
            *(bf8*)&bt[buf][chunk_at<BN>(r, bc / 8) * 8] = narrow8(v);
        }
    };

    f32x16 acc[MT][NT];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;

    const std::true_type checked;
    const std::false_type whole;
    Stage st[2];
    if (t0 < t1) {
        fetch(st[0], t0, checked);
        fetch(st[1], t0 + KT, checked);
        put(st[0], 0, rows_of(t0, checked), checked);
        fetch(st[0], t0 + 2 * KT, checked);
    }
    __syncthreads();
    auto two_tiles = [&](long long t, auto guarded) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (guarded && h && t + KT >= t1) break;
            const bool more = !guarded || t + (h + 1) * KT < t1;
            const uint32_t rows = more ? rows_of(t + (h + 1) * KT, guarded) : 0;
#pragma unroll
            for (int s = 0; s < KT / 16; ++s) {
                bf8 bf[NT];
#pragma unroll
                for (int n = 0; n < NT; ++n) bf[n] = fragment<BN>(bt[h], b_off[n], s);
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const bf8 af = fragment<BM>(at[h][p], a_off[m], s);
#pragma unroll
                        for (int n = 0; n < NT; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af, bf[n], acc[m][n], 0, 0, 0);
                    }
            }
            if (more) put(st[h ^ 1], h ^ 1, rows, guarded);
            __builtin_amdgcn_sched_barrier(0);  // one region a tile: over two the compiler reads each operand just before its product
            if (!guarded || t + (h + 3) * KT < t1) fetch(st[h ^ 1], t + (h + 3) * KT, guarded);
            __syncthreads();
        }
    };
    long long t = t0;
    for (; t + 5 * KT + 8 <= t1; t += 2 * KT) two_tiles(t, whole);
    for (; t < t1; t += 2 * KT) two_tiles(t, checked);
    store_outputs<MT, NT>(acc, a, m0 + wm, n0 + wn, split, partial);
}

// ---- large layers, dy in bfloat16 ----
// 256 x 256 outputs to a workgroup of eight waves, 128 x 64 to a wave, two waves to a SIMD. A product keeps a SIMD's matrix core for 32
// clocks and lets about four plain vector instructions of the same wave pass beside it, so all else is dealt out between the products.
// Tile i takes two phases of eight products a wave, one for each step:
//   A  products of step 0, held in registers; reads step 1; widens the second half of tile i + 1's codes
//   the one barrier of a tile
//   B  products of step 1; reads step 0 of tile i + 1; widens the first half of tile i + 2's codes; starts dy of tile i + 4 and codes of tile i + 5
// All loads go straight to LDS, dy to a ring of four tiles, codes to a ring in which every lane has its own places, from which
// it takes them a phase before it widens them. No load lands in a register, so that no wait is the compiler's; wait_loads leaves the loads
// of a tile and a half in flight.
// 16384 rows, 4096 x 4096 weights: 443 to 464 us, 1185 to 1240 TFLOP/s, 0.87 us a tile of 32 rows. The products alone take 1024 clocks, 0.47 us at
// 2.2 GHz, but the clock sinks to about 1.83 under the load, so that clocks saved come back as time only in part (the products
// alone, without loads, widening or LDS writes: 361 us). Four waves of 128 x 128, which read a third less from LDS: 487; codes and dy through
// registers: 505.
//
// Loads carry no bounds checks except near a slice's end: a chunk of dy that sticks out of its row reads the next one's start, and
// chunks past the last column repeat the first; both only reach outputs that are not stored.
constexpr int WIDE = 256, RING = 4;

// Sixteen bytes or one byte (as a word) a lane from memory to LDS, lane after lane from `lds` on. Written out because the compiler, where it
// knows of such a load, waits for all of them before any LDS access that may meet one.
__device__ __forceinline__ void start_lds16(uint32_t lds, const void* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
__device__ __forceinline__ void start_lds16(uint32_t lds, const void* p) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory", "m0");
}
__device__ __forceinline__ void start_lds1(uint32_t lds, const void* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}
template <int LEFT>
__device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

__device__ const uint32_t kZeros[4] = {0, 0, 0, 0};  // what a padded row of dy is read from

template <bool LIVE>
__global__ __launch_bounds__(512, 1) void k_wgrad_wide(const iodf_wgrad a, const Tiles tiles, float* partial) {
    constexpr int THREADS = 512, NT = 2;
    constexpr int LOADS = 4;  // of a thread and tile: sixteen codes, an exponent, two chunks of dy
    __shared__ __bf16 at[RING][KT * WIDE];
    __shared__ __bf16 bt[2][KT * WIDE];
    __shared__ u32x4 raw[RING][512];
    __shared__ uint32_t raw_e[RING][512];
    __shared__ uint32_t alive[LIVE ? kLiveRows / 32 + RING + 2 : 1];  // and of the tiles past the slice that its loop takes too
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int m0, n0, split;
    place(tiles, m0, n0, split);
    m0 *= WIDE, n0 *= WIDE;
    const int pitch = (a.cols + 31) / 32 * 32, epitch = pitch / 32;
    const long long t0 = (long long)split * tiles.slice, t1 = min((long long)a.rows, t0 + tiles.slice);
    const int wm = wave / 4 * 128, wn = wave % 4 * 64;

    // what this thread loads: chunks of eight of dy in rows ar and ar + 16, sixteen codes in row br, an exponent (each one twice a wave). A
    // chunk of dy goes to the place in LDS that its lane has, so the lane takes the chunk that belongs there.
    const int ar = tid / 32, slot = (tid % 32) ^ ((ar & 3) << 2), ac = slot ^ (slot >> 3 & 1);
    const int br = tid / 16, bc = tid % 16, er = wave * 4 + (lane >> 3 & 3), ec = n0 / 32 + (lane & 7);
    const int acol = m0 + ac * 8 < a.out ? m0 + ac * 8 : 0, bcol = n0 + bc * 16 < pitch ? n0 + bc * 16 : 0;
    const unsigned a_voff = (unsigned)(ar * (unsigned)a.dy_stride + acol) * 2, a_step = 16 * (unsigned)a.dy_stride * 2;
    const unsigned b_voff = (unsigned)(br * pitch + bcol), e_voff = (unsigned)(er * epitch + (ec < epitch ? ec : 0));
    auto lds_of = [](const void* p) { return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p; };
    const uint32_t at0 = lds_of(&at[0][0]) + wave * 1024, raw0 = lds_of(&raw[0][0]) + wave * 1024, rawe0 = lds_of(&raw_e[0][0]) + wave * 256;

    if (LIVE) {  // bit r of word k: row t0 + 32 k + r is there and no padding
        const int words = (int)((t1 - t0 + 31) / 32) + RING + 2;
        for (int k = tid; k < words; k += THREADS) {
            uint32_t w = 0;
            for (int r = 0; r < 32; ++r) {
                const long long row = t0 + k * 32ll + r;
                if (row < t1 && a.live[row]) w |= 1u << r;
            }
            alive[k] = w;
        }
        __syncthreads();
    }

    auto start_dy = [&](int to, long long t, auto guarded) {
        const char* const ab = (const char*)a.dy + t * a.dy_stride * 2;
        const uint32_t live = LIVE && !guarded ? alive[(t - t0) / 32] : 0;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = ar + 16 * i;
            if (!guarded) {
                const uint32_t lds = at0 + to * (KT * WIDE * 2) + i * (THREADS * 16);
                if (LIVE) start_lds16(lds, live >> r & 1 ? ab + (a_voff + i * a_step) : (const char*)kZeros);
                else start_lds16(lds, ab, a_voff + i * a_step);
            } else {
                const int n = t + r < t1 && (!LIVE || a.live[t + r]) ? a.out - acol : 0;
                const __bf16* const p = (const __bf16*)(ab + (a_voff + i * a_step));
                u32x4 w;
                if (n >= 8) {
                    w = *(const u32x4_any*)p;
                } else {
                    __bf16 v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = j < n ? p[j] : (__bf16)0.f;
                    __builtin_memcpy(&w, v, 16);
                }
                *(u32x4*)&at[to][(i * THREADS + tid) * 8] = w;
            }
        }
    };
    auto start_codes = [&](int to, long long t, auto guarded) {
        const char* const bb = (const char*)a.q + t * pitch;
        const uint8_t* const eb = a.e + t * epitch;
        if (!guarded) {
            start_lds16(raw0 + to * 8192, bb, b_voff);
            start_lds1(rawe0 + to * 2048, eb, e_voff);
        } else {
            raw[to][tid] = t + br < t1 ? *(const u32x4*)(bb + b_voff) : u32x4{0, 0, 0, 0};
            raw_e[to][tid] = t + er < t1 ? eb[e_voff] : 16;
        }
    };
    // A thread widens eight of its sixteen codes in either phase. Those of a padded row may stand for NaN, which would outlast the zeros that its
    // dy is: with another exponent they are finite.
    u32x2 codes[2];
    uint32_t ex[2];
    auto take_codes = [&](int half, int from, long long t) {
        codes[half] = ((const u32x2*)&raw[from][tid])[half];
        ex[half] = raw_e[from][wave * 64 + (br & 3) * 8 + bc / 2];
        if (LIVE) ex[half] = alive[(int)(t - t0) / 32] >> br & 1 ? ex[half] : 16;
    };
    auto widen = [&](int half, int to) {
        float v[8];
        decode8(codes[half], code_step(ex[half]), v);
        *(bf8*)&bt[to][chunk_at<WIDE>(br, bc * 2 + half) * 8] = narrow8(v);
    };

    int a_off[4], b_off[NT];
    const int fr = (lane >> 5) * 8 + ((lane >> 2) & 3), fc = ((lane >> 4) & 1) * 16 + (lane & 3) * 4;
#pragma unroll
    for (int m = 0; m < 4; ++m) a_off[m] = chunk_at<WIDE>(fr, (wm + m * 32 + fc) / 8) * 8 + (fc & 7);
#pragma unroll
    for (int n = 0; n < NT; ++n) b_off[n] = chunk_at<WIDE>(fr, (wn + n * 32 + fc) / 8) * 8 + (fc & 7);
    f32x16 acc[4][NT];
#pragma unroll
    for (int m = 0; m < 4; ++m)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[m][n][i] = 0.f;
    bf8 fa[2][4], fb[2][NT];
    auto read = [&](int set, int abuf, int bbuf, int step) {
#pragma unroll
        for (int n = 0; n < NT; ++n) fb[set][n] = fragment<WIDE>(bt[bbuf], b_off[n], step);
#pragma unroll
        for (int m = 0; m < 4; ++m) fa[set][m] = fragment<WIDE>(at[abuf], a_off[m], step);
    };
    auto multiply = [&](int set, int half) {
#pragma unroll
        for (int m = 2 * half; m < 2 * half + 2; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[set][m], fb[set][n], acc[m][n], 0, 0, 0);
    };
    auto barrier = [&] {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };

    const std::true_type checked;
    const std::false_type whole;
    // the loads of a tile count LOADS and follow one another as in phase B: codes two, dy two
    auto begin = [&](auto guarded) {
        start_codes(0, t0, guarded);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            start_codes(k + 1, t0 + (k + 1) * KT, guarded);
            start_dy(k, t0 + k * KT, guarded);
        }
        wait_loads<guarded ? 0 : 2 + LOADS>();  // codes of tiles 0, 1 and 2 (whose first half phase A of tile 0 takes) and dy of tile 0 have landed
        take_codes(0, 0, t0), take_codes(1, 0, t0);
        widen(0, 0), widen(1, 0);
        take_codes(0, 1, t0 + KT), take_codes(1, 1, t0 + KT);
        widen(0, 1);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        start_codes(0, t0 + 4 * KT, guarded);
        start_dy(3, t0 + 3 * KT, guarded);
    };
    if (t0 + 6 * KT < t1) begin(whole);
    else begin(checked);
    barrier();
    read(0, 0, 0, 0);

    // Half a phase: left to itself the compiler gathers reads and writes behind the products.
    auto deal = [](auto reads) {
#pragma unroll
        for (int k = 0; k < 2 * NT; ++k) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (reads) __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto four_tiles = [&](long long t, auto guarded) {
#pragma unroll
        for (int h = 0; h < RING; ++h, t += KT) {
            const int now = h & 1, next = now ^ 1;
            read(1, h, now, 1);
            take_codes(0, (h + 2) % RING, t + 2 * KT);
            widen(1, next);
            multiply(0, 0);
            deal(std::true_type());
            multiply(0, 1);
            deal(std::false_type());
            wait_loads<guarded ? 0 : 2 + LOADS>();  // dy of tile i + 1 and codes of tile i + 3 have landed
            barrier();
            __builtin_amdgcn_sched_barrier(0);
            start_codes((h + 1) % RING, t + 5 * KT, guarded);
            read(0, (h + 1) % RING, next, 0);
            take_codes(1, (h + 2) % RING, t + 2 * KT);
            widen(0, now);
            multiply(1, 0);
            deal(std::true_type());
            start_dy(h, t + 4 * KT, guarded);
            multiply(1, 1);
            deal(std::false_type());
        }
    };
    long long t = t0;
    for (; t + 9 * KT < t1; t += RING * KT) four_tiles(t, whole);
    for (; t < t1; t += RING * KT) four_tiles(t, checked);
    store_outputs<4, NT>(acc, a, m0 + wm, n0 + wn, split, partial);
}

// The slices' sums, in an order that their number alone decides: JL threads to an output, or to four neighbours (VEC). 64 slices of 512 x 512: 12 us
// for 64 MB, 5.5 TB/s.
constexpr int JL = 8;

template <int VEC>
__global__ __launch_bounds__(256) void k_wgrad_join(const iodf_wgrad a, int splits, const float* partial) {
    typedef float vec __attribute__((ext_vector_type(VEC)));
    __shared__ vec meet[JL][256 / JL];
    const int lane = threadIdx.x / (256 / JL), at = threadIdx.x % (256 / JL);
    const long long n = (long long)a.out * a.cols, i = (((long long)blockIdx.y * gridDim.x + blockIdx.x) * (256 / JL) + at) * VEC;
    vec s = 0.f;
    if (i < n) {
        int k = lane;
        for (; k + 7 * JL < splits; k += 8 * JL) {
            vec v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = *(const vec*)(partial + (k + u * JL) * n + i);
            s += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
        for (; k < splits; k += JL) s += *(const vec*)(partial + k * n + i);
    }
    meet[lane][at] = s;
    __syncthreads();
    if (lane || i >= n) return;
#pragma unroll
    for (int k = 1; k < JL; ++k) s += meet[k][at];
    const int o = (int)(i / a.cols), c = (int)(i - (long long)o * a.cols);
    float* const d = a.dw + o * a.dw_stride + c;
#pragma unroll
    for (int j = 0; j < VEC; ++j) d[j] = (a.accumulate ? d[j] : 0.f) + (a.col_scale ? a.col_scale[c + j] : 1.f) * s[j];
}

struct Plan : Tiles {
    int bm, bn;  // a tile's edges
};

// What a kind of tile costs, in microseconds: everything but the loop, a step of KT rows when a compute unit has one workgroup of the kind, and
// what each of several adds to a step. Measured with dy in bfloat16; parts of dy are multiplied one after the other.
struct TileCost {
    int bm, bn;
    float base, step, each;
};
constexpr TileCost kTiles[] = {{64, 64, 4.3f, 0.26f, 0.17f}, {64, 128, 6.3f, 0.30f, 0.24f}, {128, 64, 6.3f, 0.30f, 0.24f}, {128, 128, 8.3f, 0.36f, 0.33f},
                               {WIDE, WIDE, 14.f, 0.84f, 0.84f}};

// The tile and the number of slices of least estimated time. Large tiles read operands less often, small ones fill the chip with few outputs and
// end sooner; slices do so with few tiles, at the price of their sums' way through memory (about 0.36 us a megabyte there and back) and of a second
// launch. Over 18 shapes from 64 x 512 x 512 to 131072 x 512 x 512, timed with every tile and slices in powers of two, dy in bfloat16: at 14 the
// choice is within 7 % of the best of them, at two (16384 rows, 2048 x 512 and 66 x 896) 11 and 12 % behind, and at two it takes slices where none
// are better (1000 rows, 130 x 72: 14.0 us against 11.5; 2048 rows, 1024 x 1024: 26.0 against 19.3); with dy in 16 and 32 bits at most 24 and 20 %
// behind. One fixed rule (the largest tile that fills the chip, slices for 512 workgroups) was up to 2.7 times behind (512 x 2048 x 2048: 44 us
// against 16). A step with parts of dy takes 1.5 to 1.9 (two) and 1.8 to 2.5 times (three) as long as one without where steps are most of the time.
Plan plan_of(const iodf_wgrad& a) {
    auto up = [](long long n, long long d) { return (n + d - 1) / d; };
    const float parts = a.dy_type == IODF_T_BF16 ? 1.f : a.dy_type == IODF_T_F16 ? 1.9f : 2.7f;
    Plan best{};
    float least = 0.f;
    for (const TileCost& k : kTiles) {
        // the wide kernel has dy in bfloat16 only and 32-bit offsets within a tile; no tile is twice as large as the layer
        if (k.bm == WIDE && (a.dy_type != IODF_T_BF16 || a.dy_stride > (1 << 24) || a.out <= 128 || a.cols <= 128)) continue;
        if ((k.bm == 128 && a.out <= 64) || (k.bn == 128 && a.cols <= 64)) continue;
        const int unit = k.bm == WIDE ? RING * KT : KT;  // rows that its loop takes at a time
        const long long m = up(a.out, k.bm), n = up(a.cols, k.bn);
        const long long fill = std::max<long long>(1, 256 / (m * n));  // slices that give every unit one workgroup at most
        for (int k2 = -1; k2 <= 10; ++k2) {
            long long splits = k2 < 0 ? fill : 1ll << k2;
            if (splits > 1 && (splits > 1024 || a.rows / splits < KT)) continue;
            if (a.live) splits = std::max<long long>(splits, up(a.rows, kLiveRows));
            const long long slice = up(up(a.rows, splits), unit) * unit;
            splits = slice ? up(a.rows, slice) : 1;
            const float steps = (float)(slice / KT), a_unit = (float)up(m * n * splits, 256), outputs = 4e-6f * a.out * a.cols;
            float t = k.base + steps * parts * std::max(k.step, a_unit * k.each);
            t += splits > 1 ? 3.f + 0.36f * outputs * splits : 0.2f * outputs;
            if (!best.bm || t < least) {
                least = t;
                best.m = (int)m, best.n = (int)n, best.splits = (int)splits, best.slice = (int)slice, best.bm = k.bm, best.bn = k.bn;
            }
        }
    }
    return best;
}

template <typename TY, bool LIVE>
void run_tile(const iodf_wgrad& a, const Plan& p, float* partial, hipStream_t st) {
    const unsigned blocks = (unsigned)(p.m * p.n * p.splits);
    if (p.bm == 128 && p.bn == 128) k_wgrad<TY, 128, 128, LIVE><<<blocks, 256, 0, st>>>(a, p, partial);
    else if (p.bm == 128) k_wgrad<TY, 128, 64, LIVE><<<blocks, 256, 0, st>>>(a, p, partial);
    else if (p.bn == 128) k_wgrad<TY, 64, 128, LIVE><<<blocks, 256, 0, st>>>(a, p, partial);
    else k_wgrad<TY, 64, 64, LIVE><<<blocks, 256, 0, st>>>(a, p, partial);
}

template <typename TY>
hipError_t run(const iodf_wgrad& a, const Plan& p, float* partial, hipStream_t st) {
    const unsigned blocks = (unsigned)(p.m * p.n * p.splits);
    if (p.bm == WIDE) {
        if (a.live) k_wgrad_wide<true><<<blocks, 512, 0, st>>>(a, p, partial);
        else k_wgrad_wide<false><<<blocks, 512, 0, st>>>(a, p, partial);
    } else {
        a.live ? run_tile<TY, true>(a, p, partial, st) : run_tile<TY, false>(a, p, partial, st);
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
    // a grid of two dimensions: one holds less than 2^32 threads
    const bool fours = a.cols % 4 == 0;
    const long long n = ((long long)a.out * a.cols / (fours ? 4 : 1) + 31) / 32, x = std::min(n, 1ll << 20);
    const dim3 grid((unsigned)x, (unsigned)((n + x - 1) / x));
    if (fours) k_wgrad_join<4><<<grid, 256, 0, st>>>(a, p.splits, partial);
    else k_wgrad_join<1><<<grid, 256, 0, st>>>(a, p.splits, partial);
    return hipGetLastError();
}

}  // namespace iodf
