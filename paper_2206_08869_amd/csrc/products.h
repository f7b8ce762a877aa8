// Matrix products of 16-bit numbers with 32-bit sums, for the ends of a training step (loss.hip, orth.hip):
//   acc[m][n] = sum_k A(m, k) B(n, k)
// A workgroup computes BM x BN outputs. Operands go straight from memory to LDS in tiles of 64 along k, a tile ahead of the products, and
// each may lie in memory either way round:
//   rows   [m][k], k consecutive: a lane's fragment (eight k of one m) is one LDS read of sixteen bytes
//   sums   [k][m], m consecutive: the transposing LDS read takes the fragment out of eight rows
// so that no operand is ever transposed in memory. A number of more bits than 16 is two parts, high and low (planes of the same
// layout), and the sum of three products: high low, low high, high high (the small ones first, while the sums
// that they are rounded to are small too); or of two where only B has low parts. A 32-bit number of any size is three parts in bfloat16, exactly, and six products: those
// left out are 2^-25 of the whole and less.
//
// Tiles of 256 x 256 with eight waves are bound by power: logits of 8192 rows, 65536 classes and 4096 columns run at 1390 to 1440 TFLOP/s with random numbers
// and at 1754 with zeros. The 16 x 16 x 32 instruction moves fewer sums for an operation than the 32 x 32 x 16 one, which made 1430 of 1305. Reads that meet
// no bank twice, and reads and loads dealt out between the products by hand, were 3 percent each.
#pragma once
#include <type_traits>

#include "block_dev.h"
#include "plan.h"

namespace iodf {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 h16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// An operand, its base and leading dimension in elements. Rows (or, of a `sums` operand, columns) past `extent` repeat existing ones: they only reach
// outputs that nobody stores. Along k a `rows` operand is readable up to a multiple of 64; a `sums` operand repeats its last row past `depth`. What
// stands there must be zero in one of the operands and finite in the other. Rows start at multiples of 16 bytes.
struct Side {
    const uint16_t* p;
    long long plane;  // from the high parts to the low ones
    long long ld;
    int extent, depth;
};

template <typename T> struct Mma;
template <> struct Mma<__bf16> {
    static __device__ __forceinline__ f32x4 go(s16x8 a, s16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b16x8, a), __builtin_bit_cast(b16x8, b), c, 0, 0, 0);
    }
};
template <> struct Mma<_Float16> {
    static __device__ __forceinline__ f32x4 go(s16x8 a, s16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h16x8, a), __builtin_bit_cast(h16x8, b), c, 0, 0, 0);
    }
};

// Sixteen bytes a lane from memory to LDS, lane after lane from `lds` on. Written out because the compiler, where it knows of such a load,
// waits for all of them before any LDS access that may meet one.
__device__ __forceinline__ void to_lds16(uint32_t lds, const void* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory", "m0");
}

// A barrier that waits for LDS only: stores on their way to memory are left there.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// An address that is the same in all lanes, in scalar registers also where the compiler does not see that it is.
template <typename T>
__device__ __forceinline__ T* uniform(T* p) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    return (T*)(uintptr_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(a >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)a));
}

// One operand's way through LDS: W rows (or columns) of a tile, THREADS threads.
template <int W, int THREADS, bool SUMS>
struct Lane {
    static constexpr int LOADS = W * 8 / THREADS;      // of sixteen bytes, a thread and tile
    static constexpr int PER = W / 8;                  // chunks of a row of a `sums` tile
    uint32_t off[LOADS], ld;                           // bytes from the tile's corner (of a `sums` tile from the row's start), from row to row
    // `first`: where the workgroup's rows (columns) begin
    __device__ __forceinline__ void init(const Side& s, int first) {
        const int tid = threadIdx.x;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int p = i * THREADS + tid;
            if (!SUMS) {
                const int r = p / 8, c = (p & 7) ^ (r >> 1 & 7), at = min(r, s.extent - 1 - first);
                off[i] = (uint32_t)(at * s.ld + c * 8) * 2;
            } else {
                const int c = chunk(p / PER, p % PER);
                ld = (uint32_t)s.ld * 2;
                off[i] = (uint32_t)(first + c * 8 < s.extent ? c * 8 : 0) * 2;
            }
        }
    }
    // Where chunk c of row r lies, and which chunk lies at place c. Thirty-two lanes read 32 bytes each of rows r .. r + 3 and r + 8 .. r + 11 together: 64
    // bytes further a row and 32 every eight rows, they cover all banks.
    static __device__ __forceinline__ int chunk(int r, int c) { return c ^ (PER % 16 == 0 ? (r & 3) << 2 : (r & 2) << 1) ^ (r >> 2 & 2); }
    // tile kt (of the plane `part`): its loads i0 .. i1 - 1, to `lds`, this wave's place in the tile
    static __device__ __forceinline__ const uint16_t* corner(const Side& s, int first, int part, int kt) {
        return s.p + part * s.plane + (SUMS ? (long long)kt * PK * s.ld + first : (long long)first * s.ld + kt * PK);
    }
    // `last`: the tile's last row that exists along k; rows past it repeat it
    __device__ __forceinline__ void start(const uint16_t* corner, unsigned last, uint32_t lds, int i) const {
        to_lds16(lds + i * THREADS * 16, corner, SUMS ? __umul24(min((i * THREADS + threadIdx.x) / PER, last), ld) + off[i] : off[i]);
    }
};

// A wave's fragments of `COUNT` blocks of 16 from row (column) `w0` of the tile on: lane l holds eight numbers along k, from 8 * (l / 16) on, of row l % 16.
template <int W, int COUNT, bool SUMS>
struct Frags {
    uint32_t at[SUMS ? COUNT : 2];  // elements
    __device__ __forceinline__ void init(int w0) {
        const int lane = threadIdx.x & 63;
        if (!SUMS) {
            const int r = w0 + (lane & 15);
#pragma unroll
            for (int s = 0; s < 2; ++s) at[s] = r * PK + (((s * 4 + (lane >> 4)) ^ (r >> 1 & 7)) * 8);
        } else {
            const int r = (lane >> 4) * 8 + ((lane >> 2) & 3), c = (lane & 3) * 4;
#pragma unroll
            for (int b = 0; b < COUNT; ++b) at[b] = r * W + Lane<W, 64, true>::chunk(r, (w0 + b * 16 + c) / 8) * 8 + (c & 7);
        }
    }
    // of step `step` (32 along k) of the tile, block b
    __device__ __forceinline__ s16x8 read(const uint16_t* tile, int step, int b) const {
        if (!SUMS) return *(const s16x8*)(tile + at[step] + b * 16 * PK);
        union { s16x4 h[2]; s16x8 v; } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + at[b] + step * 32 * W));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + at[b] + (step * 32 + 4) * W));
        return u.v;
    }
};

// MW x NW waves of MT x NT blocks of 16 x 16 outputs. Low parts are held times 2^SHIFT.
template <typename T, int MW, int NW, int MT_, int NT_, bool ASUMS, bool BSUMS, int PAIRS, int SHIFT = 0>
struct Products {
    static constexpr int MT = MT_, NT = NT_, BM = MW * MT * 16, BN = NW * NT * 16, THREADS = MW * NW * 64;
    // Small tiles have all parts of both operands in LDS at a time, which takes two loads for three products; large ones, which would not fit, go over
    // the sum once for each product.
    static constexpr bool BOTH = PAIRS > 1 && BM <= (PAIRS > 3 ? 64 : 128) && BN <= (PAIRS > 3 ? 64 : 128);
    static constexpr int NA = !BOTH || PAIRS == 2 ? 1 : PAIRS > 3 ? 3 : 2, NB = !BOTH ? 1 : PAIRS > 3 ? 3 : 2;  // parts in LDS
    // of A and of B in a product: (0 2) (1 1) (2 0) (0 1) (1 0) (0 0), the last three or two of them
    static __device__ __forceinline__ constexpr int part_a(int pair) { return PAIRS == 2 ? 0 : 0x010210 >> 4 * (pair + 6 - (PAIRS > 3 ? 6 : 3)) & 3; }
    static __device__ __forceinline__ constexpr int part_b(int pair) { return PAIRS == 2 ? 1 - pair : 0x001012 >> 4 * (pair + 6 - (PAIRS > 3 ? 6 : 3)) & 3; }
    static constexpr int STAGE = (NA * BM + NB * BN) * PK;                   // elements of a tile of both operands
    static constexpr int LDS = 2 * STAGE;                                    // elements of LDS that run() wants
    f32x4 acc[MT][NT];

    static __device__ __forceinline__ int wave_m() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / NW * MT * 16; }
    static __device__ __forceinline__ int wave_n() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % NW * NT * 16; }
    // which outputs of the wave's a lane holds in acc[m][n][0..3]: rows m * 16 + row_of() and the three behind it, column n * 16 + col_of()
    static __device__ __forceinline__ int row_of() { return (threadIdx.x & 63) / 16 * 4; }
    static __device__ __forceinline__ int col_of() { return threadIdx.x & 15; }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) acc[m][n] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // What has been computed from acc is not kept for what comes: it is computed again, since it would not fit the registers.
    __device__ __forceinline__ void anew() {
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int n = 0; n < NT; ++n) asm volatile("" : "+v"(acc[m][n]));
    }

    // Tiles kt0 .. kt1 - 1 (kt1 > kt0) along k, of outputs from (m0, n0) on. Ends with a barrier: LDS is free then.
    __device__ __forceinline__ void run(const Side& a, const Side& b, int m0, int n0, int kt0, int kt1, uint16_t* lds) {
        Lane<BM, THREADS, ASUMS> la;
        Lane<BN, THREADS, BSUMS> lb;
        Frags<BM, MT, ASUMS> fa;
        Frags<BN, NT, BSUMS> fb;
        la.init(a, m0), lb.init(b, n0);
        fa.init(wave_m()), fb.init(wave_n());
        clear();
        const uint32_t lds0 = (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)lds +
                              __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * 1024;
        const int tiles = (kt1 - kt0) * (BOTH ? 1 : PAIRS);
        int pair = 0, kt = kt0;  // of the next tile to load
        const uint16_t *ca[NA], *cb[NB];
        unsigned left_a, left_b;
        auto next = [&] {
#pragma unroll
            for (int p = 0; p < NA; ++p) ca[p] = uniform(Lane<BM, THREADS, ASUMS>::corner(a, m0, BOTH ? p : PAIRS > 1 ? part_a(pair) : 0, kt));
#pragma unroll
            for (int p = 0; p < NB; ++p) cb[p] = uniform(Lane<BN, THREADS, BSUMS>::corner(b, n0, BOTH ? p : PAIRS > 1 ? part_b(pair) : 0, kt));
            left_a = a.depth - 1 - kt * PK, left_b = b.depth - 1 - kt * PK;
            if (++kt == kt1) kt = kt0, ++pair;
        };
        // loads i0 .. i1 - 1 of the tile's, of both operands; buf: where in LDS (elements) it goes
        auto start = [&](int buf, int i0, int i1) {
#pragma unroll
            for (int i = i0; i < i1; ++i) {
                const int j = i - NA * la.LOADS;
                if (j < 0) la.start(ca[i / la.LOADS], left_a, lds0 + (buf + i / la.LOADS * BM * PK) * 2, i % la.LOADS);
                else lb.start(cb[j / lb.LOADS], left_b, lds0 + (buf + (NA * BM + j / lb.LOADS * BN) * PK) * 2, j % lb.LOADS);
            }
        };
        constexpr int LOADS = NA * Lane<BM, THREADS, ASUMS>::LOADS + NB * Lane<BN, THREADS, BSUMS>::LOADS;
        auto meet = [] {
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        // A tile is two steps of MT groups of NT products. Fragments of the next step are read while this one's are multiplied: those of B and of A's last
        // SPARE blocks into registers of their own, A's other blocks into the same ones, once their products are on their way. So the last read of a
        // step has the products of the last two groups to arrive, and all of a tile is read when its second step begins. Reads (and, once a tile, the
        // loads of the tile after the next) are dealt out by hand: left to itself the compiler gathers reads just before their products.
        constexpr int SPARE = 2, ROLL = MT - SPARE, BUSY = MT > 1 ? MT / 2 : 1, EACH = (NT + SPARE + BUSY - 1) / BUSY;
        static_assert(MT >= SPARE, "two blocks of rows at least");
        s16x8 xa[NA][ROLL > 0 ? ROLL : 1], xs[2][NA][SPARE], xb[2][NB][NT];
        f32x4 low[BOTH ? MT : 1][BOTH ? NT : 1] = {};  // the small products' sums
        auto group = [&](int set, int m) {
            auto of_a = [&](int p) { return m < ROLL ? xa[p][m < ROLL ? m : 0] : xs[set][p][m < ROLL ? 0 : m - ROLL]; };
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                if (BOTH) {
#pragma unroll
                    for (int pair = 0; pair < PAIRS - 1; ++pair)
                        low[BOTH ? m : 0][BOTH ? n : 0] = Mma<T>::go(of_a(BOTH ? part_a(pair) : 0), xb[set][BOTH ? part_b(pair) : 0][n], low[BOTH ? m : 0][BOTH ? n : 0]);
                }
                acc[m][n] = Mma<T>::go(of_a(0), xb[set][0][n], acc[m][n]);
            }
        };
        auto read_a = [&](int buf, int step, int p, int m) { return fa.read(lds + buf + p * BM * PK, step, m); };
        auto reads = [&](int set, int buf, int step, int g) {  // of step `step`, before group g of the step before it
#pragma unroll
            for (int i = g * EACH; i < (g + 1) * EACH && i < NT + SPARE; ++i) {
                if (i < NT) {
#pragma unroll
                    for (int p = 0; p < NB; ++p) xb[set][p][i] = fb.read(lds + buf + (NA * BM + p * BN) * PK, step, i);
                } else {
#pragma unroll
                    for (int p = 0; p < NA; ++p) xs[set][p][i - NT] = read_a(buf, step, p, ROLL + i - NT);
                }
            }
            if (g >= 1 && g - 1 < ROLL) {
#pragma unroll
                for (int p = 0; p < NA; ++p) xa[p][g - 1] = read_a(buf, step, p, g - 1);
            }
        };
        auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
        next();
        start(0, 0, LOADS);
        meet();
        if (tiles > 1) {
            next();
            start(STAGE, 0, LOADS);
        }
#pragma unroll
        for (int g = 0; g <= MT; ++g) reads(0, 0, 0, g);
        int buf = 0;
        constexpr float DOWN = 1.f / (1 << SHIFT);
        for (int t = 0; t < tiles; ++t) {
            if (SHIFT && !BOTH && t == (PAIRS - 1) * (kt1 - kt0)) {  // the small products are done
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int n = 0; n < NT; ++n) acc[m][n] *= DOWN;
            }
#pragma unroll
            for (int g = 0; g < MT; ++g) {
                reads(1, buf, 1, g);
                group(0, g);
                fence();
            }
            const bool load = t + 2 < tiles;
            if (load) next();
            meet();  // this tile has been read by all, the next one has landed
            fence();
#pragma unroll
            for (int g = 0; g < MT; ++g) {
                reads(0, buf ^ STAGE, 0, g);  // behind the last tile of what is left there
                if (load) start(buf, g * LOADS / MT, (g + 1) * LOADS / MT);
                group(1, g);
                fence();
            }
            buf ^= STAGE;
        }
        if (BOTH) {
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[m][n] += SHIFT ? low[BOTH ? m : 0][BOTH ? n : 0] * DOWN : low[BOTH ? m : 0][BOTH ? n : 0];
        }
        lds_barrier();
    }
};

// A workgroup's outputs on their way to memory: what lanes hold as four neighbours of a row here and there goes through LDS and comes out as whole rows, sixteen
// bytes to a lane. Output rows are the products' columns n, output columns their rows m. N of the NT block columns of all waves at a time, pass by pass.
// Chunks of sixteen bytes are moved about by their row, so that the rows that a wave writes together cover all banks.
template <class P, typename E, int NW, int N>
struct Staged {
    // Of its own for every use: what one has computed for its places is not kept in registers for the next.
    unsigned tid;
    __device__ __forceinline__ Staged() : tid(threadIdx.x) { asm volatile("" : "+v"(tid)); }
    static constexpr int ROWS = NW * N * 16, CHUNKS = P::BM * (int)sizeof(E) / 16, PER = ROWS * CHUNKS / P::THREADS, OF = 16 / (int)sizeof(E);
    static constexpr int BYTES = ROWS * CHUNKS * 16, PASSES = P::NT / N;
    static constexpr int MOVE = (CHUNKS & -CHUNKS) < 32 ? (CHUNKS & -CHUNKS) - 1 : 31;
    static __device__ __forceinline__ int place(int row, int chunk) { return (row * CHUNKS + (chunk ^ (row & MOVE))) * 16; }
    // block (m, n), in pass n / N
    __device__ __forceinline__ void put(void* lds, int m, int n, const E (&v)[4]) const {
        const int row = P::wave_n() / P::NT * N + n % N * 16 + (tid & 15), c = P::wave_m() + m * 16 + (tid & 63) / 16 * 4;
        __builtin_memcpy((char*)lds + place(row, c / OF) + c % OF * sizeof(E), v, 4 * sizeof(E));
    }
    // chunk i of the thread's in a pass: its row and first column among the workgroup's outputs, and what it holds
    __device__ __forceinline__ void where(int i, int pass, int& row, int& col) const {
        const int k = i * P::THREADS + tid, r = k / CHUNKS;
        row = r / (N * 16) * (P::NT * 16) + pass * (N * 16) + r % (N * 16);
        col = k % CHUNKS * OF;
    }
    __device__ __forceinline__ u32x4 take(const void* lds, int i) const {
        const int k = i * P::THREADS + tid, r = k / CHUNKS;
        return *(const u32x4*)((const char*)lds + place(r, k % CHUNKS));
    }
    // The mirror image of 16-bit outputs, in one pass (N = NT), by the transposing read: eight neighbours of a row, which is one of the products' rows m.
    static constexpr int ACROSS = ROWS * P::BM / 8 / P::THREADS;
    __device__ __forceinline__ void where_across(int i, int& row, int& col) const {
        const int lane = tid & 63, block = i * (P::THREADS / 64) + (tid >> 6);
        row = block % (P::BM / 16) * 16 + (lane & 15);
        col = block / (P::BM / 16) * 32 + (lane >> 4) * 8;
    }
    __device__ __forceinline__ s16x8 take_across(const void* lds, int i) const {
        const int lane = tid & 63, block = i * (P::THREADS / 64) + (tid >> 6);
        const int m = block % (P::BM / 16) * 16 + (lane & 3) * 4, n = block / (P::BM / 16) * 32 + (lane >> 4) * 8 + (lane >> 2 & 3);
        union { s16x4 h[2]; s16x8 v; } u;
        u.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((const char*)lds + place(n, m / 8) + m % 8 * 2));
        u.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)((const char*)lds + place(n + 4, m / 8) + m % 8 * 2));
        return u.v;
    }
};

// Four neighbours of a row, of which n exist, at any element's address.
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));
template <typename T>
__device__ __forceinline__ void put_quad(T* to, int n, const float (&v)[4]) {
    T t[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = (T)v[j];
    if (n < 4) {
#pragma unroll
        for (int j = 0; j < 3; ++j)
            if (j < n) to[j] = t[j];
    } else if (sizeof(T) == 4) {
        u32x4 w;
        __builtin_memcpy(&w, t, 4 * sizeof(T));
        *(u32x4_any*)to = w;
    } else {
        u32x2 w;
        __builtin_memcpy(&w, t, 4 * sizeof(T));
        *(u32x2_any*)to = w;
    }
}
template <typename T>
__device__ __forceinline__ void get_quad(const T* from, int n, float (&v)[4]) {
    T t[4];
    if (n < 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) t[j] = j < n ? from[j] : (T)0.f;
    } else if (sizeof(T) == 4) {
        const u32x4 w = *(const u32x4_any*)from;
        __builtin_memcpy(t, &w, 4 * sizeof(T));
    } else {
        const u32x2 w = *(const u32x2_any*)from;
        __builtin_memcpy(t, &w, 4 * sizeof(T));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (float)t[j];
}

// Workgroups go round the eight dies (each with an L2 of its own) in turn: numbers with which a die gets neighbours.
__device__ __forceinline__ unsigned by_die(unsigned b, unsigned all) {
    const unsigned share = all / 8;
    return b < share * 8 ? b % 8 * share + b / 8 : b;
}
// Which tile of a grid of tm x tn a workgroup takes, in bands four tiles high, so that a panel of either operand is fetched into as few L2s as may be.
__device__ __forceinline__ void place_tile(unsigned b, unsigned all, unsigned tm, unsigned tn, int& m, int& n) {
    const unsigned l = by_die(b, all);
    const unsigned band = l / (4 * tn), in = l - band * 4 * tn, high = min(4u, tm - band * 4);
    m = (int)(band * 4 + in % high);
    n = (int)(in / high);
}

// Tile l of those on and below the diagonal of a square of n x n, in bands eight tiles high.
__device__ __forceinline__ void place_triangle(unsigned l, unsigned n, int& i, int& j) {
    unsigned r0 = 0;
    while (r0 + 8 < n && (r0 + 8) * (r0 + 9) / 2 <= l) r0 += 8;
    const unsigned high = min(8u, n - r0), in = l - r0 * (r0 + 1) / 2;
    if (in < high * r0) {
        i = (int)(r0 + in % high), j = (int)(in / high);
    } else {
        unsigned k = in - high * r0, r = 0;
        while (k > r) k -= ++r;
        i = (int)(r0 + r), j = (int)(r0 + k);
    }
}

}  // namespace iodf
