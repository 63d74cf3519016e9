// The layer for many rows on the binary16 matrix cores, the planes summed first.
//
//   y[r][n] = act(sum_k W[n][k] x[r][k] + bias[n]) * multiplier[r][n] + residual[r][n]
//
// W[n][k] = sum_i +-2^e_i is one binary16 number wherever the exponents of a
// (row, group) lie in [-14, 0] and q 2^(largest - smallest) <= 2^11: every partial
// sum is a multiple of the smallest factor, at most 2^11 of it, so the sum over the
// planes is exact and one matrix product serves all planes.  (Below -14 the sum may
// be subnormal, and the matrix core then drops low bits of its products: measured
// 7e-6 of sum|terms| at 2^-24.  Of subnormal activations beside these normal sums it drops
// none: rows of multiples of 2^-24 up to 3 * 2^-24 come out exact.)  A block of 128 columns
// that has any other exponents in a wave's rows is left for a second loop, two products a
// plane: +-2^e is a bfloat16 number, an activation the sum of two.
//
// Against a product a plane this takes a third of the matrix core's work for 3 planes and,
// with tiles of 256 rows x 256 outputs, an expanded key serves 256 rows: layer of
// 11008x4096, 3 planes, 4096 rows 373 us, with SiLU 377, with SiLU and multiplier 400 (923
// TFLOP/s; a library product of binary16 tensors of that size, without either, 425), 11003x4096
// 250 rows 45 us, with bias and GELU 47 (the tile kernel of gemm_mfma.hip 81 to 91 without).
// (A pass among others, weights rotated over 320 MB and more.)
//
// What bounds it.  4096 rows: power.  The same 258 thousand cycles of a 256-row tile take
// 114 us on 64 compute units (2.26 GHz) and 140 us on all (1.84 GHz); the matrix cores are
// busy 45% of the cycles, vector instructions 42%, 6.3 a product, of which 4.1 expand planes.
// Up to 32 rows: vector instructions (4096x11008, 2 planes, 16 experts of 8 to 96 rows: 75%
// of the SIMD cycles, matrix cores 19%).  Between: too few tiles for the compute units, 8
// waves each, whose expansion, LDS reads and products follow each other at the barriers.
#ifndef SHIFTADD_PANEL_H
#define SHIFTADD_PANEL_H

#include <hip/hip_runtime.h>

#include <type_traits>

#include "linear.h"

namespace sa_panel {
namespace {

using sa_linear::Layer;

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bhalf8_t __attribute__((ext_vector_type(8)));
typedef float float16_t __attribute__((ext_vector_type(16)));

constexpr int kWaves = 8;
constexpr int kThreads = 64 * kWaves;
constexpr int kTile = 32;  // outputs and rows of one matrix tile
constexpr int kFarWords = 128;

struct Args {
    Layer a;
    int n_tiles;           // tiles of outputs; they run fastest over the grid
    uint32_t group_magic;  // blocks to exponent groups: J * magic >> 32, 0: J
    int byte_offsets;      // x is below 2^32 bytes
};

__device__ inline half2_t halves(uint32_t v) { return __builtin_bit_cast(half2_t, v); }
__device__ inline half2_t both(float v) { return half2_t{(_Float16)v, (_Float16)v}; }

__device__ inline half8_t cat(const half2_t a[4]) {
    return half8_t{a[0][0], a[0][1], a[1][0], a[1][1], a[2][0], a[2][1], a[3][0], a[3][1]};
}

// A key byte is eight columns.  Half h of a key word (bytes 2 h, 2 h + 1) is spread so
// that an even position p of either 16-bit half holds bits p and p + 1 of the two bytes;
// a bit at position 10, 12 or 14 of a half is the binary16 value 2^-14, 2^-11 or 2, and
// two shifted copies bring the other positions there.
struct Spread {
    uint32_t v, v6, v12;
};
__device__ inline Spread spread(uint32_t w, int h) {
    const uint32_t v = __builtin_amdgcn_perm(w >> 1, w, h ? 0x07060302u : 0x05040100u);
    return {v, v << 6, v << 12};
}

// A factor f = 2^e, -14 <= e <= 0, as what turns the bit values into 0 or 2 f: times
// f 2^15, f 2^12 and f (normal numbers, built from e).
struct Factor {
    half2_t m10, m12, m14;
};
__device__ inline Factor factor(int e) {
    const uint32_t h = (uint32_t)(e << 10) + (30u << 10);
    const uint32_t m = h | h << 16;
    return {halves(m), halves(m - 0x0C000C00u), halves(m - 0x3C003C00u)};
}

// Pair j of byte 2 h + odd: c += (bit ? 2 f : 0).
__device__ inline half2_t add_pair(const Spread& s, const Factor& f, int odd, int j, half2_t c) {
    const uint32_t src = odd ? (j == 0 ? s.v6 : s.v) : (j < 2 ? s.v12 : s.v6);
    const int pos = odd ? (j == 0 ? 14 : 8 + 2 * j) : (j < 2 ? 12 + 2 * j : 6 + 2 * j);
    const half2_t m = pos == 10 ? f.m10 : pos == 12 ? f.m12 : f.m14;
    return __builtin_elementwise_fma(halves(src & (0x00010001u << pos)), m, c);
}

// 16 bytes a lane from memory to `lds` + 16 lane (uniform), without passing registers.
// Written as the instruction: the compiler would make every later LDS read wait for it
// (it does not tell the buffers apart).  There is no result in registers; whoever reads
// the data waits for vmcnt and a barrier first.  m0 takes effect one instruction later.
__device__ inline void copy_to_lds(uint64_t base, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds), "v"(offset), "s"(base) : "m0", "memory");
}
__device__ inline void copy_to_lds(uint64_t from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :: "s"(lds), "v"(from) : "m0", "memory");
}

// 16 bytes at any address.
__device__ inline uint4 load16(const uint8_t* p) {
    typedef uint32_t word4_t __attribute__((ext_vector_type(4), aligned(1)));
    const word4_t v = *reinterpret_cast<const word4_t*>(p);
    return uint4{v[0], v[1], v[2], v[3]};
}

__device__ inline void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Keys and exponents as loaded.  Lane (i, g) has a layer row and, of a group of two
// blocks, the 16 keys and the exponent of block g.  kPart: of one block, the 16 keys and 16
// exponents from the block's first on.  kAny: of one block, the keys of its chunks g, 2 + g,
// ..., 14 + g in w.x, w.y and their exponents in w.z, w.w.
//
// The groups a kernel takes: of whole blocks; of 8, 16, 32 or 64 columns; any.  The last two
// also take columns that end inside a block.
enum Groups { kWhole = 0, kPart = 1, kAny = 2 };
template <int Q, int GEN>
struct Keys {
    uint4 w[Q];
    uint4 x[GEN == kPart ? Q : 1];
    uint32_t e[GEN == kWhole ? Q : 1];
};

// Why these tiles: keys are expanded once per tile of rows, so a wave's 128 accumulators go
// into rows (256) before outputs (32); two waves a SIMD is what these registers leave.
//
// Work split.  Eight waves are RW sets of 32 outputs times KW shares of the columns; a
// wave has all 32 CT rows of the workgroup.  Activations of a 128-column block lie in
// LDS, double buffered and copied there without passing registers; the planes are
// expanded straight into matrix operands.  KW shares' sums meet in LDS and are added in
// order.
//
// Matrix row i of a wave is output 16 ((i >> 2) & 1) + 4 (i >> 3) + (i & 3) of its 32, so
// that a lane's 16 results are 16 consecutive outputs of one row.  Step s of a block
// multiplies its chunks 2 s (lanes 0-31) and 2 s + 1 (lanes 32-63).  A row's 16 chunks of
// a block are 256 bytes of LDS, chunk c at 16 (c ^ (row & 15)): both the copies (whole
// rows) and the reads (16 lanes at a time, one step) touch every bank once.
template <int Q, int CT, int KW, int GEN>
__device__ __forceinline__ void body(const Args& pa, uint4* xbuf, uint32_t* far_steps, int expert,
                                     int first, int end) {
    const Layer& a = pa.a;
    constexpr int RW = kWaves / KW;
    constexpr int kItems = CT * 8 / RW;  // 1 KiB copies (4 rows) of a wave a block
    constexpr int kBuf = CT * 512;       // uint4 of one block
    constexpr int kE = Q > 4 ? 2 : 1;    // words of a block's exponents
    // One row tile: with 4 column shares two workgroups a CU (64 KB of LDS, 128 registers) hide
    // more than the interleaving.  With 8 the LDS holds one workgroup; interleaving was not
    // measured there.
    constexpr bool kPipelined = Q <= 4 && CT > 1;
    const int nt = (int)(blockIdx.x % (unsigned)pa.n_tiles);
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int r = lane & 31, g = lane >> 5;
    const int rw = wave % RW, kw = wave / RW;
    const int N = a.N, C = a.K >> 3, NB = (C + 15) >> 4, NG = a.K / a.G;
    const int gper = ((NB + 1) / 2 + KW - 1) / KW;  // groups of two blocks of a column share
    const int blk0 = imin(2 * gper * kw, NB), blk1 = imin(blk0 + 2 * gper, NB);
    const int steps = imin(2 * gper, NB);
    const uint8_t* packed = a.packed + (int64_t)expert * a.q * N * C;
    const uint8_t* exps =
        reinterpret_cast<const uint8_t*>(a.exps) + (int64_t)expert * a.q * N * NG;
    const int n0 = kTile * (RW * nt + rw);  // first output of this wave
    const int n = imin(n0 + 16 * ((r >> 2) & 1) + 4 * (r >> 3) + (r & 3), N - 1);

    // rows of x that this lane copies, as 16-byte words from a.x (x is below 2^36 bytes), or
    // as bytes where these fit
    uint32_t xo[kItems];
#pragma unroll
    for (int j = 0; j < kItems; ++j) {
        const int row = 4 * (rw * kItems + j) + (lane >> 4);
        const int v = sa_linear::source_row(a, imin(first + row, end - 1));
        xo[j] = (uint32_t)imax(v, 0) * (uint32_t)C;
        if constexpr (!GEN) xo[j] += (uint32_t)((lane & 15) ^ (row & 15));
        if (pa.byte_offsets) xo[j] *= 16u;
    }
    uint4* xk = xbuf + kw * 2 * kBuf;
    const uint32_t x_lds = (uint32_t)__builtin_amdgcn_readfirstlane(
        (int)(uintptr_t)(__attribute__((address_space(3))) uint4*)(xk + rw * kItems * 64));
    auto copy_x = [&](int J, int buf) {
        const uint64_t base = (uint64_t)(uintptr_t)a.x + (GEN ? 0u : 256u * (uint64_t)J);
#pragma unroll
        for (int j = 0; j < kItems; ++j) {
            uint32_t o = xo[j];
            asm volatile("" : "+v"(o));  // (no 64-bit pointers kept over the blocks)
            if constexpr (GEN) {
                const int row = 4 * (rw * kItems + j) + (lane >> 4);
                const int c = imin(16 * J + ((lane & 15) ^ (row & 15)), C - 1);
                o += (uint32_t)c * (pa.byte_offsets ? 16u : 1u);
            }
            const uint32_t to = x_lds + 16 * (buf * kBuf + j * 64);
            if (pa.byte_offsets) copy_to_lds(base, o, to);
            else copy_to_lds(base + 16 * (uint64_t)o, to);
        }
    };
    // this lane's activations of step s, row tile c: word 512 c + ((2 s) ^ x_word)
    const uint4* xr = xk + r * 16;
    const int x_word = g ^ (r & 15);
    // the copies of this wave are done, and every wave's
    auto arrive = [] {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };

    // Planes past the last repeat it, unused.
    auto load_keys = [&](int J0, Keys<Q, GEN>& k) {
        const uint32_t eoff = (uint32_t)n * (uint32_t)NG;
        if constexpr (GEN == kPart) {
            const int T = n >> 6, R = imin(64, N - 64 * T), gb = 128 / a.G;  // groups of a block
            const bool whole = 16 * J0 + 16 <= C;                            // uniform
            const uint32_t koff = (uint32_t)(64 * T * C + 16 * J0 * R + (n & 63) * 16);
            const int64_t all = (int64_t)a.experts * a.q * N * NG;
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const int pi = imin(i, a.q - 1);
                const uint8_t* kp = packed + (size_t)pi * (size_t)N * (size_t)C;
                if (whole) {
                    k.w[i] = load16(kp + koff);
                } else {
                    uint32_t b[2] = {0, 0};
#pragma unroll
                    for (int s = 0; s < 8; ++s) {
                        const int c = imin(16 * J0 + 2 * s + g, C - 1);
                        b[s >> 2] |= (uint32_t)kp[layout_offset(0, n, c, N, C)] << (8 * (s & 3));
                    }
                    k.w[i] = uint4{b[0], b[1], 0, 0};
                }
                // 16 bytes of the whole exponents, one at a time where these end
                const int64_t at = ((int64_t)(expert * a.q + pi) * N + n) * NG + (int64_t)J0 * gb;
                const uint8_t* ep = reinterpret_cast<const uint8_t*>(a.exps) + at;
                if (at + 16 <= all) {
                    k.x[i] = load16(ep);
                } else {
                    uint32_t x[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int b = 0; b < 16; ++b)
                        if (at + b < all) x[b >> 2] |= (uint32_t)ep[b] << (8 * (b & 3));
                    k.x[i] = uint4{x[0], x[1], x[2], x[3]};
                }
            }
        } else if constexpr (GEN == kAny) {
            const int gc = a.G >> 3;
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                const int pi = imin(i, a.q - 1);
                const uint8_t* ep = exps + (size_t)pi * (size_t)N * (size_t)NG;
                uint32_t b[2] = {0, 0}, e[2] = {0, 0};
#pragma unroll
                for (int s = 0; s < 8; ++s) {
                    const int c = imin(16 * J0 + 2 * s + g, C - 1);
                    b[s >> 2] |= (uint32_t)packed[layout_offset(pi, n, c, N, C)] << (8 * (s & 3));
                    e[s >> 2] |= (uint32_t)ep[eoff + (uint32_t)(c / gc)] << (8 * (s & 3));
                }
                k.w[i] = uint4{b[0], b[1], e[0], e[1]};
            }
        } else {
            const int J = imin(J0 + g, NB - 1);
            const uint32_t group =
                pa.group_magic ? __umulhi((uint32_t)J, pa.group_magic) : (uint32_t)J;
            const int T = n >> 6, R = imin(64, N - 64 * T);
            uint32_t koff = (uint32_t)(64 * T * C + 16 * (n & 63) + 16 * J * R);
            asm volatile("" : "+v"(koff));
#pragma unroll
            for (int i = 0; i < Q; ++i)
                k.e[i] = (exps + (size_t)imin(i, a.q - 1) * (size_t)N * (size_t)NG)[eoff + group];
#pragma unroll
            for (int i = 0; i < Q; ++i)
                k.w[i] = *reinterpret_cast<const uint4*>(
                    packed + (size_t)imin(i, a.q - 1) * (size_t)N * (size_t)C + koff);
        }
    };

    float16_t acc[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[c][v] = 0.0f;

    // GEN: columns past the last hold no weight
    auto inside = [&](int J, int s) { return !GEN || 16 * J + 2 * s + g < C; };
    // May these exponents' planes not be summed?
    auto is_far = [&](const int (&e)[Q]) {
        constexpr int kSpread = Q == 1 ? 127 : Q == 2 ? 10 : Q <= 4 ? 9 : 8;
        int hi = e[0], lo = e[0];
#pragma unroll
        for (int i = 1; i < Q; ++i) {
            hi = max(hi, e[i]);
            lo = imin(lo, e[i]);
        }
        return hi > 0 || lo < -14 || hi - lo > kSpread;
    };
    // Matrix operands of steps 2 q and 2 q + 1 of a block (q < 4): w(i, h) is plane i's key
    // word of steps 4 h .. 4 h + 3, e(i, s) its exponent in step s.
    auto expand = [&](int J, int q, auto w, auto e, half8_t (&W)[2]) {
        half2_t p[2][4];
        Factor f[2][Q];
#pragma unroll
        for (int o = 0; o < 2; ++o) {
            half2_t sum;
#pragma unroll
            for (int i = 0; i < Q; ++i) {
                f[o][i] = factor(e(i, 2 * q + o));
                if (Q > 4 || GEN) {
                    const half2_t z = both(i < a.q && inside(J, 2 * q + o) ? 1.0f : 0.0f);
                    f[o][i] = {f[o][i].m10 * z, f[o][i].m12 * z, f[o][i].m14 * z};
                }
                sum = i == 0 ? -f[o][i].m14 : sum - f[o][i].m14;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) p[o][j] = sum;
        }
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const Spread sp = spread(w(i, q >> 1), q & 1);
#pragma unroll
            for (int o = 0; o < 2; ++o)
#pragma unroll
                for (int j = 0; j < 4; ++j) p[o][j] = add_pair(sp, f[o][i], o, j, p[o][j]);
        }
        W[0] = cat(p[0]);
        W[1] = cat(p[1]);
    };
    // Products of a block, activations read kAhead of them before they are used, X[i % kRing]
    // those of product i = step * CT + row tile.
    constexpr int kAhead = 2, kRing = kAhead + 1, kProducts = 8 * CT;
    auto read_x = [&](const uint4* xs, int xw, int i, half8_t (&X)[kRing]) {
        X[i % kRing] = __builtin_bit_cast(half8_t, xs[512 * (i % CT) + ((2 * (i / CT)) ^ xw)]);
    };
    auto products = [&](const uint4* xs, int xw, int q, const half8_t (&W)[2], half8_t (&X)[kRing]) {
#pragma unroll
        for (int i = 2 * CT * q; i < 2 * CT * (q + 1); ++i) {
            if (i + kAhead < kProducts) read_x(xs, xw, i + kAhead, X);
            acc[i % CT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(W[(i / CT) & 1], X[i % kRing],
                                                                 acc[i % CT], 0, 0, 0);
        }
    };
    auto first_x = [&](const uint4* xs, int* xw, half8_t (&X)[kRing]) {
        *xw = x_word;
        asm volatile("" : "+v"(*xw));  // (addresses are not kept over the blocks)
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read_x(xs, *xw, i, X);
    };
    auto summed = [&](int J, const uint4* xs, auto w, auto e) {
        half8_t X[kRing], W[2];
        int xw;
        first_x(xs, &xw, X);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            expand(J, q, w, e, W);
            __builtin_amdgcn_sched_barrier(0);
            products(xs, xw, q, W, X);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // The same with the next quarter's operands expanded between one quarter's products, a
    // piece after each: a product takes the matrix core 32 cycles, in which the two waves of
    // a SIMD issue the expansion's vector instructions (11008x4096, nothing after the product,
    // 4096 rows 402 -> 373 us, 250 rows 48 -> 45; 4096x4096 64 rows, one row tile, the same; the
    // compiler's own order of the same code puts the LDS reads last and gains nothing).  Pieces
    // 0 .. Q - 1 spread a plane's word, the others are a pair each, by the position of its bits
    // (add_pair).
    struct Next {
        Spread sp[Q];
        half2_t m10[Q], m[Q];  // factors of the block for position 10, and for the position at hand
        half2_t sum;
        half2_t p[2][4];
    };
    auto new_block = [&](Next& x, auto e) {
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const Factor f = factor(e(i, 0));
            x.m10[i] = f.m10;
            x.sum = i == 0 ? -f.m14 : x.sum - f.m14;
        }
    };
    constexpr int kPieces = Q + 8;
    auto piece = [&](Next& x, int k, int q, auto w) {
        constexpr int kOdd[8] = {0, 1, 0, 0, 1, 0, 1, 1}, kPair[8] = {2, 1, 0, 3, 2, 1, 0, 3};
        if (k < Q) {
            x.sp[k] = spread(w(k, q >> 1), q & 1);
            return;
        }
        const int o = kOdd[k - Q], j = kPair[k - Q];
        if (k == Q || k == Q + 2 || k == Q + 5) {
            const uint32_t down = k == Q ? 0u : k == Q + 2 ? 0x0C000C00u : 0x3C003C00u;
#pragma unroll
            for (int i = 0; i < Q; ++i)
                x.m[i] = halves(__builtin_bit_cast(uint32_t, x.m10[i]) - down);
        }
        half2_t c = x.sum;
#pragma unroll
        for (int i = 0; i < Q; ++i) c = add_pair(x.sp[i], {x.m[i], x.m[i], x.m[i]}, o, j, c);
        x.p[o][j] = c;
    };
    auto take = [&](const Next& x, half8_t (&W)[2]) {
        W[0] = cat(x.p[0]);
        W[1] = cat(x.p[1]);
    };
    // (a block without the interleaving)
    auto in_turn = [&](const uint4* xs, auto w, auto e) {
        half8_t X[kRing], W[2];
        Next x;
        int xw;
        first_x(xs, &xw, X);
        new_block(x, e);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#pragma unroll
            for (int u = 0; u < kPieces; ++u) piece(x, u, q, w);
            take(x, W);
            __builtin_amdgcn_sched_barrier(0);
            products(xs, xw, q, W, X);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto quarter = [&](const uint4* xs, int xw, int q, const half8_t (&W)[2], half8_t (&X)[kRing],
                       auto next) {
        constexpr int n = 2 * CT;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < n; ++u) {
            const int i = n * q + u;
            if (i + kAhead < kProducts) read_x(xs, xw, i + kAhead, X);
            acc[i % CT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(W[(i / CT) & 1], X[i % kRing],
                                                                 acc[i % CT], 0, 0, 0);
#pragma unroll
            for (int k = (u * kPieces + n - 1) / n; k < ((u + 1) * kPieces + n - 1) / n; ++k) next(k);
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    // Any exponents: a product a plane in bfloat16, whose range holds +-2^e, with the
    // activations as two exact pieces.  A group's sum may be finite where a factor times one
    // activation is not: factors above 2^kTop have their block's sum apart, at 2^-kTopShift.
    constexpr int kTop = 100, kTopShift = 64;
    struct Planes {
        uint64_t keys[Q], ex[Q];  // a byte per step, the next one lowest
    };
    auto planes_of = [&](auto w, auto e) {
        Planes p;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            p.keys[i] = (uint64_t)w(i, 1) << 32 | w(i, 0);
            p.ex[i] = 0;
#pragma unroll
            for (int s = 0; s < (GEN ? 8 : 1); ++s)
                p.ex[i] |= (uint64_t)(uint8_t)e(i, s) << (8 * s);
        }
        return p;
    };
    // The planes' operands of step s; `apart`: those above kTop alone, else the others alone.
    auto next_step = [&](int J, int s, bool apart, Planes& p, bhalf8_t (&W)[Q]) {
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            const Spread sp = spread((uint32_t)p.keys[i], 0);
            const int own = (int)(int8_t)p.ex[i], ei = apart ? own - kTopShift : own;
            // 2^-127 and 2^-128 are subnormal
            uint32_t mag = ei > -127 ? (uint32_t)(ei + 127) << 7 : ei == -127 ? 0x40u : 0x20u;
            mag |= mag << 16;
            const bool none = i >= a.q || !inside(J, s) || (own > kTop) != apart;
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                v[j] = none ? 0u : ((sp.v << (15 - 2 * j)) & 0x80008000u) ^ (mag | 0x80008000u);
            W[i] = __builtin_bit_cast(bhalf8_t, uint4{v[0], v[1], v[2], v[3]});
            p.keys[i] >>= 8;
            if constexpr (GEN) p.ex[i] >>= 8;
        }
    };
    auto add_planes = [&](const uint4* xs, int s, int c, const bhalf8_t (&W)[Q], float16_t sum) {
        const half8_t X = __builtin_bit_cast(half8_t, xs[512 * c + ((2 * s) ^ x_word)]);
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            // eight significant bits, and the at most three behind them
            const float f0 = (float)X[2 * j], f1 = (float)X[2 * j + 1];
            const uint32_t h0 = __builtin_bit_cast(uint32_t, f0) & 0xffff0000u;
            const uint32_t h1 = __builtin_bit_cast(uint32_t, f1) & 0xffff0000u;
            const float l0 = f0 - __builtin_bit_cast(float, h0);
            const float l1 = f1 - __builtin_bit_cast(float, h1);
            hi[j] = h0 >> 16 | h1;
            lo[j] = __builtin_bit_cast(uint32_t, l0) >> 16 |
                    (__builtin_bit_cast(uint32_t, l1) & 0xffff0000u);
        }
        const bhalf8_t H = __builtin_bit_cast(bhalf8_t, uint4{hi[0], hi[1], hi[2], hi[3]});
        const bhalf8_t L = __builtin_bit_cast(bhalf8_t, uint4{lo[0], lo[1], lo[2], lo[3]});
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(W[i], H, sum, 0, 0, 0);
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(W[i], L, sum, 0, 0, 0);
        }
        return sum;
    };
    auto plane_by_plane = [&](int J, const uint4* xs, auto w, auto e) {
        Planes p = planes_of(w, e);
        bool top = false;
#pragma unroll
        for (int i = 0; i < Q; ++i)
#pragma unroll
            for (int s = 0; s < (GEN ? 8 : 1); ++s) top |= e(i, s) > kTop;
#pragma unroll 1
        for (int s = 0; s < 8; ++s) {
            bhalf8_t W[Q];
            next_step(J, s, false, p, W);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                acc[c] = add_planes(xs, s, c, W, acc[c]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (!__any(top)) return;
        // (not unrolled: the row tiles take turns in acc[0], and no registers are added)
#pragma unroll 1
        for (int c = 0; c < CT; ++c) {
            p = planes_of(w, e);
            float16_t sum;
#pragma unroll
            for (int v = 0; v < 16; ++v) sum[v] = 0.0f;
#pragma unroll 1
            for (int s = 0; s < 8; ++s) {
                bhalf8_t W[Q];
                next_step(J, s, true, p, W);
                sum = add_planes(xs, s, c, W, sum);
            }
#pragma unroll
            for (int v = 0; v < 16; ++v) sum[v] = acc[0][v] + ldexpf(sum[v], kTopShift);
#pragma unroll
            for (int i = 0; i + 1 < CT; ++i) acc[i] = acc[i + 1];
            acc[CT - 1] = sum;
        }
    };

    // a row's 16 keys of a block are stored rotated by the row
    const uint32_t rot = (uint32_t)(16 - (n & 15)) & 15u;
    const uint32_t rot_bytes = rot & 3u, rot_bits = 4u * (rot & 4u);
    const bool rot_swap = rot & 8u;
    // A group of two blocks as words in step order: wd[block][plane][half], ew the planes'
    // exponents of a block; returns whether this lane's row has a block to do plane by plane.
    auto unpack = [&](const Keys<Q, GEN>& k, uint32_t (&wd)[2][Q][2], uint32_t (&ew)[2][kE]) {
        int ex[Q];
        uint32_t own[kE] = {};
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            // rotated by rot: the part of whole bytes first, then even and odd chunks as two
            // rows of 8 bytes, each by half of the rest
            const uint32_t in[4] = {k.w[i].x, k.w[i].y, k.w[i].z, k.w[i].w};
            uint32_t c[4], ev[2], od[2];
#pragma unroll
            for (int d = 0; d < 4; ++d)
                c[d] = __builtin_amdgcn_alignbyte(in[(d + 1) & 3], in[d], rot_bytes);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ev[h] = __builtin_amdgcn_perm(c[2 * h + 1], c[2 * h], 0x06040200u);
                od[h] = __builtin_amdgcn_perm(c[2 * h + 1], c[2 * h], 0x07050301u);
            }
            auto turn = [&](uint32_t (&v)[2]) {
                const uint32_t lo = __builtin_amdgcn_alignbit(v[1], v[0], rot_bits);
                const uint32_t hi = __builtin_amdgcn_alignbit(v[0], v[1], rot_bits);
                v[0] = rot_swap ? hi : lo;
                v[1] = rot_swap ? lo : hi;
            };
            turn(ev);
            turn(od);
            // lanes 0-31 keep the even chunks of both blocks, lanes 32-63 the odd ones
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto sw = __builtin_amdgcn_permlane32_swap(ev[h], od[h], false, false);
                wd[0][i][h] = sw[0];
                wd[1][i][h] = sw[1];
            }
            ex[i] = (int)(int8_t)k.e[i];
            own[i >> 2] |= k.e[i] << (8 * (i & 3));
        }
#pragma unroll
        for (int d = 0; d < kE; ++d) {
            const auto sw = __builtin_amdgcn_permlane32_swap(own[d], own[d], false, false);
            ew[0][d] = sw[0];
            ew[1][d] = sw[1];
        }
        return is_far(ex);
    };
    // kPart: chunk 2 s + g of a block has exponent (2 s + g) / gc of those loaded, byte s & 3
    // of selector s / 4; with groups of one chunk the second four lie 8 bytes further
    const int gc = imax(a.G >> 3, 1);
    uint32_t sel[2] = {0, 0};
    if constexpr (GEN == kPart) {
#pragma unroll
        for (int s = 0; s < 8; ++s)
            sel[s >> 2] |= (uint32_t)(((2 * s + g) / gc) & 7) << (8 * (s & 3));
    }
    // kPart: one block's keys and exponents in the form of kAny
    auto spread_out = [&](const Keys<Q, GEN>& k, int J) {
        Keys<Q, GEN> out;
#pragma unroll
        for (int i = 0; i < Q; ++i) {
            uint4 w = k.w[i];
            if (16 * J + 16 <= C) {
                const uint32_t in[4] = {w.x, w.y, w.z, w.w};
                uint32_t c[4];
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    c[d] = __builtin_amdgcn_alignbyte(in[(d + 1) & 3], in[d], rot_bytes);
                const uint32_t pick = g ? 0x07050301u : 0x06040200u;
                const uint32_t v0 = __builtin_amdgcn_perm(c[1], c[0], pick);
                const uint32_t v1 = __builtin_amdgcn_perm(c[3], c[2], pick);
                const uint32_t lo = __builtin_amdgcn_alignbit(v1, v0, rot_bits);
                const uint32_t hi = __builtin_amdgcn_alignbit(v0, v1, rot_bits);
                w.x = rot_swap ? hi : lo;
                w.y = rot_swap ? lo : hi;
            }
            const uint4 x = k.x[GEN == kPart ? i : 0];
            w.z = __builtin_amdgcn_perm(x.y, x.x, sel[0]);
            w.w = gc == 1 ? __builtin_amdgcn_perm(x.w, x.z, sel[1])
                          : __builtin_amdgcn_perm(x.y, x.x, sel[1]);
            out.w[i] = w;
        }
        return out;
    };
    auto word_of = [](const Keys<Q, GEN>& k, int i, int h) { return h ? k.w[i].y : k.w[i].x; };
    auto exponent_of = [](const Keys<Q, GEN>& k, int i, int s) {
        return (int)(int8_t)((s & 4 ? k.w[i].w : k.w[i].z) >> (8 * (s & 3)));
    };
    auto block_far = [&](const Keys<Q, GEN>& k) {
        bool far = false;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            int ex[Q];
#pragma unroll
            for (int i = 0; i < Q; ++i) ex[i] = exponent_of(k, i, s);
            far |= is_far(ex);
        }
        return far;
    };

    // Blocks left for the second loop, a bit per two steps (steps far apart share one): it
    // visits those alone (11008x4096, 250 rows: 45 us, one such group in the layer 57, where a
    // loop over all blocks took 79; every block 197).
    bool left = false;
    auto leave = [&](int s) {
        left = true;
        if (lane == 0) atomicOr(&far_steps[(s >> 6) & (kFarWords - 1)], 1u << ((s >> 1) & 31));
    };
    if ((int)threadIdx.x < kFarWords) far_steps[threadIdx.x] = 0u;
    Keys<Q, GEN> k;
    if (blk0 < blk1) {
        copy_x(blk0, 0);
        load_keys(blk0, k);
    }
    arrive();
    if constexpr (GEN) {
#pragma unroll 1
        for (int s = 0; s < steps; ++s) {
            const int J = blk0 + s;
            if (J + 1 < blk1) copy_x(J + 1, (s + 1) & 1);
            if (J < blk1) {
                const Keys<Q, GEN> now = GEN == kPart ? spread_out(k, J) : k;
                if (J + 1 < blk1) load_keys(J + 1, k);
                if (__any(block_far(now)))
                    leave(s);
                else
                    summed(J, xr + (s & 1) * kBuf,
                           [&](int i, int h) { return word_of(now, i, h); },
                           [&](int i, int st) { return exponent_of(now, i, st); });
            }
            arrive();
        }
    } else {
        // groups of two blocks; the next group's keys are requested in the second
#pragma unroll 1
        for (int s0 = 0; s0 < steps; s0 += 2) {
            uint32_t wd[2][Q][2], ew[2][kE];
            const bool far = __any(unpack(k, wd, ew) && blk0 + s0 + g < blk1);
            if (far) leave(s0);
            const int J0 = blk0 + s0;
            auto e0 = [&](int i, int) { return (int)(int8_t)(ew[0][i >> 2] >> (8 * (i & 3))); };
            auto e1 = [&](int i, int) { return (int)(int8_t)(ew[1][i >> 2] >> (8 * (i & 3))); };
            auto w0 = [&](int i, int h) { return wd[0][i][h]; };
            auto w1 = [&](int i, int h) { return wd[1][i][h]; };
            const bool run = J0 < blk1 && !far;
            if (J0 + 1 < blk1) copy_x(J0 + 1, 1);
            half8_t W[2], X[kRing];
            Next x;
            int xw;
            if constexpr (kPipelined) {
                if (run) {
                    first_x(xr, &xw, X);
                    new_block(x, e0);
#pragma unroll
                    for (int u = 0; u < kPieces; ++u) piece(x, u, 0, w0);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        take(x, W);
                        if (q == 3) new_block(x, e1);  // (unused if there is no second block)
                        quarter(xr, xw, q, W, X, [&](int u) {
                            if (q < 3) piece(x, u, q + 1, w0);
                            else piece(x, u, 0, w1);
                        });
                    }
                }
            } else if (run) {
                if constexpr (Q <= 4) in_turn(xr, w0, e0);
                else summed(J0, xr, w0, e0);
            }
            arrive();
            if (s0 + 1 >= steps) break;
            if (J0 + 2 < blk1) {
                copy_x(J0 + 2, 0);
                load_keys(J0 + 2, k);
            }
            const uint4* xs = xr + kBuf;
            if (run && J0 + 1 < blk1) {
                if constexpr (kPipelined) {
                    first_x(xs, &xw, X);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        take(x, W);
                        quarter(xs, xw, q, W, X, [&](int u) {
                            if (q < 3) piece(x, u, q + 1, w1);
                        });
                    }
                } else if constexpr (Q <= 4) {
                    in_turn(xs, w1, e1);
                } else {
                    summed(J0 + 1, xs, w1, e1);
                }
            }
            arrive();
        }
    }
    // the second loop runs the groups that the first one left, the same in every way
    if (__syncthreads_or(left)) {
#pragma unroll 1
        for (int s = 0; s < steps; ++s) {
            const uint32_t word = (uint32_t)__builtin_amdgcn_readfirstlane(
                (int)far_steps[(s >> 6) & (kFarWords - 1)]);
            if (!(word >> ((s >> 1) & 31) & 1u)) continue;  // uniform over the workgroup
            const int J = blk0 + s;
            if (J < blk1) copy_x(J, 0);
            arrive();
            if (J < blk1) {
                if constexpr (GEN) {
                    load_keys(J, k);
                    if constexpr (GEN == kPart) k = spread_out(k, J);
                    if (__any(block_far(k)))
                        plane_by_plane(J, xr, [&](int i, int h) { return word_of(k, i, h); },
                                       [&](int i, int st) { return exponent_of(k, i, st); });
                } else {
                    uint32_t wd[2][Q][2], ew[2][kE];
                    load_keys(J & ~1, k);
                    if (__any(unpack(k, wd, ew) && (J & ~1) + g < blk1)) {
                        // block J & 1, by selects (values the compiler cannot turn into an
                        // indexed array in memory)
                        auto pick = [&](uint32_t w0, uint32_t w1) {
                            asm volatile("" : "+v"(w0), "+v"(w1));
                            return J & 1 ? w1 : w0;
                        };
                        plane_by_plane(
                            J, xr, [&](int i, int h) { return pick(wd[0][i][h], wd[1][i][h]); },
                            [&](int i, int) {
                                const uint32_t e = pick(ew[0][i >> 2], ew[1][i >> 2]);
                                return (int)(int8_t)(e >> (8 * (i & 3)));
                            });
                    }
                }
            }
            __syncthreads();
        }
    }

    // Through LDS to outputs: lane (r, g) of row tile c has row r of it and 16 consecutive
    // outputs from nb.  Loops that are not unrolled: what follows the product is a lot of
    // code.  KW = 1: a wave's own space takes half its row tiles at a time.
    constexpr int kPasses = KW > 1 ? 1 : 2, kPass = CT / kPasses;
    constexpr int kVals = kPass * 1024;
    static_assert(CT % kPasses == 0 && kWaves * kVals <= KW * 2 * kBuf * 4, "sums fit the buffers");
    float* red = reinterpret_cast<float*>(xbuf) + lane;
    const int nb = n0 + 16 * g;
    const sa_epi::Epilogue& epi = a.epi;
    // (KW > 1: a wave's vectors are all first or all second halves of the 16)
    constexpr int kHalves = KW > 1 ? 1 : 2;
    float bias[kHalves][8];
#pragma unroll
    for (int j = 0; j < 8 * kHalves; ++j) {
        const int nn = nb + (KW > 1 ? 8 * (kw & 1) : 0) + j;
        bias[j >> 3][j & 7] = epi.bias ? epi.bias[(int64_t)expert * N + imin(nn, N - 1)] : 0.0f;
    }
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
#pragma unroll
        for (int c = 0; c < kPass; ++c)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                red[wave * kVals + (c * 16 + v) * 64] = acc[pass * kPass + c][v];
        if constexpr (KW > 1) __syncthreads();
        else wave_fence();
        // kUnroll vectors of 8 outputs at a time, their operands requested together
        constexpr int kVectors = (2 * kPass + KW - 1) / KW, kUnroll = kVectors < 4 ? kVectors : 4;
#pragma unroll 1
        for (int o0 = KW > 1 ? kw : 0; o0 < 2 * kPass; o0 += kUnroll * KW) {
            sa_epi::Operands8 operands[kUnroll];
            int64_t at[kUnroll];
            int count[kUnroll];  // outputs of the vector, at most 0: none
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int o = o0 + u * KW, nn = nb + 8 * (o & 1);
                const int row = first + kTile * (pass * kPass + (o >> 1)) + r;
                at[u] = (int64_t)row * N + nn;
                count[u] = o < 2 * kPass && row < end && sa_linear::source_row(a, row) >= 0
                               ? N - nn
                               : 0;
                if (count[u] >= 8) sa_epi::fetch(epi, at[u], &operands[u]);
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                if (count[u] < 1) continue;
                const int o = o0 + u * KW;
                float v[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float* p = red + rw * kVals + (o * 8 + j) * 64;
                    v[j] = p[0];
#pragma unroll
                    for (int x = 1; x < KW; ++x) v[j] += p[x * RW * kVals];
                }
                if (count[u] >= 8) sa_epi::finish(epi, at[u], bias[u % kHalves], operands[u], v);
                else sa_epi::finish_some(epi, at[u], bias[u % kHalves], count[u], v);
            }
        }
        if constexpr (kPasses > 1) wave_fence();
    }
}

template <int Q, int CT, int KW, int GEN>
__global__ __launch_bounds__(kThreads, CT == 1 && Q <= 4 && !GEN ? 4 : 2)
void k_panel(Args pa) {
    __shared__ uint4 xbuf[KW * 2 * CT * 512];
    __shared__ uint32_t far_steps[kFarWords];
    int expert, first, end;
    if (!sa_linear::find_tile(pa.a, kTile * CT, (int)(blockIdx.x / (unsigned)pa.n_tiles), &expert,
                              &first, &end))
        return;
    // a tile of fewer rows runs the body of their height
    const int rows = end - first;
    if constexpr (CT == 8) {
        if (rows <= 2 * kTile) return body<Q, 2, KW, GEN>(pa, xbuf, far_steps, expert, first, end);
        if (rows <= 4 * kTile) return body<Q, 4, KW, GEN>(pa, xbuf, far_steps, expert, first, end);
        if (rows <= 6 * kTile) return body<Q, 6, KW, GEN>(pa, xbuf, far_steps, expert, first, end);
    } else if constexpr (CT == 4 || (CT == 2 && KW > 1)) {
        if (rows <= CT / 2 * kTile) return body<Q, CT / 2, KW, GEN>(pa, xbuf, far_steps, expert, first, end);
    }
    body<Q, CT, KW, GEN>(pa, xbuf, far_steps, expert, first, end);
}

template <int Q, int CT, int KW, int GEN>
void start(Args& pa, hipStream_t s) {
    const int cols = kTile * (kWaves / KW);
    pa.n_tiles = (pa.a.N + cols - 1) / cols;
    const int64_t tiles = sa_linear::most_tiles(pa.a, kTile * CT);
    hipLaunchKernelGGL((k_panel<Q, CT, KW, GEN>), dim3((unsigned)(tiles * pa.n_tiles)),
                       dim3(kThreads), 0, s, pa);
}

// Tiles of a workgroup: 32 ct rows and 256 / kw outputs, with what its time is made of.
struct Form {
    int ct, kw;
    double base, alone, alone_q, shared, shared_q, end;
};

template <int Q, int GEN>
void start_form(Args& pa, const Form& f, hipStream_t s) {
    switch (10 * f.ct + f.kw) {
        case 81:
            if constexpr (Q <= 4 && GEN == kWhole) start<Q, 8, 1, GEN>(pa, s);
            break;
        case 41:
            if constexpr (Q <= 4 && GEN != kAny) start<Q, 4, 1, GEN>(pa, s);
            break;
        case 42:
            if constexpr (Q <= 4 && GEN != kAny) start<Q, 4, 2, GEN>(pa, s);
            break;
        case 22: start<Q, 2, 2, GEN>(pa, s); break;
        case 24: start<Q, 2, 4, GEN>(pa, s); break;
        case 14: start<Q, 1, 4, GEN>(pa, s); break;
        default: start<Q, 1, 8, GEN>(pa, s); break;
    }
}

// The arguments of a layer whose groups are whole blocks, and of any other.
inline Args other_args(const Layer& a) {
    Args pa{};
    pa.a = a;
    pa.byte_offsets = (int64_t)a.x_rows * a.K < (int64_t)1 << 31;
    return pa;
}
inline Args whole_args(const Layer& a) {
    Args pa = other_args(a);
    const uint32_t d = (uint32_t)(a.G / 128);
    pa.group_magic = d <= 1 ? 0u : (uint32_t)(((1ull << 32) + d - 1) / d);
    return pa;
}

}  // namespace
}  // namespace sa_panel

#endif
