// What every kernel of the layer needs to read keys and exponents of the packed
// layout (16-byte key rows, rotated by the row).
#ifndef SHIFTADD_KEYS_H
#define SHIFTADD_KEYS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

__host__ __device__ inline int imin(int a, int b) { return a < b ? a : b; }
__host__ __device__ inline int imax(int a, int b) { return a > b ? a : b; }

// Byte offset of the key of (plane i, row n, chunk c) in the packed layout.
// Rows come in tiles of 64 and chunks in blocks of 16; a 64-row tile of one
// block is a contiguous piece, 16 bytes per row.  Inside a full block the 16
// keys of row r are rotated by r: position p holds chunk (p + r) mod 16, so
// that the lanes of a wave querying position p touch 16 different tables.
__host__ __device__ inline int64_t layout_offset(int i, int n, int c, int N, int C) {
    const int T = n >> 6, r = n & 63;
    const int R = imin(64, N - 64 * T);
    const int J = c >> 4, u = c & 15;
    const int U = imin(16, C - 16 * J);
    const int p = (U == 16) ? ((u - r) & 15) : u;
    return ((int64_t)i * N + (int64_t)64 * T) * C + (int64_t)16 * J * R +
           (int64_t)r * U + p;
}

// Bytes of v rotated so that byte p of the result is byte (p + r) mod 16 of v.  The
// key at position p of a row is chunk (p + row) mod 16 of its block: rotating 16
// exponents in chunk order by the row lines them up with the keys, rotating the
// keys by 16 - row puts them in chunk order.
__device__ inline void rotate16(const uint4 v, int r, uint32_t out[4]) {
    const uint32_t in[4] = {v.x, v.y, v.z, v.w};
    const uint32_t b = (uint32_t)(r & 3);
    uint32_t t[4], u[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) t[d] = __builtin_amdgcn_alignbyte(in[(d + 1) & 3], in[d], b);
#pragma unroll
    for (int d = 0; d < 4; ++d) u[d] = (r & 4) ? t[(d + 1) & 3] : t[d];
#pragma unroll
    for (int d = 0; d < 4; ++d) out[d] = (r & 8) ? u[(d + 2) & 3] : u[d];
}

// T consecutive bytes (exponents or signs of a group's terms), one per byte of the
// result; 2 and 4 are aligned to their size (checked on the host).
__device__ inline uint32_t load_terms(const int8_t* p, int T) {
    const uint8_t* b = reinterpret_cast<const uint8_t*>(p);
    if (T == 4) return *reinterpret_cast<const uint32_t*>(b);
    if (T == 2) return *reinterpret_cast<const uint16_t*>(b);
    if (T == 3) return (uint32_t)b[0] | ((uint32_t)b[1] << 8) | ((uint32_t)b[2] << 16);
    return b[0];
}

#endif
