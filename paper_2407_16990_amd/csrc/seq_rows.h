// Rows of fp32 or bf16 elements at any address, 16 bytes of them a thread: whole loads and stores wherever a row has them.
#pragma once
#include "seq_common.h"

// 16 bytes of a row of `cols` elements from element c on, of which the row may have fewer: all lanes load whole pieces that lie in the
// row, the last ones from further ahead, and row_place moves those to their place, with zeros behind.  (A branch for them, element by
// element, was a way to memory of its own: 14720 x 4092 of bf16 126 us, now 108.)
template <typename T, int E>
__device__ __forceinline__ u32x4 row_load(const T* row, int c, int cols)
{
    if (cols >= E) return seq_load<u32x4>(row + (c < cols - E ? c : cols - E));
    u32x4 w = {0, 0, 0, 0};                                  // a row shorter than a piece
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (c + i < cols) w[i * (int)sizeof(T) / 4] |= sizeof(T) == 4 ? *(const uint32_t*)(row + c + i) : (uint32_t)*(const uint16_t*)(row + c + i) << (16 * (i & 1));
    return w;
}
template <typename T, int E>
__device__ __forceinline__ void row_place(u32x4 w, int c, int cols, float (&v)[E])
{
    const int s = cols >= E && c > cols - E ? c - (cols - E) : 0;            // elements that w is ahead by
    if (__any(s)) {
        constexpr int W = 4 / sizeof(T);                     // elements of a word
        if (s & 2 * W) w = u32x4{w[2], w[3], 0, 0};
        if (s & W) w = u32x4{w[1], w[2], w[3], 0};
        if (W == 2 && (s & 1))
            w = u32x4{w[0] >> 16 | w[1] << 16, w[1] >> 16 | w[2] << 16, w[2] >> 16 | w[3] << 16, w[3] >> 16};
        if (s >= E) w = u32x4{0, 0, 0, 0};
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[2 * i] = seq_bf16_lo(w[i]); v[2 * i + 1] = seq_bf16_hi(w[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
    }
}

// the first `bytes` of w, or all 16; whole elements of B bytes
template <int B>
__device__ __forceinline__ void row_put(uint8_t* p, int bytes, u32x4 w)
{
    if (bytes >= 16) { seq_store(p, w); return; }
    if (bytes & 8) { seq_store(p, make_uint2(w[0], w[1])); p += 8; w = u32x4{w[2], w[3], 0, 0}; }
    if (bytes & 4) { seq_store(p, w[0]); p += 4; w[0] = w[1]; }
    if (B < 4 && (bytes & 2)) { seq_store(p, (uint16_t)w[0]); p += 2; w[0] >>= 16; }
    if (B < 2 && (bytes & 1)) *p = (uint8_t)w[0];
}

// past: whole pieces past the L2, for what the kernel does not read again and the L2s do not hold anyway
template <typename T, int E>
__device__ __forceinline__ void row_store(T* p, int n, const float (&v)[E], bool past = false)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if constexpr (sizeof(T) == 2) w[i] = seq_pack_bf16(v[2 * i], v[2 * i + 1]); else w[i] = __float_as_uint(v[i]);
    if (past && n >= E) seq_store_past(p, w);
    else row_put<(int)sizeof(T)>((uint8_t*)p, n * (int)sizeof(T), w);
}
#define ROWS_PAST (32ll << 20)   // bytes of output from which on: as many as the eight L2s have
