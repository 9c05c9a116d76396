// Eight columns of a row in a lane's registers: loads, stores and sums shared by the kernels of the history encoder, and the
// arithmetic of rows in 8 bits.
#pragma once

#include "fs_device.h"
#include "freescale_encoder.h"

namespace fs {

// The GPU of a context for the time of a call, whatever device is current.
struct device_scope {
    int before = -1;
    bool ok = true;
    explicit device_scope(int device) {
        int cur = device;
        ok = hipGetDevice(&cur) == hipSuccess;
        if (ok && cur != device) {
            ok = hipSetDevice(device) == hipSuccess;
            if (ok) before = cur;
        }
    }
    ~device_scope() {
        if (before >= 0) (void)hipSetDevice(before);
    }
};

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline int elem_size(int dt) { return dt == FS_F32 ? 4 : 2; }

struct bf16_t {
    uint16_t bits;
};

// Eight consecutive elements, the first `left` of which exist (any number; in fours for fp32 rows, in eights for bf16 rows).
__device__ __forceinline__ void load8(const float *__restrict__ p, int left, float (&v)[8]) {
    const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
    const f32x4 a = left >= 4 ? *reinterpret_cast<const f32x4 *>(p) : zero;
    const f32x4 b = left >= 8 ? *reinterpret_cast<const f32x4 *>(p + 4) : zero;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a[i];
        v[4 + i] = b[i];
    }
}
__device__ __forceinline__ void load8(const bf16_t *__restrict__ p, int left, float (&v)[8]) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    const u32x4 a = left >= 8 ? *reinterpret_cast<const u32x4 *>(p) : zero;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_lo(a[i]);
        v[2 * i + 1] = bf16_hi(a[i]);
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    return f32_to_bf16_bits(lo) | (f32_to_bf16_bits(hi) << 16);
}
__device__ __forceinline__ void store8(float *p, int left, const float (&v)[8]) {
    const f32x4 a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
    if (left >= 4) *reinterpret_cast<f32x4 *>(p) = a;
    if (left >= 8) *reinterpret_cast<f32x4 *>(p + 4) = b;
}
__device__ __forceinline__ void store8(bf16_t *p, int left, const float (&v)[8]) {
    u32x4 a;
#pragma unroll
    for (int i = 0; i < 4; ++i) a[i] = pack_bf16(v[2 * i], v[2 * i + 1]);
    if (left >= 8) *reinterpret_cast<u32x4 *>(p) = a;
}
// the value an element has once it is stored
__device__ __forceinline__ float as_stored(float x, const float *) { return x; }
__device__ __forceinline__ float as_stored(float x, const bf16_t *) { return __uint_as_float(f32_to_bf16_bits(x) << 16); }

// sum over the LPR lanes that share a row, in every one of them; fixed order
template <int LPR>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int m = LPR / 2; m >= 1; m >>= 1) x += __shfl_xor(x, m, kWave);
    return x;
}

// ---- rows in 8 bits: groups of 32 columns are four neighbouring lanes of eight columns --------------------------------------
// The exponent byte of a group whose largest magnitude has these bits.  Six bits below its own power of two the magnitude
// lies in [64, 128) steps; from 127.5 steps on it would round to 128, and the step doubles - but for the top power of two, where
// 128 steps are beyond fp32 and the code stays at 127.  Integer comparisons order NaN behind infinity behind every number.
__device__ __forceinline__ uint32_t rows8_exp(uint32_t top_bits) {
    const uint32_t e = top_bits >> 23;
    if (e == 255u) return 255u;
    if (e < 7u) return 1u;
    return e - 6u + ((top_bits & 0x7FFFFFu) >= 0x7F0000u && e < 254u ? 1u : 0u);
}
__device__ __forceinline__ float rows8_step(uint32_t exp) {
    return exp == 0u ? __uint_as_float(0x00400000u) : exp == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(exp << 23);
}
// Codes of a lane's eight columns and the exponent byte of its group (the same in its four lanes).  The factor is a power of
// two, so a product is exact wherever it rounds to anything but zero.
__device__ __forceinline__ u32x2 rows8_encode(const float (&v)[8], uint32_t &exp) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = __float_as_uint(v[i]) & 0x7FFFFFFFu;
        top = b > top ? b : top;
    }
    uint32_t o = (uint32_t)__shfl_xor((int)top, 1, kWave);
    top = o > top ? o : top;
    o = (uint32_t)__shfl_xor((int)top, 2, kWave);
    top = o > top ? o : top;
    exp = rows8_exp(top);
    const float inv = exp == 255u ? 0.f : __uint_as_float((254u - exp) << 23);
    u32x2 codes = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = exp == 255u ? 0.f : v[i];
        const uint32_t c = (uint32_t)(int)fminf(fmaxf(rintf(x * inv), -127.f), 127.f) & 255u;
        codes[i / 4] |= c << (8 * (i % 4));
    }
    return codes;
}
__device__ __forceinline__ void rows8_decode(u32x2 codes, uint32_t exp, float (&v)[8]) {
    const float step = rows8_step(exp);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(int)(int8_t)(codes[i / 4] >> (8 * (i % 4))) * step;
}

}  // namespace fs
