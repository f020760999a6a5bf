// Rotary positions: a vector's dimensions in pairs, each turned by its token's position times the pair's frequency.
//
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),  t = position * frequency
//
// Frequencies are kept as fractions of a turn, in units of 2^-64.  Their product with a position, modulo 2^64, is the angle
// modulo a turn without any rounding but the frequency's own (below 2^-64 of a turn per position: 2^-33 at the farthest), in two
// integer multiplications; only what is left of the angle within an eighth of a turn goes to a float.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"

namespace scoot_dev {

// What the kernels take of a scoot_rotation, and how a head's dimensions fall into tasks: task j of D / 16 has the chunks (of
// eight dimensions) chunk_a(j) and chunk_b(j), which hold the pairs 8 j .. 8 j + 7 if they turn at all (j < turned).
struct Rotation {
    const uint64_t* turns;
    int32_t turned;       // rot_dim / 16
    int32_t interleaved;
    float magnitude, sign;
    __device__ __forceinline__ int chunk_a(int j) const { return interleaved || j >= turned ? 2 * j : j; }
    __device__ __forceinline__ int chunk_b(int j) const { return interleaved || j >= turned ? 2 * j + 1 : j + turned; }
};

// magnitude (cos, sin) of position * turns.
__device__ __forceinline__ float2 rotation_at(const Rotation& r, int pair, int32_t position) {
    const uint64_t t = __ldg(reinterpret_cast<const unsigned long long*>(r.turns) + pair) * (uint64_t)(int64_t)position;
    const uint32_t q = (uint32_t)((t + (1ull << 61)) >> 62);  // the nearest quarter, and what is left: at most an eighth
    const float x = (float)(int32_t)((t >> 32) - ((uint64_t)q << 30)) * 0x1p-31f;  // in units of pi
    float s, c;
    sincospif(x, &s, &c);
    const float cq = q & 1u ? s : c, sq = q & 1u ? c : s;
    const float cn = (q + 1u) & 2u ? -cq : cq, sn = q & 2u ? -sq : sq;
    return make_float2(cn * r.magnitude, sn * (r.magnitude * r.sign));
}

// The cosines and sines of a token in shared memory: [4][turned] float4, the pairs 8 j + 2 i, 8 j + 2 i + 1 at i * turned + j,
// so that the tasks of a head read consecutive pieces.
__device__ __forceinline__ int rotation_place(const Rotation& r, int pair) {
    const int j = pair >> 3, i = (pair >> 1) & 3;
    return 2 * (i * r.turned + j) + (pair & 1);  // as float2
}

template <bool kBf16>
__device__ __forceinline__ float2 unpack16(uint32_t w) {
    if (kBf16) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack16_rn(float lo, float hi) {
    if (kBf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// A task's two chunks in fp32, turned by the cosines and sines cs of its token.
template <bool kBf16>
__device__ __forceinline__ void turn_task(const Rotation& r, const float4* cs, int j, uint4 ra, uint4 rb, float* a, float* b) {
    const uint32_t wa[4] = {ra.x, ra.y, ra.z, ra.w}, wb[4] = {rb.x, rb.y, rb.z, rb.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 x = unpack16<kBf16>(wa[i]), y = unpack16<kBf16>(wb[i]);
        a[2 * i] = x.x;
        a[2 * i + 1] = x.y;
        b[2 * i] = y.x;
        b[2 * i + 1] = y.y;
    }
    if (j >= r.turned) return;
    auto turn = [](float& x, float& y, float c, float s) {
        const float u = x;
        x = fmaf(u, c, -(y * s));
        y = fmaf(y, c, u * s);
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 t = cs[i * r.turned + j];
        if (r.interleaved) {  // neighbours: the pairs of the first chunk, then those of the second
            float* x = i < 2 ? a + 4 * i : b + 4 * (i - 2);
            turn(x[0], x[1], t.x, t.y);
            turn(x[2], x[3], t.z, t.w);
        } else {
            turn(a[2 * i], b[2 * i], t.x, t.y);
            turn(a[2 * i + 1], b[2 * i + 1], t.z, t.w);
        }
    }
}

}  // namespace scoot_dev

// Checks a rotation for heads of head_dim, and what the kernels take of it.
scoot_status scoot_check_rotation(scoot_ctx* ctx, const scoot_rotation* rotation, int32_t head_dim, bool inverse,
                                  scoot_dev::Rotation* out);
