// Rotary positions: a vector's dimensions in pairs, each turned by its token's position times the pair's frequency.
//
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),  t = position * frequency
//
// Frequencies are kept as fractions of a turn, in units of 2^-64.  Their product with a position, modulo 2^64, is the angle
// modulo a turn without any rounding but the frequency's own (below 2^-64 of a turn per position: 2^-33 at the farthest), in two
// integer multiplications; only what is left of the angle within an eighth of a turn goes to a float, in units of 2^-32 (up
// to 2^-29 of a sine).
//
// What bounds it, in a graph: 2 bytes in and 2 out of an element.  32 k tokens with their keys and values into the cache (28 and 4
// heads of 128, fp16): 96 us, 6.2 TB/s, 92% of the copy rate; gradients of as many tokens turned back: 39 us, 88%.  256 tokens: 2.8
// us, a launch.  The angles are computed once per token and pair for all heads.
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

constexpr int kRotaryThreads = 256;
constexpr int kRotaryWindow = 16;   // tokens of a block of threads
constexpr int kRotaryPer = 2;       // tasks of a thread under way at once

struct Heads {
    const uint16_t* p;
    int64_t ld_token, ld_head;
};

struct RotaryArgs {
    Rotation rot;
    int32_t n_q, n_k, n_v;      // heads turned in place of y's, turned into the cache, copied into it
    int32_t tasks;              // of a head: head_dim / 16
    int32_t window;
    int64_t n_tokens;
    const int32_t* position;
    Heads q, k, v;
    uint16_t* y;
    int64_t y_ld_token, y_ld_head;
    const int64_t* slot;        // NULL: no cache
    int32_t bs_log;
    int64_t n_slots, ld_block, ld_token, ld_head;
    uint16_t* k_cache;
    uint16_t* v_cache;
    uint32_t* err;
};

// A block takes `window` tokens: their cosines and sines once for all heads, into shared memory, then a task (16 dimensions of
// a head: two chunks of eight that hold whole pairs) per thread, kRotaryPer of them in flight.
template <bool kBf16>
__device__ __forceinline__ void rotary_block(const RotaryArgs& a, int64_t block, float4* cs) {
    const int64_t t0 = block * a.window;
    const int n = (int)min((int64_t)a.window, a.n_tokens - t0), pairs = 8 * a.rot.turned;
    for (int e = threadIdx.x; e < n * pairs; e += kRotaryThreads) {
        const int t = e / pairs, pair = e - t * pairs;
        reinterpret_cast<float2*>(cs)[t * pairs + rotation_place(a.rot, pair)] = rotation_at(a.rot, pair, a.position[t0 + t]);
    }
    __syncthreads();
    const uint32_t per_token = (uint32_t)(a.n_q + a.n_k + a.n_v) * a.tasks, all = n * per_token;
    for (uint32_t e0 = threadIdx.x; e0 < all; e0 += kRotaryThreads * kRotaryPer) {
        uint4 ra[kRotaryPer], rb[kRotaryPer];
        uint16_t* to[kRotaryPer];
        int task[kRotaryPer], tok[kRotaryPer];
#pragma unroll
        for (int i = 0; i < kRotaryPer; ++i) {
            const uint32_t e = e0 + i * kRotaryThreads;
            to[i] = nullptr;
            if (e >= all) continue;
            const uint32_t t = e / per_token, c = e - t * per_token;
            int head = (int)(c / a.tasks);
            const int j = (int)(c - head * a.tasks);
            const int64_t token = t0 + t;
            int64_t s = 0;
            if (a.slot) {
                s = a.slot[token];
                if (s >= a.n_slots && c == 0) atomicOr(a.err, SCOOT_DEVERR_INDEX);
                if (s < 0 || s >= a.n_slots) continue;
            }
            const bool isq = head < a.n_q, isv = head >= a.n_q + a.n_k;
            Heads src = a.q;
            if (!isq) {
                head -= a.n_q;
                src = a.k;
                if (isv) {
                    head -= a.n_k;
                    src = a.v;
                }
                to[i] = (isv ? a.v_cache : a.k_cache) + (s >> a.bs_log) * a.ld_block + (s & ((1 << a.bs_log) - 1)) * a.ld_token + head * a.ld_head;
            } else {
                to[i] = a.y + token * a.y_ld_token + head * a.y_ld_head;
            }
            task[i] = isv ? j | 0x40000000 : j;
            tok[i] = (int)t;
            const uint16_t* p = src.p + token * src.ld_token + head * src.ld_head;
            ra[i] = *reinterpret_cast<const uint4*>(p + 8 * (isv ? 2 * j : a.rot.chunk_a(j)));
            rb[i] = *reinterpret_cast<const uint4*>(p + 8 * (isv ? 2 * j + 1 : a.rot.chunk_b(j)));
        }
#pragma unroll
        for (int i = 0; i < kRotaryPer; ++i) {
            if (!to[i]) continue;
            const bool isv = task[i] & 0x40000000;
            const int j = task[i] & 0x3FFFFFFF;
            if (!isv && j < a.rot.turned) {
                float x[8], y[8];
                turn_task<kBf16>(a.rot, cs + tok[i] * (pairs / 2), j, ra[i], rb[i], x, y);
                ra[i] = make_uint4(pack16_rn<kBf16>(x[0], x[1]), pack16_rn<kBf16>(x[2], x[3]), pack16_rn<kBf16>(x[4], x[5]), pack16_rn<kBf16>(x[6], x[7]));
                rb[i] = make_uint4(pack16_rn<kBf16>(y[0], y[1]), pack16_rn<kBf16>(y[2], y[3]), pack16_rn<kBf16>(y[4], y[5]), pack16_rn<kBf16>(y[6], y[7]));
            }
            *reinterpret_cast<uint4*>(to[i] + 8 * (isv ? 2 * j : a.rot.chunk_a(j))) = ra[i];
            *reinterpret_cast<uint4*>(to[i] + 8 * (isv ? 2 * j + 1 : a.rot.chunk_b(j))) = rb[i];
        }
    }
}

// Tokens of a block, few where there are few, so that there are blocks for all multiprocessors; with a cache, whose blocks
// take longer, two to four times as many blocks (32 k tokens of 28 and 4 heads of 128: 96 us, 98 with windows twice as long).
inline int rotary_window(scoot_ctx* ctx, int64_t n_tokens, int most, bool cache) {
    const int64_t blocks = (cache ? 32ll : 8ll) * scoot_sms(ctx);
    int window = 1;
    while (window < most && (n_tokens + window - 1) / window > blocks) window *= 2;
    return window;
}

}  // namespace scoot_dev

// Checks a rotation for heads of head_dim, and what the kernels take of it.
scoot_status scoot_check_rotation(scoot_ctx* ctx, const scoot_rotation* rotation, int32_t head_dim, bool inverse,
                                  scoot_dev::Rotation* out);
