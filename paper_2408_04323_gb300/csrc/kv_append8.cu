// Keys and values into a paged cache of 8-bit floats (four exponent and three fraction bits) with a scale per block of tokens
// and head.
//
//   s = least power of two with amax <= 448 s,   code = rn(x / s)
//
// over all that the block holds of the head.  A power of two, so that a scale that grows (new tokens with larger numbers in a
// block that held some) changes only the exponents of the older codes: they are exact still, but for those that get so
// small that they lose fraction bits, whose error stays below half of the least step.  With any other scale every growth would
// round all of them again.  The format's steps are relative, so that nothing is lost by not using the scale's fraction.
//
// A run, the batch's tokens of one block, and a head are a warp's, so that scale and codes need no atomics: a block of threads
// takes the runs that begin among its window of tokens.  Queries are turned by blocks of their own.
//
// What bounds it: 32 k tokens of prompts, 32 heads of queries over 8 of 128, bf16: 136 us in a graph, 5.4 TB/s, 79% of the copy rate
// (queries alone 88 us, keys and values alone 60): issue slots and DRAM both two thirds busy.  Runs staged in shared memory took
// longer; held in registers between the two looks, with half as many blocks per multiprocessor, 189 us; values after keys 141.
// A token each for 256 requests: 5.2 us, of decodes and chunks with heads of 64 13.2 us: the chain slot - numbers - scale - older
// codes - codes.
#include <cuda_fp8.h>

#include <algorithm>

#include "rotary.cuh"

namespace {

using namespace scoot_dev;

constexpr int kThreads = kRotaryThreads, kWarps = kThreads / 32;
constexpr int kMaxWindow = 32;   // tokens among which a block of threads looks for the first ones of its runs
constexpr int kMaxBlock = 256;   // the largest block_size
constexpr int kWords = (kMaxWindow + kMaxBlock) / 32 + 1;

struct Append8Args {
    Rotation rot;               // turned = 0: none
    int32_t n_kv_heads, bs_log, window;
    int64_t kv_blocks;          // blocks of threads that take keys and values; the others queries
    int64_t n_tokens, n_slots;
    const int32_t* position;
    const uint16_t* kv[2];
    int64_t kv_ld_token[2], kv_ld_head[2];
    const int64_t* slot;
    int64_t ld_block, ld_token, ld_head;
    uint8_t* cache[2];
    float* scale[2];
    uint32_t* err;
    RotaryArgs queries;
};

// Two numbers as codes (of magnitude 448 at most), and back.
__device__ __forceinline__ uint32_t encode2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float2 decode2(uint32_t w) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)w));
    return __half22float2(*reinterpret_cast<const __half2*>(&r));
}

// The least power of two s >= 2^-100 with amax <= 448 s = 1.75 * 2^8 s; amax finite.
__device__ __forceinline__ float least_scale(float amax) {
    const uint32_t b = __float_as_uint(amax);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)max(e, 27) << 23);
}

// The largest magnitude; NaN if there is one.
__device__ __forceinline__ float max_nan(float a, float b) {
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void finite(float* x) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (!(fabsf(x[e]) < INFINITY)) x[e] = 0.0f;
}

template <bool kBf16, int D>
__global__ void __launch_bounds__(kThreads, 4) kv_append8_kernel(const Append8Args a) {
    constexpr int kTasks = D / 16, kTokens = 32 / kTasks;
    extern __shared__ float4 cs[];
    if (blockIdx.x >= a.kv_blocks) {
        rotary_block<kBf16>(a.queries, blockIdx.x - a.kv_blocks, cs);
        return;
    }
    __shared__ uint32_t goes_on[kWords], begins[kWords];  // bit i: token t0 + i continues a run; begins one
    __shared__ int run_at[kMaxWindow], run_n[kMaxWindow];
    __shared__ int n_runs, last;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t t0 = (int64_t)blockIdx.x * a.window;
    const int bs = 1 << a.bs_log;
    if (tid == 0) n_runs = last = 0;
    for (int i = tid; i < kWords * 32; i += kThreads) {  // (whole warps)
        bool on = false, first = false;
        if (i < a.window + bs && t0 + i < a.n_tokens) {
            const int64_t s = a.slot[t0 + i];
            const bool there = s >= 0 && s < a.n_slots;
            if (s >= a.n_slots && i < a.window) atomicOr(a.err, SCOOT_DEVERR_INDEX);
            on = there && (s & (bs - 1)) && t0 + i > 0 && a.slot[t0 + i - 1] == s - 1;
            first = there && !on;
        }
        const uint32_t w_on = __ballot_sync(0xffffffffu, on), w_first = __ballot_sync(0xffffffffu, first);
        if (lane == 0) {
            goes_on[i >> 5] = w_on;
            begins[i >> 5] = w_first;
        }
    }
    __syncthreads();
    if (tid < a.window && begins[tid >> 5] >> (tid & 31) & 1u) {
        int n = 1;
        while (tid + n < kWords * 32) {  // up to the next token that does not go on: at most bs - 1 further
            const int i = tid + n;
            const uint32_t stops = ~goes_on[i >> 5] >> (i & 31);
            if (stops) {
                n += __ffs(stops) - 1;
                break;
            }
            n += 32 - (i & 31);
        }
        const int at = atomicAdd(&n_runs, 1);
        run_at[at] = tid;
        run_n[at] = n;
        atomicMax(&last, tid + n);
    }
    __syncthreads();
    const int end = last, pairs = 8 * a.rot.turned;
    if (a.rot.turned) {
        for (int e = tid; e < end * pairs; e += kThreads) {
            const int t = e / pairs, pair = e - t * pairs;
            reinterpret_cast<float2*>(cs)[t * pairs + rotation_place(a.rot, pair)] = rotation_at(a.rot, pair, a.position[t0 + t]);
        }
        __syncthreads();
    }

    const int sub = lane / kTasks, j = lane % kTasks;
    const int units = n_runs * a.n_kv_heads, ka = 8 * a.rot.chunk_a(j), kb = 8 * a.rot.chunk_b(j);
    Rotation none = a.rot;
    none.turned = 0;
    bool odd = false;
#pragma unroll 1
    for (int u = warp; u < units; u += kWarps) {
        const int r = u / a.n_kv_heads, head = u - r * a.n_kv_heads;
        const int at = run_at[r], n = run_n[r];
        const int64_t t1 = t0 + at, s1 = a.slot[t1], block = s1 >> a.bs_log;
        const int in_block = (int)(s1 & (bs - 1));
        const int64_t scale_at = block * a.n_kv_heads + head;
        const uint16_t* src[2] = {a.kv[0] + t1 * a.kv_ld_token[0] + head * a.kv_ld_head[0], a.kv[1] + t1 * a.kv_ld_token[1] + head * a.kv_ld_head[1]};
        const int64_t to = block * a.ld_block + in_block * a.ld_token + head * a.ld_head;
        // (a power of two may be any number where the caller made the scale)
        float held = 0.0f;  // lanes 0 and 1: of keys and of values
        if (in_block && lane < 2) held = a.scale[lane][scale_at];
        // The lane's sixteen numbers of token t, of keys (turned) or of values.
        auto numbers = [&](int kv, int t, float* x) {
            const uint16_t* p = src[kv] + t * a.kv_ld_token[kv];
            if (kv == 0) turn_task<kBf16>(a.rot, cs + (at + t) * (pairs / 2), j, *reinterpret_cast<const uint4*>(p + ka), *reinterpret_cast<const uint4*>(p + kb), x, x + 8);
            else turn_task<kBf16>(none, nullptr, j, *reinterpret_cast<const uint4*>(p + 16 * j), *reinterpret_cast<const uint4*>(p + 16 * j + 8), x, x + 8);
        };
        // All of the run's lines on their way at once, without registers (prompts of 32 k tokens: 139 us without, 136 with).
        constexpr int kLines = D * 2 / 128;
        for (int e = lane; e < 2 * kLines * n; e += 32) {
            const int kv = e & 1, t = (e >> 1) / kLines, i = (e >> 1) % kLines;
            asm volatile("prefetch.global.L1 [%0];" ::"l"(src[kv] + t * a.kv_ld_token[kv] + 64 * i));
        }
        // Twice over the run's numbers, the second time from L1: for the largest, and for the codes.
        float top[2] = {0.0f, 0.0f};
        uint32_t top16 = 0;  // of values, which nothing turns: as bits of 16, two at a time
#pragma unroll 1
        for (int t = sub; t < n; t += kTokens) {
            const uint4* pv = reinterpret_cast<const uint4*>(src[1] + t * a.kv_ld_token[1] + 16 * j);
            const uint4 v0 = pv[0], v1 = pv[1];
            float x[16];
            numbers(0, t, x);
#pragma unroll
            for (int e = 0; e < 16; ++e) top[0] = max_nan(top[0], fabsf(x[e]));
            const uint32_t w[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) top16 = __vmaxu2(top16, w[e] & 0x7FFF7FFFu);
        }
        top[1] = unpack16<kBf16>(max(top16 & 0xFFFFu, top16 >> 16)).x;  // (what is not finite is above the others)
        const bool bad = __any_sync(0xffffffffu, !(top[0] < INFINITY) || !(top[1] < INFINITY));
        if (bad) {  // once more, without it
            odd = true;
            top[0] = top[1] = 0.0f;
#pragma unroll 1
            for (int t = sub; t < n; t += kTokens)
#pragma unroll
                for (int kv = 0; kv < 2; ++kv) {
                    float x[16];
                    numbers(kv, t, x);
                    finite(x);
#pragma unroll
                    for (int e = 0; e < 16; ++e) top[kv] = fmaxf(top[kv], fabsf(x[e]));
                }
        }
        float inv[2];
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], d));
            top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], d));
        }
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            float s = least_scale(top[kv]);
            if (in_block) {
                const float h = __shfl_sync(0xffffffffu, held, kv);
                const bool wrong = !(h >= 0.0f && h < INFINITY);
                odd |= wrong;
                if (h >= s && !wrong) {
                    s = h;
                } else {
                    // the scale has grown: the older tokens' codes by the growth
                    const float f = h / s;
                    for (int i = sub; i < in_block; i += kTokens) {
                        uint4* p = reinterpret_cast<uint4*>(a.cache[kv] + to + (int64_t)(i - in_block) * a.ld_token + 16 * j);
                        const uint4 w = *p;
                        auto again = [&](uint32_t v) {
                            const float2 lo = decode2(v & 0xFFFFu), hi = decode2(v >> 16);
                            return encode2(lo.x * f, lo.y * f) | encode2(hi.x * f, hi.y * f) << 16;
                        };
                        // (under a scale that cannot be, zeros: what is a NaN stays one when multiplied)
                        *p = wrong ? make_uint4(0, 0, 0, 0) : make_uint4(again(w.x), again(w.y), again(w.z), again(w.w));
                    }
                }
            }
            if (lane == 0) a.scale[kv][scale_at] = s;
            inv[kv] = 1.0f / s;
        }
#pragma unroll 1
        for (int t = sub; t < n; t += kTokens)
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                float x[16];
                numbers(kv, t, x);
                if (bad) finite(x);
                uint8_t* p = a.cache[kv] + to + t * a.ld_token;
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    w[e] = encode2(x[4 * e] * inv[kv], x[4 * e + 1] * inv[kv]) | encode2(x[4 * e + 2] * inv[kv], x[4 * e + 3] * inv[kv]) << 16;
                *reinterpret_cast<uint2*>(p + (kv ? 16 * j : ka)) = make_uint2(w[0], w[1]);
                *reinterpret_cast<uint2*>(p + (kv ? 16 * j + 8 : kb)) = make_uint2(w[2], w[3]);
            }
    }
    if (odd) atomicOr(a.err, SCOOT_DEVERR_VALUE);
}

template <bool kBf16, int D>
scoot_status launch(scoot_ctx* ctx, Append8Args& a, cudaStream_t st) {
    a.window = rotary_window(ctx, a.n_tokens, kMaxWindow, true);
    a.kv_blocks = (a.n_tokens + a.window - 1) / a.window;
    int64_t q_blocks = 0;
    size_t smem = (size_t)(a.window + (1 << a.bs_log)) * a.rot.turned * 8 * sizeof(float2);
    if (a.queries.n_q) {
        a.queries.window = rotary_window(ctx, a.n_tokens, kRotaryWindow, true);
        q_blocks = (a.n_tokens + a.queries.window - 1) / a.queries.window;
        smem = std::max(smem, (size_t)a.queries.window * a.rot.turned * 8 * sizeof(float2));
    }
    auto kern = kv_append8_kernel<kBf16, D>;
    const uint32_t bit = 1u << (5 + 2 * kBf16 + (D == 128));
    if (!(ctx->smem_set & bit)) {  // once per context, for the largest window and block
        SCOOT_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (kMaxWindow + kMaxBlock) * D / 2 * (int)sizeof(float2)));
        ctx->smem_set |= bit;
    }
    kern<<<(unsigned)(a.kv_blocks + q_blocks), kThreads, smem, st>>>(a);
    SCOOT_LAUNCHED(ctx);
    return SCOOT_OK;
}

}  // namespace

scoot_status scoot_check_kv8(scoot_ctx* ctx, const scoot_kv_layout* L, const void* k_cache, const void* v_cache, const float* k_scale,
                             const float* v_scale) {
    if (!L) return scoot_fail(ctx, SCOOT_EINVAL, "layout is NULL");
    if (L->dtype != SCOOT_E4M3) return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "the cache's dtype = %d is not SCOOT_E4M3", L->dtype);
    scoot_kv_layout as16 = *L;
    as16.dtype = SCOOT_BF16;
    scoot_status s = scoot_check_kv(ctx, &as16, k_cache, v_cache);
    if (s != SCOOT_OK) return s;
    if ((L->ld_block | L->ld_token | L->ld_head) & 15)
        return scoot_fail(ctx, SCOOT_EINVAL, "the cache's strides %lld, %lld and %lld must be multiples of 16", (long long)L->ld_block,
                          (long long)L->ld_token, (long long)L->ld_head);
    if (!k_scale || !v_scale) return scoot_fail(ctx, SCOOT_EINVAL, "k_scale or v_scale is NULL");
    if ((reinterpret_cast<uintptr_t>(k_scale) | reinterpret_cast<uintptr_t>(v_scale)) & 3u)
        return scoot_fail(ctx, SCOOT_EINVAL, "k_scale or v_scale is not 4-byte aligned");
    return SCOOT_OK;
}

extern "C" scoot_status scoot_kv_append8(scoot_ctx* ctx, const scoot_kv_layout* layout, int32_t dtype, const scoot_rotation* rotation,
                                         const void* q, int64_t q_ld_token, int64_t q_ld_head, int32_t n_heads, void* q_out,
                                         int64_t q_out_ld_token, int64_t q_out_ld_head, const void* k, int64_t k_ld_token,
                                         int64_t k_ld_head, const void* v, int64_t v_ld_token, int64_t v_ld_head,
                                         const int64_t* slot, const int32_t* position, int64_t n_tokens, void* k_cache,
                                         void* v_cache, float* k_scale, float* v_scale, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if ((s = scoot_check_kv8(ctx, layout, k_cache, v_cache, k_scale, v_scale)) != SCOOT_OK) return s;
    if (dtype != SCOOT_F16 && dtype != SCOOT_BF16)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "dtype = %d is neither SCOOT_F16 nor SCOOT_BF16", dtype);
    const int D = layout->head_dim;
    Append8Args a = {};
    if (n_heads < 0 || (n_heads && !rotation)) return scoot_fail(ctx, SCOOT_EINVAL, "n_heads = %d: queries come with a rotation", n_heads);
    if (rotation && (s = scoot_check_rotation(ctx, rotation, D, false, &a.rot)) != SCOOT_OK) return s;
    if ((s = scoot_check_tokens(ctx, n_tokens, (int64_t)n_heads + 2ll * layout->n_kv_heads)) != SCOOT_OK) return s;
    if (n_tokens == 0) return SCOOT_OK;
    if (n_heads) {
        if ((s = scoot_check_heads(ctx, "q", q, q_ld_token, q_ld_head, D)) != SCOOT_OK) return s;
        if ((s = scoot_check_heads(ctx, "q_out", q_out, q_out_ld_token, q_out_ld_head, D)) != SCOOT_OK) return s;
    }
    if ((s = scoot_check_heads(ctx, "k", k, k_ld_token, k_ld_head, D)) != SCOOT_OK) return s;
    if ((s = scoot_check_heads(ctx, "v", v, v_ld_token, v_ld_head, D)) != SCOOT_OK) return s;
    if (!slot || (rotation && !position)) return scoot_fail(ctx, SCOOT_EINVAL, "slot or position is NULL");
    a.n_kv_heads = layout->n_kv_heads;
    while ((1 << a.bs_log) < layout->block_size) ++a.bs_log;
    a.n_tokens = n_tokens;
    a.n_slots = layout->n_blocks << a.bs_log;
    a.position = position;
    a.queries.rot = a.rot;
    a.queries.n_q = n_heads;
    a.queries.tasks = D / 16;
    a.queries.n_tokens = n_tokens;
    a.queries.position = position;
    a.queries.q = {static_cast<const uint16_t*>(q), q_ld_token, q_ld_head};
    a.queries.y = static_cast<uint16_t*>(q_out);
    a.queries.y_ld_token = q_out_ld_token;
    a.queries.y_ld_head = q_out_ld_head;
    a.queries.slot = slot;
    a.queries.n_slots = a.n_slots;
    a.queries.err = ctx->d_err;
    a.kv[0] = static_cast<const uint16_t*>(k);
    a.kv[1] = static_cast<const uint16_t*>(v);
    a.kv_ld_token[0] = k_ld_token;
    a.kv_ld_token[1] = v_ld_token;
    a.kv_ld_head[0] = k_ld_head;
    a.kv_ld_head[1] = v_ld_head;
    a.slot = slot;
    a.ld_block = layout->ld_block;
    a.ld_token = layout->ld_token;
    a.ld_head = layout->ld_head;
    a.cache[0] = static_cast<uint8_t*>(k_cache);
    a.cache[1] = static_cast<uint8_t*>(v_cache);
    a.scale[0] = k_scale;
    a.scale[1] = v_scale;
    a.err = ctx->d_err;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == SCOOT_BF16) return D == 128 ? launch<true, 128>(ctx, a, st) : launch<true, 64>(ctx, a, st);
    return D == 128 ? launch<false, 128>(ctx, a, st) : launch<false, 64>(ctx, a, st);
}
