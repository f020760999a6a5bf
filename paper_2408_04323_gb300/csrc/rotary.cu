// Rotary positions, alone and on the way into a paged key-value cache.
#include <algorithm>
#include <cmath>

#include "rotary.cuh"

namespace {

using namespace scoot_dev;

constexpr int kThreads = 256;
constexpr int kMaxWindow = 16;  // tokens of a block of threads
constexpr int kPer = 2;         // tasks of a thread under way at once

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
// a head: two chunks of eight that hold whole pairs) per thread, kPer of them in flight.
template <bool kBf16>
__global__ void __launch_bounds__(kThreads) rotary_kernel(const RotaryArgs a) {
    extern __shared__ float4 cs[];
    const int64_t t0 = (int64_t)blockIdx.x * a.window;
    const int n = (int)min((int64_t)a.window, a.n_tokens - t0), pairs = 8 * a.rot.turned;
    for (int e = threadIdx.x; e < n * pairs; e += kThreads) {
        const int t = e / pairs, pair = e - t * pairs;
        reinterpret_cast<float2*>(cs)[t * pairs + rotation_place(a.rot, pair)] = rotation_at(a.rot, pair, a.position[t0 + t]);
    }
    __syncthreads();
    const uint32_t per_token = (uint32_t)(a.n_q + a.n_k + a.n_v) * a.tasks, all = n * per_token;
    for (uint32_t e0 = threadIdx.x; e0 < all; e0 += kThreads * kPer) {
        uint4 ra[kPer], rb[kPer];
        uint16_t* to[kPer];
        int task[kPer], tok[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const uint32_t e = e0 + i * kThreads;
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
        for (int i = 0; i < kPer; ++i) {
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

scoot_status launch(scoot_ctx* ctx, RotaryArgs& a, bool bf16, cudaStream_t st) {
    // few tokens: one each, so that there are blocks for all multiprocessors
    const int64_t most = 8ll * scoot_sms(ctx);
    a.window = 1;
    while (a.window < kMaxWindow && (a.n_tokens + a.window - 1) / a.window > most) a.window *= 2;
    a.err = ctx->d_err;
    const int64_t blocks = (a.n_tokens + a.window - 1) / a.window;
    const size_t smem = (size_t)a.window * a.rot.turned * 8 * sizeof(float2);
    (bf16 ? rotary_kernel<true> : rotary_kernel<false>)<<<(unsigned)blocks, kThreads, smem, st>>>(a);
    SCOOT_LAUNCHED(ctx);
    return SCOOT_OK;
}

}  // namespace

scoot_status scoot_check_rotation(scoot_ctx* ctx, const scoot_rotation* rotation, int32_t head_dim, bool inverse, Rotation* out) {
    if (!rotation) return scoot_fail(ctx, SCOOT_EINVAL, "rotation is NULL");
    if (!rotation->turns || (reinterpret_cast<uintptr_t>(rotation->turns) & 7u))
        return scoot_fail(ctx, SCOOT_EINVAL, "rotation: turns is NULL or not 8-byte aligned");
    if (rotation->rot_dim < 16 || rotation->rot_dim % 16)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "rot_dim = %d is not a positive multiple of 16", rotation->rot_dim);
    if (rotation->rot_dim > head_dim)
        return scoot_fail(ctx, SCOOT_EINVAL, "rot_dim = %d is more than the head's %d", rotation->rot_dim, head_dim);
    if (!std::isfinite(rotation->magnitude)) return scoot_fail(ctx, SCOOT_EINVAL, "rotation: magnitude is not finite");
    out->turns = rotation->turns;
    out->turned = rotation->rot_dim / 16;
    out->interleaved = rotation->interleaved != 0;
    out->magnitude = rotation->magnitude;
    out->sign = inverse ? -1.0f : 1.0f;
    return SCOOT_OK;
}

scoot_status scoot_check_tokens(scoot_ctx* ctx, int64_t n_tokens, int64_t heads) {
    if (n_tokens < 0 || n_tokens > 0x7FFFFFFFll)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_tokens = %lld outside 0..2^31-1", (long long)n_tokens);
    if (heads < 1 || heads > 262140) return scoot_fail(ctx, SCOOT_EINVAL, "%lld heads outside 1..262140", (long long)heads);
    return SCOOT_OK;
}

extern "C" {

scoot_status scoot_rotary_frequencies(int32_t rot_dim, double base, int32_t stretch, double factor, double low, double high,
                                      double original_len, double* h_frequency) {
    if (rot_dim < 2 || rot_dim % 2 || !h_frequency || !(base > 0.0) || !std::isfinite(base)) return SCOOT_EINVAL;
    if (stretch != SCOOT_STRETCH_NONE && (!(factor > 0.0) || !std::isfinite(factor))) return SCOOT_EINVAL;
    if (stretch == SCOOT_STRETCH_PARTS && (!(high > low) || !std::isfinite(high - low) || !(original_len > 0.0) || !std::isfinite(original_len)))
        return SCOOT_EINVAL;
    if (stretch == SCOOT_STRETCH_BASE && rot_dim == 2) return SCOOT_EINVAL;  // the only frequency is 1
    if (stretch < SCOOT_STRETCH_NONE || stretch > SCOOT_STRETCH_PARTS) return SCOOT_EUNSUPPORTED;
    if (stretch == SCOOT_STRETCH_BASE) base *= std::pow(factor, (double)rot_dim / (rot_dim - 2));
    for (int i = 0; i < rot_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / rot_dim);
        if (stretch == SCOOT_STRETCH_LINEAR) f /= factor;
        if (stretch == SCOOT_STRETCH_PARTS) {
            const double turns = original_len * f / (2.0 * M_PI);
            const double keep = std::min(1.0, std::max(0.0, (turns - low) / (high - low)));
            f = f * keep + f / factor * (1.0 - keep);
        }
        h_frequency[i] = f;
    }
    return SCOOT_OK;
}

scoot_status scoot_rotary_turns(const double* h_frequency, int32_t n, uint64_t* h_turns) {
    if (n < 1 || !h_frequency || !h_turns) return SCOOT_EINVAL;
    for (int i = 0; i < n; ++i)
        if (!std::isfinite(h_frequency[i])) return SCOOT_EINVAL;
    for (int i = 0; i < n; ++i) {
        const double turns = std::fabs(h_frequency[i]) / (2.0 * M_PI), part = turns - std::floor(turns);
        const uint64_t t = (uint64_t)std::ldexp(part, 64);  // part < 1, so below 2^64; its last places, below 2^-64, are dropped
        h_turns[i] = h_frequency[i] < 0.0 ? 0 - t : t;
    }
    return SCOOT_OK;
}

scoot_status scoot_rotary(scoot_ctx* ctx, const scoot_rotation* rotation, int32_t dtype, const void* x, int64_t x_ld_token,
                          int64_t x_ld_head, int32_t n_heads, int32_t head_dim, const int32_t* position, int64_t n_tokens,
                          int32_t inverse, void* y, int64_t y_ld_token, int64_t y_ld_head, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if (dtype != SCOOT_F16 && dtype != SCOOT_BF16)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "dtype = %d is neither SCOOT_F16 nor SCOOT_BF16", dtype);
    if (head_dim < 16 || head_dim > 256 || head_dim % 16)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "head_dim = %d is not a multiple of 16 from 16 to 256", head_dim);
    RotaryArgs a = {};
    if ((s = scoot_check_rotation(ctx, rotation, head_dim, inverse != 0, &a.rot)) != SCOOT_OK) return s;
    if ((s = scoot_check_tokens(ctx, n_tokens, n_heads)) != SCOOT_OK) return s;
    if (n_tokens == 0) return SCOOT_OK;
    if ((s = scoot_check_heads(ctx, "x", x, x_ld_token, x_ld_head, head_dim)) != SCOOT_OK) return s;
    if ((s = scoot_check_heads(ctx, "y", y, y_ld_token, y_ld_head, head_dim)) != SCOOT_OK) return s;
    if (!position) return scoot_fail(ctx, SCOOT_EINVAL, "position is NULL");
    a.n_q = n_heads;
    a.tasks = head_dim / 16;
    a.n_tokens = n_tokens;
    a.position = position;
    a.q = {static_cast<const uint16_t*>(x), x_ld_token, x_ld_head};
    a.y = static_cast<uint16_t*>(y);
    a.y_ld_token = y_ld_token;
    a.y_ld_head = y_ld_head;
    return launch(ctx, a, dtype == SCOOT_BF16, static_cast<cudaStream_t>(stream));
}

scoot_status scoot_kv_append_rotary(scoot_ctx* ctx, const scoot_kv_layout* layout, const scoot_rotation* rotation, const void* q,
                                    int64_t q_ld_token, int64_t q_ld_head, int32_t n_heads, void* q_out, int64_t q_out_ld_token,
                                    int64_t q_out_ld_head, const void* k, int64_t k_ld_token, int64_t k_ld_head, const void* v,
                                    int64_t v_ld_token, int64_t v_ld_head, const int64_t* slot, const int32_t* position,
                                    int64_t n_tokens, void* k_cache, void* v_cache, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if ((s = scoot_check_kv(ctx, layout, k_cache, v_cache)) != SCOOT_OK) return s;
    const int D = layout->head_dim;
    RotaryArgs a = {};
    if ((s = scoot_check_rotation(ctx, rotation, D, false, &a.rot)) != SCOOT_OK) return s;
    if (n_heads < 0) return scoot_fail(ctx, SCOOT_EINVAL, "n_heads = %d < 0", n_heads);
    if ((s = scoot_check_tokens(ctx, n_tokens, (int64_t)n_heads + 2ll * layout->n_kv_heads)) != SCOOT_OK) return s;
    if (n_tokens == 0) return SCOOT_OK;
    if (n_heads) {
        if ((s = scoot_check_heads(ctx, "q", q, q_ld_token, q_ld_head, D)) != SCOOT_OK) return s;
        if ((s = scoot_check_heads(ctx, "q_out", q_out, q_out_ld_token, q_out_ld_head, D)) != SCOOT_OK) return s;
    }
    if ((s = scoot_check_heads(ctx, "k", k, k_ld_token, k_ld_head, D)) != SCOOT_OK) return s;
    if ((s = scoot_check_heads(ctx, "v", v, v_ld_token, v_ld_head, D)) != SCOOT_OK) return s;
    if (!slot || !position) return scoot_fail(ctx, SCOOT_EINVAL, "slot or position is NULL");
    a.n_q = n_heads;
    a.n_k = a.n_v = layout->n_kv_heads;
    a.tasks = D / 16;
    a.n_tokens = n_tokens;
    a.position = position;
    a.q = {static_cast<const uint16_t*>(q), q_ld_token, q_ld_head};
    a.k = {static_cast<const uint16_t*>(k), k_ld_token, k_ld_head};
    a.v = {static_cast<const uint16_t*>(v), v_ld_token, v_ld_head};
    a.y = static_cast<uint16_t*>(q_out);
    a.y_ld_token = q_out_ld_token;
    a.y_ld_head = q_out_ld_head;
    a.slot = slot;
    while ((1 << a.bs_log) < layout->block_size) ++a.bs_log;
    a.n_slots = layout->n_blocks << a.bs_log;
    a.ld_block = layout->ld_block;
    a.ld_token = layout->ld_token;
    a.ld_head = layout->ld_head;
    a.k_cache = static_cast<uint16_t*>(k_cache);
    a.v_cache = static_cast<uint16_t*>(v_cache);
    return launch(ctx, a, layout->dtype == SCOOT_BF16, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
