// Rotary positions, alone and on the way into a paged key-value cache.
#include <algorithm>
#include <cmath>

#include "rotary.cuh"

namespace {

using namespace scoot_dev;

template <bool kBf16>
__global__ void __launch_bounds__(kRotaryThreads) rotary_kernel(const RotaryArgs a) {
    extern __shared__ float4 cs[];
    rotary_block<kBf16>(a, blockIdx.x, cs);
}

scoot_status launch(scoot_ctx* ctx, RotaryArgs& a, bool bf16, cudaStream_t st) {
    a.window = rotary_window(ctx, a.n_tokens, kRotaryWindow, a.slot != nullptr);
    a.err = ctx->d_err;
    const int64_t blocks = (a.n_tokens + a.window - 1) / a.window;
    const size_t smem = (size_t)a.window * a.rot.turned * 8 * sizeof(float2);
    (bf16 ? rotary_kernel<true> : rotary_kernel<false>)<<<(unsigned)blocks, kRotaryThreads, smem, st>>>(a);
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
    // 1 / 2 pi in two words (off by 2^-110): the product in two words as well, whose whole turns are dropped one by one.
    const double inverse = 0x1.45f306dc9c883p-3, inverse_low = -0x1.6b01ec5417056p-57;
    for (int i = 0; i < n; ++i) {
        const double f = std::fabs(h_frequency[i]);
        const double turns = std::fma(f, inverse, 0.0);  // (rounded here on every machine, and not fused into what follows)
        double low = std::fma(f, inverse_low, std::fma(f, inverse, -turns));
        low -= std::floor(low + 0.5);
        const double units = std::ldexp(turns - std::floor(turns), 64), whole = std::floor(units);  // below 2^64
        const double rest = units - whole + std::ldexp(low, 64);                                    // of either sign
        uint64_t t = (uint64_t)whole;
        t = rest < 0.0 ? t - (uint64_t)(0.5 - rest) : t + (uint64_t)(0.5 + rest);
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
