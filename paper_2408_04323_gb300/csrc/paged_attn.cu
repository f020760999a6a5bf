// Attention of a batch of new tokens over a paged key-value cache.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"

namespace {

struct AttnArgs {
    scoot_kv_layout L;
    int32_t bs_log, n_heads, group, n_req, causal, window;
    const void* q;
    int64_t q_ld_token, q_ld_head, n_tokens;
    const int32_t* query_start;
    const int32_t* kv_len;
    const int32_t* table;
    int64_t ld_table;
    const void* k;
    const void* v;
    float scale;
    void* out;
    int64_t out_ld_token, out_ld_head;
    float* lse;
    uint32_t* err;
};

__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float x, __half& y) { y = __float2half_rn(x); }
__device__ __forceinline__ void from_float(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }

// One warp per (token, query head): the keys that it sees one after another,
// with the running maximum and sum of the softmax; a lane holds D / 32
// consecutive dimensions.
template <typename T, int D>
__global__ void __launch_bounds__(256) attn_row_kernel(const AttnArgs a) {
    constexpr int kE = D / 32;
    const int lane = threadIdx.x & 31;
    const int64_t rows = a.n_tokens * a.n_heads;
    if (blockIdx.x == 0)
        for (int r = threadIdx.x; r < a.n_req; r += blockDim.x)
            if (a.query_start[r] > a.query_start[r + 1]) atomicOr(a.err, SCOOT_DEVERR_INDEX);
    for (int64_t w = ((int64_t)blockIdx.x * blockDim.x + threadIdx.x) >> 5; w < rows;
         w += ((int64_t)gridDim.x * blockDim.x) >> 5) {
        const int64_t t = w / a.n_heads;
        const int h = (int)(w - t * a.n_heads);
        // the request: the last one that starts at or before t
        int lo = 0, hi = a.n_req - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (a.query_start[mid] <= t) lo = mid;
            else hi = mid - 1;
        }
        const int64_t q0 = a.query_start[lo], q1 = a.query_start[lo + 1], kv = a.kv_len[lo];
        if (q0 < 0 || q1 > a.n_tokens || kv < 0 || kv > a.ld_table << a.bs_log) {
            if (lane == 0) atomicOr(a.err, SCOOT_DEVERR_INDEX);
            continue;
        }
        if (t < q0 || t >= q1) continue;
        const int64_t pos = kv - (q1 - q0) + (t - q0);
        const int64_t end = a.causal ? min(kv, pos + 1) : kv;
        const int64_t begin = a.window > 0 ? max((int64_t)0, pos + 1 - a.window) : 0;
        float qf[kE], o[kE], m = -INFINITY, l = 0.0f;
        const T* qp = static_cast<const T*>(a.q) + t * a.q_ld_token + h * a.q_ld_head + lane * kE;
#pragma unroll
        for (int e = 0; e < kE; ++e) {
            qf[e] = to_float(qp[e]);
            o[e] = 0.0f;
        }
        const int64_t head_at = (int64_t)(h / a.group) * a.L.ld_head + lane * kE;
        for (int64_t i = begin; i < end; ++i) {
            const int32_t id = a.table[lo * a.ld_table + (i >> a.bs_log)];
            if (id < 0 || id >= a.L.n_blocks) {
                if (lane == 0) atomicOr(a.err, SCOOT_DEVERR_INDEX);
                continue;
            }
            const int64_t at = id * a.L.ld_block + (i & ((1 << a.bs_log) - 1)) * a.L.ld_token + head_at;
            const T* kp = static_cast<const T*>(a.k) + at;
            const T* vp = static_cast<const T*>(a.v) + at;
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < kE; ++e) s = fmaf(qf[e], to_float(kp[e]), s);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
            s *= a.scale;
            const float mn = fmaxf(m, s), ms = mn == -INFINITY ? 0.0f : mn;
            const float f = expf(m - ms), p = expf(s - ms);
            l = fmaf(l, f, p);
#pragma unroll
            for (int e = 0; e < kE; ++e) o[e] = fmaf(o[e], f, p * to_float(vp[e]));
            m = mn;
        }
        T* op = static_cast<T*>(a.out) + t * a.out_ld_token + h * a.out_ld_head + lane * kE;
#pragma unroll
        for (int e = 0; e < kE; ++e) from_float(end > begin ? o[e] / l : 0.0f, op[e]);
        if (a.lse && lane == 0) a.lse[t * a.n_heads + h] = end > begin ? m + logf(l) : -INFINITY;
    }
}

template <typename T>
scoot_status launch_rows(scoot_ctx* ctx, const AttnArgs& a, cudaStream_t st) {
    int sms = 0;
    SCOOT_CUDA(ctx, cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, ctx->device));
    int64_t blocks = (a.n_tokens * a.n_heads + 7) / 8;
    if (blocks > sms * 64) blocks = sms * 64;
    if (a.L.head_dim == 64) attn_row_kernel<T, 64><<<(unsigned)blocks, 256, 0, st>>>(a);
    else attn_row_kernel<T, 128><<<(unsigned)blocks, 256, 0, st>>>(a);
    SCOOT_LAUNCHED(ctx);
    return SCOOT_OK;
}

}  // namespace

extern "C" scoot_status scoot_paged_attention(scoot_ctx* ctx, const scoot_kv_layout* layout, const void* q,
                                              int64_t q_ld_token, int64_t q_ld_head, int32_t n_heads, int64_t n_tokens,
                                              const int32_t* query_start, const int32_t* kv_len, int32_t n_req,
                                              const int32_t* block_table, int64_t ld_table, const void* k_cache,
                                              const void* v_cache, float scale, int32_t causal, int32_t window, void* out,
                                              int64_t out_ld_token, int64_t out_ld_head, float* lse, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if ((s = scoot_check_kv(ctx, layout, k_cache, v_cache)) != SCOOT_OK) return s;
    if (n_heads < 1 || n_heads % layout->n_kv_heads)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_heads = %d is not a multiple of n_kv_heads = %d", n_heads, layout->n_kv_heads);
    if (n_heads / layout->n_kv_heads > SCOOT_MAX_GROUP)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "%d query heads per key-value head, more than %d",
                          n_heads / layout->n_kv_heads, SCOOT_MAX_GROUP);
    if (n_tokens < 0 || n_tokens > 0x7FFFFFFFll / n_heads || n_req < 0 || ld_table < 0 || ld_table > (0x7FFFFFFFll / layout->block_size))
        return scoot_fail(ctx, SCOOT_EINVAL, "n_tokens = %lld, n_req = %d or ld_table = %lld out of range", (long long)n_tokens,
                          n_req, (long long)ld_table);
    if (!(scale > 0.0f) || scale > 3.0e38f) return scoot_fail(ctx, SCOOT_EINVAL, "scale = %g must be positive and finite", scale);
    if (window < 0) return scoot_fail(ctx, SCOOT_EINVAL, "window = %d < 0", window);
    if (n_tokens == 0 || n_req == 0) return SCOOT_OK;
    if ((s = scoot_check_heads(ctx, "q", q, q_ld_token, q_ld_head, n_tokens, n_heads, layout->head_dim)) != SCOOT_OK) return s;
    if ((s = scoot_check_heads(ctx, "out", out, out_ld_token, out_ld_head, n_tokens, n_heads, layout->head_dim)) != SCOOT_OK)
        return s;
    if (!query_start || !kv_len || (ld_table && !block_table)) return scoot_fail(ctx, SCOOT_EINVAL, "an array is NULL");
    AttnArgs a;
    a.L = *layout;
    a.bs_log = 0;
    while ((1 << a.bs_log) < layout->block_size) ++a.bs_log;
    a.n_heads = n_heads;
    a.group = n_heads / layout->n_kv_heads;
    a.n_req = n_req;
    a.causal = causal != 0;
    a.window = window;
    a.q = q;
    a.q_ld_token = q_ld_token;
    a.q_ld_head = q_ld_head;
    a.n_tokens = n_tokens;
    a.query_start = query_start;
    a.kv_len = kv_len;
    a.table = block_table;
    a.ld_table = ld_table;
    a.k = k_cache;
    a.v = v_cache;
    a.scale = scale;
    a.out = out;
    a.out_ld_token = out_ld_token;
    a.out_ld_head = out_ld_head;
    a.lse = lse;
    a.err = ctx->d_err;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return layout->dtype == SCOOT_BF16 ? launch_rows<__nv_bfloat16>(ctx, a, st) : launch_rows<__half>(ctx, a, st);
}
