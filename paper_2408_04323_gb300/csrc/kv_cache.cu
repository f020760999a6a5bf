// A paged key-value cache: block tables and slot maps of a serving step from
// its requests' lengths, and the new tokens' keys and values into their slots.
#include <algorithm>

#include "internal.h"

namespace {

constexpr int kTabThreads = 1024;
constexpr uint32_t kTabSmemBit = 1u << 4;  // of scoot_ctx::smem_set
constexpr int kTabStaged = 16384;  // requests whose lengths go to shared memory (139 KB with the gaps)

// What scoot_kv_tables takes, by value.
struct TabArgs {
    const int32_t* cached;
    const int32_t* fresh;
    int32_t n_req, bs_log;
    int64_t longest;  // tokens that a row of the table and a 32-bit length hold
    int64_t n_blocks;
    int32_t* table;
    int64_t ld_table;
    const int32_t* free_blocks;
    int64_t n_free;
    int32_t* query_start;
    int32_t* kv_len;
    int64_t* slot;
    int32_t* position;
    int64_t n_tokens;
    int32_t* counts;
    uint32_t* err;
};

// One request: its tokens, the blocks it holds and the blocks it lacks.
struct TabRequest {
    int32_t cached, fresh, held, need;
    bool bad;
};

// (k_log: a thread's requests, for the gap after each thread's in shared memory that keeps their reads on
// different banks.)
__device__ __forceinline__ TabRequest tab_request(const TabArgs& a, const int2* staged, int k_log, int64_t r) {
    TabRequest q;
    const int2 len = staged ? staged[r + (r >> k_log)] : make_int2(a.cached[r], a.fresh[r]);
    q.cached = len.x;
    q.fresh = len.y;
    const int64_t total = (int64_t)q.cached + q.fresh;
    q.bad = q.cached < 0 || q.fresh < 0 || total > a.longest;
    q.fresh = max(q.fresh, 0);  // a bad request's tokens still have their places in the batch
    const int64_t mask = (1 << a.bs_log) - 1;
    q.held = q.bad ? 0 : (int32_t)((q.cached + mask) >> a.bs_log);
    q.need = q.bad ? 0 : (int32_t)((total + mask) >> a.bs_log) - q.held;
    return q;
}

// One launch.  Token t belongs to the request whose running sum of new tokens
// passes t, and its block, when the request does not hold it yet, is the free
// one at the running sum of the blocks lacked before it: both sums run over
// all requests.  Every block of the grid takes them for itself (thread i over
// k consecutive requests, k a power of two, then a scan of the 1024 threads' sums), which costs
// a read of 8 bytes per request from L2 where passing them on would cost a
// second launch, and then serves its own share of the batch's tokens: a binary
// search of the threads' sums, and a walk over the k requests of the one found.
// The lengths stay in shared memory up to kTabStaged requests, with a gap after
// each thread's (14.4 us without the gaps, 12.4 with them, for 8192 requests and
// 65,413 tokens).  The first token of a block that the request lacks writes its
// table entry.  Bound by latency: a launch, the lengths, the scan, an entry, a
// slot; 4.1 us for 48 requests of one token each among ten calls of a captured
// graph, 10.8 for the 8192 (a call through the binding 7.7 and 12.3).  Sums of 32
// bits in the walk and twice the blocks measured the same (12.4 us).
__global__ void __launch_bounds__(kTabThreads) kv_tables_kernel(const TabArgs a) {
    extern __shared__ int2 staged_s[];
    __shared__ int64_t tok_end[kTabThreads], blk_end[kTabThreads];  // sums up to and with each thread
    __shared__ int64_t warp_tok[32], warp_blk[32];
    __shared__ unsigned long long taken, refused;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int k_log = 0;
    while (((int64_t)kTabThreads << k_log) < a.n_req) ++k_log;
    const int64_t k = (int64_t)1 << k_log;
    const int64_t r0 = min((int64_t)a.n_req, tid * k), r1 = min((int64_t)a.n_req, r0 + k);
    if (tid == 0) taken = refused = 0;
    const int2* staged = a.n_req <= kTabStaged ? staged_s : nullptr;
    if (staged) {
        for (int r = tid; r < a.n_req; r += kTabThreads) staged_s[r + (r >> k_log)] = make_int2(a.cached[r], a.fresh[r]);
        __syncthreads();
    }
    int64_t tok = 0, blk = 0;
    for (int64_t r = r0; r < r1; ++r) {
        const TabRequest q = tab_request(a, staged, k_log, r);
        tok += q.fresh;
        blk += q.need;
    }
    const int64_t my_tok = tok, my_blk = blk;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, tok, d), b = __shfl_up_sync(0xffffffffu, blk, d);
        if (lane >= d) {
            tok += t;
            blk += b;
        }
    }
    if (lane == 31) {
        warp_tok[warp] = tok;
        warp_blk[warp] = blk;
    }
    __syncthreads();
    if (warp == 0) {
        int64_t t = warp_tok[lane], b = warp_blk[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t tu = __shfl_up_sync(0xffffffffu, t, d), bu = __shfl_up_sync(0xffffffffu, b, d);
            if (lane >= d) {
                t += tu;
                b += bu;
            }
        }
        warp_tok[lane] = t;
        warp_blk[lane] = b;
    }
    __syncthreads();
    if (warp > 0) {
        tok += warp_tok[warp - 1];
        blk += warp_blk[warp - 1];
    }
    tok_end[tid] = tok;
    blk_end[tid] = blk;
    __syncthreads();

    // Per-request outputs, each thread's requests by one block of the grid, and the counts by the first.
    const int64_t total_tok = warp_tok[31];
    const bool mine = blockIdx.x == (int64_t)tid * gridDim.x / kTabThreads;
    int64_t my_got = 0, my_lost = 0;
    if (mine || blockIdx.x == 0) {
        int64_t t = tok - my_tok, b = blk - my_blk, got = 0, lost = 0;
        for (int64_t r = r0; r < r1; ++r) {
            const TabRequest q = tab_request(a, staged, k_log, r);
            const bool fits = !q.bad && (q.need == 0 || b + q.need <= a.n_free);
            if (mine) {
                a.query_start[r] = (int32_t)t;
                a.kv_len[r] = fits ? q.cached + q.fresh : 0;
                if (q.bad) atomicOr(a.err, SCOOT_DEVERR_INDEX);
            }
            got += fits ? q.need : 0;
            lost += !fits;
            t += q.fresh;
            b += q.need;
        }
        my_got = got;
        my_lost = lost;
    }
    if (blockIdx.x == 0) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            my_got += __shfl_xor_sync(0xffffffffu, my_got, d);
            my_lost += __shfl_xor_sync(0xffffffffu, my_lost, d);
        }
        if (lane == 0) {
            atomicAdd(&taken, (unsigned long long)my_got);
            atomicAdd(&refused, (unsigned long long)my_lost);
        }
        __syncthreads();
        if (tid == 0) {
            a.counts[0] = (int32_t)taken;
            a.counts[1] = (int32_t)refused;
            a.query_start[a.n_req] = (int32_t)total_tok;
            if (total_tok > a.n_tokens) atomicOr(a.err, SCOOT_DEVERR_INDEX);
        }
    }

    // Tokens.
    const int64_t mask = (1 << a.bs_log) - 1;
    for (int64_t t = (int64_t)blockIdx.x * kTabThreads + tid; t < a.n_tokens; t += (int64_t)gridDim.x * kTabThreads) {
        int64_t slot = -1;
        int32_t pos = 0;
        if (t < total_tok) {
            int lo = 0, hi = kTabThreads - 1;  // the first thread whose sum passes t
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (tok_end[mid] > t) hi = mid;
                else lo = mid + 1;
            }
            int64_t start = lo ? tok_end[lo - 1] : 0, base = lo ? blk_end[lo - 1] : 0;
            int64_t r = lo * k;
            TabRequest q = tab_request(a, staged, k_log, r);
            while (start + q.fresh <= t) {
                start += q.fresh;
                base += q.need;
                q = tab_request(a, staged, k_log, ++r);
            }
            const int64_t p = q.cached + (t - start);
            const bool fits = !q.bad && (q.need == 0 || base + q.need <= a.n_free);
            pos = (int32_t)max(p, (int64_t)0);
            if (fits) {
                const int64_t j = p >> a.bs_log;
                int32_t* entry = a.table + r * a.ld_table + j;
                const int32_t id = j < q.held ? *entry : a.free_blocks[base + j - q.held];
                if (id < 0 || id >= a.n_blocks) atomicOr(a.err, SCOOT_DEVERR_INDEX);
                else slot = ((int64_t)id << a.bs_log) + (p & mask);
                if (j >= q.held && (p & mask) == 0) *entry = id;
            }
        }
        a.slot[t] = slot;
        a.position[t] = pos;
    }
}

// A block takes kAppend consecutive 16-byte pieces of the tokens' keys, and the same of their values; a thread two of
// them, 256 apart, with all its loads under way before the first store.  Bound by HBM: 134 MB of keys and as much of values,
// read and written (537 MB), in 82 us.  (A piece per thread with its token by a 64-bit division: 88 us.)
constexpr int kAppendThreads = 256, kAppendPer = 2, kAppend = kAppendThreads * kAppendPer;

__global__ void __launch_bounds__(kAppendThreads)
kv_append_kernel(const scoot_kv_layout L, int bs_log, const uint4* __restrict__ k, int64_t k_ld_token, int64_t k_ld_head,
                 const uint4* __restrict__ v, int64_t v_ld_token, int64_t v_ld_head, const int64_t* __restrict__ slot,
                 int64_t n_tokens, uint4* __restrict__ k_cache, uint4* __restrict__ v_cache, uint32_t* err) {
    const int head_log = L.head_dim == 128 ? 4 : 3;
    const uint32_t per_token = (uint32_t)L.n_kv_heads << head_log;
    const int64_t n_slots = L.n_blocks << bs_log;
    const int64_t first = (int64_t)blockIdx.x * kAppend, t0 = first / per_token;
    const uint32_t r0 = (uint32_t)(first - t0 * per_token);
    uint4 kk[kAppendPer], vv[kAppendPer];
    int64_t at[kAppendPer];
#pragma unroll
    for (int i = 0; i < kAppendPer; ++i) {
        const uint32_t e = r0 + threadIdx.x + i * kAppendThreads, dt = e / per_token, c = e - dt * per_token;
        const int64_t t = t0 + dt;
        const int head = (int)(c >> head_log), w = (int)(c & ((1u << head_log) - 1u));
        at[i] = -1;
        if (t >= n_tokens) continue;
        const int64_t s = slot[t];
        if (s >= n_slots) atomicOr(err, SCOOT_DEVERR_INDEX);
        if (s < 0 || s >= n_slots) continue;
        at[i] = ((s >> bs_log) * L.ld_block + (s & ((1 << bs_log) - 1)) * L.ld_token + head * L.ld_head) / 8 + w;
        kk[i] = __ldcs(k + (t * k_ld_token + head * k_ld_head) / 8 + w);
        vv[i] = __ldcs(v + (t * v_ld_token + head * v_ld_head) / 8 + w);
    }
#pragma unroll
    for (int i = 0; i < kAppendPer; ++i)
        if (at[i] >= 0) {
            k_cache[at[i]] = kk[i];
            v_cache[at[i]] = vv[i];
        }
}

int log2_block(int32_t bs) {
    int l = 0;
    while ((1 << l) < bs) ++l;
    return l;
}

scoot_status check_block_size(scoot_ctx* ctx, int32_t bs, int64_t n_blocks) {
    if (bs < 8 || bs > 256 || (bs & (bs - 1)))
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "block_size = %d is not a power of two from 8 to 256", bs);
    if (n_blocks < 1 || n_blocks > 0x7FFFFFFFll)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_blocks = %lld outside 1..2^31-1", (long long)n_blocks);
    return SCOOT_OK;
}

}  // namespace

int32_t scoot_sms(scoot_ctx* ctx) {
    if (!ctx->sms && (cudaDeviceGetAttribute(&ctx->sms, cudaDevAttrMultiProcessorCount, ctx->device) != cudaSuccess || ctx->sms < 1)) {
        cudaGetLastError();
        ctx->sms = 1;
    }
    return ctx->sms;
}

scoot_status scoot_check_heads(scoot_ctx* ctx, const char* name, const void* p, int64_t ld_token, int64_t ld_head,
                               int32_t head_dim) {
    if (!p) return scoot_fail(ctx, SCOOT_EINVAL, "%s is NULL", name);
    if (!scoot_aligned16(p)) return scoot_fail(ctx, SCOOT_EINVAL, "%s is not 16-byte aligned", name);
    const int64_t most = int64_t(1) << 38;  // 2^39 bytes
    if (ld_token < head_dim || ld_head < head_dim || (ld_token & 7) || (ld_head & 7) || ld_token > most || ld_head > most)
        return scoot_fail(ctx, SCOOT_EINVAL, "%s: strides %lld (token) and %lld (head) must be multiples of 8 from %d to 2^38",
                          name, (long long)ld_token, (long long)ld_head, head_dim);
    return SCOOT_OK;
}

scoot_status scoot_check_kv(scoot_ctx* ctx, const scoot_kv_layout* L, const void* k_cache, const void* v_cache) {
    if (!L) return scoot_fail(ctx, SCOOT_EINVAL, "layout is NULL");
    if (L->dtype != SCOOT_F16 && L->dtype != SCOOT_BF16)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "dtype = %d is neither SCOOT_F16 nor SCOOT_BF16", L->dtype);
    if (L->head_dim != 64 && L->head_dim != 128)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "head_dim = %d is neither 64 nor 128", L->head_dim);
    if (L->n_kv_heads < 1 || L->n_kv_heads > 65535)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_kv_heads = %d outside 1..65535", L->n_kv_heads);
    scoot_status s = check_block_size(ctx, L->block_size, L->n_blocks);
    if (s != SCOOT_OK) return s;
    s = scoot_check_heads(ctx, "k_cache", k_cache, L->ld_token, L->ld_head, L->head_dim);
    if (s != SCOOT_OK) return s;
    s = scoot_check_heads(ctx, "v_cache", v_cache, L->ld_token, L->ld_head, L->head_dim);
    if (s != SCOOT_OK) return s;
    return scoot_check_heads(ctx, "cache blocks", k_cache, L->ld_block, L->ld_head, L->head_dim);
}

extern "C" {

scoot_status scoot_kv_tables(scoot_ctx* ctx, const int32_t* cached_len, const int32_t* new_len, int32_t n_req,
                             int32_t block_size, int64_t n_blocks, int32_t* block_table, int64_t ld_table,
                             const int32_t* free_blocks, int64_t n_free, int32_t* query_start, int32_t* kv_len,
                             int64_t* slot, int32_t* position, int64_t n_tokens, int32_t* counts, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if ((s = check_block_size(ctx, block_size, n_blocks)) != SCOOT_OK) return s;
    if (n_req < 0 || n_tokens < 0 || n_tokens > 0x7FFFFFFFll || n_free < 0 || ld_table < 0 || ld_table > 0x7FFFFFFFll)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_req = %d, n_tokens = %lld, n_free = %lld or ld_table = %lld out of range", n_req,
                          (long long)n_tokens, (long long)n_free, (long long)ld_table);
    if (!query_start || !counts || (n_tokens && (!slot || !position)) || (n_free && !free_blocks) ||
        (n_req && (!cached_len || !new_len || !kv_len || (ld_table && !block_table))))
        return scoot_fail(ctx, SCOOT_EINVAL, "an array is NULL");
    TabArgs a;
    a.cached = cached_len;
    a.fresh = new_len;
    a.n_req = n_req;
    a.bs_log = log2_block(block_size);
    a.longest = std::min<int64_t>(ld_table << a.bs_log, 0x7FFFFFFFll);
    a.n_blocks = n_blocks;
    a.table = block_table;
    a.ld_table = ld_table;
    a.free_blocks = free_blocks;
    a.n_free = n_free;
    a.query_start = query_start;
    a.kv_len = kv_len;
    a.slot = slot;
    a.position = position;
    a.n_tokens = n_tokens;
    a.counts = counts;
    a.err = ctx->d_err;
    int64_t blocks = (n_tokens + kTabThreads - 1) / kTabThreads;
    if (blocks > scoot_sms(ctx)) blocks = scoot_sms(ctx);
    if (blocks < 1) blocks = 1;
    const size_t smem = n_req <= kTabStaged ? (size_t)(n_req + std::min(n_req, kTabThreads)) * sizeof(int2) : 0;
    if (!(ctx->smem_set & kTabSmemBit)) {  // once per context, whatever this call's size: the static part counts as well
        SCOOT_CUDA(ctx, cudaFuncSetAttribute(kv_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                             (int)((kTabStaged + kTabThreads) * sizeof(int2))));
        ctx->smem_set |= kTabSmemBit;
    }
    kv_tables_kernel<<<(unsigned)blocks, kTabThreads, smem, static_cast<cudaStream_t>(stream)>>>(a);
    SCOOT_LAUNCHED(ctx);
    return SCOOT_OK;
}

scoot_status scoot_kv_append(scoot_ctx* ctx, const scoot_kv_layout* layout, const void* k, int64_t k_ld_token,
                             int64_t k_ld_head, const void* v, int64_t v_ld_token, int64_t v_ld_head,
                             const int64_t* slot, int64_t n_tokens, void* k_cache, void* v_cache, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if ((s = scoot_check_kv(ctx, layout, k_cache, v_cache)) != SCOOT_OK) return s;
    if (n_tokens < 0 || n_tokens > 0x7FFFFFFFll)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_tokens = %lld outside 0..2^31-1", (long long)n_tokens);
    if (n_tokens == 0) return SCOOT_OK;
    s = scoot_check_heads(ctx, "k", k, k_ld_token, k_ld_head, layout->head_dim);
    if (s != SCOOT_OK) return s;
    s = scoot_check_heads(ctx, "v", v, v_ld_token, v_ld_head, layout->head_dim);
    if (s != SCOOT_OK) return s;
    if (!slot) return scoot_fail(ctx, SCOOT_EINVAL, "slot is NULL");
    const int64_t total = n_tokens * layout->n_kv_heads * (layout->head_dim / 8), blocks = (total + kAppend - 1) / kAppend;
    if (blocks > 0x7FFFFFFFll) return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "%lld tokens are too many for one call", (long long)n_tokens);
    kv_append_kernel<<<(unsigned)blocks, kAppendThreads, 0, static_cast<cudaStream_t>(stream)>>>(
        *layout, log2_block(layout->block_size), static_cast<const uint4*>(k), k_ld_token, k_ld_head,
        static_cast<const uint4*>(v), v_ld_token, v_ld_head, slot, n_tokens, static_cast<uint4*>(k_cache),
        static_cast<uint4*>(v_cache), ctx->d_err);
    SCOOT_LAUNCHED(ctx);
    return SCOOT_OK;
}

}  // extern "C"
