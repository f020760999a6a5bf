// Attention of a batch of new tokens over a paged key-value cache of 8-bit floats, a scale per block of tokens and head.
//
//   out_t = sum_i softmax_i(scale s_b(i) q_t . k_i) s'_b(i) v_i,   lse_t = ln sum_i exp(scale s_b(i) q_t . k_i)
//
// over the keys i that token t sees; k_i, v_i are codes, s_b and s'_b their blocks' scales.
//
// This kernel serves requests of few rows (a row is a token's query head; single tokens above all), which bytes bound: a
// warp is a worker of its own, with 8 or 16 rows against tiles of 32 keys (64 with heads of 64).  Codes become fp16, which
// holds all of them, on their way from shared memory into the operands of the tensor cores (mma.m16n8k16: the tcgen05 forms
// take 64 or 128 rows, and their operands would have to be written back to shared memory).  Keys, and values by dimensions, are
// the products' first operand, sixteen at a time, and the rows the second, eight at a time: with rows as the first a group
// of four heads left twelve of sixteen empty.  Queries become fp16 as well, bf16 ones divided by a power of two of their row
// so that the largest is below 2^15: what that rounds is below 2^-39 of the row's largest.
//
// Dimensions and keys are dealt to the operands' places as the loads want them.  Q K^T: lane (g, c) = (lane / 4, lane % 4) has
// of sixteen keys g and g + 8, and of each D / 4 dimensions in a row, four per step, and the same ones of row g.  The result's
// transpose (movmatrix) is P as the second operand.  P V: rows g and g + 8 of product t are dimensions g D / 8 + 2 t and
// the next, so that a lane reads whole pieces of four keys' values, and has D / 8 consecutive dimensions of two rows' results.
//
// Running maximum m and sum l as elsewhere: p = 2^(c s - m), and O is rescaled only where a maximum has grown by more than 2^8.
// The values' scales go into the probabilities: fp16 of p s'_b / r * 2^7, r the largest scale of values that the row has seen so
// far, which stays below 2^15 (2^15 129 / 128 where r is let be) and rounds what is below 2^-21 of r with an error of 2^-32 r at
// most; O is in units of r 2^-7.  r is each row's own: a tile's values may be hidden from some.
//
// Work: items (request, key-value head, rows) in a row, each costing its tiles and a constant, are cut into equal ranges for as
// many teams as the work is worth, the same number on each multiprocessor (a cut close to an item's start or end moves
// there).  A team is a warp, or `share` warps for the same tokens of as many heads.  A warp copies its tiles, page by page
// by TMA and their scales beside them, into a ring of its own, ahead across items; where its next item lies is kept in
// shared memory, out of the registers of the loop over tiles.  An item that lies in several ranges leaves its parts (O, m, l)
// in the workspace.  Of few parts the warp that comes last joins them.  Of many, the block joins its own at its end, and the
// last of an item's blocks joins the blocks', in the ranges' order: results do not depend on who was last.
//
// What bounds it, as measured per call in a captured graph, on tensors in use one after the other:
//   * 256 sequences of 64 to 2560 tokens, 32 heads over 8 of 128, one new token each, bf16: 118 to 123 us, 5.6 to 5.9 TB/s, 83
//     to 87% of the copy rate.  A warp takes 3000 cycles for a tile of 8 KB with eleven others beside it, which is DRAM's rate; costs
//     and ranges (2.5 us), the first tiles, and the ends of items (queries, parts, counters) are the rest.
//   * three sequences of 20,000 to 65,535, 28 heads over 4, fp16: 44 to 47 us, 3.2 TB/s: as much again for the first tile and the joins
//     of parts within and across blocks (7 us) as for the keys and values.
//   * one token over 777: 15.4 to 16.1 us (over a 16-bit cache 14.0 to 14.5): a chain of latencies, two thirds of it before the first
//     product.
//   * 128 sequences of 1500 with 4 new tokens each: 95 to 98 us, products of sixteen rows.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "mbarrier.cuh"
#include "paged_attn8.cuh"

namespace {

// An item's start and end, in tiles.  With 2 and with 4, in turn on one device: 256 sequences to 2560 tokens 122 us both, one of 4000
// 18.2 and 16.4, 128 of 500 39.8 and 37.1, of 1500 79.6 and 82.6, three of 40,000 41.7 and 40.3.
constexpr int kItemCost = 4;
constexpr int kMinRange = 2;    // cost that a warp takes at least (a token over 777 keys, 8 heads: 15.6 us, with 3 16.1)
constexpr int kSnap = 2;        // a cut this close to the start or end of an item's tiles moves there
constexpr int kMaxBlocks = 256;
constexpr int kShare = 4;       // warps that take as many heads' keys of the same tokens at a time, at most
// Counters, apart: two per block of the tiles kernel, one per warp of this, kShare per block of this.
constexpr int kWarpCounts = 2 * kMaxBlocks, kBlockCounts = kWarpCounts + 12 * kMaxBlocks;
static_assert(kBlockCounts + kShare * kMaxBlocks <= (int)SCOOT_COUNTS, "counters");
constexpr int kFewParts = 16;   // parts that the warp that comes last joins by itself
constexpr int kItems = 8;       // items of a warp between its copies and their attention
// Requests of up to so many items per head are this kernel's.  Each item reads the keys again, mostly from DRAM; the tiles kernel
// reads them once, but makes tiles for 128 rows.  128 sequences of 1500 keys, 32 heads of 128, each kernel made to take them: over 8
// heads of keys, items of eight rows, 79 us with one (a token), 140 with two, 234 with three and 293 with four, of sixteen rows
// 95 and 180, the tiles kernel 232 to 242 whatever the rows; over 2 heads, items of sixteen, 42 and 66 against 67 and 69; 16 heads
// over one 35 and 49 against 32 and 34.
constexpr int kFewItems = 2;
constexpr float kMaxScale = 2.3e38f;  // times log2 e it is still finite
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;

template <int D, int NT>
struct Shape {
    static constexpr int kRows = 8 * NT;                 // of an item: the products' N
    static constexpr int kWarps = NT == 1 ? 12 : 8, kThreads = 32 * kWarps;  // as many as have the registers
    static constexpr int kKeys = D == 128 ? 32 : 64;     // of a tile
    static constexpr int kTile = kKeys * D;              // bytes of a tile's keys, or values
    static constexpr int kStage = 2 * kTile;
    static constexpr int kStages = NT == 1 ? 2 : 3;
    static constexpr int kScales = kWarps * kStages * kStage;     // after the warps' rings those of their tiles' scales
    static constexpr int kScale = kKeys;                 // bytes of them: groups of eight keys, and of values
    static constexpr int kSmem = kScales + kWarps * kStages * kScale;
    static constexpr int kPart = kRows * (D + 2);        // floats of a part: O, then (m, l) of each row
};

// Boxes of up to 32 tokens of a block and head.
struct KvMaps {
    CUtensorMap k, v;
};

struct Item {
    int32_t r, h;          // request, key-value head
    int32_t tok, head;     // first token (of the batch), first query head
    int32_t rows;          // row = token * group + head
    int32_t pos, kv;       // position of the first token, length of the sequence
    int32_t begin, end;    // keys that some row sees
    int32_t u0, u1;        // this part's tiles
    int32_t first, n_parts;  // team of the first part, and how many parts
};

__device__ __forceinline__ float exp2_hw(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.0f : m; }
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.0f ? 0.0f : __fdividef(1.0f, l); }

// 128 / x of a scale, infinite for zero.  (In quarters: __fdividef takes divisors up to 2^126.)
__device__ __forceinline__ float unit_of(float x) { return __fdividef(32.0f, 0.25f * x); }

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (!kBf16) return half2_bits(lo, hi);
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Two codes of a word as fp16 (exact).
__device__ __forceinline__ uint32_t decode_lo(uint32_t w) {
    uint32_t r;
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ uint32_t decode_hi(uint32_t w) { return decode_lo(w >> 16); }
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// The codes that the format reserves for NaN as 448.
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
    const uint32_t nan = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
    return w & ~(nan >> 7);
}
__device__ __forceinline__ void mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void copy4(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(there ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void lds(uint32_t addr, uint32_t* w) {
    if (N == 4) asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(addr));
    else asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(addr));
}

// Where piece j (16 bytes) of key `row` of a tile lies (the copies' swizzle of 128 or 64 bytes).
template <int D>
__device__ __forceinline__ uint32_t piece_at(int row, int j) {
    return D == 128 ? row * 128 + ((j ^ (row & 7)) << 4) : row * 64 + ((j ^ ((row >> 1) & 3)) << 4);
}

struct Req {
    int32_t q0, n, kv;
};
// One request's lengths, empty if they are bad.
__device__ __forceinline__ Req load_req(const Attn8Args& a, int r, bool flag) {
    Req q{0, 0, 0};
    if (r >= a.n_req) return q;
    const int q0 = a.query_start[r], q1 = a.query_start[r + 1], kv = a.kv_len[r];
    if (q0 < 0 || q1 < q0 || q1 > a.n_tokens || kv < 0 || kv > a.ld_table << a.bs_log || (a.max_new > 0 && q1 - q0 > a.max_new)) {
        if (flag) atomicOr(a.err, SCOOT_DEVERR_INDEX);
        return q;
    }
    if (q1 - q0 > a.few) return q;
    q.q0 = q0;
    q.n = q1 - q0;
    q.kv = kv;
    return q;
}

__device__ __forceinline__ int item_count(const Attn8Args& a, int n) { return (n + a.toks - 1) / a.toks; }
// The keys [begin, end) that some row of item j sees.
__device__ __forceinline__ void seen_keys(const Attn8Args& a, int kv, int n, int j, int& begin, int& end) {
    const int tok = j * a.toks, nt = min(a.toks, n - tok);
    const int64_t p0 = (int64_t)kv - n + tok;
    end = a.causal ? (int)min((int64_t)kv, p0 + nt) : kv;
    begin = a.window > 0 ? (int)max((int64_t)0, p0 + 1 - a.window) : 0;
    if (end <= begin) begin = end = 0;
}
template <int kKeys>
__device__ __forceinline__ int item_cost(const Attn8Args& a, int kv, int n, int j) {
    int begin, end;
    seen_keys(a, kv, n, j, begin, end);
    return kItemCost + (end + kKeys - 1) / kKeys - begin / kKeys;
}
// The cost of a head's items of a request, by the whole warp.
template <int kKeys>
__device__ __forceinline__ int64_t head_cost(const Attn8Args& a, int kv, int n) {
    const int m = item_count(a, n);
    int64_t c = 0;
    for (int j = threadIdx.x & 31; j < m; j += 32) c += item_cost<kKeys>(a, kv, n, j);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) c += __shfl_xor_sync(0xffffffffu, c, d);
    return c;
}

__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

__device__ __forceinline__ uint16_t* out_row(const Attn8Args& a, const Item& it, int q) {
    const int t = q / a.group;
    return a.out + (int64_t)(it.tok + t) * a.out_ld_token + (int64_t)(it.head + q - t * a.group) * a.out_ld_head;
}
__device__ __forceinline__ float* lse_row(const Attn8Args& a, const Item& it, int q) {
    const int t = q / a.group;
    return a.lse + (int64_t)(it.tok + t) * a.n_heads + it.head + q - t * a.group;
}

// n parts of an item, of which `first` is the first: the others lie `step` floats apart from `second` on.
struct Parts {
    const float *first, *second;
    int64_t step;
    int32_t n;
    __device__ __forceinline__ const float* at(int i) const { return i == 0 ? first : second + (i - 1) * step; }
};

// Parts joined, T tasks of a thread at once with P parts of each in flight.  Task e < total is four columns of a row of one of
// `count` items; source(i, to) gives item i's parts, and where its rows go if they are parts again (else to the outputs).
template <bool kBf16, int D, int kRows, int kThreads, int T, int P, typename F>
__device__ __forceinline__ void join(const Attn8Args& a, const Item* items, int count, int total, int me, F&& source) {
    constexpr int kQuads = D / 4;
#pragma unroll 1
    for (int e0 = me; e0 < total; e0 += T * kThreads) {
        Parts parts[T];
        float* to[T];
        int at[T], row[T], most = 0;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const int e = e0 + t * kThreads;
            int q = e / kQuads, i = 0;
            while (i < count && q >= (items[i].n_parts ? items[i].rows : 0)) q -= items[i].n_parts ? items[i].rows : 0, ++i;
            at[t] = i;
            row[t] = q;
            to[t] = nullptr;
            parts[t].n = 0;
            if (i < count) parts[t] = source(i, to[t]);
            most = max(most, parts[t].n);
        }
        const int c = me % kQuads;  // (of all tasks: kThreads is a multiple)
        float M[T], L[T];
        float4 o[T];
#pragma unroll
        for (int t = 0; t < T; ++t) {
            M[t] = -INFINITY;
            L[t] = 0.0f;
            o[t] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll 1
        for (int i0 = 0; i0 < most; i0 += P) {
            float2 ml[T][P];
            float4 v[T][P];
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    ml[t][i] = make_float2(-INFINITY, 0.0f);
                    v[t][i] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (i0 + i < parts[t].n) {
                        const float* p = parts[t].at(i0 + i);
                        ml[t][i] = __ldcg(reinterpret_cast<const float2*>(p + kRows * D) + row[t]);
                        v[t][i] = __ldcg(reinterpret_cast<const float4*>(p + row[t] * D) + c);
                    }
                }
#pragma unroll
            for (int t = 0; t < T; ++t) {
                float Mn = M[t];
#pragma unroll
                for (int i = 0; i < P; ++i) Mn = fmaxf(Mn, ml[t][i].x);
                const float Ms = finite_or_zero(Mn), f = exp2_hw(M[t] - Ms);
                L[t] *= f;
                o[t] = make_float4(o[t].x * f, o[t].y * f, o[t].z * f, o[t].w * f);
                M[t] = Mn;
#pragma unroll
                for (int i = 0; i < P; ++i) {
                    const float w = exp2_hw(ml[t][i].x - Ms);
                    L[t] = fmaf(w, ml[t][i].y, L[t]);
                    o[t] = make_float4(fmaf(w, v[t][i].x, o[t].x), fmaf(w, v[t][i].y, o[t].y), fmaf(w, v[t][i].z, o[t].z), fmaf(w, v[t][i].w, o[t].w));
                }
            }
        }
#pragma unroll
        for (int t = 0; t < T; ++t) {
            if (parts[t].n == 0) continue;
            if (to[t]) {
                reinterpret_cast<float4*>(to[t] + row[t] * D)[c] = o[t];
                if (c == 0) reinterpret_cast<float2*>(to[t] + kRows * D)[row[t]] = make_float2(M[t], L[t]);
            } else {
                const Item& it = items[at[t]];
                const float inv = inverse_sum(L[t]);
                *reinterpret_cast<uint2*>(out_row(a, it, row[t]) + 4 * c) =
                    make_uint2(pack16<kBf16>(o[t].x * inv, o[t].y * inv), pack16<kBf16>(o[t].z * inv, o[t].w * inv));
                if (c == 0 && a.lse) *lse_row(a, it, row[t]) = L[t] == 0.0f ? -INFINITY : (M[t] + __log2f(L[t])) * kLn2;
            }
        }
    }
}

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// Where a warp is among the items of its range, in shared memory: what is done per item stays out of the registers of what is
// done per tile.
struct Cursor {
    int64_t at, begin, end, range;  // start of the next item; the range; its length
    int32_t r, h, j, team;          // the next item: request, heads, which of the heads'
    int32_t member;                 // the head is h share + member
    Req req;                        // r's lengths
};

// The ids of 32 blocks of an item's request in the lanes; INT32_MIN for those that no row sees any of, and for no other: negative
// ids are -1.
__device__ __forceinline__ int fetch_ids(const Attn8Args& a, const Item& it, int group) {
    const int block = group * 32 + (threadIdx.x & 31);
    const int64_t key = (int64_t)block << a.bs_log;
    return key < it.end && key + (1 << a.bs_log) > it.begin ? max(__ldg(a.table + (int64_t)it.r * a.ld_table + block), -1) : INT32_MIN;
}

// A range's next item with keys goes to *to; false if there is none.  reqs: the requests' lengths, or NULL where they are many.  Those without keys get their zeros here.  By a warp.
template <int D, int kKeys>
__device__ __noinline__ bool next_item(const Attn8Args& a, Cursor* cur, Item* to, const Req* reqs) {
    const int lane = threadIdx.x & 31;
    Cursor c = *cur;
    bool found = false;
    while (c.at < c.end) {
        if (c.j >= item_count(a, c.req.n)) {  // the next head, or the next request with a token
            c.j = 0;
            if (c.req.n > 0 && ++c.h < a.n_kv_heads / a.share) continue;
            c.h = 0;
            for (++c.r; c.r < a.n_req;) {
                const Req q = !reqs ? load_req(a, c.r + lane, false) : c.r + lane < a.n_req ? reqs[c.r + lane] : Req{0, 0, 0};
                const uint32_t some = __ballot_sync(0xffffffffu, q.n > 0);
                if (some) {
                    const int src = __ffs(some) - 1;
                    c.r += src;
                    c.req = Req{__shfl_sync(0xffffffffu, q.q0, src), __shfl_sync(0xffffffffu, q.n, src), __shfl_sync(0xffffffffu, q.kv, src)};
                    break;
                }
                c.r += 32;
            }
            if (c.r >= a.n_req) {
                c.at = c.end;
                break;
            }
        }
        Item it;
        it.r = c.r;
        it.h = c.h * a.share + c.member;
        const int tok = c.j * a.toks;
        it.rows = min(a.toks, c.req.n - tok) * a.group;
        it.tok = c.req.q0 + tok;
        it.head = it.h * a.group;
        it.pos = c.req.kv - c.req.n + tok;
        it.kv = c.req.kv;
        seen_keys(a, c.req.kv, c.req.n, c.j, it.begin, it.end);
        const int tile0 = it.begin / kKeys, units = (it.end + kKeys - 1) / kKeys - tile0;
        const int64_t start = c.at, s0 = start + kItemCost;  // where its tiles start
        auto cut = [&](int64_t b) { return b >= s0 + units ? units : b - s0 < kSnap ? 0 : s0 + units - b < kSnap ? units : (int)(b - s0); };
        const int lo = cut(c.begin), hi = cut(c.end);
        c.at = s0 + units;
        ++c.j;
        if (units == 0 && start >= c.begin) {
            for (int e = lane; e < it.rows * (D / 8); e += 32)
                *reinterpret_cast<uint4*>(out_row(a, it, e / (D / 8)) + 8 * (e % (D / 8))) = make_uint4(0, 0, 0, 0);
            if (a.lse)
                for (int q = lane; q < it.rows; q += 32) *lse_row(a, it, q) = -INFINITY;
        }
        if (hi <= lo) continue;
        it.first = c.team;
        it.n_parts = 1;
        if (hi - lo < units) {
            it.first = (int)quotient(s0 + kSnap - 1, c.range);
            it.n_parts = (int)quotient(s0 + units - kSnap, c.range) - it.first + 1;
        }
        it.u0 = tile0 + lo;
        it.u1 = tile0 + hi;
        if (lane == 0) *to = it;
        // queries on their way to the L2 cache
        for (int e = lane; e < it.rows * (D / 64); e += 32) {
            const int q = e / (D / 64), t = q / a.group;
            asm volatile("prefetch.global.L2 [%0];" ::"l"(a.q + (int64_t)(it.tok + t) * a.q_ld_token + (int64_t)(it.head + q - t * a.group) * a.q_ld_head +
                                                          e % (D / 64) * 64));
        }
        found = true;
        break;
    }
    __syncwarp();
    if (lane == 0) *cur = c;
    __syncwarp();
    return found;
}

template <bool kBf16, int D, int NT>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) attn8_rows_kernel(const __grid_constant__ Attn8Args a, const __grid_constant__ KvMaps maps) {
    using Sh = Shape<D, NT>;
    constexpr int kRows = Sh::kRows, kWarps = Sh::kWarps, kThreads = Sh::kThreads, kKeys = Sh::kKeys, kM = kKeys / 16, kG = kKeys / 8, kSteps = D / 16, kDims = D / 16;  // steps of Q K^T; sixteens of dimensions of O
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int64_t cost_s[kThreads];
    __shared__ Item items[kShare + kWarps];  // of the block's items of many parts: those that came in, and one that begins with each warp's last
    __shared__ Item queue_s[kWarps][kItems];
    __shared__ Item ends_s[kWarps][2];  // of a range's two split items, those of few parts
    __shared__ Cursor cursor_s[kWarps];
    __shared__ Attn8Args args_s;       // for next_item: a call reads the parameters' own memory slowly
    __shared__ Req req_s[kThreads];    // with at most kThreads requests: theirs
    __shared__ int last_s[kShare + kWarps], failed, many;
    __shared__ __align__(8) uint64_t bars[kWarps * Sh::kStages];
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int g = lane >> 2, c = lane & 3;

    // The cost of all items: each thread k consecutive requests, then a scan.
    const int k = (a.n_req + kThreads - 1) / kThreads;
    if (tid < kShare + kWarps) items[tid].n_parts = 0;
    if (tid < 2 * kWarps) ends_s[tid / 2][tid % 2].n_parts = 0;
    if (tid == 0) failed = many = 0;
    if (tid < 2) asm volatile("prefetch.tensormap [%0];" ::"l"(tid ? &maps.v : &maps.k) : "memory");
    for (int i = tid; i < (int)(sizeof(Attn8Args) / 4); i += kThreads) reinterpret_cast<uint32_t*>(&args_s)[i] = reinterpret_cast<const uint32_t*>(&a)[i];
    if (tid < kWarps * Sh::kStages) scoot_dev::mbar_init(&bars[tid], 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    int64_t mine = 0;
#pragma unroll 1
    for (int i = 0; i < k; ++i) {
        const Req q = load_req(a, tid * k + i, blockIdx.x == 0);
        if (k == 1) req_s[tid] = q;
        const bool one = item_count(a, q.n) == 1;
        if (one) mine += item_cost<kKeys>(a, q.kv, q.n, 0);
        uint32_t big = __ballot_sync(0xffffffffu, q.n > 0 && !one);
        while (big) {
            const int src = __ffs(big) - 1;
            big &= big - 1;
            const int64_t cost = head_cost<kKeys>(a, __shfl_sync(0xffffffffu, q.kv, src), __shfl_sync(0xffffffffu, q.n, src));
            if (lane == src) mine += cost;
        }
    }
    const int heads = a.n_kv_heads / a.share;
    mine *= heads;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, mine, d);
        if (lane >= d) mine += t;
    }
    cost_s[tid] = mine;  // up to and with this thread, of its warp
    __syncthreads();
    int64_t upto = lane < kWarps ? cost_s[lane * 32 + 31] : 0;
#pragma unroll
    for (int d = 1; d < kWarps; d <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += t;
    }
    const int64_t total = __shfl_sync(0xffffffffu, upto, kWarps - 1);
    const int n_workers = gridDim.x * kWarps, n_teams = n_workers / a.share;
    // The kernel of the requests of more rows may begin on each multiprocessor that is done here (without items it begins after
    // this one, on all of them at once: taking them up one by one cost 1 % of a prefill of 619 us).
    if (total > 0) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // As many teams as the work is worth, the same number on each multiprocessor.
    const int64_t range = max(quotient(total + n_teams - 1, n_teams), (int64_t)kMinRange);
    const int teams = (int)quotient(quotient(total + range - 1, range) + gridDim.x - 1, gridDim.x);
    const int nth = warp / a.share, member = warp % a.share, team = blockIdx.x * teams + nth;
    const int64_t B0 = nth < teams ? min(total, team * range) : total, B1 = min(total, B0 + range);

    int cached = -1;  // requests 32 cached .. are in the lanes
    Req in_lane{0, 0, 0};
    auto get = [&](int r) {
        if (k == 1) return req_s[r];
        if ((r >> 5) != cached) {
            cached = r >> 5;
            in_lane = load_req(a, cached * 32 + lane, false);
        }
        return Req{__shfl_sync(0xffffffffu, in_lane.q0, r & 31), __shfl_sync(0xffffffffu, in_lane.n, r & 31),
                   __shfl_sync(0xffffffffu, in_lane.kv, r & 31)};
    };
    int r = 0, h = 0, j = 0;
    int64_t p = B0;  // where item (r, h, j) starts
    if (B0 < B1) {
        // the warp's sum that passes B0, then the thread's, then the request, its head and its item
        const int w = __ffs(__ballot_sync(0xffffffffu, lane < kWarps && upto > B0)) - 1;
        int64_t at = __shfl_sync(0xffffffffu, upto, w) - cost_s[w * 32 + 31];
        const int64_t in_warp = cost_s[w * 32 + lane];
        const int t = __ffs(__ballot_sync(0xffffffffu, at + in_warp > B0)) - 1;
        const int64_t before = __shfl_sync(0xffffffffu, in_warp, (t + 31) & 31);
        if (t > 0) at += before;
        r = (w * 32 + t) * k;
        while (r < a.n_req) {
            const Req q = get(r);
            const int64_t one = q.n == 0 ? 0 : item_count(a, q.n) == 1 ? item_cost<kKeys>(a, q.kv, q.n, 0) : head_cost<kKeys>(a, q.kv, q.n);
            if (at + one * heads > B0) {
                h = (int)quotient(B0 - at, one);
                at += h * one;
                break;
            }
            at += one * heads;
            ++r;
        }
        const Req q = get(min(r, a.n_req - 1));
        const int m = item_count(a, q.n);
        for (int j0 = 0; m > 1 && j0 < m; j0 += 32) {
            const int64_t cost = j0 + lane < m ? item_cost<kKeys>(a, q.kv, q.n, j0 + lane) : 0;
            int64_t s = cost;
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const int64_t up = __shfl_up_sync(0xffffffffu, s, d);
                if (lane >= d) s += up;
            }
            const uint32_t past = __ballot_sync(0xffffffffu, at + s > B0);
            if (past) {
                const int src = __ffs(past) - 1;
                j = j0 + src;
                at += __shfl_sync(0xffffffffu, s - cost, src);
                break;
            }
            at += __shfl_sync(0xffffffffu, s, 31);
        }
        p = at;
        if (lane == 0) cursor_s[warp] = Cursor{p, B0, B1, range, r, h, j, team, member, q};
    } else if (lane == 0) {
        cursor_s[warp] = Cursor{0, 0, 0, range, 0, 0, 0, team, member, Req{0, 0, 0}};
    }
    __syncwarp();

    const uint32_t ring = scoot_dev::smem_u32(smem) + warp * Sh::kStages * Sh::kStage;
    const uint32_t ring_scales = scoot_dev::smem_u32(smem) + Sh::kScales + warp * Sh::kStages * Sh::kScale;
    const uint32_t bar0 = scoot_dev::smem_u32(&bars[warp * Sh::kStages]);
    const bool one_lane = elect_one();
    uint32_t to_load = 0, stage = 0, phase = 0;  // places in the ring: of the next load, and of the next tile with its barrier's phase
    bool ok = true;
    bool bad_id = false, bad_scale = false;
    const int bs = 1 << a.bs_log;
    // An item's n parts from that of team t on: a warp's first buffer has the part of an item that began before it, the second that
    // of one that begins with it and goes on.
    auto parts_at = [&](int t, int begun, int who, int n) {
        return Parts{a.parts + (size_t)(2 * (t * a.share + who) + (t == begun)) * Sh::kPart, a.parts + (size_t)2 * ((t + 1) * a.share + who) * Sh::kPart,
                     (int64_t)2 * a.share * Sh::kPart, n};
    };

    // Of a split item's few parts, how many were there before the warp's.  By a lane; the warp's other lanes' stores are before it.
    auto add_one = [&](const Item& it) {
        __threadfence();
        return atomicAdd(a.warp_count + it.first * a.share + member, 1u);
    };
    uint32_t came = 0;
    uint32_t n_made = 0, n_taken = 0;  // items found, and those whose copies have begun
    int first_ids = 0;                 // ids of the first 32 blocks of the last one found, in the lanes
    auto find = [&]() {
        Item* to = &queue_s[warp][n_made % kItems];
        if (!next_item<D, kKeys>(args_s, &cursor_s[warp], to, k == 1 ? req_s : nullptr)) return;
        ++n_made;
        first_ids = fetch_ids(a, *to, (to->u0 * kKeys >> a.bs_log) >> 5);
    };

    // The next tile's copies: of keys and of values per page, and the scales of its groups of eight keys.
    int group = 0, ids = 0, ids_next = 0, load_u = 0, load_u1 = 0;
    auto use = [&](int raw) {
        const bool out = raw < 0 || raw >= a.n_blocks;
        bad_id |= out && raw != INT32_MIN;
        ids = out ? (int)a.n_blocks : raw;  // past the end: the copy reads nothing and writes zeros
    };
    auto load = [&]() {
        bool taken = false;
        if (load_u == load_u1) {
            if (n_taken == n_made) return;
            const Item& it = queue_s[warp][n_taken % kItems];
            load_u = it.u0;
            load_u1 = it.u1;
            group = (load_u * kKeys >> a.bs_log) >> 5;
            use(first_ids);
            ids_next = fetch_ids(a, it, group + 1);
            ++n_taken;
            taken = true;
        }
        const Item& it = queue_s[warp][(n_taken - 1) % kItems];
        const int key0 = load_u++ * kKeys, b0 = key0 >> a.bs_log, head = it.h;
        if (b0 >> 5 != group) {
            use(ids_next);
            group = b0 >> 5;
            ids_next = fetch_ids(a, it, group + 1);
        }
        const uint32_t bar = bar0 + 8 * to_load, dst = ring + to_load * Sh::kStage;
        if (one_lane)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)Sh::kStage) : "memory");
        auto copy = [&](int id, int within, uint32_t at) {
            if (!one_lane) return;
            asm volatile(
                "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(at),
                "l"(&maps.k), "r"(0), "r"(head), "r"(within), "r"(id), "r"(bar)
                : "memory");
            asm volatile(
                "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(at + Sh::kTile),
                "l"(&maps.v), "r"(0), "r"(head), "r"(within), "r"(id), "r"(bar)
                : "memory");
        };
        auto pages = [&](auto n) {
            constexpr int N = decltype(n)::value;
            int id[N];
#pragma unroll
            for (int i = 0; i < N; ++i) id[i] = __shfl_sync(0xffffffffu, ids, (b0 + i) & 31);
#pragma unroll
            for (int i = 0; i < N; ++i) copy(id[i], N == 1 ? key0 & (bs - 1) : 0, dst + i * (Sh::kTile / N));
        };
        if (bs >= kKeys) pages(std::integral_constant<int, 1>());
        else if (bs == 16) pages(std::integral_constant<int, kKeys / 16>());
        else if (bs == 8) pages(std::integral_constant<int, kKeys / 8>());
        else pages(std::integral_constant<int, kKeys / 32>());
        const int key = key0 + 8 * (lane & (kG - 1)), id = __shfl_sync(0xffffffffu, ids, (key >> a.bs_log) & 31);
        if (lane < 2 * kG) {
            const bool there = id < a.n_blocks && key + 8 > it.begin && key < it.end;
            copy4(ring_scales + to_load * Sh::kScale + 4 * lane, (lane < kG ? a.k_scale : a.v_scale) + (there ? (int64_t)id * a.n_kv_heads + head : 0), there);
        }
        if (++to_load == Sh::kStages) to_load = 0;
        if (taken) find();  // (after the copies, which wait for nothing of it)
    };

    find();
#pragma unroll 1
    for (int i = 0; i < Sh::kStages; ++i) {
        load();
        copies_end();
    }
    // The copies run ahead of the products by the ring's places, across items.
#pragma unroll 1
    for (uint32_t n_done = 0; n_done < n_taken && ok; ++n_done) {
        const Item& it = queue_s[warp][n_done % kItems];
        uint32_t qb[NT][kSteps][2];
        float c_row[NT][2];              // scale of a row's scores, to log2
        int k0[NT][2], k1[NT][2];        // keys that a row sees
        int all0, all1;                  // keys that all rows see
        const bool several = it.rows > a.group;  // tokens, so that some rows see keys that others do not
        bool large;                      // a product with a scale may pass fp32
        float o[NT][kDims][4], m[NT][2], l[NT][2], inv_ref[NT][2];  // O in units of 1 / inv_ref
        all0 = it.begin;
        all1 = it.end;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int row = 8 * nt + 2 * c + i, pos = it.pos + row / a.group;
                const bool live = row < it.rows;
                k1[nt][i] = live ? (a.causal ? min(it.kv, pos + 1) : it.kv) : 0;
                k0[nt][i] = live && a.window > 0 ? (int)max((int64_t)0, (int64_t)pos + 1 - a.window) : 0;
                if (live) {
                    all0 = max(all0, k0[nt][i]);
                    all1 = min(all1, k1[nt][i]);
                }
            }
            const int row = 8 * nt + g, t = row / a.group;
            const uint16_t* src = a.q + (int64_t)(it.tok + t) * a.q_ld_token + (int64_t)(it.head + row - t * a.group) * a.q_ld_head;
#pragma unroll
            for (int s = 0; s < kSteps; s += 2) {
                const uint4 x = row < it.rows ? *reinterpret_cast<const uint4*>(src + (D / 4) * c + 4 * s) : make_uint4(0, 0, 0, 0);
                qb[nt][s][0] = x.x;
                qb[nt][s][1] = x.y;
                qb[nt][s + 1][0] = x.z;
                qb[nt][s + 1][1] = x.w;
            }
            float cr = a.scale_log2;
            if (kBf16) {
                uint32_t top = 0;  // the largest magnitude, as bits
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
#pragma unroll
                    for (int e = 0; e < 2; ++e) top = __vmaxu2(top, qb[nt][s][e] & 0x7FFF7FFFu);
                top = max(top & 0xFFFFu, top >> 16);
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
                top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
                // 2^(14 - its exponent), and its inverse; a row of zeros, or with what is not finite, as it is
                const int e = (int)(top >> 7), up = top == 0 || e == 255 ? 0 : min(14 + 127 - e, 126);
                const float f = __uint_as_float((uint32_t)(127 + up) << 23);
                cr = fminf(cr * __uint_as_float((uint32_t)(127 - up) << 23), FLT_MAX);
#pragma unroll
                for (int s = 0; s < kSteps; ++s)
#pragma unroll
                    for (int e2 = 0; e2 < 2; ++e2)
                        qb[nt][s][e2] = half2_bits(__uint_as_float(qb[nt][s][e2] << 16) * f, __uint_as_float(qb[nt][s][e2] & 0xFFFF0000u) * f);
            }
            c_row[nt][0] = __shfl_sync(0xffffffffu, cr, 8 * c);      // (lane 4 g' has row g')
            c_row[nt][1] = __shfl_sync(0xffffffffu, cr, 8 * c + 4);
        }
        all0 = __reduce_max_sync(0xffffffffu, all0);
        all1 = __reduce_min_sync(0xffffffffu, all1);
        large = false;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) large |= c_row[nt][0] > 1.0f || c_row[nt][1] > 1.0f;
        large = __any_sync(0xffffffffu, large);

#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
            for (int t = 0; t < kDims; ++t)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][t][e] = 0.0f;
            m[nt][0] = m[nt][1] = -INFINITY;
            l[nt][0] = l[nt][1] = inv_ref[nt][0] = inv_ref[nt][1] = 0.0f;
        }
#pragma unroll 1
        for (int u = it.u0, u1 = it.u1, u_first = it.u0; u < u1; ++u) {
            const uint32_t st = ring + stage * Sh::kStage, sc = ring_scales + stage * Sh::kScale;
            copies_wait<Sh::kStages - 1>();
            ok = __all_sync(0xffffffffu, scoot_dev::mbar_wait_tries(bar0 + 8 * stage, phase));
            __syncwarp();
            if (!ok) break;
            uint32_t ks[kG], vs[kG];
#pragma unroll
            for (int t = 0; t < kG; t += 4) {
                lds<4>(sc + 4 * t, ks + t);
                lds<4>(sc + 4 * kG + 4 * t, vs + t);
            }
            if (lane < 2 * kG) {
                float own;
                asm volatile("ld.shared.f32 %0, [%1];" : "=f"(own) : "r"(sc + 4 * lane));
                bad_scale |= !(own >= 0.0f && own < INFINITY);
            }
#pragma unroll
            for (int t = 0; t < kG; ++t) {
                // (as bits: what is not finite, or negative, is above the others)
                if (ks[t] >= 0x7F800000u) ks[t] = 0u;
                if (vs[t] >= 0x7F800000u) vs[t] = 0u;
            }
            // scores: sixteen keys by eight rows a product
            float x[kM][NT][4];
#pragma unroll
            for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) x[mt][nt][0] = x[mt][nt][1] = x[mt][nt][2] = x[mt][nt][3] = 0.0f;
#pragma unroll
            for (int half = 0; half < D / 64; ++half) {
                uint32_t w[kM][2][4];
#pragma unroll
                for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) lds<4>(st + piece_at<D>(16 * mt + 8 * i + g, D / 64 * c + half), w[mt][i]);
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int mt = 0; mt < kM; ++mt) {
                        const uint32_t ka[4] = {decode_lo(w[mt][0][s]), decode_lo(w[mt][1][s]), decode_hi(w[mt][0][s]), decode_hi(w[mt][1][s])};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma(x[mt][nt], ka, qb[nt][4 * half + s][0], qb[nt][4 * half + s][1]);
                    }
            }
            // softmax: x[mt][nt][2 i + e] is of key 16 mt + 8 i + g and row 8 nt + 2 c + e
            const bool partial = u * kKeys < all0 || (u + 1) * kKeys > all1;
            float ck[kM][2][NT][2];
#pragma unroll
            for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) ck[mt][i][nt][e] = c_row[nt][e] * __uint_as_float(ks[2 * mt + i]);
            // the largest scale of the values that a row sees
            float vmax = fmaxf(__uint_as_float(vs[0]), __uint_as_float(vs[1])), vt[NT][2];
#pragma unroll
            for (int t = 2; t < kG; t += 2) vmax = max3(vmax, __uint_as_float(vs[t]), __uint_as_float(vs[t + 1]));
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) vt[nt][0] = vt[nt][1] = vmax;
            if (partial || large) {
                if (partial && several) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            vt[nt][e] = 0.0f;
#pragma unroll
                            for (int t = 0; t < kG; ++t) {
                                const int key = u * kKeys + 8 * t;
                                if (max(k0[nt][e], key) < min(k1[nt][e], key + 8)) vt[nt][e] = fmaxf(vt[nt][e], __uint_as_float(vs[t]));
                            }
                        }
                }
                const int key0 = u * kKeys + g;
#pragma unroll
                for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int key = key0 + 16 * mt + 8 * i;
                                if (key < k0[nt][e] || key >= k1[nt][e]) x[mt][nt][2 * i + e] = -INFINITY;
                                // (not zero, so that what is masked stays -inf; finite, so that a score of zero stays zero)
                                ck[mt][i][nt][e] = fminf(fmaxf(ck[mt][i][nt][e], 1e-37f), FLT_MAX);
                            }
            }
            float mx[NT][2];
            bool grown = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float y = fmaxf(x[0][nt][e] * ck[0][0][nt][e], x[0][nt][2 + e] * ck[0][1][nt][e]);
#pragma unroll
                    for (int mt = 1; mt < kM; ++mt) y = max3(y, x[mt][nt][e] * ck[mt][0][nt][e], x[mt][nt][2 + e] * ck[mt][1][nt][e]);
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 4));
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 8));
                    y = fmaxf(y, __shfl_xor_sync(0xffffffffu, y, 16));
                    mx[nt][e] = y;
                    grown |= y > m[nt][e] + 8.0f || vt[nt][e] * inv_ref[nt][e] > 129.0f;  // (128 and a rounding: nothing new)
                }
            if (u == u_first) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        m[nt][e] = mx[nt][e];
                        inv_ref[nt][e] = unit_of(fmaxf(vt[nt][e], 0x1p-100f));
                    }
            } else if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float mn = fmaxf(m[nt][e], mx[nt][e]), inv = fminf(inv_ref[nt][e], unit_of(vt[nt][e]));
                        f[e] = mn == -INFINITY ? 1.0f : exp2_hw(m[nt][e] - mn);
                        m[nt][e] = mn;
                        l[nt][e] *= f[e];
                        f[e] *= __fdividef(inv, inv_ref[nt][e]);
                        inv_ref[nt][e] = inv;
                    }
#pragma unroll
                    for (int t = 0; t < kDims; ++t)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[nt][t][e] *= f[e & 1];
                }
            }
            // P of sixteen keys by eight rows, turned round to be the other operand: lane (g, c) gets keys 2 c and the next of row g
            uint32_t pb[kM][NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float2 ms = make_float2(-finite_or_zero(m[nt][0]), -finite_or_zero(m[nt][1]));
                float2 sum = make_float2(0.f, 0.f);
#pragma unroll
                for (int mt = 0; mt < kM; ++mt)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float v = __uint_as_float(vs[2 * mt + i]);
                        const float2 z = __ffma2_rn(make_float2(x[mt][nt][2 * i], x[mt][nt][2 * i + 1]),
                                                    make_float2(ck[mt][i][nt][0], ck[mt][i][nt][1]), ms);
                        const float2 e = make_float2(exp2_hw(z.x), exp2_hw(z.y));
                        sum = __fadd2_rn(sum, e);
                        // (in this order what is hidden is zero, however large its scale over the row's)
                        const float2 pf = __fmul2_rn(__fmul2_rn(e, make_float2(inv_ref[nt][0], inv_ref[nt][1])), make_float2(v, v));
                        const uint32_t w = half2_bits(pf.x, pf.y);
                        asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(pb[mt][nt][i]) : "r"(w));
                    }
                l[nt][0] += sum.x;
                l[nt][1] += sum.y;
            }
            // values: sixteen dimensions by eight rows a product
#pragma unroll
            for (int mt = 0; mt < kM; ++mt) {
                constexpr int kW = D / 32;  // words of a key's piece
                uint32_t w[4][kW];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = 16 * mt + 2 * c + (i & 1) + 8 * (i >> 1);
                    if (D == 128) lds<kW>(st + Sh::kTile + piece_at<D>(row, g), w[i]);
                    else lds<kW>(st + Sh::kTile + piece_at<D>(row, g >> 1) + 8 * (g & 1), w[i]);
                    if (partial) {  // (a value that some row does not see, times its zero)
#pragma unroll
                        for (int e = 0; e < kW; ++e) w[i][e] = without_nan(w[i][e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < kW; ++e) {
#pragma unroll
                    for (int h2 = 0; h2 < 2; ++h2) {
                        const uint32_t lo2 = __byte_perm(w[0][e], w[1][e], h2 ? 0x7362 : 0x5140), hi2 = __byte_perm(w[2][e], w[3][e], h2 ? 0x7362 : 0x5140);
                        const uint32_t va[4] = {decode_lo(lo2), decode_hi(lo2), decode_lo(hi2), decode_hi(hi2)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) mma(o[nt][2 * e + h2], va, pb[mt][nt][0], pb[mt][nt][1]);
                    }
                }
            }
            __syncwarp();  // the tile has been read
            if (++stage == Sh::kStages) {
                stage = 0;
                phase ^= 1u;
            }
            load();
            copies_end();
        }
        if (!ok) break;
        // ---- the end of the item: the lane has 16 (8) dimensions in a row of rows 8 nt + 2 c and the next
        const bool whole = it.n_parts == 1;
        const bool begins = it.first == team;
        float* part = a.parts + (size_t)(2 * (team * a.share + member) + begins) * Sh::kPart;
        if (!whole && lane == 0) {
            if (it.n_parts <= kFewParts) ends_s[warp][begins] = it;
            else many = 1;
            if (it.n_parts > kFewParts && (begins || warp < a.share)) items[begins ? kShare + warp : member] = it;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 4);
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 8);
                l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], 16);
                const int row = 8 * nt + 2 * c + e;
                if (row >= it.rows) continue;
                const float unit = __fdividef(1.0f, inv_ref[nt][e]);
                if (whole) {
                    const float f = inverse_sum(l[nt][e]);
                    uint16_t* dst = out_row(a, it, row) + g * (D / 8);
#pragma unroll
                    for (int t = 0; t < kDims; t += 4) {
                        uint32_t w[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) w[i] = pack16<kBf16>(o[nt][t + i][e] * f * unit, o[nt][t + i][2 + e] * f * unit);
                        *reinterpret_cast<uint4*>(dst + 2 * t) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                    if (g == 0 && a.lse) *lse_row(a, it, row) = l[nt][e] == 0.0f ? -INFINITY : (m[nt][e] + __log2f(l[nt][e])) * kLn2;
                } else {
                    float* dst = part + row * D + g * (D / 8);
#pragma unroll
                    for (int t = 0; t < kDims; t += 2)
                        *reinterpret_cast<float4*>(dst + 2 * t) =
                            make_float4(o[nt][t][e] * unit, o[nt][t][2 + e] * unit, o[nt][t + 1][e] * unit, o[nt][t + 1][2 + e] * unit);
                    if (g == 0) reinterpret_cast<float2*>(part + kRows * D)[row] = make_float2(m[nt][e], l[nt][e]);
                }
            }
        if (!whole && !begins && it.n_parts <= kFewParts) {
            __syncwarp();
            if (lane == 0) came = add_one(it);  // (its result is not waited for here)
        }
    }
    // Of the range's split items, the one that began before it and the one that goes on after it: whether the other parts are there.
    __syncwarp();
    if (ok) {
        bool last = false;
        if (lane < 2 && ends_s[warp][lane].n_parts) {
            const Item& it = ends_s[warp][lane];
            if (lane == 1) came = add_one(it);
            last = came == (uint32_t)it.n_parts - 1;
            if (last) a.warp_count[it.first * a.share + member] = 0;
            __threadfence();
        }
        uint32_t done = __ballot_sync(0xffffffffu, last);
        __syncwarp();
#pragma unroll 1
        for (; done; done &= done - 1) {
            const Item* it = &ends_s[warp][__ffs(done) - 1];
            join<kBf16, D, kRows, 32, 4, 4>(a, it, 1, it->rows * (D / 4), lane, [&](int, float*&) {
                return parts_at(it->first, it->first, member, it->n_parts);
            });
        }
    }
    if (!ok) {  // a copy did not come: what is under way lands before the block ends
        if (lane == 0) atomicOr(a.err, SCOOT_DEVERR_TIMEOUT);
        failed = 1;
#pragma unroll 1
        for (int i = 0; i < Sh::kStages; ++i)
            if (i != (int)stage) scoot_dev::mbar_wait_tries(bar0 + 8 * i, i < (int)stage ? phase ^ 1u : phase);
    }
    if (bad_id) atomicOr(a.err, SCOOT_DEVERR_INDEX);
    if (bad_scale) atomicOr(a.err, SCOOT_DEVERR_VALUE);

    // ---- split items: the block's parts of each, then the blocks'
    __syncthreads();
    if (failed || !many) return;
    const int t0 = blockIdx.x * teams, t1 = t0 + teams - 1;
    float* joined = a.parts + (size_t)2 * n_workers * Sh::kPart;  // 2 kShare per block
    int rows = 0;
#pragma unroll 1
    for (int i = 0; i < kShare + kWarps; ++i) rows += items[i].n_parts ? items[i].rows : 0;
    const auto source = [&](int i, float*& to) {
        const Item& it = items[i];
        const int first = max(it.first, t0), n = min(it.first + it.n_parts - 1, t1) - first + 1, who = it.h % a.share;
        if (n < it.n_parts) to = joined + (size_t)((2 * blockIdx.x + (it.first >= t0 ? 1 : 0)) * kShare + who) * Sh::kPart;
        return parts_at(first, it.first, who, n);
    };
    if (rows * (D / 4) <= kThreads) join<kBf16, D, kRows, kThreads, 1, 8>(a, items, kShare + kWarps, rows * (D / 4), tid, source);
    else join<kBf16, D, kRows, kThreads, 4, 2>(a, items, kShare + kWarps, rows * (D / 4), tid, source);
    __syncthreads();
    // Of the items that lie in other blocks as well: whether this was the last.
    if (tid < kShare + kWarps) {
        const Item& it = items[tid];
        bool last = false;
        if (it.n_parts && (it.first < t0 || it.first + it.n_parts - 1 > t1)) {
            __threadfence();  // (the block's other threads' stores are before it by the barrier)
            const int b0 = it.first / teams, b1 = (it.first + it.n_parts - 1) / teams;
            uint32_t* count = a.block_count + b0 * kShare + it.h % a.share;
            last = atomicAdd(count, 1u) == (uint32_t)(b1 - b0);
            if (last) *count = 0;
            __threadfence();
        }
        last_s[tid] = last;
    }
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < kShare + kWarps; ++i) {
        if (!last_s[i]) continue;
        join<kBf16, D, kRows, kThreads, 1, 16>(a, items + i, 1, items[i].rows * (D / 4), tid, [&](int, float*&) {
            const int b0 = items[i].first / teams, b1 = (items[i].first + items[i].n_parts - 1) / teams, who = items[i].h % a.share;
            return Parts{joined + (size_t)((2 * b0 + 1) * kShare + who) * Sh::kPart, joined + (size_t)((2 * b0 + 2) * kShare + who) * Sh::kPart,
                         2 * kShare * Sh::kPart, b1 - b0 + 1};
        });
    }
}

template <bool kBf16, int D, int NT>
scoot_status launch(scoot_ctx* ctx, const Attn8Args& a, const KvMaps& maps, int sms, cudaStream_t st) {
    using Sh = Shape<D, NT>;
    auto kern = attn8_rows_kernel<kBf16, D, NT>;
    const uint32_t bit = 1u << (17 + 4 * (NT - 1) + 2 * kBf16 + (D == 128));
    if (!(ctx->smem_set & bit)) {  // once per context: the call is short
        SCOOT_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::kSmem));
        ctx->smem_set |= bit;
    }
    kern<<<(unsigned)sms, Sh::kThreads, Sh::kSmem, st>>>(a, maps);
    SCOOT_LAUNCHED(ctx);
    return SCOOT_OK;
}
template <int NT>
scoot_status launch(scoot_ctx* ctx, const Attn8Args& a, const KvMaps& maps, bool bf16, int D, int sms, cudaStream_t st) {
    if (bf16) return D == 128 ? launch<true, 128, NT>(ctx, a, maps, sms, st) : launch<true, 64, NT>(ctx, a, maps, sms, st);
    return D == 128 ? launch<false, 128, NT>(ctx, a, maps, sms, st) : launch<false, 64, NT>(ctx, a, maps, sms, st);
}

}  // namespace

extern "C" scoot_status scoot_paged_attention8(scoot_ctx* ctx, const scoot_kv_layout* layout, int32_t dtype, const void* q,
                                               int64_t q_ld_token, int64_t q_ld_head, int32_t n_heads, int64_t n_tokens,
                                               const int32_t* query_start, const int32_t* kv_len, int32_t n_req,
                                               const int32_t* block_table, int64_t ld_table, const void* k_cache,
                                               const void* v_cache, const float* k_scale, const float* v_scale, float scale,
                                               int32_t causal, int32_t window, int32_t max_new, void* out, int64_t out_ld_token,
                                               int64_t out_ld_head, float* lse, void* stream) {
    scoot_status s = scoot_enter(ctx);
    if (s != SCOOT_OK) return s;
    if ((s = scoot_check_kv8(ctx, layout, k_cache, v_cache, k_scale, v_scale)) != SCOOT_OK) return s;
    if (dtype != SCOOT_F16 && dtype != SCOOT_BF16)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "dtype = %d is neither SCOOT_F16 nor SCOOT_BF16", dtype);
    if (n_heads < 1 || n_heads % layout->n_kv_heads)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_heads = %d is not a multiple of n_kv_heads = %d", n_heads, layout->n_kv_heads);
    if (n_heads / layout->n_kv_heads > SCOOT_MAX_GROUP)
        return scoot_fail(ctx, SCOOT_EUNSUPPORTED, "%d query heads per key-value head, more than %d",
                          n_heads / layout->n_kv_heads, SCOOT_MAX_GROUP);
    if (n_tokens < 0 || n_tokens > 0x40000000ll || n_tokens > 0x7FFFFFFFll / n_heads || n_req < 0 || n_req > 0x40000000 ||
        ld_table < 0 || ld_table > 0x40000000ll / layout->block_size)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_tokens = %lld, n_req = %d or ld_table = %lld out of range", (long long)n_tokens,
                          n_req, (long long)ld_table);
    if (!(scale > 0.0f) || scale > kMaxScale)
        return scoot_fail(ctx, SCOOT_EINVAL, "scale = %g must be positive and at most %g", scale, kMaxScale);
    if (window < 0 || max_new < 0) return scoot_fail(ctx, SCOOT_EINVAL, "window = %d or max_new = %d < 0", window, max_new);
    if (n_tokens == 0 || n_req == 0) return SCOOT_OK;
    const int D = layout->head_dim, G = n_heads / layout->n_kv_heads;
    if ((s = scoot_check_heads(ctx, "q", q, q_ld_token, q_ld_head, D)) != SCOOT_OK) return s;
    if ((s = scoot_check_heads(ctx, "out", out, out_ld_token, out_ld_head, D)) != SCOOT_OK) return s;
    if (!query_start || !kv_len || (ld_table && !block_table)) return scoot_fail(ctx, SCOOT_EINVAL, "an array is NULL");
    const int sms = std::min(scoot_sms(ctx), kMaxBlocks);
    Attn8Args a = {};
    while ((1 << a.bs_log) < layout->block_size) ++a.bs_log;
    a.n_heads = n_heads;
    a.n_kv_heads = layout->n_kv_heads;
    a.group = G;
    a.n_req = n_req;
    a.causal = causal != 0;
    a.window = window < ld_table * layout->block_size ? window : 0;  // no sequence is longer
    a.max_new = max_new;
    // Items of sixteen rows where the group needs them, or all requests may have more than eight and are this kernel's (above);
    // else of eight, for which twelve warps have the registers and not eight: single tokens of the first of those in 82 us, not 88.
    const int row_tiles = G > 8 || (max_new * (int64_t)G > 8 && max_new <= kFewItems * (16 / G)) ? 2 : 1, item_rows = 8 * row_tiles;
    a.toks = std::max(1, item_rows / G);
    // Heads of the same tokens lie side by side in most caches: together they are read at 5.7 TB/s, one after the other at 4.7
    // (256 sequences, 8 heads of 128).  With fewer items than warps each is split into many parts instead, whose joins would fall
    // to the same blocks: three long sequences of 4 heads take 45 us alone, 76 together.
    const int warps = row_tiles == 1 ? Shape<64, 1>::kWarps : Shape<64, 2>::kWarps;
    a.share = (int64_t)n_req * layout->n_kv_heads < (int64_t)sms * warps ? 1 : kShare;
    while (layout->n_kv_heads % a.share) a.share /= 2;
    a.n_tokens = n_tokens;
    a.n_blocks = layout->n_blocks;
    a.query_start = query_start;
    a.kv_len = kv_len;
    a.table = block_table;
    a.ld_table = ld_table;
    a.q = static_cast<const uint16_t*>(q);
    a.q_ld_token = q_ld_token;
    a.q_ld_head = q_ld_head;
    a.k = static_cast<const uint8_t*>(k_cache);
    a.v = static_cast<const uint8_t*>(v_cache);
    a.ld_block = layout->ld_block;
    a.ld_token = layout->ld_token;
    a.ld_head = layout->ld_head;
    a.k_scale = k_scale;
    a.v_scale = v_scale;
    a.scale_log2 = scale * kLog2e;
    a.out = static_cast<uint16_t*>(out);
    a.out_ld_token = out_ld_token;
    a.out_ld_head = out_ld_head;
    a.lse = lse;
    a.warp_count = ctx->d_count + kWarpCounts;
    a.block_count = ctx->d_count + kBlockCounts;
    a.tile_count = ctx->d_count;
    a.err = ctx->d_err;
    a.few = G <= item_rows ? kFewItems * a.toks : 0;
    // The host does not know the lengths: without max_new both kernels are launched, and one may find nothing to do.
    const bool rows = a.few > 0, tiles = max_new == 0 || max_new > a.few;
    const size_t part = (size_t)item_rows * (D + 2) * sizeof(float);
    const size_t row_bytes = rows ? (size_t)sms * 2 * (warps + kShare) * part : 0;
    s = scoot_workspace(ctx, row_bytes + (tiles ? sms * scoot_attn8_tile_bytes(D) : 0), stream);
    if (s != SCOOT_OK) return s;
    a.parts = static_cast<float*>(ctx->ws);
    a.tile_parts = a.parts + row_bytes / sizeof(float);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool bf16 = dtype == SCOOT_BF16;
    if (rows) {
        KvMaps maps;
        const int keys = D == 128 ? Shape<128, 1>::kKeys : Shape<64, 1>::kKeys;
        if (!scoot_encode_codes(&maps.k, layout, k_cache, keys) || !scoot_encode_codes(&maps.v, layout, v_cache, keys))
            return scoot_fail(ctx, SCOOT_EINVAL, "the cache's layout has no tensor map");
        s = row_tiles == 1 ? launch<1>(ctx, a, maps, bf16, D, sms, st) : launch<2>(ctx, a, maps, bf16, D, sms, st);
        if (s != SCOOT_OK) return s;
    }
    return tiles ? scoot_attn8_tiles(ctx, layout, a, bf16, sms, st, rows) : SCOOT_OK;
}
