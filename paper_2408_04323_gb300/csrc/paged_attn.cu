// Attention of a batch of new tokens over a paged key-value cache, on the fifth-generation tensor cores.
//
//   out_t = sum_i softmax_i(scale q_t . k_i) v_i,   lse_t = ln sum_i exp(scale q_t . k_i)
//
// over the keys i that token t sees.  The keys go by in tiles of 128: S = Q K^T [128 x 128] by tcgen05.mma into tensor
// memory, then per row the running maximum m and sum l of the softmax (in log2 units: p = 2^(c s - m), c = scale log2 e),
// P rounded to the cache's type back into tensor memory over S, and O += P V.  O is rescaled only when a row's maximum
// has grown by more than 2^8 since it was last: until then p stays below 2^8, which the 16-bit types and the fp32 sums
// hold, and l and O carry the same factor, so that O / l is unchanged.
//
// Rows.  A query head's tokens and the G heads that share a key-value head are all rows of one product (row = token * G +
// head), so keys and values are read once for the group.  A CTA has two slots of 128 rows, each with its own O and four
// softmax warps:
//   * more than 128 rows (a chunk of a prompt): a pair, both slots against the same tile, so that one's softmax runs
//     under the other's products;
//   * up to 128 rows: one slot, the slots taking successive items in turn.  With at most 64 or 32 rows (single tokens) the
//     rows are loaded two or four times over, and the copy in lanes 32 w .. serves the w-th part of the tile's keys as
//     rows of its own, with its own m, l and O: the exponentials, which one warp would have taken for the whole tile,
//     are spread over the four.  The copies are joined at the end like the parts of a split item.
// Scores go to two buffers in tensor memory in turn, three with heads of 64, so that the next ones are computed under a
// softmax.
//
// Work.  An item is a (key-value head, request, up to 256 rows), its units the tiles of keys that its rows see.  All
// units in a row, head by head and request by request, with an extra cost per item, are cut into equal ranges, one per
// SM (a cut close to an item's start or end moves there): long sequences are split, short ones follow one another,
// whatever the batch.  Each CTA takes the sums over the requests for itself (lengths are on the device), so the call is
// one launch.  Items without keys (a sequence of no token, tokens before their sequence) are written by the warp that finds
// them and go no further: the product warp holds back up to kBuf products until the next units' scores are issued, and
// relies on every item that it is handed having a unit.  An item that lies in several ranges leaves its parts (O, m, l) in the workspace, and the CTA that comes last
// (a counter per item) joins them in the ranges' order, so that the result does not depend on who was last.
//
// Warps 0-3 and 4-7: softmax of slots 0 and 1.  Warp 8: the products.  Warp 9: the items, and the copies of queries and
// keys; warp 10: those of values.  A tile comes page by page through the block table, by TMA into a ring (128-byte
// swizzle), a box of up to 128 tokens x 64 dimensions per page and half head.
//
// Values that are not finite: a probability of 0 times an infinity or NaN is NaN, and so
//   * the value tiles at the ends of the sequence and along the diagonal, whose keys some row may not see, are looked through
//     first: rows past the ends are set to zero, and a value that is not finite is replaced by zero and the item marked;
//   * where a row's probability of a key that it sees has rounded to zero, and where a copy of a row has zeros at the keys of
//     the other copies, the product leaves a NaN.
// By the definition each probability is positive, and an infinity or NaN that a row sees is its sum's, whatever its weight.
// So an item that is marked, or whose sums are not all finite, has the values of its keys looked through at its end, and
// each row's sums set by those that it sees (odd_values); the joins give a weight of zero no say over such sums.
//
// What bounds it, as measured in calls one after the other (heads of 128 in blocks of 16, four query heads per key-value
// head, bf16):
//   * 256 sequences of 64 to 2560 tokens, one new token each: 220 us, 6.3 TB/s, 92% of the copy rate: HBM (a tile of
//     64 KB per SM in 2700 cycles; scores, softmax and products of one row group take 1500).
//   * a chunk of 8192 tokens over 8192 cached ones: 1.10 to 1.17 ms as the card's power allows, 1410 to 1500 TFLOP/s, 76 to
//     80% of the library's large product; the tensor pipe is busy in 68% of the cycles.  The rest is, as reckoned, the way
//     scores - softmax - values of a slot (3000 cycles for 2048 of products) and the shared memory that feeds both operands
//     of Q K^T.
//   * prompts in a window (heads of 64): 54 us, the tensor pipe busy in 27% and the schedulers in 40% of the active cycles:
//     1400 cycles of softmax per tile, and starts and ends of items (about 5 us of a call: ranges, first tile, last join).
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "internal.h"
#include "mbarrier.cuh"

namespace {

using namespace scoot_dev;

constexpr int kRows = 128;         // rows of a slot: the MMA's M and the TMEM lanes
constexpr int kKeys = 128;         // keys of a tile
constexpr int kThreads = 384;      // three warpgroups: the two softmax ones take registers from the third
constexpr int kSoftmaxRegs = 200, kOtherRegs = 104;  // 2 * 200 + 104 = 3 * 168, what the block is launched with
constexpr int kMmaWarp = 8, kLoadWarp = 9, kValueWarp = 10;
constexpr int kRing = 4;         // items handed from the load warp to the others
constexpr int kItemCost = 1;     // an item's start and end, in units,
constexpr int kPairCost = 5;     // and a pair's, with the tiles along its diagonal
constexpr int kMinRange = 4;     // units that a CTA takes at least
constexpr int kSnapMin = 2;      // a cut this close to an item's ends moves there; and up to this close, if it is
constexpr int kSnapMax = 6;      // a quarter of a range: writing, counting and joining parts costs five to nine units
constexpr int kBufs = 4;         // part buffers of a CTA
constexpr int kScratch = 16384;  // bytes of a slot's scratch: 32 columns of sums of its rows, or weights of parts
constexpr int kHalf = kKeys * 128;  // bytes of a tile's half: 128 keys x 64 dimensions
constexpr int kMaxCtas = (int)(SCOOT_COUNTS / 2);
constexpr float kMaxScale = 2.3e38f;  // times log2 e it is still finite
constexpr float kLn2 = 0.69314718055994531f, kLog2e = 1.4426950408889634f;

template <int D>
struct Shape {
    static constexpr int kTile = kKeys * D * 2;           // bytes of a tile of keys, values or queries
    static constexpr int kStages = (D == 128 ? 4 : 10);   // tiles of keys or values in flight
    // Tensor memory: score buffers of 128 columns from 0 on, then the slots' O.
    static constexpr uint32_t kBuf = D == 128 ? 2 : 3, kO = 512 - 2 * D;
    static constexpr int kSmem = 2 * kTile + kStages * kTile + 2 * kScratch;  // and the static part, up to 227 KB
};

struct AttnArgs {
    CUtensorMap kmap, vmap, qmap[3];  // qmap[i]: tokens of 128 >> i rows
    int32_t bs_log, n_heads, n_kv_heads, group, n_req, causal, window;
    int32_t toks;         // tokens of a slot: 128 / group
    int32_t inv_group;    // row / group = row * inv_group >> 16, for rows below 128
    int64_t n_tokens, n_blocks;
    const int32_t* query_start;
    const int32_t* kv_len;
    const int32_t* table;
    int64_t ld_table;
    const uint16_t* v;    // for the marked items
    int64_t ld_block, ld_token, ld_head;
    float scale_log2;
    uint16_t* out;
    int64_t out_ld_token, out_ld_head;
    float* lse;
    float* parts;         // kBufs part buffers per CTA (part_buf)
    uint32_t* count;      // arrivals per split item and slot, zero between calls
    uint32_t* err;
};

// What the load warp tells the others about an item, or a part of it.
struct Item {
    int32_t h, r, tok, ntok;   // key-value head, request, first row of q, tokens
    int32_t pos, kv;           // position of the first token, length of the sequence
    int32_t begin, end;        // keys that some row of the item sees
    int32_t u0, nu;            // this part's tiles: u0 .. u0 + nu - 1
    int32_t slot;              // 0 or 1; 2: a pair
    int32_t rep_log;           // copies of the rows: 1 << rep_log
    int32_t first, n_parts;    // CTA of the first part, and how many parts
    int32_t poison;            // a value that is not finite was replaced
    int32_t stop;
};

// The first three are [slot][number of the slot's unit mod 3, of 4]: up to three units of a slot are under way at once.
enum {
    kSFull = 0, kPFull = 8, kPvDone = 16, kQFull = 24, kQEmpty = 26, kWg = 28, kItemFull = 30, kItemEmpty = 34, kDrain = 38,
    kKvFull = 40, kKvEmpty = 50, kBars = 60
};

// The swizzled K-major tile of queries or keys: rows of 128 bytes, 8-row groups 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_k(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// The value tile, whose product runs over keys (rows): 64-dimension halves kHalf bytes apart, 8-key groups 1024.
__device__ __forceinline__ uint64_t desc_v(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFFu) | ((uint64_t)(kHalf >> 4) << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// kind::f16, fp32 accumulator, M = 128; b_mn: B runs along its N in memory.
__device__ __forceinline__ uint32_t idesc(bool bf16, uint32_t n, bool b_mn) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) | ((n >> 3) << 17) | (8u << 24);
}

// 32 consecutive columns of the calling warp's 32 lanes of tensor memory, to and from registers (lane i of the warp
// holds its lane's row); a load is complete after tmem_wait_ld.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* x) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15]), "=r"(x[16]), "=r"(x[17]), "=r"(x[18]), "=r"(x[19]), "=r"(x[20]), "=r"(x[21]), "=r"(x[22]), "=r"(x[23]), "=r"(x[24]), "=r"(x[25]), "=r"(x[26]), "=r"(x[27]), "=r"(x[28]), "=r"(x[29]), "=r"(x[30]), "=r"(x[31])
        : "r"(addr));
}

__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* x) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]), "=r"(x[8]), "=r"(x[9]), "=r"(x[10]), "=r"(x[11]), "=r"(x[12]), "=r"(x[13]), "=r"(x[14]), "=r"(x[15])
        : "r"(addr));
}

__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* x) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]), "r"(x[8]), "r"(x[9]), "r"(x[10]), "r"(x[11]), "r"(x[12]), "r"(x[13]), "r"(x[14]), "r"(x[15]));
}

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

__device__ __forceinline__ float exp2_hw(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float finite_or_zero(float m) { return m == -INFINITY ? 0.0f : m; }

// 1 / l, 0 for a row that sees nothing (NaN stays).
__device__ __forceinline__ float inverse_sum(float l) { return l == 0.0f ? 0.0f : __fdividef(1.0f, l); }

template <bool kBf16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    if (kBf16) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&v);
    }
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// A pair's halves that are infinite or NaN: their bits set.  (The exponent's complement is zero in them.)
template <bool kBf16>
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    const uint32_t e = kBf16 ? 0x7F807F80u : 0x7C007C00u;
    return __vcmpeq2(~w & e, 0u);
}
// Bits 15 and 31 set where a half's exponent is all ones (a carry out of it), other bits anything.
template <bool kBf16>
__device__ __forceinline__ uint32_t top_exponent(uint32_t w) {
    return kBf16 ? (w & 0x7F807F80u) + 0x00800080u : (w & 0x7C007C00u) + 0x04000400u;
}
// x of a sum whose weight is zero: what is finite has none, the rest all of it.
__device__ __forceinline__ float weightless(float x) { return fabsf(x) < INFINITY ? 0.0f : x; }

// One request's lengths, empty if they are bad.
struct Req {
    int32_t q0, n, kv;
};
__device__ __forceinline__ Req load_req(const AttnArgs& a, int r, bool flag) {
    Req q{0, 0, 0};
    if (r >= a.n_req) return q;
    const int q0 = a.query_start[r], q1 = a.query_start[r + 1], kv = a.kv_len[r];
    if (q0 < 0 || q1 < q0 || q1 > a.n_tokens || kv < 0 || kv > a.ld_table << a.bs_log) {
        if (flag) atomicOr(a.err, SCOOT_DEVERR_INDEX);
        return q;
    }
    q.q0 = q0;
    q.n = q1 - q0;
    q.kv = kv;
    return q;
}

// The keys [begin, end) that tokens tok0 .. tok0 + nt - 1 of n new ones see, all together.
__device__ __forceinline__ void seen_keys(const AttnArgs& a, int kv, int n, int tok0, int nt, int& begin, int& end) {
    const int64_t p0 = (int64_t)kv - n + tok0;
    end = a.causal ? (int)min((int64_t)kv, p0 + nt) : kv;
    begin = a.window > 0 ? (int)max((int64_t)0, p0 + 1 - a.window) : 0;
    if (end <= begin) begin = end = 0;
}
// The cost, in units, of item j of n tokens beside its units.
__device__ __forceinline__ int item_cost(const AttnArgs& a, int n, int j) {
    return n - j * 2 * a.toks > a.toks ? kPairCost : kItemCost;
}
__device__ __forceinline__ int item_units(const AttnArgs& a, int kv, int n, int j) {
    const int per = 2 * a.toks;
    int begin, end;
    seen_keys(a, kv, n, j * per, min(per, n - j * per), begin, end);
    return (end + kKeys - 1) / kKeys - begin / kKeys;
}

// a / b of a >= 0, b > 0, in 32 bits where they fit.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
    return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Part buffers: 128 rows of D sums, then (m, l) of each.  A CTA has one per half (slot of a pair) for the part of an item
// that an earlier CTA began, and one for the part that begins an item that goes on in the next; the parts of an item of
// CTAs c, c + 1, .. are buffers 2 c + 1, 2 c + 2, 2 c + 4, ..: from 2 c + 2 on every second.
template <int D>
constexpr int kPartFloats = kRows * (D + 2);
template <int D>
__device__ __forceinline__ float* part_buf(float* first, int i) {  // of part i, first that of part 0
    return first + (size_t)(i == 0 ? 0 : 2 * i - 1) * kPartFloats<D>;
}
template <int D>
__device__ __forceinline__ const float* part_buf(const float* first, int i) {
    return first + (size_t)(i == 0 ? 0 : 2 * i - 1) * kPartFloats<D>;
}

// Bounded waits that pass at once after the first that gave up.  A lane's `ok` is its own until all() makes it the warp's:
// between the two the role goes on as if the wait had ended, on memory that is its own all the same.
struct Waiter {
    bool ok = true;
    __device__ __forceinline__ void warp(uint64_t* b, uint32_t use) { at(smem_u32(b), use & 1u); }
    __device__ __forceinline__ void at(uint32_t b, uint32_t parity) {
        if (ok) ok = mbar_wait_tries(b, parity);
    }
    __device__ __forceinline__ bool all() { return ok = __all_sync(0xffffffffu, ok) != 0; }
};

// Softmax of NCH chunks of 32 columns from chunk ch0 on of a row's scores, P over them and zeros in the other chunks.
// [c0, c1): the columns that the row sees, if not all.  rescale(f) multiplies the row's O by f and returns when that
// is done; called by whole warps.
template <bool kBf16, int NCH, typename F>
__device__ __forceinline__ void softmax_tile(uint32_t tS, int ch0, bool full, int c0, int c1, float c, bool first, bool live,
                                             float& m, float& l, F&& rescale) {
    uint32_t x[NCH * 32];
#pragma unroll
    for (int q = 0; q < NCH; ++q) tmem_ld32(tS + 32 * (ch0 + q), x + 32 * q);
    tmem_wait_ld();
    if (!full) {
#pragma unroll
        for (int q = 0; q < NCH; ++q) {
            // the columns of this chunk that the row sees, as bits; most chunks are seen by all the warp's rows
            const int lo = min(max(c0 - 32 * (ch0 + q), 0), 32), hi = min(max(c1 - 32 * (ch0 + q), 0), 32);
            const uint32_t bits = hi <= lo ? 0u : (0xFFFFFFFFu >> (32 - hi)) & (0xFFFFFFFFu << lo);
            if (__all_sync(0xffffffffu, bits == 0xFFFFFFFFu)) continue;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (!(bits & (1u << i))) x[32 * q + i] = 0xFF800000u;
        }
    }
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int i = 0; i < NCH * 32; ++i) mx[i & 3] = fmaxf(mx[i & 3], __uint_as_float(x[i]));
    const float mt = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * c;
    if (first) {
        m = mt;
    } else if (__any_sync(0xffffffffu, live && mt > m + 8.0f)) {
        const float mn = fmaxf(m, mt);
        const float f = mn == -INFINITY ? 1.0f : exp2_hw(m - mn);
        m = mn;
        l *= f;
        rescale(f);
    }
    const float ms = finite_or_zero(m);
    const float2 cc = make_float2(c, c), mm = make_float2(-ms, -ms);
    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
    for (int q = 0; q < NCH; ++q) {
        uint32_t p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 s = make_float2(__uint_as_float(x[32 * q + 2 * i]), __uint_as_float(x[32 * q + 2 * i + 1]));
            const float2 t = __ffma2_rn(s, cc, mm);
            const float2 e = make_float2(exp2_hw(t.x), exp2_hw(t.y));
            sum[i & 1] = __fadd2_rn(sum[i & 1], e);
            p[i] = pack16<kBf16>(e.x, e.y);
        }
        tmem_st16(tS + 16 * (ch0 + q), p);
    }
    if (NCH < 4) {
        uint32_t z[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0u;
#pragma unroll
        for (int q = 0; q < 4; ++q)
            if (q < ch0 || q >= ch0 + NCH) tmem_st16(tS + 16 * q, z);
    }
    l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
    tmem_wait_st();
}

// One step of a product (16 of its inner dimension), both operands in shared memory, or A in tensor memory.  The upper
// halves of the operands' descriptors are constants.
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t da, uint32_t db, uint32_t upper, uint32_t id, bool acc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 da, {%1, %3};\n\t"
                 "mov.b64 db, {%2, %3};\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, p;\n\t}" ::"r"(d),
                 "r"(da), "r"(db), "r"(upper), "r"(id), "r"((uint32_t)acc));
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t ta, uint32_t db, uint32_t upper, uint32_t id, bool acc) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 db;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 db, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %4, p;\n\t}" ::"r"(d),
                 "r"(ta), "r"(db), "r"(upper), "r"(id), "r"((uint32_t)acc));
}

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// A warp that copies the tiles of keys or of values, loads `at`, at + 2, .. of the ring.  One lane issues (a copy takes its
// operands from the warp's uniform registers: 32 lanes with a copy each took 66 cycles per copy).  The lanes hold the
// block ids of 32 pages, four tiles' at 16 tokens a block, and those of the next 32 in flight.
template <int D>
struct TileLoader {
    const AttnArgs& a;
    const CUtensorMap* map;
    uint64_t* bars;
    uint32_t tiles;  // shared address of the ring
    uint32_t st, phase;         // the next load's place in the ring, and of its barriers
    uint32_t at;
    int box, n_page, page_log;  // tokens of a page, pages of a tile
    int group;                  // ids: of pages 32 group ..
    int ids, ids_next;
    bool bad = false;
    static constexpr int kNone = INT32_MIN, kCopies = 4;
    __device__ __forceinline__ TileLoader(const AttnArgs& a_, const CUtensorMap* m, uint64_t* b, uint32_t t, uint32_t first)
        : a(a_), map(m), bars(b), tiles(t), st(first), phase(0), at(first) {
        page_log = a.bs_log < 7 ? 7 - a.bs_log : 0;
        n_page = 1 << page_log;
        box = kKeys >> page_log;
    }
    // This lane's id of the pages of group g; kNone if no row sees any of its tokens.
    __device__ __forceinline__ int fetch(const Item& it, int g) const {
        const int64_t key = ((int64_t)g * 32 + (threadIdx.x & 31)) * box;
        return key < it.end && key + box > it.begin ? __ldg(a.table + (int64_t)it.r * a.ld_table + (key >> a.bs_log)) : kNone;
    }
    __device__ __forceinline__ void use(int raw) {
        const bool out = raw < 0 || raw >= a.n_blocks;
        bad |= out && raw != kNone;
        ids = out ? (int)a.n_blocks : raw;  // past the end: the copy reads nothing and writes zeros
    }
    __device__ __forceinline__ void begin(const Item& it) {
        group = (it.u0 << page_log) >> 5;
        use(fetch(it, group));
        ids_next = fetch(it, group + 1);
    }
    __device__ __forceinline__ void tile(const Item& it, int u, Waiter& wait) {
        constexpr uint32_t kNS = Shape<D>::kStages;
        const int page = u << page_log;
        if (page >> 5 != group) {
            group = page >> 5;
            use(ids_next);
            ids_next = fetch(it, group + 1);
        }
        const uint32_t bar = smem_u32(&bars[kKvFull + st]);
        if (at >= kNS) wait.warp(&bars[kKvEmpty + st], phase ^ 1u);
        if (!wait.all()) return;
        at += 2;
        const bool one = elect_one();
        if (one)
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)Shape<D>::kTile) : "memory");
        const uint32_t dst = tiles + st * Shape<D>::kTile;
        const int within = (u * kKeys) & ((1 << a.bs_log) - 1);
        auto copy = [&](int i, int id) {
#pragma unroll
            for (int half = 0; half < D / 64; ++half)
                asm volatile(
                    "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, "
                    "%5}], [%6];" ::"r"(dst + i * box * 128 + half * kHalf),
                    "l"(map), "r"(half * 64), "r"(it.h), "r"(within), "r"(id), "r"(bar)
                    : "memory");
        };
        // (straight code for kCopies pages at a time: with a branch per page a copy took 150 cycles)
        int i = 0;
#pragma unroll 1
        for (; i + kCopies <= n_page; i += kCopies) {
            int id[kCopies];
#pragma unroll
            for (int j = 0; j < kCopies; ++j) id[j] = __shfl_sync(0xffffffffu, ids, (page & 31) + i + j);
            if (one) {
#pragma unroll
                for (int j = 0; j < kCopies; ++j) copy(i + j, id[j]);
            }
        }
#pragma unroll 1
        for (; i < n_page; ++i) {
            const int id = __shfl_sync(0xffffffffu, ids, (page & 31) + i);
            if (one) copy(i, id);
        }
        __syncwarp();
        if ((st += 2) >= kNS) {
            st -= kNS;
            phase ^= 1u;
        }
    }
    // After a wait that gave up: the copies in flight land before the block ends.
    __device__ __forceinline__ void drain() const {
        constexpr uint32_t kNS = Shape<D>::kStages;
#pragma unroll 1
        for (uint32_t i = at & 1u; i < at; i += 2)
            if (i + kNS >= at) mbar_wait_tries(smem_u32(&bars[kKvFull + i % kNS]), (i / kNS) & 1u);
    }
};

// A slot's four warps meet (bounded): warps of one that gave up do not hold the others.
struct SlotSync {
    uint64_t* bar;
    uint32_t n;
    Waiter wait;
    __device__ __forceinline__ void operator()() {
        warp_arrive(bar);
        wait.warp(bar, n++);
    }
};

// O of a warp's rows, each of which sees the keys [k0, k1), after a part of nu tiles with values that are not finite: an
// infinity or NaN among those that the row sees (a copy: of its own keys in a tile) decides its sum, and a copy's NaN that
// only the others' keys account for was a zero times theirs.  The keys are [begin, end), 32 at a time, a lane each.
template <bool kBf16, int D>
__device__ __noinline__ void odd_values(const AttnArgs& a, uint32_t tO, int h, int r, int u0, int nu, int begin, int end, int k0, int k1,
                                        int rep_log, int copy) {
    const int lane = threadIdx.x & 31;
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
        uint32_t pos = 0, neg = 0, others = 0;  // columns with +inf, -inf, both (a NaN counts as both); with any of other copies
#pragma unroll 1
        for (int key0 = max(u0 * kKeys, begin & ~31); key0 < min((u0 + nu) * kKeys, end); key0 += 32) {
            const int key = key0 + lane;
            uint4 w[4] = {};
            if (key >= begin && key < end) {
                const int id = a.table[(int64_t)r * a.ld_table + (key >> a.bs_log)];
                if (id >= 0 && id < a.n_blocks) {
                    const uint4* v = reinterpret_cast<const uint4*>(a.v + id * a.ld_block + (key & ((1 << a.bs_log) - 1)) * a.ld_token +
                                                                    h * a.ld_head + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = v[i];
                }
            }
            const uint32_t* x = reinterpret_cast<const uint32_t*>(w);
            uint32_t p = 0, n = 0;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t odd = not_finite<kBf16>(x[i]);
                const uint32_t nan = odd & ~__vcmpeq2(x[i] & (kBf16 ? 0x007F007Fu : 0x03FF03FFu), 0u);
                const uint32_t sign = __vcmpgeu2(x[i], 0x80008000u);
                const uint32_t up = nan | (odd & ~sign), down = nan | (odd & sign);
                p |= ((up & 1u) | (up >> 30 & 2u)) << (2 * i);
                n |= ((down & 1u) | (down >> 30 & 2u)) << (2 * i);
            }
            uint32_t some = __ballot_sync(0xffffffffu, (p | n) != 0);
            const bool own = rep_log == 0 || (key0 % kKeys) >> (7 - rep_log) == copy;
            while (some) {
                const int src = __ffs(some) - 1;
                some &= some - 1;
                const uint32_t ps = __shfl_sync(0xffffffffu, p, src), ns = __shfl_sync(0xffffffffu, n, src);
                const bool sees = key0 + src >= k0 && key0 + src < k1;
                if (sees && own) {
                    pos |= ps;
                    neg |= ns;
                } else if (sees) {
                    others |= ps | ns;
                }
            }
        }
        if (!__any_sync(0xffffffffu, (pos | neg | others) != 0)) continue;
#pragma unroll 1
        for (int half = 0; half < 32; half += 16) {
            uint32_t o[16];
            tmem_ld16(tO + c + half, o);
            tmem_wait_ld();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t bit = 1u << (half + i), up = pos & bit, down = neg & bit;
                if (up | down) o[i] = up && down ? 0x7FFFFFFFu : up ? 0x7F800000u : 0xFF800000u;
                else if ((others & bit) && __uint_as_float(o[i]) != __uint_as_float(o[i])) o[i] = 0u;
            }
            tmem_st16(tO + c + half, o);
        }
        tmem_wait_st();
    }
}

// Row q of a slot, tokens from tok on, the group's first head `head`: where it goes.
__device__ __forceinline__ uint16_t* out_row(const AttnArgs& a, int tok, int head, int q) {
    const int t = q * a.inv_group >> 16;
    return a.out + (int64_t)(tok + t) * a.out_ld_token + (int64_t)(head + q - t * a.group) * a.out_ld_head;
}
__device__ __forceinline__ float* lse_row(const AttnArgs& a, int tok, int head, int q) {
    const int t = q * a.inv_group >> 16;
    return a.lse + (int64_t)(tok + t) * a.n_heads + head + q - t * a.group;
}

// Four columns (at: in groups of four) of a row's V parts by their weights, where some of the sums are not finite.
template <int D>
__device__ __noinline__ float4 join_odd(const float* part, const float* w, int V, int at) {
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
    for (int p = 0; p < V; ++p) {
        float4 v = __ldcg(reinterpret_cast<const float4*>(part_buf<D>(part, p)) + at);
        float f = w[p];
        if (f == 0.0f) {
            v = make_float4(weightless(v.x), weightless(v.y), weightless(v.z), weightless(v.w));
            f = 1.0f;
        }
        acc = make_float4(fmaf(f, v.x, acc.x), fmaf(f, v.y, acc.y), fmaf(f, v.z, acc.z), fmaf(f, v.w, acc.w));
    }
    return acc;
}

// The weighted sums of V parts of rows q0 .. q0 + nq - 1 (weights w [row][V]).  A thread has four columns of R rows, 128 /
// (D / 4) apart, with P parts of each in flight.
template <bool kBf16, int D, int R, int P>
__device__ __forceinline__ void join_rows(const AttnArgs& a, const float* part, const float* w, int V, int q0, int nq, int tok,
                                          int head) {
    constexpr int kGroups = D / 4, kStep = kRows / kGroups;
    const int row = threadIdx.x & (kRows - 1), c = row % kGroups;
#pragma unroll 1
    for (int q = row / kGroups; q < nq; q += R * kStep) {
        float4 acc[R];
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int p0 = 0; p0 < V; p0 += P) {
            float4 v[P][R];
            float f[P][R];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const int pt = min(p0 + p, V - 1);  // past the last part, or row: the last one's, not used
                const float4* src = reinterpret_cast<const float4*>(part_buf<D>(part, pt)) + q0 * kGroups + c;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    const int r = min(q + i * kStep, nq - 1);
                    v[p][i] = __ldcg(src + r * kGroups);
                    f[p][i] = w[r * V + pt];
                }
            }
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (p0 + p < V)
#pragma unroll
                    for (int i = 0; i < R; ++i)
                        acc[i] = make_float4(fmaf(f[p][i], v[p][i].x, acc[i].x), fmaf(f[p][i], v[p][i].y, acc[i].y),
                                             fmaf(f[p][i], v[p][i].z, acc[i].z), fmaf(f[p][i], v[p][i].w, acc[i].w));
        }
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (q + i * kStep < nq) {
                if (const float sum = (acc[i].x + acc[i].y) + (acc[i].z + acc[i].w); sum != sum)
                    acc[i] = join_odd<D>(part, w + (q + i * kStep) * V, V, (q0 + q + i * kStep) * kGroups + c);
                *reinterpret_cast<uint2*>(out_row(a, tok, head, q0 + q + i * kStep) + 4 * c) =
                    make_uint2(pack16<kBf16>(acc[i].x, acc[i].y), pack16<kBf16>(acc[i].z, acc[i].w));
            }
    }
}

// The V parts of a split item's rows, joined by the slot whose part came last: per row the parts' common maximum and sum
// and each part's weight (a thread per row, into the scratch), then the weighted sums, a warp over several rows.
template <bool kBf16, int D>
__device__ __noinline__ SlotSync join_parts(const AttnArgs& a, const float* part, int V, int rows, int tok, int head, float* w,
                                            SlotSync sync) {
    const int row = threadIdx.x & (kRows - 1), batch = min(kRows, kScratch / 4 / V);
#pragma unroll 1
    for (int q0 = 0; q0 < rows; q0 += batch) {
        const int nq = min(batch, rows - q0);
        if (q0 > 0) sync();
        if (nq <= 8) {
            // few rows: a warp per row, a lane per part
#pragma unroll 1
            for (int q = row >> 5; q < nq; q += kRows / 32) {
                float M = -INFINITY, L = 0.0f;
#pragma unroll 1
                for (int i = row & 31; i < V; i += 32) {
                    const float2 v = __ldcg(reinterpret_cast<const float2*>(part_buf<D>(part, i) + kRows * D) + q0 + q);
                    const float Mn = fmaxf(M, v.x), Ms = finite_or_zero(Mn);
                    L = fmaf(L, exp2_hw(M - Ms), exp2_hw(v.x - Ms) * v.y);
                    M = Mn;
                    w[q * V + i] = v.x;
                }
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) {
                    const float Mo = __shfl_xor_sync(0xffffffffu, M, d), Lo = __shfl_xor_sync(0xffffffffu, L, d);
                    const float Mn = fmaxf(M, Mo), Ms = finite_or_zero(Mn);
                    L = L * exp2_hw(M - Ms) + Lo * exp2_hw(Mo - Ms);
                    M = Mn;
                }
                const float inv = inverse_sum(L), Ms = finite_or_zero(M);
#pragma unroll 1
                for (int i = row & 31; i < V; i += 32) w[q * V + i] = exp2_hw(w[q * V + i] - Ms) * inv;
                if (a.lse && (row & 31) == 0) *lse_row(a, tok, head, q0 + q) = L == 0.0f ? -INFINITY : (M + __log2f(L)) * kLn2;
            }
        } else if (row < nq) {
            float M = -INFINITY, L = 0.0f;
#pragma unroll 1
            for (int i0 = 0; i0 < V; i0 += 8) {
                float2 v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[i] = i0 + i < V ? __ldcg(reinterpret_cast<const float2*>(part_buf<D>(part, i0 + i) + kRows * D) + q0 + row)
                                      : make_float2(-INFINITY, 0.0f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float Mn = fmaxf(M, v[i].x), Ms = finite_or_zero(Mn);
                    L = fmaf(L, exp2_hw(M - Ms), exp2_hw(v[i].x - Ms) * v[i].y);
                    M = Mn;
                    if (i0 + i < V) w[row * V + i0 + i] = v[i].x;
                }
            }
            const float inv = inverse_sum(L), Ms = finite_or_zero(M);
#pragma unroll 1
            for (int i = 0; i < V; ++i) w[row * V + i] = exp2_hw(w[row * V + i] - Ms) * inv;
            if (a.lse) *lse_row(a, tok, head, q0 + row) = L == 0.0f ? -INFINITY : (M + __log2f(L)) * kLn2;
        }
        sync();
        if (nq <= 8) join_rows<kBf16, D, 2, 8>(a, part, w, V, q0, nq, tok, head);
        else join_rows<kBf16, D, 4, 2>(a, part, w, V, q0, nq, tok, head);
    }
    return sync;
}

// Zeros and -inf for the rows of an item without keys, by one warp.
template <int D>
__device__ __forceinline__ void no_keys(const AttnArgs& a, const Item& it) {
    const int lane = threadIdx.x & 31, rows = it.ntok * a.group;
#pragma unroll 1
    for (int e = lane; e < rows * (D / 8); e += 32) {
        const int q = e / (D / 8), t = q / a.group;
        *reinterpret_cast<uint4*>(a.out + (int64_t)(it.tok + t) * a.out_ld_token + (int64_t)(it.h * a.group + q - t * a.group) * a.out_ld_head +
                                  8 * (e % (D / 8))) = make_uint4(0, 0, 0, 0);
    }
    if (a.lse)
#pragma unroll 1
        for (int q = lane; q < rows; q += 32) {
            const int t = q / a.group;
            a.lse[(int64_t)(it.tok + t) * a.n_heads + it.h * a.group + q - t * a.group] = -INFINITY;
        }
}

template <bool kBf16, int D>
__global__ void __launch_bounds__(kThreads, 1) paged_attn_kernel(const __grid_constant__ AttnArgs a) {
    using Sh = Shape<D>;
    constexpr int kNS = Sh::kStages, kNH = D / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* sQ = smem;
    uint8_t* sKV = sQ + 2 * Sh::kTile;
    uint8_t* sScratch = sKV + kNS * Sh::kTile;
    __shared__ __align__(8) uint64_t bars[kBars];
    __shared__ Item items[kRing];
    __shared__ uint32_t tslot;
    // the threads' sums of costs and requests, in the ring's last tile until the load warp has found its first item
    int64_t* cost_s = reinterpret_cast<int64_t*>(sKV + (kNS - 1) * Sh::kTile);
    Req* req_s = reinterpret_cast<Req*>(cost_s + kThreads);
    __shared__ int last_flag[2];
    __shared__ float2 ml_s[2][kRows];
    // (the same for all lanes, and by the shuffle known to be)
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);

    if (tid == 0) {
        for (int s = 0; s < 8; ++s) {
            mbar_init(&bars[kSFull + s], 1);
            mbar_init(&bars[kPFull + s], 4);
            mbar_init(&bars[kPvDone + s], 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbar_init(&bars[kQFull + s], 1);
            mbar_init(&bars[kQEmpty + s], 1);
            mbar_init(&bars[kWg + s], 4);
        }
        for (int s = 0; s < kRing; ++s) {
            mbar_init(&bars[kItemFull + s], 1);
            mbar_init(&bars[kItemEmpty + s], 10);  // eight softmax warps, the product thread and the value warp
        }
        mbar_init(&bars[kDrain], 1);
        for (int s = 0; s < kNS; ++s) {
            mbar_init(&bars[kKvFull + s], 1);
            mbar_init(&bars[kKvEmpty + s], 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kLoadWarp && lane < 5 && (lane < 3 || kRows >> (lane - 2) >= a.group)) {  // (maps that are in use)
        const CUtensorMap* map = lane == 0 ? &a.kmap : lane == 1 ? &a.vmap : &a.qmap[lane - 2];
        asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tslot)), "r"(512u));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }

    // The cost of all items of one head: each thread k consecutive requests, then a scan.  A request of several items is
    // summed by its warp.
    const int k = (a.n_req + kThreads - 1) / kThreads, per = 2 * a.toks;
    int64_t mine = 0;
#pragma unroll 1
    for (int i = 0; i < k; ++i) {
        const int r = tid * k + i;
        const Req q = load_req(a, r, blockIdx.x == 0);
        if (k == 1) req_s[tid] = q;
        if (q.n > 0 && q.n <= per) mine += item_cost(a, q.n, 0) + item_units(a, q.kv, q.n, 0);
        uint32_t big = __ballot_sync(0xffffffffu, q.n > per);
        while (big) {
            const int src = __ffs(big) - 1;
            big &= big - 1;
            const int kv = __shfl_sync(0xffffffffu, q.kv, src), n = __shfl_sync(0xffffffffu, q.n, src);
            int64_t c = 0;
            const int m = (n + per - 1) / per;
#pragma unroll 1
            for (int j = lane; j < m; j += 32) c += item_cost(a, n, j) + item_units(a, kv, n, j);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) c += __shfl_xor_sync(0xffffffffu, c, d);
            if (lane == src) mine += c;
        }
    }
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, mine, d);
        if (lane >= d) mine += t;
    }
    cost_s[tid] = mine;  // up to and with this thread, of its warp
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tslot;
    Waiter wait;

    if (warp >= kMmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == kLoadWarp) {
            // ---- items, and the copies of their tiles
            uint32_t n_item = 0, n_q[2] = {0, 0};
            int cached = -1;  // requests 32 cached .. are in the lanes
            Req in_lane{0, 0, 0};
            auto get = [&](int r) {
                if ((r >> 5) != cached) {
                    cached = r >> 5;
                    in_lane = load_req(a, cached * 32 + lane, false);
                }
                return Req{__shfl_sync(0xffffffffu, in_lane.q0, r & 31), __shfl_sync(0xffffffffu, in_lane.n, r & 31),
                           __shfl_sync(0xffffffffu, in_lane.kv, r & 31)};
            };
            // The warps' sums, one per lane, and their running sum: a head's cost at the last.  All heads' items in a row are cut
            // into ranges of `range` units; this CTA's is [B0, B1).
            int64_t upto = lane < kThreads / 32 ? cost_s[lane * 32 + 31] : 0;
#pragma unroll
            for (int d = 1; d < kThreads / 32; d <<= 1) {
                const int64_t t = __shfl_up_sync(0xffffffffu, upto, d);
                if (lane >= d) upto += t;
            }
            const int64_t head_cost = __shfl_sync(0xffffffffu, upto, kThreads / 32 - 1), total = head_cost * a.n_kv_heads;
            const int64_t range = max(quotient(total + gridDim.x - 1, gridDim.x), (int64_t)kMinRange);
            const int64_t B0 = min(total, blockIdx.x * range), B1 = min(total, B0 + range);
            const int snap = (int)max((int64_t)kSnapMin, min((int64_t)kSnapMax, range / 4));
            int h = 0, r = 0, j = 0;
            int64_t p = B0;  // where item (h, r, j) starts
            if (B0 < B1) {
                // the warp, then the thread, whose sum passes y, then the request, then its item
                h = (int)quotient(B0, head_cost);
                const int64_t y = B0 - h * head_cost;
                const int w = __ffs(__ballot_sync(0xffffffffu, lane < kThreads / 32 && upto > y)) - 1;
                int64_t at = __shfl_sync(0xffffffffu, upto, w) - cost_s[w * 32 + 31];
                const int64_t in_warp = cost_s[w * 32 + lane];
                const int t = __ffs(__ballot_sync(0xffffffffu, at + in_warp > y)) - 1;
                const int64_t before = __shfl_sync(0xffffffffu, in_warp, (t + 31) & 31);
                if (t > 0) at += before;
                r = (w * 32 + t) * k;
                if (k == 1) {
                    cached = w;
                    in_lane = req_s[w * 32 + lane];
                }
                for (bool found = false; !found;) {
                    const Req q = get(r);
#pragma unroll 1
                    for (int j0 = 0; j0 * per < q.n && !found; j0 += 32) {
                        const int64_t c = (j0 + lane) * per < q.n ? item_cost(a, q.n, j0 + lane) + item_units(a, q.kv, q.n, j0 + lane) : 0;
                        int64_t s = c;
                        if (q.n > per) {
#pragma unroll
                            for (int d = 1; d < 32; d <<= 1) {
                                const int64_t up = __shfl_up_sync(0xffffffffu, s, d);
                                if (lane >= d) s += up;
                            }
                        }
                        const uint32_t past = __ballot_sync(0xffffffffu, at + s > y);
                        if (past) {
                            const int src = __ffs(past) - 1;
                            j = j0 + src;
                            at += __shfl_sync(0xffffffffu, s - c, src);
                            found = true;
                        } else {
                            at += __shfl_sync(0xffffffffu, s, q.n > per ? 31 : 0);
                        }
                    }
                    if (!found && ++r >= a.n_req) found = true;  // not reached: y is below the sum of all
                }
                p = h * head_cost + at;
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the tile may be copied over
                __syncwarp();
            }
            TileLoader<D> keys(a, &a.kmap, bars, smem_u32(sKV), 0);
            auto load_q = [&](const Item& it, int s, int tok, int head) {
                if (n_q[s] > 0) wait.warp(&bars[kQEmpty + s], n_q[s] - 1);
                if (!wait.all()) return;
                const uint32_t bar = smem_u32(&bars[kQFull + s]);
                const int rows = kRows >> it.rep_log, boxed = (rows * a.inv_group >> 16) * a.group, copies = 1 << it.rep_log;
                const CUtensorMap* map = &a.qmap[it.rep_log];
                if (elect_one()) {
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar),
                                 "r"((uint32_t)(copies * kNH * boxed * 128))
                                 : "memory");
#pragma unroll 1
                    for (int c = 0; c < copies; ++c)
#pragma unroll
                        for (int half = 0; half < kNH; ++half)
                            asm volatile(
                                "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, "
                                "%3, %4}], [%5];" ::"r"(smem_u32(sQ) + s * Sh::kTile + half * kHalf + c * rows * 128),
                                "l"(map), "r"(half * 64), "r"(head * a.group), "r"(tok), "r"(bar)
                                : "memory");
                }
                __syncwarp();
                ++n_q[s];
            };
            int turn = 0;
            while (p < B1 && wait.ok) {
                const Req q = get(r);
                if (j * per >= q.n) {  // the next request with a token, in the next head if need be
                    const uint32_t more = __ballot_sync(0xffffffffu, in_lane.n > 0) & ~((2u << (r & 31)) - 1u);
                    r = more ? (r & ~31) + __ffs(more) - 1 : (r & ~31) + 32;
                    j = 0;
                    if (r >= a.n_req) {
                        r = 0;
                        ++h;
                        if (h >= a.n_kv_heads) break;
                    }
                    continue;
                }
                Item it;
                it.h = h;
                it.r = r;
                it.ntok = min(per, q.n - j * per);
                it.tok = q.q0 + j * per;
                it.pos = q.kv - q.n + j * per;
                it.kv = q.kv;
                seen_keys(a, q.kv, q.n, j * per, it.ntok, it.begin, it.end);
                it.rep_log = it.ntok * a.group <= kRows / 4 ? 2 : it.ntok * a.group <= kRows / 2 ? 1 : 0;
                it.poison = it.stop = 0;
                const int t0 = it.begin / kKeys, units = (it.end + kKeys - 1) / kKeys - t0;
                const int64_t s = p + item_cost(a, q.n, j);  // where its units start
                auto cut = [&](int64_t b) {
                    return b >= s + units ? units : b - s < snap ? 0 : s + units - b < snap ? units : (int)(b - s);
                };
                const int lo = cut(B0), hi = cut(B1);
                const bool here = units ? hi > lo : p >= B0;
                p = s + units;
                ++j;
                if (!here) continue;
                if (units == 0) {  // not into the ring: no unit of such an item would make the product warp issue what it holds back
                    no_keys<D>(a, it);
                    continue;
                }
                it.u0 = t0 + lo;
                it.nu = hi - lo;
                it.first = blockIdx.x;
                it.n_parts = 1;
                if (it.nu < units) {
                    it.first = (int)quotient(s + snap - 1, range);
                    it.n_parts = (int)quotient(s + units - snap, range) - it.first + 1;
                }
                it.slot = it.ntok > a.toks ? 2 : turn;
                if (it.slot < 2) turn ^= 1;
                const uint32_t ring = n_item % kRing;
                if (n_item >= kRing) wait.warp(&bars[kItemEmpty + ring], n_item / kRing - 1);
                if (!wait.all()) break;
                if (lane == 0) {
                    items[ring] = it;
                    mbar_arrive(&bars[kItemFull + ring]);
                }
                __syncwarp();
                ++n_item;
                keys.begin(it);
#pragma unroll 1
                for (int u = 0; u < it.nu && wait.ok; ++u) {
                    keys.tile(it, it.u0 + u, wait);
                    if (u == 0) {
#pragma unroll
                        for (int sl = 0; sl < 2; ++sl)
                            if (it.slot == 2 || it.slot == sl) load_q(it, sl, it.tok + (it.slot == 2 ? sl * a.toks : 0), h);
                    }
                }
            }
            if (wait.ok && n_item >= kRing) wait.warp(&bars[kItemEmpty + n_item % kRing], n_item / kRing - 1);
            if (wait.all() && lane == 0) {
                items[n_item % kRing].stop = 1;
                mbar_arrive(&bars[kItemFull + n_item % kRing]);
            }
            if (keys.bad) atomicOr(a.err, SCOOT_DEVERR_INDEX);
            __syncwarp();
            if (!wait.ok) {
                // gave up: the copies in flight land before the block ends
                if (lane == 0) atomicOr(a.err, SCOOT_DEVERR_TIMEOUT);
                keys.drain();
#pragma unroll
                for (int s = 0; s < 2; ++s)
                    if (n_q[s] > 0) mbar_wait_tries(smem_u32(&bars[kQFull + s]), (n_q[s] - 1) & 1u);
            }
        } else if (warp == kValueWarp) {
            // ---- the copies of the values
            TileLoader<D> vals(a, &a.vmap, bars, smem_u32(sKV), 1);
            for (uint32_t n_item = 0; wait.ok; ++n_item) {
                wait.warp(&bars[kItemFull + n_item % kRing], n_item / kRing);
                if (!wait.all()) break;
                const Item it = items[n_item % kRing];
                if (it.stop) break;
                warp_arrive(&bars[kItemEmpty + n_item % kRing]);
                vals.begin(it);
#pragma unroll 1
                for (int u = 0; u < it.nu && wait.ok; ++u) vals.tile(it, it.u0 + u, wait);
            }
            if (!wait.ok) {
                if (lane == 0) atomicOr(a.err, SCOOT_DEVERR_TIMEOUT);
                vals.drain();
            }
        } else if (warp == kMmaWarp) {
            // ---- the products.  The warp runs as one, so that the operands stay in its uniform registers, and one lane issues.
            {
                // The scores of successive (unit, slot)s go to the buffers in turn, and the product with V of the P that replaces
                // them is issued before the buffer's next scores: the scores of the next one or two run under a softmax.  todo0
                // is the oldest such product still to be issued, of n_todo, each a word: its slot and the slot's unit mod 3
                // (kSlotUnit, as the barriers are laid out), their phase, ...  This warp's instructions, six to nine cycles each, are
                // on the way of every unit: its places in the rings are counted along, and the code is short (with more
                // copies of it, it did not stay in the instruction cache).
                enum : uint32_t { kSlotUnit = 7, kPhase = 8, kAcc = 16, kRelease = 32, kVPhase = 64, kVStage = 8, kBufAt = 12 };
                constexpr uint32_t kTileDesc = Sh::kTile >> 4;
                uint32_t n_todo = 0, todo0 = 0, todo1 = 0, todo2 = 0;
                uint32_t buf = 0, n_q0 = 0, n_q1 = 0;
                uint32_t next0 = 0, next1 = 4;        // the slots' next units, as in a word
                uint32_t v_word = 1u << kVStage;      // this unit's values: stage and phase, as in a word
                const uint32_t id_s = idesc(kBf16, kKeys, false), id_o = idesc(kBf16, D, true), bar0 = smem_u32(bars);
                const uint32_t q_desc = (uint32_t)desc_k(smem_u32(sQ)), k_desc0 = (uint32_t)desc_k(smem_u32(sKV)),
                               v_desc = (uint32_t)desc_v(smem_u32(sKV));
                uint32_t k_desc = k_desc0, k_bar = bar0 + 8 * kKvFull;  // this unit's keys
                const bool leader = elect_one();
                auto commit = [&](uint32_t b) {
                    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(b) : "memory");
                };
                auto ready = [&](uint32_t b, uint32_t parity) { return __all_sync(0xffffffffu, mbar_test(b, parity)) != 0; };
                auto k_phase = [&]() { return v_word & kVPhase ? 1u : 0u; };
                auto p_bar = [&]() { return bar0 + 8 * kPFull + 8 * (todo0 & kSlotUnit); };
                auto p_phase = [&]() { return todo0 & kPhase ? 1u : 0u; };
                auto v_bar = [&]() { return bar0 + 8 * kKvFull + 8 * (todo0 >> kVStage & 15u); };
                auto v_phase = [&]() { return todo0 & kVPhase ? 1u : 0u; };
                auto issue_values = [&]() {  // by the leader: the oldest product with V
                    const uint32_t dv = v_desc + (todo0 >> kVStage & 15u) * kTileDesc;
                    const uint32_t o = tmem + Sh::kO + (todo0 & 4u ? D : 0), pp = tmem + (todo0 >> kBufAt) * kKeys;
#pragma unroll
                    for (int i = 0; i < kKeys / 16; ++i)
                        mma_ts(o, pp + 8 * i, dv + 128 * i, (uint32_t)(desc_v(0) >> 32), id_o, i > 0 || (todo0 & kAcc));
                    commit(bar0 + 8 * kPvDone + 8 * (todo0 & kSlotUnit));
                    if (todo0 & kRelease) commit(v_bar() + 8 * (kKvEmpty - kKvFull));
                };
                auto issue_scores = [&](uint32_t sl, uint32_t next, bool item_end, bool last) {
                    const uint32_t dq = q_desc + sl * kTileDesc, d = tmem + buf * kKeys;
#pragma unroll
                    for (int i = 0; i < D / 16; ++i) {
                        const uint32_t off = (i / 4) * (kHalf >> 4) + (i % 4) * 2;
                        mma_ss(d, dq + off, k_desc + off, (uint32_t)(desc_k(0) >> 32), id_s, i > 0);
                    }
                    commit(bar0 + 8 * kSFull + 8 * (next & kSlotUnit));
                    if (last) commit(k_bar + 8 * (kKvEmpty - kKvFull));
                    if (item_end) commit(bar0 + 8 * (kQEmpty + sl));
                };
                auto pop = [&]() {
                    todo0 = todo1;
                    todo1 = todo2;
                    --n_todo;
                };
                auto push = [&](uint32_t w) {
                    if (n_todo == 0) todo0 = w;
                    else if (n_todo == 1) todo1 = w;
                    else todo2 = w;
                    ++n_todo;
                    buf = buf + 1 == Sh::kBuf ? 0 : buf + 1;
                };
                auto advance = [&](uint32_t next) { return (next & 3u) == 2u ? (next - 2u) ^ kPhase : next + 1u; };
                auto values = [&]() {
                    wait.at(p_bar(), p_phase());
                    wait.at(v_bar(), v_phase());
                    fence_after();
                    if (leader) issue_values();
                    __syncwarp();
                    pop();
                };
                auto scores = [&](uint32_t sl, int u, int nu, bool last) {  // last: of this tile's users
                    if (u == 0) {
                        wait.at(bar0 + 8 * (kQFull + sl), (sl ? n_q1 : n_q0) & 1u);
                        n_q0 += sl == 0;
                        n_q1 += sl;
                    }
                    const uint32_t next = sl ? next1 : next0;
                    fence_after();
                    if (leader) issue_scores(sl, next, u == nu - 1, last);
                    __syncwarp();
                    push(next | v_word | (u > 0 ? kAcc : 0) | (last ? kRelease : 0) | buf << kBufAt);
                    if (sl) next1 = advance(next);
                    else next0 = advance(next);
                };
                for (uint32_t n_item = 0;; ++n_item) {
                    wait.at(bar0 + 8 * (kItemFull + n_item % kRing), n_item / kRing & 1u);
                    if (!wait.all()) break;
                    const volatile Item& it = items[n_item % kRing];
                    const int stop = __reduce_max_sync(0xffffffffu, it.stop), nu = __reduce_max_sync(0xffffffffu, it.nu),
                              slot = __reduce_max_sync(0xffffffffu, it.slot);
                    if (stop) break;
                    warp_arrive(&bars[kItemEmpty + n_item % kRing]);
#pragma unroll 1
                    for (int u = 0; u < nu; ++u) {
                        if (slot == 2) {
                            if (n_todo == Sh::kBuf) values();
                            wait.at(k_bar, k_phase());
                            scores(0, u, nu, false);
                            if (n_todo == Sh::kBuf) values();
                            scores(1, u, nu, true);
                        } else if (u > 0 && n_todo == Sh::kBuf &&
                                   __all_sync(0xffffffffu, mbar_test3(p_bar(), p_phase(), v_bar(), v_phase(), k_bar, k_phase()))) {
                            // all that the oldest product and these scores need is there
                            const uint32_t next = slot ? next1 : next0;
                            fence_after();
                            if (leader) {
                                issue_values();
                                issue_scores(slot, next, u == nu - 1, true);
                            }
                            __syncwarp();
                            pop();
                            push(next | v_word | kAcc | kRelease | buf << kBufAt);
                            if (slot) next1 = advance(next);
                            else next0 = advance(next);
                        } else {
                            if (n_todo == Sh::kBuf) values();
                            // a product that gets ready while the keys are on their way goes first
                            for (uint32_t i = 0; !ready(k_bar, k_phase()); ++i) {
                                if (n_todo && ready(p_bar(), p_phase())) values();
                                else wait.ok &= i < (1u << 22);
                                if (!wait.all()) break;
                            }
                            scores(slot, u, nu, true);
                        }
                        k_desc += 2 * kTileDesc;
                        k_bar += 16;
                        v_word += 2u << kVStage;
                        if (k_bar == bar0 + 8 * (kKvFull + kNS)) {
                            k_desc = k_desc0;
                            k_bar = bar0 + 8 * kKvFull;
                            v_word = (v_word - ((uint32_t)kNS << kVStage)) ^ kVPhase;
                        }
                        if (!wait.all()) break;
                    }
                    if (!wait.ok) break;
                }
                while (n_todo && wait.all()) values();
                if (!wait.ok && lane == 0) atomicOr(a.err, SCOOT_DEVERR_TIMEOUT);
                if (leader) commit(bar0 + 8 * kDrain);
                __syncwarp();
                mbar_wait_tries(smem_u32(&bars[kDrain]), 0);
            }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ---- softmax of slot s; this thread's row of tensor memory is lane row
        const int s = warp >> 2, row = tid & (kRows - 1);
        const uint32_t lane_at = (uint32_t)(32 * (warp & 3)) << 16;
        const uint32_t tO = tmem + Sh::kO + s * D + lane_at;
        // units of all slots; the next unit's score buffer; this slot's next unit mod 3, and its barriers' phase
        uint32_t n_unit = 0, buf = 0, unit = 0, uphase = 0;
        const uint32_t slot_bars = smem_u32(bars) + 32 * s;
        SlotSync wg_sync{&bars[kWg + s], 0, {}};
        for (uint32_t n_item = 0;; ++n_item) {
            const uint32_t ring = n_item % kRing;
            wait.warp(&bars[kItemFull + ring], n_item / kRing);
            wait.ok &= wg_sync.wait.ok;
            if (!wait.all()) break;
            const Item it = items[ring];
            if (it.stop) break;
            if (it.slot != 2 && it.slot != s) {
                warp_arrive(&bars[kItemEmpty + ring]);
                n_unit += it.nu;
                buf = (buf + it.nu) % Sh::kBuf;
                continue;
            }
            const int half = it.slot == 2 ? s : 0;
            const int tok0 = half * a.toks, ntok = min(a.toks, it.ntok - tok0), rows = ntok * a.group;
            const int per_copy = kRows >> it.rep_log, rr = row & (per_copy - 1), copy = row / per_copy;
            const int j = rr * a.inv_group >> 16;
            const bool live = rr < rows;
            const bool busy = __any_sync(0xffffffffu, live);
            // keys that this row sees; that every row of the slot sees
            const int pos = it.pos + tok0 + j;
            int k0, k1;
            {
                k1 = a.causal ? min(it.kv, pos + 1) : it.kv;
                k0 = a.window > 0 ? (int)max((int64_t)0, (int64_t)pos + 1 - a.window) : 0;
                if (!live) k0 = k1 = 0;
            }
            const int all1 = a.causal ? min(it.kv, it.pos + tok0 + 1) : it.kv;
            const int all0 = a.window > 0 ? (int)max((int64_t)0, (int64_t)it.pos + tok0 + ntok - a.window) : 0;
            float m = -INFINITY, l = 0.0f;
            const uint32_t step = it.slot == 2 ? 2 : 1;
            uint32_t b = (buf + (it.slot == 2 ? s : 0)) % Sh::kBuf;
            buf = (buf + step * it.nu) % Sh::kBuf;
            int t0 = it.u0 * kKeys;
#pragma unroll 1
            for (int u = 0; u < it.nu; ++u, ++n_unit, t0 += kKeys) {
                const bool full = t0 >= all0 && t0 + kKeys <= all1;
                const uint32_t at = slot_bars + 8 * unit, tS = tmem + b * kKeys + lane_at;  // the unit's barriers
                b += step;
                if (b >= Sh::kBuf) b -= Sh::kBuf;
                wait.at(at + 8 * kSFull, uphase);
                fence_after();
                if (busy) {
                    auto rescale = [&](float f) {
                        wait.warp(&bars[kPvDone + 4 * s + (unit ? unit - 1 : 2)], unit ? uphase : uphase ^ 1u);
                        fence_after();
#pragma unroll 1
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            tmem_ld16(tO + c, o);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st16(tO + c, o);
                        }
                    };
                    if (it.rep_log == 0)
                        softmax_tile<kBf16, 4>(tS, 0, full, k0 - t0, k1 - t0, a.scale_log2, u == 0, live, m, l, rescale);
                    else if (it.rep_log == 1)
                        softmax_tile<kBf16, 2>(tS, 2 * copy, full, k0 - t0, k1 - t0, a.scale_log2, u == 0, live, m, l, rescale);
                    else
                        softmax_tile<kBf16, 1>(tS, copy, full, k0 - t0, k1 - t0, a.scale_log2, u == 0, live, m, l, rescale);
                }
                if (!full) {
                    // values that some row may not see: this thread looks through those of key t0 + row
                    const uint32_t load = 2 * n_unit + 1, st = load % kNS;
                    wait.warp(&bars[kKvFull + st], load / kNS);
                    const int key = t0 + row;
                    uint4* v = reinterpret_cast<uint4*>(sKV + st * Sh::kTile + row * 128);
                    if (key < it.begin || key >= it.end) {
#pragma unroll 4
                        for (int c = 0; c < D / 8; ++c) v[(c / 8) * (kHalf / 16) + (c ^ row) % 8] = make_uint4(0, 0, 0, 0);
                    } else if (key < all0 || key >= all1) {
                        uint32_t any = 0;
#pragma unroll 4
                        for (int c = 0; c < D / 8; ++c) {
                            const uint4 w = v[(c / 8) * (kHalf / 16) + (c ^ row) % 8];
                            any |= top_exponent<kBf16>(w.x) | top_exponent<kBf16>(w.y) | top_exponent<kBf16>(w.z) | top_exponent<kBf16>(w.w);
                        }
                        if (any & 0x80008000u) {
                            *reinterpret_cast<volatile int32_t*>(&items[ring].poison) = 1;  // before the zeros can be seen
                            __threadfence_block();
#pragma unroll 1
                            for (int c = 0; c < D / 2; ++c) {
                                uint32_t* at32 = reinterpret_cast<uint32_t*>(v + (c / 32) * (kHalf / 16)) + c % 32;
                                *at32 &= ~not_finite<kBf16>(*at32);
                            }
                        }
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive_at(at + 8 * kPFull);
                if (++unit == 3) {
                    unit = 0;
                    uphase ^= 1u;
                }
            }
            // ---- the end of the item: O and l of this part
            wait.warp(&bars[kPvDone + 4 * s + (unit ? unit - 1 : 2)], unit ? uphase : uphase ^ 1u);
            fence_after();
            const bool poison = *reinterpret_cast<volatile int32_t*>(&items[ring].poison) != 0;
            if (busy) {
                // 0 times the sums: NaN if one of them is not finite (those of a row whose scores are NaN stay as they are)
                float y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    uint32_t x[32];
                    tmem_ld32(tO + c, x);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) y[i & 3] = fmaf(__uint_as_float(x[i]), 0.0f, y[i & 3]);
                }
                if (__any_sync(0xffffffffu, poison || (live && l == l && (y[0] + y[1]) + (y[2] + y[3]) != 0.0f)))
                    odd_values<kBf16, D>(a, tO, it.h, it.r, it.u0, it.nu, it.begin, it.end, k0, k1, it.rep_log, copy);
            }
            auto load_o = [&](int c, float* o) {  // columns c .. c + 31
                uint32_t x[32];
                tmem_ld32(tO + c, x);
                tmem_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = __uint_as_float(x[i]);
            };
            const int head = it.h * a.group, tok = it.tok + tok0;
            const bool whole = it.n_parts == 1;
            // parts of half 0, then those of half 1, of all CTAs
            float* part0 = a.parts + (size_t)(half * 2 * gridDim.x + 2 * it.first + 1) * kPartFloats<D>;
            float* buf = part_buf<D>(part0, blockIdx.x - it.first);
            float* scratch = reinterpret_cast<float*>(sScratch + s * kScratch);
            if (it.rep_log > 0) {
                // Copies of the rows: their common maximum and sum, then the weighted sums of their O through the scratch
                // (16-byte groups swizzled by the row), as many columns at a time as it holds of the rows in use.
                const int copies = 1 << it.rep_log, used = rows << it.rep_log;
                ml_s[s][row] = live ? make_float2(m, l) : make_float2(-INFINITY, 0.0f);
                wg_sync();
                float M = -INFINITY, L = 0.0f;
#pragma unroll 1
                for (int c = 0; c < copies; ++c) M = fmaxf(M, ml_s[s][c * per_copy + rr].x);
                const float Ms = finite_or_zero(M);
#pragma unroll 1
                for (int c = 0; c < copies; ++c) {
                    const float2 v = ml_s[s][c * per_copy + rr];
                    L = fmaf(exp2_hw(v.x - Ms), v.y, L);
                }
                const float w = exp2_hw(m - Ms), f = whole ? w * inverse_sum(L) : w, g = f == 0.0f ? 1.0f : f;
                if (copy == 0 && live) {
                    if (!whole) *reinterpret_cast<float2*>(buf + kRows * D + 2 * rr) = make_float2(M, L);
                    else if (a.lse) *lse_row(a, tok, head, rr) = L == 0.0f ? -INFINITY : (M + __log2f(L)) * kLn2;
                }
                const int width = used <= 32 ? min(D, 128) : used <= 64 ? 64 : 32, groups = width / 4;
                const int g_log = 31 - __clz(groups);
#pragma unroll 1
                for (int c0 = 0; c0 < D; c0 += width) {
                    if (busy)
#pragma unroll 1
                        for (int c = 0; c < width; c += 32) {
                            float o[32];
                            load_o(c0 + c, o);
                            if (live) {
                                if (f == 0.0f)
#pragma unroll
                                    for (int i = 0; i < 32; ++i) o[i] = weightless(o[i]);
                                const int at = copy * rows + rr;
                                float4* dst = reinterpret_cast<float4*>(scratch) + at * groups;
#pragma unroll
                                for (int i = 0; i < 8; ++i)
                                    dst[(c / 4 + i) ^ (at & 7)] = make_float4(o[4 * i] * g, o[4 * i + 1] * g, o[4 * i + 2] * g, o[4 * i + 3] * g);
                            }
                        }
                    wg_sync();
#pragma unroll 1
                    for (int e = row; e < rows << g_log; e += kRows) {
                        const int q = e >> g_log, gq = e & (groups - 1);
                        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
                        for (int c = 0; c < copies; ++c) {
                            const int at = c * rows + q;
                            const float4 v = reinterpret_cast<const float4*>(scratch)[at * groups + (gq ^ (at & 7))];
                            t = make_float4(t.x + v.x, t.y + v.y, t.z + v.z, t.w + v.w);
                        }
                        if (whole) *reinterpret_cast<uint2*>(out_row(a, tok, head, q) + c0 + 4 * gq) = make_uint2(pack16<kBf16>(t.x, t.y), pack16<kBf16>(t.z, t.w));
                        else *reinterpret_cast<float4*>(buf + q * D + c0 + 4 * gq) = t;
                    }
                    if (c0 + width < D) wg_sync();
                }
            } else if (whole) {
                const float inv = inverse_sum(l);
                if (busy) {
                    uint16_t* dst = out_row(a, tok, head, rr);
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        float o[32];
                        load_o(c, o);
                        if (live) {
#pragma unroll
                            for (int i = 0; i < 32; i += 8)
                                *reinterpret_cast<uint4*>(dst + c + i) =
                                    make_uint4(pack16<kBf16>(o[i] * inv, o[i + 1] * inv), pack16<kBf16>(o[i + 2] * inv, o[i + 3] * inv),
                                               pack16<kBf16>(o[i + 4] * inv, o[i + 5] * inv), pack16<kBf16>(o[i + 6] * inv, o[i + 7] * inv));
                        }
                    }
                    if (live && a.lse) *lse_row(a, tok, head, rr) = l == 0.0f ? -INFINITY : (m + __log2f(l)) * kLn2;
                }
            } else if (busy) {
#pragma unroll 1
                for (int c = 0; c < D; c += 32) {
                    float o[32];
                    load_o(c, o);
                    if (live) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4)
                            *reinterpret_cast<float4*>(buf + row * D + c + i) = make_float4(o[i], o[i + 1], o[i + 2], o[i + 3]);
                    }
                }
                if (live) *reinterpret_cast<float2*>(buf + kRows * D + 2 * row) = make_float2(m, l);
            }
            warp_arrive(&bars[kItemEmpty + ring]);
            if (whole) continue;
            wg_sync();
            if (row == 0) {
                __threadfence();  // (the slot's other threads' stores are before it by the barrier)
                uint32_t* cnt = a.count + 2 * it.first + half;
                const bool last = atomicAdd(cnt, 1u) == (uint32_t)it.n_parts - 1;
                if (last) *cnt = 0;
                __threadfence();
                *reinterpret_cast<volatile int*>(&last_flag[s]) = last;
            }
            wg_sync();
            if (*reinterpret_cast<volatile int*>(&last_flag[s]) == 0) continue;
            wg_sync = join_parts<kBf16, D>(a, part0, it.n_parts, rows, tok, head, scratch, wg_sync);
        }
        if (!wait.ok && lane == 0) atomicOr(a.err, SCOOT_DEVERR_TIMEOUT);
    }
    fence_before();
    __syncthreads();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u));
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// cuTensorMapEncodeTiled, from the driver (the library does not link it).
EncodeTiled encode_tiled() {
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            p = nullptr;
        }
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

// A map of n_dim dimensions, the first of 64-element rows (128-byte swizzle); strides in elements.
bool encode(CUtensorMap* map, bool bf16, const void* base, int n_dim, const cuuint64_t* dims, const int64_t* ld,
            const cuuint32_t* box) {
    cuuint64_t strides[4];
    const cuuint32_t step[4] = {1, 1, 1, 1};
    for (int i = 0; i + 1 < n_dim; ++i) strides[i] = (cuuint64_t)ld[i] * 2;
    return encode_tiled()(map, bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, n_dim,
                          const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                          CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                          CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool kBf16, int D>
scoot_status launch(scoot_ctx* ctx, AttnArgs& a, int sms, cudaStream_t st) {
    scoot_status s = scoot_workspace(ctx, (size_t)sms * kBufs * kRows * (D + 2) * sizeof(float), st);
    if (s != SCOOT_OK) return s;
    a.parts = static_cast<float*>(ctx->ws);
    auto kern = paged_attn_kernel<kBf16, D>;
    const uint32_t bit = 1u << (2 * kBf16 + (D == 128));
    if (!(ctx->smem_set & bit)) {  // once per context: the call is short
        SCOOT_CUDA(ctx, cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D>::kSmem));
        ctx->smem_set |= bit;
    }
    kern<<<(unsigned)sms, kThreads, Shape<D>::kSmem, st>>>(a);
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
    if (n_tokens < 0 || n_tokens > 0x40000000ll || n_tokens > 0x7FFFFFFFll / n_heads || n_req < 0 || n_req > 0x40000000 ||
        ld_table < 0 || ld_table > 0x40000000ll / layout->block_size)
        return scoot_fail(ctx, SCOOT_EINVAL, "n_tokens = %lld, n_req = %d or ld_table = %lld out of range", (long long)n_tokens,
                          n_req, (long long)ld_table);
    if (!(scale > 0.0f) || scale > kMaxScale)
        return scoot_fail(ctx, SCOOT_EINVAL, "scale = %g must be positive and at most %g", scale, kMaxScale);
    if (window < 0) return scoot_fail(ctx, SCOOT_EINVAL, "window = %d < 0", window);
    if (n_tokens == 0 || n_req == 0) return SCOOT_OK;
    if ((s = scoot_check_heads(ctx, "q", q, q_ld_token, q_ld_head, layout->head_dim)) != SCOOT_OK) return s;
    if ((s = scoot_check_heads(ctx, "out", out, out_ld_token, out_ld_head, layout->head_dim)) != SCOOT_OK)
        return s;
    if (!query_start || !kv_len || (ld_table && !block_table)) return scoot_fail(ctx, SCOOT_EINVAL, "an array is NULL");
    const int D = layout->head_dim, G = n_heads / layout->n_kv_heads;
    if (!encode_tiled()) return scoot_fail(ctx, SCOOT_ECUDA, "the driver has no cuTensorMapEncodeTiled");
    const int sms = std::min(scoot_sms(ctx), kMaxCtas);
    AttnArgs a = {};
    const bool bf16 = layout->dtype == SCOOT_BF16;
    {
        const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)layout->n_kv_heads, (cuuint64_t)layout->block_size,
                                    (cuuint64_t)layout->n_blocks};
        const int64_t ld[3] = {layout->ld_head, layout->ld_token, layout->ld_block};
        const cuuint32_t box[4] = {64, 1, (cuuint32_t)(layout->block_size < kKeys ? layout->block_size : kKeys), 1};
        if (!encode(&a.kmap, bf16, k_cache, 4, dims, ld, box) || !encode(&a.vmap, bf16, v_cache, 4, dims, ld, box))
            return scoot_fail(ctx, SCOOT_EINVAL, "the cache's layout has no tensor map");
    }
    for (int i = 0; i < 3; ++i) {
        const int toks = (kRows >> i) / G;
        if (toks == 0) continue;  // a token's rows do not fit: no item uses it
        const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)n_heads, (cuuint64_t)n_tokens};
        const int64_t ld[2] = {q_ld_head, q_ld_token};
        const cuuint32_t box[3] = {64, (cuuint32_t)G, (cuuint32_t)toks};
        if (!encode(&a.qmap[i], bf16, q, 3, dims, ld, box)) return scoot_fail(ctx, SCOOT_EINVAL, "q's layout has no tensor map");
    }
    while ((1 << a.bs_log) < layout->block_size) ++a.bs_log;
    a.n_heads = n_heads;
    a.n_kv_heads = layout->n_kv_heads;
    a.group = G;
    a.n_req = n_req;
    a.causal = causal != 0;
    a.window = window < ld_table * layout->block_size ? window : 0;  // no sequence is longer
    a.toks = kRows / G;
    a.inv_group = (65536 + G - 1) / G;
    a.n_tokens = n_tokens;
    a.n_blocks = layout->n_blocks;
    a.query_start = query_start;
    a.kv_len = kv_len;
    a.table = block_table;
    a.ld_table = ld_table;
    a.v = static_cast<const uint16_t*>(v_cache);
    a.ld_block = layout->ld_block;
    a.ld_token = layout->ld_token;
    a.ld_head = layout->ld_head;
    a.scale_log2 = scale * kLog2e;
    a.out = static_cast<uint16_t*>(out);
    a.out_ld_token = out_ld_token;
    a.out_ld_head = out_ld_head;
    a.lse = lse;
    a.count = ctx->d_count;
    a.err = ctx->d_err;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (bf16) return D == 128 ? launch<true, 128>(ctx, a, sms, st) : launch<true, 64>(ctx, a, sms, st);
    return D == 128 ? launch<false, 128>(ctx, a, sms, st) : launch<false, 64>(ctx, a, sms, st);
}
