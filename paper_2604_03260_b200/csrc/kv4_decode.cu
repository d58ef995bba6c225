// focus_kv4_decode_step: one new query per sequence against the pages of the 4-bit cache, under the rule of focus_decode_step (the new
// token at position len-1 attends key j when len-1-j <= w or its groups meet the key's groups), sequences of their own lengths.
//
// HBM-bound by its bytes (D + D / 8 per attended key of a KV head, a quarter of bf16's 4 D), but only just: at the card's copy rate an SM
// takes in 24 bytes a cycle, 16 keys of D = 128 in 96 cycles, in which its four integer pipes, which turn codes into fp16 (2 cycles a
// pair, measured) and move them about, have time for 192 warp instructions.  So the kernel is laid out for few instructions per code:
//   - The order in which a contraction meets its dimensions is free, so a lane's operands are the codes of one 16-byte piece of a key row,
//     and of one piece of a value row, in the order in which they lie there.
//   - Keys are the row operand, the query heads of the group (at most 8) the column operand: no row of a tile is padding.
//   - A code times its scale has six significant bits at most: exact in fp16, so the products with Q are the products of the values that
//     the codes stand for.  Q goes to fp16 with a power of two per head (exact but for elements 2^27 smaller than the head's largest),
//     probabilities carry a factor 2^10 into fp16, so that they lose bits only below 2^-24 of the largest.
//   - The operand of P V holds two keys per register.  Their codes are put side by side four at a time, before they are converted (2
//     instructions for 8 numbers; after it, 8).
//   - The maximum that probabilities are relative to follows the scores only when one of them is 2^5 beyond it: a vote per tile instead
//     of six exchanges.
//   - A warp walks the masks.  32 keys (16 at D = 256) that lie together, of which three quarters are attended, are a tile as they lie; of the
//     others the attended ones are listed, and as many off the list are a tile.
// Rows come through a ring in shared memory, private to a warp, by asynchronous copies: one address per 16 bytes, none for the operands.
// Every warp keeps its own maximum, sum and O; a CTA joins its warps, a second kernel the CTAs.
// Measured (32 + 8 heads of 128): 131072 keys 42.8 us, of which 11 are the plan, the first masks and copies, the joins (24 at the copy rate of all
// bytes; issue slots 61 %); 24 sequences of 1 to 16385 keys 50.5 us (25.7); 2049 keys 8.1 us.  65536 keys, 16 + 8 heads of 256, 44 % of them
// attended, with a cap: 38.8 us (11.2); there half of the issue slots are free and latency is what is left.
#include "kv4_common.cuh"
#include "f32x2.cuh"

#include <float.h>

#include <type_traits>

namespace focus {

constexpr int KD_GMAX = 8;
constexpr int KD_WARPS = 4;
constexpr int KD_SMS = 148;
constexpr int KD_MAX_BATCH = 1024;
constexpr int KD_ALONE = 256;            // keys up to which a head is one CTA's even when there are more heads than CTAs, see kd_alone
constexpr int KD_LIST = 256;             // ring of listed keys: at most 31 left over, 64 new, and those of the tiles under way
constexpr int KD_BATCH = 64;             // keys whose masks a warp looks at together (128: six registers more, 2 % slower)
constexpr float KD_LOG2E = 1.4426950408889634f;
constexpr float KD_LN2 = 0.6931471805599453f;
constexpr float KD_PSHIFT = 10.f;
constexpr float KD_SLACK = 5.f;          // 2^15 < 65504, the largest fp16 number (`limit` is rounded down, and differences of scores taken before they are scaled)

template <int D> struct KdCfg {
    static constexpr int PER_SM = D == 256 ? 3 : 4;           // CTAs that fit an SM
    static constexpr int CTAS = KD_SMS * PER_SM;
    static constexpr int SUB = D == 256 ? 1 : 2;              // a tile of the walk: 16 or 32 keys, whose copies, flags and vote are one
    static constexpr int KEYS = 16 * SUB;
    static constexpr int UNIT = KEYS * KD_WARPS;              // keys: the grain of the split over CTAs, a tile per warp
    static constexpr int TURN = (320 + UNIT - 1) / UNIT;      // units that a range loses when it enters another head, see below
    static constexpr int WHOLE = KEYS * 3 / 4;                // attended keys of an aligned tile from which on all are loaded
    static constexpr int STAGES = D == 128 ? 2 : 3;           // tiles in a warp's ring
    // a stage: rows of key codes, of value codes, of scales.  A lane reads 16 bytes of a key row (8 at D = 64), eight lanes two whole rows
    // (half rows at D = 256, where the halves of odd rows are swapped): no bank is asked twice.  Of a value row a lane reads an eighth, 4 rows
    // two apart at once: the rows are 16 bytes longer.
    static constexpr int KROW = D / 2, VROW = D / 2 + 16, SROW = D / 8;
    static constexpr int V_AT = KEYS * KROW, S_AT = V_AT + KEYS * VROW, STAGE = S_AT + KEYS * SROW;
    static constexpr int RING = KD_WARPS * STAGES * STAGE;
    static constexpr int JOIN = KD_WARPS * KD_GMAX * (D + 2) * (int)sizeof(float);         // over the rings, when they are through
    static constexpr size_t SMEM = RING > JOIN ? RING : JOIN;
};

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t kd_transpose(uint32_t x) {           // an 8 x 8 matrix of fp16
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
// (lo, lo) and (hi, hi) of a pair (lo, hi): half selections that a multiplication takes along
__device__ __forceinline__ void kd_halves(uint32_t two, uint32_t& lo, uint32_t& hi) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tmov.b32 %0, {l, l};\n\tmov.b32 %1, {h, h};\n\t}" : "=r"(lo), "=r"(hi) : "r"(two));
}
__device__ __forceinline__ uint32_t kd_pack(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float kd_exp2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// a scale of a value that is NaN (the key's are too, and make the scores NaN) counts as 0 here, so that it does not reach the heads
// that do not attend the token
__device__ __forceinline__ uint32_t kd_no_nan(uint32_t s) {
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(s), "r"(0u));
    return r;
}

__device__ __forceinline__ void kd_copy16(uint32_t dst, const unsigned char* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void kd_copy8(uint32_t dst, const unsigned char* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint32_t kd_low_high(uint32_t x, uint32_t y) { return (x & 0x0f0f0f0fu) | (y & 0xf0f0f0f0u); }

// `WORDS` words of shared memory; a key row's second half at D = 256 is 64 bytes away, in the direction that the row's place says
template <int WORDS>
__device__ __forceinline__ void kd_read(uint32_t (&r)[WORDS], const unsigned char* p) {
    if constexpr (WORDS == 1) {
        r[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (WORDS == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        r[0] = x.x; r[1] = x.y;
    } else {
        const uint4 x = *reinterpret_cast<const uint4*>(p);
        r[0] = x.x; r[1] = x.y; r[2] = x.z; r[3] = x.w;
    }
}

__host__ __device__ __forceinline__ int kd_cdiv(int a, int b) { return (a + b - 1) / b; }

// Where the flags of key x of a tile are: those of the keys x % 8, + 8, ... that one lane has, side by side.
template <int KEYS>
__device__ __forceinline__ int kd_spot(int x) { return (x & ~(KEYS - 1)) + (x & 7) * (KEYS / 8) + ((x & (KEYS - 1)) >> 3); }

// How the work is cut.  Every KV head of a sequence has ceil(len / UNIT) units; the units of all heads form one list, dealt out in equal
// contiguous ranges of `per` units.  A CTA whose range enters another head writes one more partial result and starts over, which takes as
// long as TURN units: every head ends with that many empty ones, so that such a CTA gets the fewer keys (24 ragged sequences of D = 128: 58 -> 52 us;
// 64 and 256 take the same 320 keys).
// Where whole ranges per head make no longer ranges, the heads are padded to them instead; where no sequence can be longer than a CTA's share (kd_alone),
// they are padded to `span` units, its length, and a range is whole heads (one each, CTA by CTA and with nothing to work out, where there
// are no more of them than CTAs: `direct`).  The lengths are on the device, and so every CTA works this out
// for itself (every warp for itself, up to 32 sequences); the sums are over the sequences of the batch.
struct KdPlan {
    int per, pad;                        // units of a range; heads are padded to multiples of `pad`, or by TURN (0)
};

__device__ __forceinline__ int kd_length(const Kv4View& c, int b, int n, int32_t* status) {
    const int len = dep_load(c.lens + b);
    if (len < 0 || len > n) {
        kv4_report(status, KV4_BAD_LENGTH, b, len, n);
        return 0;                        // as if it were empty
    }
    return len;
}

// units of a head in the list
template <int D>
__device__ __forceinline__ int kd_padded(int len, const KdPlan& p) {
    const int u = kd_cdiv(len, KdCfg<D>::UNIT);
    return u == 0 ? 0 : p.pad > 0 ? kd_cdiv(u, p.pad) * p.pad : u + KdCfg<D>::TURN;
}

// GP: query heads per KV head, G, rounded up to a power of two; CAP: with a cap on the scores (kernels of their own: 2049 keys
// without one 9.0 -> 8.5 us, 131072 43.7 -> 42.8)
template <int D, int GP, bool CAP>
__global__ void __launch_bounds__(KD_WARPS * 32, KdCfg<D>::PER_SM)
kv4_decode_kernel(const Kv4View c, const __nv_bfloat16* q, int64_t q_sb, int64_t q_sh, const uint32_t* mq_new, int batch, int Hq, int G, int n, int span, FixedDiv by_ctas, int w,
                  float scale, float softcap, float* part, int2* ranges, __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, float* lse, int32_t* status) {
    using C = KdCfg<D>;
    constexpr int SUB = C::SUB, KEYS = C::KEYS, STAGES = C::STAGES;
    constexpr int KW = D == 64 ? 2 : 4, KH = D == 256 ? 2 : 1;     // words a lane reads of a key row at once, and how often
    constexpr int VW = D / 64;                                 // words of a value row
    constexpr int MT = D / 16;                                 // 16-row tiles of O
    constexpr int CPT = D / 16;                                // 16-byte pieces of a token's codes
    constexpr int COPIES = 16 * CPT / 32, ROWSTEP = 32 / CPT;  // copies per lane and 16 keys; tokens apart
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int chunk_s[KD_MAX_BATCH / 32 + 1];             // first unit of every 32 sequences (more than 32 of them)
    __shared__ int red_s[KD_WARPS][5];
    __shared__ float wgt_s[KD_GMAX][KD_WARPS], sum_s[KD_GMAX][2];
    __shared__ uint2 key_s[KD_WARPS][KD_LIST];                 // listed keys: where their codes are (in 16 bytes) and scales (in 8)
    __shared__ uint2 tile_s[KD_WARPS][KD_BATCH / 16];          // where the 16 keys start of tiles that are taken as they lie
    // which heads attend a key: of the listed keys, and of the last four batches that had whole tiles (the tiles under way, at most two, are
    // of two of them, and a third is being written)
    __shared__ __align__(4) uint8_t bit_s[KD_WARPS][KD_LIST + 4 * KD_BATCH];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, qd = lane & 3;
    const int Hkv = c.Hkv, lgP = c.lgP;
    const uint32_t pmask = (1u << lgP) - 1u, lower = (1u << lane) - 1u;
    unsigned char* ring = smem + warp * STAGES * C::STAGE;
    dep_wait();
    dep_trigger();

    // ---- the plan (the host has seen to it that the list has fewer than 2^29 units)
    KdPlan plan;
    int total;
    const bool direct = span > 0 && (int)gridDim.x == batch * Hkv;
    int len0 = 0;                                              // lengths of the first 32 sequences
    if (direct) {
        plan.per = plan.pad = span;
        total = batch * Hkv * span;
    } else {
        len0 = lane < batch ? kd_length(c, lane, n, blockIdx.x == 0 && warp == 0 ? status : nullptr) : 0;
        const int ctas = gridDim.x;
        int sum = kd_cdiv(len0, C::UNIT), turns = len0 > 0 ? C::TURN : 0;
        // a wider batch: the warps share the rest out (every warp has the first 32)
        if (batch > 32) {
            int more = 0, more_turns = 0;
            for (int b = 32 + threadIdx.x; b < batch; b += KD_WARPS * 32) {
                const int len = kd_length(c, b, n, blockIdx.x == 0 ? status : nullptr);
                more += kd_cdiv(len, C::UNIT);
                more_turns += len > 0 ? C::TURN : 0;
            }
            more = __reduce_add_sync(0xffffffffu, more);
            more_turns = __reduce_add_sync(0xffffffffu, more_turns);
            if (lane == 0) { red_s[warp][0] = more; red_s[warp][4] = more_turns; }
            __syncthreads();
            if (lane < KD_WARPS) { sum += red_s[lane][0]; turns += red_s[lane][4]; }
        }
        total = (int)__reduce_add_sync(0xffffffffu, sum) * Hkv;
        const int with_turns = total + (int)__reduce_add_sync(0xffffffffu, turns) * Hkv;
        const int per0 = total > ctas ? (int)by_ctas(total + ctas - 1) : 1;
        // three lengths of a range to try with whole ranges per head: the shortest, an eighth and a quarter longer
        const int cand[3] = {per0, per0 + kd_cdiv(per0, 8), per0 + kd_cdiv(per0, 4)};
        int cnt[3];
#pragma unroll
        for (int i = 0; i < 3; ++i) cnt[i] = kd_cdiv(kd_cdiv(len0, C::UNIT), cand[i]);
        if (batch > 32) {
            int more[3] = {0, 0, 0};
            for (int b = 32 + threadIdx.x; b < batch; b += KD_WARPS * 32) {
                const int u = kd_cdiv(kd_length(c, b, n, nullptr), C::UNIT);
#pragma unroll
                for (int i = 0; i < 3; ++i) more[i] += kd_cdiv(u, cand[i]);
            }
#pragma unroll
            for (int i = 0; i < 3; ++i) {
                more[i] = __reduce_add_sync(0xffffffffu, more[i]);
                if (lane == 0) red_s[warp][1 + i] = more[i];
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (lane < KD_WARPS) cnt[i] += red_s[lane][1 + i];
        }
        plan.per = (int)by_ctas(with_turns + ctas - 1);
        plan.pad = 0;
#pragma unroll
        for (int i = 2; i >= 0; --i)
            if ((int)__reduce_add_sync(0xffffffffu, cnt[i]) * Hkv <= ctas && cand[i] <= plan.per) plan.per = plan.pad = cand[i];
        // lengths that turn out so short are left whole too (8 sequences of 200 keys of 4296 possible ones 11.6 -> 9.0 us; of 500: ragged 10.7 -> 11.3)
        if (span == 0 && batch <= 32) {
            const int longest = (int)__reduce_max_sync(0xffffffffu, kd_cdiv(len0, C::UNIT));
            if (longest <= 2 && (with_turns - total) / C::TURN <= ctas) plan.per = plan.pad = max(longest, 1);
        }
        if (span > 0) {                                        // (with_turns - total: TURN for every head that has keys)
            plan.pad = span;
            plan.per = span * max(kd_cdiv((with_turns - total) / C::TURN, ctas), 1);
        }
        int u = kd_padded<D>(len0, plan) * Hkv;
        if (batch > 32) {
            // first unit of every 32 sequences, by the first warp
            if (warp == 0) {
                int base = 0;
                for (int b0 = 0; b0 < batch; b0 += 32) {
                    if (b0 > 0) u = b0 + lane < batch ? kd_padded<D>(kd_length(c, b0 + lane, n, nullptr), plan) * Hkv : 0;
                    if (lane == 0) chunk_s[b0 / 32] = base;
                    base += __reduce_add_sync(0xffffffffu, u);
                }
                if (lane == 0) chunk_s[kd_cdiv(batch, 32)] = base;
            }
            __syncthreads();
            total = chunk_s[kd_cdiv(batch, 32)];
        } else {
            total = __reduce_add_sync(0xffffffffu, u);
        }
    }

    const int f_end = min(((int)blockIdx.x + 1) * plan.per, total);
    for (int f = (int)blockIdx.x * plan.per; f < f_end;) {
        // ---- the sequence and head of unit f (every warp for itself)
        int b, len, start;
        if (direct) {
            b = (int)blockIdx.x / Hkv;
            len = kd_length(c, b, n, status);
            start = b * Hkv * span;
            if (len == 0) break;
        } else if (batch == 1) {                               // (nothing to search: 2049 keys 8.4 -> 8.2 us)
            b = 0;
            len = __shfl_sync(0xffffffffu, len0, 0);
            start = 0;
        } else {
            int ch = 0, base = 0, l = len0;
            if (batch > 32) {
                while (ch < kd_cdiv(batch, 32) - 1 && chunk_s[ch + 1] <= f) ++ch;      // (lengths that change under the kernel do not lead beyond it)
                base = chunk_s[ch];
                if (ch > 0) l = ch * 32 + lane < batch ? kd_length(c, ch * 32 + lane, n, nullptr) : 0;
            }
            const int u = kd_padded<D>(l, plan) * Hkv;
            int incl = u;
#pragma unroll
            for (int off = 1; off < 32; off <<= 1) {
                const int t = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl += t;
            }
            incl += base;
            const uint32_t beyond = __ballot_sync(0xffffffffu, incl > f);
            if (beyond == 0) break;
            const int at = __ffs(beyond) - 1;
            b = ch * 32 + at;
            len = __shfl_sync(0xffffffffu, l, at);
            start = __shfl_sync(0xffffffffu, incl - u, at);
        }
        const int units = kd_cdiv(len, C::UNIT), stride = direct ? span : kd_padded<D>(len, plan);
        const int hk = (f - start) / stride;
        const int f0 = start + hk * stride;                    // the head's first unit
        const int bh = b * Hkv + hk;
        const int u0 = f - f0, u1 = min(units, u0 + (f_end - f));
        f = min(f_end, f0 + stride);
        if (u0 == 0 && threadIdx.x == 0) ranges[bh] = make_int2(f0 / plan.per, (f0 + units - 1) / plan.per);
        if (u0 >= u1) continue;                                // (the padding of a head)
        const int t0 = u0 * C::UNIT, t1 = min(u1 * C::UNIT, len), near = len - 1 - w;      // keys from `near` on are local

        // ---- this warp's keys: a quarter of the range, in whole tiles.  Pages are on their way two batches ahead, masks one
        const int32_t* table = c.table + (size_t)b * c.max_pages;
        const unsigned char* masks = c.pages + c.mask_off + ((size_t)hk << lgP) * 4;
        const uint32_t page16 = (uint32_t)(c.page_bytes / 16);
        const int quarter = kd_cdiv(t1 - t0, KEYS * KD_WARPS) * KEYS;
        const int k_end = min(t0 + (warp + 1) * quarter, t1);
        int next = t0 + warp * quarter;                        // keys looked at so far
        uint32_t pg[2], pg_next[2], mk[2];                     // pages of the next batch (beyond any where there is no key) and of the one after, masks
        auto fetch_pages = [&](int from) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int j = from + 32 * k + lane;
                pg_next[k] = j < k_end ? (uint32_t)dep_load(table + (j >> lgP)) : 0xffffffffu;
            }
        };
        auto fetch_masks = [&](int from) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int j = from + 32 * k + lane;
                pg[k] = pg_next[k];
                mk[k] = 0u;
                if (pg[k] < (uint32_t)c.num_pages)
                    mk[k] = dep_load(reinterpret_cast<const uint32_t*>(masks + (size_t)(pg[k] * page16) * 16) + (j & pmask));
                else if (j < k_end)
                    kv4_report(status, KV4_BAD_PAGE, b, j >> lgP, (int)pg[k]);     // its keys are passed over
            }
        };
        fetch_pages(next);
        uint32_t mq_all[GP];
#pragma unroll
        for (int gg = 0; gg < GP; ++gg) mq_all[gg] = gg < G ? dep_load(mq_new + (size_t)b * Hq + hk * G + gg) : 0u;
        fetch_masks(next);
        fetch_pages(next + KD_BATCH);
        int tail = 0, taken = 0;                               // keys listed, and taken off the list
        uint32_t whole = 0, batches = 0;                       // whole tiles of the batch still to come; batches that had some
        uint32_t under_way = 0, depth = 0;                     // where the tiles under way have their flags, 10 bits each; how many they are
        const int spot = kd_spot<KEYS>(lane);
        // look at the next batch: its whole tiles, and its other attended keys for the list
        auto look = [&] {
            uint32_t bits[2], any[2];
            whole = 0;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int j = next + 32 * k + lane;
                bits[k] = 0;                                   // (a key without a page has no group either)
#pragma unroll
                for (int gg = 0; gg < GP; ++gg)
                    if (mq_all[gg] & mk[k]) bits[k] |= 1u << gg;
                if (next + KD_BATCH > near && j >= near && pg[k] < (uint32_t)c.num_pages) bits[k] = (1u << G) - 1u;
                any[k] = __ballot_sync(0xffffffffu, bits[k] != 0u);
                if constexpr (SUB == 2) {
                    if (__popc(any[k]) >= C::WHOLE) { whole |= 1u << k; any[k] = 0; }
                } else {
                    if (__popc(any[k] & 0xffffu) >= C::WHOLE) { whole |= 1u << (2 * k); any[k] &= 0xffff0000u; }
                    if (__popc(any[k] >> 16) >= C::WHOLE) { whole |= 2u << (2 * k); any[k] &= 0xffffu; }
                }
            }
            const uint32_t slot = next + lane;
            if (whole) {
                uint8_t* flags = &bit_s[warp][KD_LIST + (batches & 3u) * KD_BATCH + spot];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    flags[32 * k] = (uint8_t)bits[k];
                    // (used where the tile is whole: then either 16 of its keys hold an attended one, and with it their first has a page)
                    if ((lane & 15) == 0) {
                        const uint32_t sl = (slot + 32 * k) & pmask;
                        tile_s[warp][2 * k + (lane >> 4)] = make_uint2(pg[k] * page16 + sl * (D / 16), pg[k] * (2 * page16) + sl * (D / 64));
                    }
                }
                ++batches;
            }
            if (any[0] | any[1]) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    if ((any[k] >> lane) & 1u) {
                        const int at = (tail + __popc(any[k] & lower)) & (KD_LIST - 1);
                        const uint32_t sl = (slot + 32 * k) & pmask;
                        key_s[warp][at] = make_uint2(pg[k] * page16 + sl * (D / 16), pg[k] * (2 * page16) + sl * (D / 64));
                        bit_s[warp][kd_spot<KEYS>(at)] = (uint8_t)bits[k];
                    }
                    tail += __popc(any[k]);
                }
            }
            next += KD_BATCH;
            if (next < k_end) {
                fetch_masks(next);
                fetch_pages(next + KD_BATCH);
            }
            __syncwarp();
        };
        // copies of 16 keys: piece `lane % CPT` of token `lane / CPT`, and on by ROWSTEP tokens; then the scales
        const int ctok = lane / CPT, piece = lane % CPT;
        const bool cv = piece >= CPT / 2;
        const unsigned char* csrc = c.pages + ((size_t)hk << lgP) * D + piece * 16;
        // (at D = 256 ROWSTEP is 2: the row's parity, which says how its halves lie, is the lane's)
        const int cdst = cv ? C::V_AT + ctok * C::VROW + (piece - CPT / 2) * 16 : ctok * C::KROW + (D == 256 ? (piece ^ ((ctok & 1) << 2)) * 16 : piece * 16);
        const int cstep = ROWSTEP * (cv ? C::VROW : C::KROW);
        constexpr int SP = D == 256 ? 2 : 1;                   // pieces of a row of scales
        const unsigned char* scales = c.pages + c.scale_off + ((size_t)hk << lgP) * (D / 8);
        const uint32_t ring_u32 = (uint32_t)__cvta_generic_to_shared(ring);
        uint32_t into = ring_u32;                              // the stage of the next tile's copies
        // the next tile's copies, if there is one: a whole tile, or KEYS keys off the list
        auto issue = [&] {
            while (whole == 0 && tail - taken < KEYS && next < k_end) look();
            uint32_t flags;
            if (whole) {
                const int t = __ffs(whole) - 1;
                whole &= whole - 1;
#pragma unroll
                for (int u = 0; u < SUB; ++u) {
                    const unsigned char* src = csrc + ctok * D + (size_t)tile_s[warp][t * SUB + u].x * 16;
#pragma unroll
                    for (int i = 0; i < COPIES; ++i) kd_copy16(into + cdst + (u * COPIES + i) * cstep, src + i * ROWSTEP * D);
                }
                // the scales: 32 rows of 8 or 16 bytes, or 16 of 32
                {
                    const unsigned char* sc = scales + (size_t)tile_s[warp][t * SUB + (SUB == 2 ? lane >> 4 : 0)].y * 8;
                    if constexpr (D == 64) kd_copy8(into + C::S_AT + lane * 8, sc + (lane & 15) * 8);
                    else kd_copy16(into + C::S_AT + lane * 16, sc + (D == 256 ? lane : lane & 15) * 16);
                }
                flags = KD_LIST + ((batches - 1) & 3u) * KD_BATCH + KEYS * t;
            } else if (tail > taken) {
                if (tail - taken < KEYS) {                     // the last ones: filled up with the last key, attended by no head
                    const uint2 pad = key_s[warp][(tail - 1) & (KD_LIST - 1)];
                    if (lane < taken + KEYS - tail) {
                        key_s[warp][(tail + lane) & (KD_LIST - 1)] = pad;
                        bit_s[warp][kd_spot<KEYS>((tail + lane) & (KD_LIST - 1))] = 0;
                    }
                    tail = taken + KEYS;
                    __syncwarp();
                }
                flags = taken & (KD_LIST - 1);
                const uint2* keys = &key_s[warp][flags];
#pragma unroll
                for (int i = 0; i < COPIES * SUB; ++i) kd_copy16(into + cdst + i * cstep, csrc + (size_t)keys[ctok + i * ROWSTEP].x * 16);
                {
                    const unsigned char* sc = scales + (size_t)keys[lane / SP].y * 8;
                    if constexpr (D == 64) kd_copy8(into + C::S_AT + lane * 8, sc);
                    else kd_copy16(into + C::S_AT + lane * 16, sc + (lane % SP) * 16);
                }
                taken += KEYS;
            } else {
                asm volatile("cp.async.commit_group;" ::: "memory");
                return;
            }
            under_way |= flags << (10 * depth);
            ++depth;
            into = into == ring_u32 + (STAGES - 1) * C::STAGE ? ring_u32 : into + C::STAGE;
            asm volatile("cp.async.commit_group;" ::: "memory");
        };
        // ---- Q as the column operand: this lane has, of head g, the dimensions of its pieces of a key row
        uint32_t raw[D / 8];
        {
            const __nv_bfloat16* qrow = q + (size_t)b * q_sb + (size_t)(hk * G + (g < G ? g : 0)) * q_sh;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                const int d = (i / (4 * KW)) * (D / 2) + qd * (8 * KW) + 2 * (i % (4 * KW));
                raw[i] = g < G ? *reinterpret_cast<const uint32_t*>(qrow + d) : 0u;
            }
        }
#pragma unroll
        for (int i = 0; i < STAGES - 1; ++i) issue();
        uint32_t qb[MT][2];
        // a score is y = S (or, with a cap, tanh(S * cap_in)) times `mul`, in log2 units; per head of this lane's two.  `mul` is kept a positive
        // number, so that a key that is not attended (y = -inf) is -inf after it and a score of 0 is 0: the sums S are below 2^35, and what is lost at
        // the lower end is below 2^-91
        float mul[2], cap_in[2];
        {
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw[i] << 16)), fabsf(__uint_as_float(raw[i] & 0xffff0000u))));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^13 <= top * up < 2^14 (a head of zeros or of denormal numbers: as if its largest were 2^-100)
            const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100);
            const float up = __uint_as_float((uint32_t)(13 - e + 127) << 23), down = __uint_as_float((uint32_t)(e - 13 + 127) << 23);
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                qb[i >> 1][i & 1] = kd_pack(__uint_as_float(raw[i] << 16) * up, __uint_as_float(raw[i] & 0xffff0000u) * up);
            // scores come out as (key, head) with heads 2 qd and 2 qd + 1 in this lane
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float x = fminf(__shfl_sync(0xffffffffu, down, (2 * qd + i) * 4) * scale * c.k_scale, FLT_MAX);
                mul[i] = fminf(fmaxf((CAP ? softcap : x) * KD_LOG2E, FLT_MIN), FLT_MAX);
                cap_in[i] = CAP ? fminf(x / softcap, FLT_MAX) : 0.f;
            }
        }

        // of heads 2 qd, 2 qd + 1; l: this lane's keys alone.  The reference is a y: near it the difference of two is exact, where products with `mul`
        // differ by their own rounding, at 2^26 by more than fp16 has room for.  One that no key has moved yet is FLT_MAX below
        // everything, and its limit such that any score but minus infinity is beyond it
        F2 n_ref = f2(FLT_MAX, FLT_MAX);                       // (minus the reference)
        float limit[2] = {-FLT_MAX, -FLT_MAX};
        F2 l_run = f2(0.f, 0.f);
        float acc[MT][4];                                      // O: dimensions (D / 8) g + 2 i (elements 0, 1) and + 1 (2, 3), heads 2 qd, 2 qd + 1
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;

        const unsigned char* st = ring;
        while (true) {
            issue();                                           // into the stage that the tile before has left
            if (depth == 0) break;
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            __syncwarp();
            uint32_t flags;                                    // of this lane's keys g, g + 8, ... a byte each; from the bit of head 2 qd on
            {
                const uint8_t* at = &bit_s[warp][(under_way & 1023u) + g * (2 * SUB)];
                flags = (SUB == 2 ? *reinterpret_cast<const uint32_t*>(at) : (uint32_t) * reinterpret_cast<const uint16_t*>(at)) >> (2 * qd);
            }
            under_way >>= 10;
            --depth;
            // ---- S = K Q^T: keys g (elements 0, 1) and g + 8 (2, 3) of 16 for heads 2 qd, 2 qd + 1; two sums in turn
            float y[SUB][4];
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                float s0[4], s1[4];
#pragma unroll
                for (int h = 0; h < KH; ++h) {
                    uint32_t kr[2][KW], sc[2][2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const int row = u * 16 + g + 8 * i;
                        kd_read<KW>(kr[i], st + row * C::KROW + (KH == 2 ? (h ^ (g & 1)) * 64 : 0) + qd * (4 * KW));
                        const unsigned char* sp = st + C::S_AT + row * C::SROW;
                        const uint32_t two = kv4_scales(D == 64 ? (uint32_t)sp[qd] : (uint32_t) * reinterpret_cast<const uint16_t*>(sp + 8 * h + 2 * qd));
                        kd_halves(two, sc[i][0], sc[i][1]);
                    }
#pragma unroll
                    for (int wd = 0; wd < KW; ++wd) {
                        uint32_t a[2][4];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            kv4_unpack8(kr[i][wd], a[i]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) a[i][e] = kv4_mul2(a[i][e], sc[i][wd >> 1]);
                        }
                        const uint32_t(*qx)[2] = &qb[2 * (h * KW + wd)];
                        if (h == 0 && wd == 0) {
                            mma_f16_16816_first(s0, a[0][0], a[1][0], a[0][1], a[1][1], qx[0][0], qx[0][1]);
                            mma_f16_16816_first(s1, a[0][2], a[1][2], a[0][3], a[1][3], qx[1][0], qx[1][1]);
                        } else {
                            mma_f16_16816(s0, a[0][0], a[1][0], a[0][1], a[1][1], qx[0][0], qx[0][1]);
                            mma_f16_16816(s1, a[0][2], a[1][2], a[0][3], a[1][3], qx[1][0], qx[1][1]);
                        }
                    }
                }
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float2 t = f2_get(f2_add(f2(s0[e], s0[e + 1]), f2(s1[e], s1[e + 1])));
                    y[u][e] = t.x;
                    y[u][e + 1] = t.y;
                }
            }
            if constexpr (CAP) {
#pragma unroll
                for (int u = 0; u < SUB; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[u][e] = tanhf(y[u][e] * cap_in[e & 1]);
            }
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
#pragma unroll
                for (int e = 0; e < 4; ++e) y[u][e] = flags & (1u << (16 * u + 8 * (e >> 1) + (e & 1))) ? y[u][e] : -INFINITY;
#pragma unroll
                for (int e = 0; e < 2; ++e) top[e] = fmaxf(top[e], fmaxf(y[u][e], y[u][e + 2]));
            }
            if (__any_sync(0xffffffffu, top[0] > limit[0] || top[1] > limit[1])) {
                float fac[2], y_ref[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    y_ref[e] = e ? -f2_get(n_ref).y : -f2_get(n_ref).x;
#pragma unroll
                    for (int off = 4; off <= 16; off <<= 1) top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], off));
                    const float y_new = fmaxf(y_ref[e], top[e]);
                    fac[e] = kd_exp2((y_ref[e] - y_new) * mul[e]);
                    y_ref[e] = y_new;
                    limit[e] = y_new == -FLT_MAX ? -FLT_MAX : __fadd_rd(y_new, KD_SLACK / mul[e]);
                }
                n_ref = f2(-y_ref[0], -y_ref[1]);
                l_run = f2_mul(l_run, f2(fac[0], fac[1]));
#pragma unroll
                for (int i = 0; i < MT; ++i) { acc[i][0] *= fac[0]; acc[i][1] *= fac[1]; acc[i][2] *= fac[0]; acc[i][3] *= fac[1]; }
            }
#pragma unroll
            for (int u = 0; u < SUB; ++u) {
                float p[4];
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const float2 t = f2_get(f2_fma(f2_add(f2(y[u][e], y[u][e + 1]), n_ref), f2(mul[0], mul[1]), f2(KD_PSHIFT, KD_PSHIFT)));
                    p[e] = kd_exp2(t.x);
                    p[e + 1] = kd_exp2(t.y);
                    l_run = f2_add(l_run, f2(p[e], p[e + 1]));
                }
                // probabilities as the column operand (key, head): two transposed 8 x 8 blocks
                const uint32_t pb0 = kd_transpose(kd_pack(p[0], p[1])), pb1 = kd_transpose(kd_pack(p[2], p[3]));
                // ---- O += V^T P: keys 2 qd, 2 qd + 1 (A, B) and 2 qd + 8, 2 qd + 9 (C, D) of 16
                uint32_t vr[4][VW], vs[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int row = u * 16 + 2 * qd + (i & 1) + 8 * (i >> 1);
                    kd_read<VW>(vr[i], st + C::V_AT + row * C::VROW + g * (D / 16));
                    const unsigned char* sp = st + C::S_AT + row * C::SROW + D / 16;
                    vs[i] = D == 64 ? sp[g >> 1] : D == 128 ? sp[g] : *reinterpret_cast<const uint16_t*>(sp + 2 * g);
                }
                uint32_t sab[D == 256 ? 2 : 1], scd[D == 256 ? 2 : 1];
#pragma unroll
                for (int i = 0; i < (D == 256 ? 2 : 1); ++i) {
                    sab[i] = kd_no_nan(kv4_scales(__byte_perm(vs[0], vs[1], 0x0040 + 0x11 * i)));
                    scd[i] = kd_no_nan(kv4_scales(__byte_perm(vs[2], vs[3], 0x0040 + 0x11 * i)));
                }
#pragma unroll
                for (int wd = 0; wd < VW; ++wd) {
                    // codes of the same dimension of two keys in a byte: even dimensions, odd ones
                    uint32_t ab[2][4], cd[2][4];
                    kv4_unpack8(kd_low_high(vr[0][wd], vr[1][wd] << 4), ab[0]);
                    kv4_unpack8(kd_low_high(vr[0][wd] >> 4, vr[1][wd]), ab[1]);
                    kv4_unpack8(kd_low_high(vr[2][wd], vr[3][wd] << 4), cd[0]);
                    kv4_unpack8(kd_low_high(vr[2][wd] >> 4, vr[3][wd]), cd[1]);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        mma_f16_16816(acc[4 * wd + e], kv4_mul2(ab[0][e], sab[wd >> 1]), kv4_mul2(ab[1][e], sab[wd >> 1]), kv4_mul2(cd[0][e], scd[wd >> 1]),
                                      kv4_mul2(cd[1][e], scd[wd >> 1]), pb0, pb1);
                }
            }
            st = st == ring + (STAGES - 1) * C::STAGE ? ring : st + C::STAGE;
            __syncwarp();                                      // the stage and its place in the list are free
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");

        // ---- join the warps
#pragma unroll
        for (int off = 4; off <= 16; off <<= 1) {
            const float2 l = f2_get(l_run);
            l_run = f2_add(l_run, f2(__shfl_xor_sync(0xffffffffu, l.x, off), __shfl_xor_sync(0xffffffffu, l.y, off)));
        }
        __syncthreads();                                       // the rings are through
        auto xw = reinterpret_cast<float(*)[KD_GMAX][D + 2]>(smem);
        if (g == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float y_ref = e ? -f2_get(n_ref).y : -f2_get(n_ref).x;
                xw[warp][2 * qd + e][0] = y_ref == -FLT_MAX ? -FLT_MAX : fmaxf(y_ref * mul[e], -FLT_MAX);      // in log2 units from here on
                xw[warp][2 * qd + e][1] = e ? f2_get(l_run).y : f2_get(l_run).x;
            }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<float2*>(&xw[warp][2 * qd + e][2 + (D / 8) * g + 2 * i]) = make_float2(acc[i][e], acc[i][2 + e]);
        }
        __syncthreads();
        // what each warp's sums count for, by the first warp: lane (head, warp)
        if (warp == 0) {
            const int gg = lane >> 2, ww = lane & 3;
            const float m = xw[ww][gg][0];
            float M = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
            M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 2));
            const float wgt = exp2f(m - M);
            float L = xw[ww][gg][1] * wgt;
            L += __shfl_xor_sync(0xffffffffu, L, 1);
            L += __shfl_xor_sync(0xffffffffu, L, 2);
            wgt_s[gg][ww] = wgt;
            if (ww == 0) { sum_s[gg][0] = M; sum_s[gg][1] = L; }
        }
        __syncthreads();
        const bool alone = u0 == 0 && u1 == units;             // the head's only range: its result, no partial one
        for (int idx = threadIdx.x; idx < G * (D / 2); idx += KD_WARPS * 32) {
            const int gg = idx / (D / 2), d = idx % (D / 2) * 2;
            float2 a = make_float2(0.f, 0.f);
#pragma unroll
            for (int ww = 0; ww < KD_WARPS; ++ww) {
                const float2 x = *reinterpret_cast<const float2*>(&xw[ww][gg][2 + d]);
                const float wgt = wgt_s[gg][ww];
                a.x = fmaf(x.x, wgt, a.x);
                a.y = fmaf(x.y, wgt, a.y);
            }
            const float M = sum_s[gg][0], L = sum_s[gg][1];
            if (alone) {
                const float f = L == 0.f ? 0.f : c.v_scale / L;
                __nv_bfloat16* dst = o + (size_t)b * o_sb + (size_t)(hk * G + gg) * o_sh + d;
                dst[0] = __float2bfloat16(L == 0.f ? 0.f : a.x * f);
                dst[1] = __float2bfloat16(L == 0.f ? 0.f : a.y * f);
                if (d == 0) lse[(size_t)b * Hq + hk * G + gg] = L == 0.f ? -INFINITY : (M + log2f(L) - KD_PSHIFT) * KD_LN2;
            } else {
                float* dst = part + ((size_t)(bh + (int)blockIdx.x) * G + gg) * (D + 2);
                if (d == 0) *reinterpret_cast<float2*>(dst) = make_float2(M, L);
                *reinterpret_cast<float2*>(dst + 2 + d) = a;
            }
        }
        __syncthreads();                                       // the next head's rows and results
    }
    // empty sequences: nothing to attend
    for (int b = blockIdx.x; b < batch; b += gridDim.x) {
        if (kd_length(c, b, n, nullptr) > 0) continue;
        for (int i = threadIdx.x; i < Hq * D; i += KD_WARPS * 32) o[(size_t)b * o_sb + (size_t)(i / D) * o_sh + i % D] = __float2bfloat16(0.f);
        for (int i = threadIdx.x; i < Hq; i += KD_WARPS * 32) lse[(size_t)b * Hq + i] = -INFINITY;
    }
}

// Joins the partial results of a query head whose keys went to several CTAs by their maxima; a block per 2 LANES dimensions: 32 where that
// leaves room for all blocks at once (ragged, 24 sequences of 32 heads: 63 us with it, 58 without), else all.  Partial result s of KV
// head bh is in place bh + s of the list: each step along the list of ranges moves to another head or to another CTA.  Latency is all of it:
// the threads form 256 / LANES rows, row r taking every so many partials, eight of a thread's loads are under way while the weights are worked out
// (74 partials of 32 heads: 3.6 us behind the partial pass; a block per head with 4 rows 7.4).
template <int D, int LANES>
__global__ void __launch_bounds__(256)
kv4_merge_kernel(const Kv4View c, const float* part, const int2* ranges, int Hq, int G, int n, __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, float* lse) {
    constexpr int ROWS = 256 / LANES, AHEAD = 8, SLICES = D / (2 * LANES);
    __shared__ float wgt_s[KD_SMS * 4 + 1];
    __shared__ float red_s[2][8];
    __shared__ float2 acc_s[ROWS][LANES + 1];
    const int head = blockIdx.x / SLICES, slice = blockIdx.x % SLICES;
    const int b = head / Hq, hq = head - b * Hq, t = threadIdx.x, row = t / LANES, col = t % LANES;
    const int hk = hq / G, bh = b * c.Hkv + hk;
    dep_wait();
    dep_trigger();
    __nv_bfloat16* dst = o + (size_t)b * o_sb + (size_t)hq * o_sh + slice * (2 * LANES) + 2 * col;
    const int len = dep_load(c.lens + b);
    const int2 rg = ranges[bh];                                // (of an empty sequence: not written, not used)
    const int cnt = rg.y - rg.x + 1;
    if (len <= 0 || len > n || cnt == 1) return;               // written by a CTA of the partial pass
    const float* p = part + ((size_t)(bh + rg.x) * G + (hq - hk * G)) * (D + 2);
    const float* pv = p + 2 + slice * (2 * LANES) + 2 * col;
    const size_t step = (size_t)G * (D + 2);
    float2 v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int s = row + j * ROWS;
        v[j] = s < cnt ? *reinterpret_cast<const float2*>(pv + s * step) : make_float2(0.f, 0.f);
    }
    float2 ml[3];                                              // maxima and sums: at most 592 partials
#pragma unroll
    for (int j = 0; j < 3; ++j) ml[j] = t + 256 * j < cnt ? *reinterpret_cast<const float2*>(p + (size_t)(t + 256 * j) * step) : make_float2(-FLT_MAX, 0.f);
    float m = fmaxf(ml[0].x, fmaxf(ml[1].x, ml[2].x));
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    if ((t & 31) == 0) red_s[0][t >> 5] = m;
    __syncthreads();
    float M = red_s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) M = fmaxf(M, red_s[0][i]);
    float l = 0.f;
#pragma unroll
    for (int j = 0; j < 3; ++j) {
        const float wg = exp2f(ml[j].x - M);
        if (t + 256 * j < cnt) wgt_s[t + 256 * j] = wg;
        l = fmaf(ml[j].y, wg, l);
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    if ((t & 31) == 0) red_s[1][t >> 5] = l;
    __syncthreads();
    float2 acc = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int s = row + j * ROWS;
        const float wg = s < cnt ? wgt_s[s] : 0.f;
        acc.x = fmaf(v[j].x, wg, acc.x);
        acc.y = fmaf(v[j].y, wg, acc.y);
    }
#pragma unroll 8
    for (int s = row + AHEAD * ROWS; s < cnt; s += ROWS) {
        const float2 x = *reinterpret_cast<const float2*>(pv + s * step);
        const float wg = wgt_s[s];
        acc.x = fmaf(x.x, wg, acc.x);
        acc.y = fmaf(x.y, wg, acc.y);
    }
    acc_s[row][col] = acc;
    __syncthreads();
    if (t >= LANES) return;
    float L = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) L += red_s[1][i];
#pragma unroll
    for (int r = 1; r < ROWS; ++r) { acc.x += acc_s[r][col].x; acc.y += acc_s[r][col].y; }
    const float f = L == 0.f ? 0.f : c.v_scale / L;
    dst[0] = __float2bfloat16(L == 0.f ? 0.f : acc.x * f);
    dst[1] = __float2bfloat16(L == 0.f ? 0.f : acc.y * f);
    if (t == 0 && slice == 0) lse[head] = L == 0.f ? -INFINITY : (M + log2f(L) - KD_PSHIFT) * KD_LN2;
}

// the partial results, one more than ranges per head, and the ranges of the heads; a function of the shape without its length
size_t kv4_decode_workspace_bytes(const focus_shape* s) {
    const size_t heads = (size_t)s->batch * s->Hkv;
    const int ctas = s->D == 256 ? KdCfg<256>::CTAS : KdCfg<128>::CTAS;
    return align_up(heads * sizeof(int2), 16) + (heads + ctas) * (s->Hq / s->Hkv) * (s->D + 2) * sizeof(float);
}

// Whether every head is one CTA's, so that nothing is merged (3 us and more), by the longest length alone.  Heads that have a CTA each: up to 8 units
// of keys, where few heads leave the machine empty up to 4 (before -> now at D = 128, us: 1 sequence of 300 keys, 8 KV heads 7.6 -> 6.8, of 600 stays 7.9, would
// be 8.9; 8 sequences of 500 12.6 -> 8.4, of 900 13.3 -> 12.1; 64 of 1000 30.6 -> 25.3, of 1800 45.7 and would be 40.0, but 30.4 -> 31.9
// when their lengths differ).  More heads than CTAs: up to KD_ALONE keys (150 sequences of 500: 45.8, would be 44.9, but 32.4 -> 37.5 when they differ).
template <int D>
static bool kd_alone(int heads, int n) {
    const int units = cdiv(n, KdCfg<D>::UNIT);
    return heads > KdCfg<D>::CTAS ? n <= KD_ALONE : units <= (heads >= 32 ? 8 : 4);
}

template <int D, int GP, bool CAP>
static int decode_dg(const focus_shape* s, const Kv4View& c, const focus_tensor& q, const uint32_t* mq_new, const focus_tensor& o, float* lse, void* ws,
                    float scale, int32_t* status, cudaStream_t st) {
    const int span = kd_alone<D>(s->batch * s->Hkv, s->n) ? cdiv(s->n, KdCfg<D>::UNIT) : 0;
    const long long most = (long long)s->batch * s->Hkv * (span > 0 ? 1 : cdiv(s->n, KdCfg<D>::UNIT));
    const int grid = (int)(most < KdCfg<D>::CTAS ? most : KdCfg<D>::CTAS);
    const int G = s->Hq / s->Hkv;
    int2* ranges = reinterpret_cast<int2*>(ws);
    float* part = reinterpret_cast<float*>((char*)ws + align_up((size_t)s->batch * s->Hkv * sizeof(int2), 16));
    int rc = check_cuda(allow_smem<kv4_decode_kernel<D, GP, CAP>>(KdCfg<D>::SMEM, true), "cudaFuncSetAttribute(kv4 decode)");
    if (rc) return rc;
    rc = check_cuda(launch_dependent(kv4_decode_kernel<D, GP, CAP>, dim3(grid), dim3(KD_WARPS * 32), KdCfg<D>::SMEM, st, c, reinterpret_cast<const __nv_bfloat16*>(q.ptr),
                                         q.stride_b, q.stride_h, mq_new, s->batch, s->Hq, G, s->n, span, fixed_div(grid), s->window, scale, s->softcap, part, ranges,
                                         reinterpret_cast<__nv_bfloat16*>(o.ptr), o.stride_b, o.stride_h, lse, status), "kv4 decode kernel launch");
    if (rc || span > 0) return rc;                             // (every head is one CTA's)
    const bool narrow = (long long)s->batch * s->Hq * (D / 32) <= KD_SMS * 8;
    const dim3 blocks(s->batch * s->Hq * (narrow ? D / 32 : 1));
    return check_cuda(launch_dependent(narrow ? kv4_merge_kernel<D, 16> : kv4_merge_kernel<D, D / 2>, blocks, dim3(256), 0, st, c, part, ranges, s->Hq, G,
                                       s->n, reinterpret_cast<__nv_bfloat16*>(o.ptr), o.stride_b, o.stride_h, lse), "kv4 merge kernel launch");
}

template <int D>
static int decode_d(const focus_shape* s, const Kv4View& c, const focus_tensor& q, const uint32_t* mq_new, const focus_tensor& o, float* lse, void* ws,
                    float scale, int32_t* status, cudaStream_t st) {
    const int G = s->Hq / s->Hkv;
    const bool cap = s->softcap > 0.f;
    auto go = [&](auto gp) {
        constexpr int GP = decltype(gp)::value;
        return cap ? decode_dg<D, GP, true>(s, c, q, mq_new, o, lse, ws, scale, status, st) : decode_dg<D, GP, false>(s, c, q, mq_new, o, lse, ws, scale, status, st);
    };
    if (G == 1) return go(std::integral_constant<int, 1>());
    if (G == 2) return go(std::integral_constant<int, 2>());
    if (G <= 4) return go(std::integral_constant<int, 4>());
    return go(std::integral_constant<int, 8>());
}

int kv4_decode_check(const focus_shape* s, const Kv4View& c) {
    if (s->scale > FLT_MAX || s->softcap > FLT_MAX) return fail(FOCUS_ERR_INVALID_ARG, "kv4 decode: scale and softcap must be finite");
    if (s->Hq / s->Hkv > KD_GMAX) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: more than %d query heads per KV head", KD_GMAX);
    if (s->batch > KD_MAX_BATCH) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: more than %d sequences in one call", KD_MAX_BATCH);
    if ((long long)s->batch * s->Hkv * cdiv(s->n, 64) >= (1ll << 28)) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: batch * Hkv * n is too large");
    // listed keys say where their codes are in 16 bytes and their scales in 8
    if ((size_t)c.num_pages * c.page_bytes >= (1ull << 35)) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: a pool of 32 GiB or more");
    return FOCUS_OK;
}

int launch_kv4_decode(const focus_shape* s, const Kv4View& c, const focus_tensor& q, const uint32_t* mq_new, const focus_tensor& o, float* lse, void* ws,
                      float scale, int32_t* status, cudaStream_t st) {
    switch (s->D) {
        case 64: return decode_d<64>(s, c, q, mq_new, o, lse, ws, scale, status, st);
        case 128: return decode_d<128>(s, c, q, mq_new, o, lse, ws, scale, status, st);
        default: return decode_d<256>(s, c, q, mq_new, o, lse, ws, scale, status, st);
    }
}

}  // namespace focus
