// focus_kv4_decode_step: one new query per sequence against the pages of the 4-bit cache, under the rule of focus_decode_step (the new
// token at position len-1 attends key j when len-1-j <= w or its groups meet the key's groups), sequences of their own lengths.
//
// HBM-bound by its bytes (D + D / 8 per attended key of a KV head, a quarter of bf16's 4 D), but only just: at the card's copy rate an SM
// takes in 24 bytes a cycle, 43 codes, and each costs an SM about 1.5 thread instructions to become an operand of the matrix unit, where
// it has 128 a cycle.  So the kernel is laid out for few instructions per code:
//   - The rows are loaded straight into the registers of the matrix instruction that needs them.  The order in which a contraction
//     meets its dimensions is free, so lane q of a quad takes the contiguous quarter q of a key row (16 bytes at D = 128, two whole
//     blocks of scales), and lane row r of the warp the contiguous eighth r of a value row.
//   - Keys are the row operand, the query heads of the group (at most 8) the column operand: no row of a tile is padding.
//   - A code times its scale has six significant bits at most: exact in fp16, so the products with Q are the products of the values that
//     the codes stand for.  Q goes to fp16 with a power of two per head (exact but for elements 2^27 smaller than the head's largest),
//     probabilities carry a factor 2^10 into fp16, so that they lose bits only below 2^-24 of the largest.
//   - Only attended keys become rows of a tile: a warp walks the masks, lists the attended keys, and takes 16 off the list at a time.
// Every warp keeps its own maximum, sum and O; a CTA joins its warps, a second kernel the CTAs.
#include "kv4_common.cuh"

namespace focus {

constexpr int KD_GMAX = 8;
constexpr int KD_WARPS = 4;
constexpr int KD_UNIT = 64;              // keys: the grain of the split over CTAs, 16 per warp
constexpr int KD_SMS = 148;
constexpr int KD_MAX_BATCH = 1024;
constexpr int KD_LIST = 16 + 128;        // attended keys a warp has listed: what is left of a tile, and 128 more
constexpr float KD_LOG2E = 1.4426950408889634f;
constexpr float KD_LN2 = 0.6931471805599453f;
constexpr float KD_PSHIFT = 10.f;

template <int D> struct KdCfg {
    static constexpr int PER_SM = D == 256 ? 3 : 4;           // CTAs that fit an SM by their registers
    static constexpr int CTAS = KD_SMS * PER_SM;
};

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t kd_transpose(uint32_t x) {           // an 8 x 8 matrix of fp16
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
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

// words per lane: of a key row, of a value row
template <int WORDS>
__device__ __forceinline__ void kd_load(uint32_t (&r)[WORDS], const unsigned char* p) {
    if constexpr (WORDS == 1) {
        r[0] = *reinterpret_cast<const uint32_t*>(p);
    } else if constexpr (WORDS == 2) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        r[0] = x.x; r[1] = x.y;
    } else {
#pragma unroll
        for (int i = 0; i < WORDS / 4; ++i) {
            const uint4 x = reinterpret_cast<const uint4*>(p)[i];
            r[4 * i] = x.x; r[4 * i + 1] = x.y; r[4 * i + 2] = x.z; r[4 * i + 3] = x.w;
        }
    }
}

__host__ __device__ __forceinline__ int kd_cdiv(int a, int b) { return (a + b - 1) / b; }

// How the work is cut.  Every KV head of a sequence has ceil(len / 64) units of 64 keys; the units of all heads form one list, dealt out
// in equal contiguous ranges of `per` units.  A CTA whose range enters another head writes one more partial result and starts over, so
// the heads are padded to whole ranges where that still leaves no more ranges than CTAs.  The lengths are on the device, and so every
// CTA works this out for itself (a microsecond; the sums are over the sequences of the batch).
struct KdPlan {
    long long per;
    int aligned;
};

__device__ __forceinline__ int kd_length(const Kv4View& c, int b, int n, int32_t* status) {
    const int len = dep_load(c.lens + b);
    if (len < 0 || len > n) {
        kv4_report(status, KV4_BAD_LENGTH, b, len, n);
        return 0;                        // as if it were empty
    }
    return len;
}

template <int D>
__global__ void __launch_bounds__(KD_WARPS * 32, KdCfg<D>::PER_SM)
kv4_decode_kernel(const Kv4View c, const __nv_bfloat16* q, int64_t q_sb, int64_t q_sh, const uint32_t* mq_new, int batch, int Hq, int G, int n, int w,
                  float scale, float softcap, float* part, int2* ranges, __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, float* lse, int32_t* status) {
    constexpr int KW = D / 32, VW = D / 64;                    // words per lane of a key row, of a value row
    constexpr int MT = D / 16;                                 // 16-row tiles of O
    constexpr int KSB = D / 64;                                // blocks of scales in a lane's part of a key row
    __shared__ long long start_s[KD_MAX_BATCH + 1];            // first unit of each sequence
    __shared__ int len_s[KD_MAX_BATCH];
    __shared__ long long red_s[KD_WARPS][4];
    __shared__ uint32_t key_s[KD_WARPS][KD_LIST];              // listed keys: page * P + slot
    __shared__ uint8_t bit_s[KD_WARPS][KD_LIST];               // and which heads attend them
    __shared__ float xw[KD_WARPS][KD_GMAX][D + 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int g = lane >> 2, qd = lane & 3;
    const int Hkv = c.Hkv, lgP = c.lgP;
    const uint32_t pmask = (1u << lgP) - 1u;
    dep_wait();
    dep_trigger();

    // ---- the plan
    KdPlan plan;
    long long total;
    {
        const int ctas = gridDim.x;
        long long sum = 0;
        for (int b = threadIdx.x; b < batch; b += KD_WARPS * 32) {
            const int len = kd_length(c, b, n, blockIdx.x == 0 ? status : nullptr);
            len_s[b] = len;
            sum += kd_cdiv(len, KD_UNIT);
        }
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
        if (lane == 0) red_s[warp][0] = sum;
        __syncthreads();
        total = 0;
#pragma unroll
        for (int i = 0; i < KD_WARPS; ++i) total += red_s[i][0];
        total *= Hkv;
        const long long per0 = total > ctas ? (total + ctas - 1) / ctas : 1;
        // three lengths of a range to try with whole ranges per head: the shortest, an eighth and a quarter longer
        const long long cand[3] = {per0, per0 + (per0 + 7) / 8, per0 + (per0 + 3) / 4};
        long long cnt[3] = {0, 0, 0};
        for (int b = threadIdx.x; b < batch; b += KD_WARPS * 32) {
            const int u = kd_cdiv(len_s[b], KD_UNIT);
#pragma unroll
            for (int i = 0; i < 3; ++i) cnt[i] += (u + (uint32_t)cand[i] - 1u) / (uint32_t)cand[i];
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) {
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) cnt[i] += __shfl_xor_sync(0xffffffffu, cnt[i], off);
            if (lane == 0) red_s[warp][1 + i] = cnt[i];
        }
        __syncthreads();
        plan.per = per0;
        plan.aligned = 0;
#pragma unroll
        for (int i = 2; i >= 0; --i) {
            long long ranges_needed = 0;
#pragma unroll
            for (int j = 0; j < KD_WARPS; ++j) ranges_needed += red_s[j][1 + i];
            if (ranges_needed * Hkv <= ctas) { plan.per = cand[i]; plan.aligned = 1; }
        }
        // first unit of each sequence: a scan of the padded heads, by the first warp
        if (warp == 0) {
            long long base = 0;
            for (int b0 = 0; b0 < batch; b0 += 32) {
                const int b = b0 + lane;
                long long u = 0;
                if (b < batch) {
                    u = kd_cdiv(len_s[b], KD_UNIT);
                    if (plan.aligned) u = (u + plan.per - 1) / plan.per * plan.per;
                    u *= Hkv;
                }
                long long incl = u;
#pragma unroll
                for (int off = 1; off < 32; off <<= 1) {
                    const long long t = __shfl_up_sync(0xffffffffu, incl, off);
                    if (lane >= off) incl += t;
                }
                if (b < batch) start_s[b] = base + incl - u;
                base += __shfl_sync(0xffffffffu, incl, 31);
            }
            if (lane == 0) start_s[batch] = base;
        }
        __syncthreads();
        total = start_s[batch];
    }

    const long long f_end = min((long long)(blockIdx.x + 1) * plan.per, total);
    for (long long f = (long long)blockIdx.x * plan.per; f < f_end;) {
        // ---- the sequence and head of unit f
        int b;
        {
            int lo = 0, hi = batch;                            // start_s[lo] <= f < start_s[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (start_s[mid] <= f) lo = mid; else hi = mid;
            }
            b = lo;
        }
        const int len = len_s[b], units = kd_cdiv(len, KD_UNIT);
        const long long stride = plan.aligned ? (units + plan.per - 1) / plan.per * plan.per : units;
        const int hk = (int)((f - start_s[b]) / stride);
        const long long f0 = start_s[b] + hk * stride;         // the head's first unit
        const int bh = b * Hkv + hk;
        const int u0 = (int)(f - f0);
        const int u1 = (int)min((long long)units, u0 + (f_end - f));
        f = min(f_end, f0 + stride);
        if (u0 == 0 && threadIdx.x == 0)
            ranges[bh] = make_int2((int)(f0 / plan.per), (int)((f0 + units - 1) / plan.per));
        if (u0 >= u1) continue;                                // (the padding of a head)
        const int t0 = u0 * KD_UNIT, t1 = min(u1 * KD_UNIT, len), last = len - 1;

        // ---- Q as the column operand: this lane has quarter qd of head g
        uint32_t qb[MT][2];
        float qf;                                              // what a score of this lane's head is multiplied by
        {
            const __nv_bfloat16* qrow = q + (size_t)b * q_sb + (size_t)(hk * G + (g < G ? g : 0)) * q_sh + qd * (D / 4);
            uint32_t raw[D / 8];
            float top = 0.f;
#pragma unroll
            for (int i = 0; i < D / 8; ++i) {
                raw[i] = g < G ? *reinterpret_cast<const uint32_t*>(qrow + 2 * i) : 0u;
                top = fmaxf(top, fmaxf(fabsf(__uint_as_float(raw[i] << 16)), fabsf(__uint_as_float(raw[i] & 0xffff0000u))));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // 2^13 <= top * up < 2^14 (a head of zeros or of denormal numbers: as if its largest were 2^-100)
            const int e = max((int)(__float_as_uint(top) >> 23) - 127, -100);
            const float up = __uint_as_float((uint32_t)(13 - e + 127) << 23);
            qf = __uint_as_float((uint32_t)(e - 13 + 127) << 23);
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
                qb[i >> 1][i & 1] = kd_pack(__uint_as_float(raw[i] << 16) * up, __uint_as_float(raw[i] & 0xffff0000u) * up);
        }
        // scores come out as (key, head) with heads 2 qd and 2 qd + 1 in this lane; in log2 units they are S * mul, or tanh(S * cap_in) * sl2
        float mul[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float x = __shfl_sync(0xffffffffu, qf, (2 * qd + e) * 4) * c.k_scale * scale;
            mul[e] = softcap > 0.f ? x / softcap : x * KD_LOG2E;
        }
        const float cap2 = softcap * KD_LOG2E;
        uint32_t mq_all[KD_GMAX];
#pragma unroll
        for (int gg = 0; gg < KD_GMAX; ++gg) mq_all[gg] = gg < G ? dep_load(mq_new + (size_t)b * Hq + hk * G + gg) : 0u;

        const unsigned char* codes = c.pages + ((size_t)hk << lgP) * D;
        const unsigned char* scales = c.pages + c.scale_off + ((size_t)hk << lgP) * (D / 8);
        const unsigned char* masks = c.pages + c.mask_off + ((size_t)hk << lgP) * 4;
        const int32_t* table = c.table + (size_t)b * c.max_pages;

        // ---- this warp's keys: blocks of 16, every fourth one; x-th key -> position
        const int blocks = kd_cdiv(t1 - t0, 16);
        const int mine = (blocks - warp + KD_WARPS - 1) / KD_WARPS * 16;           // (may pass the end: checked per key)
        auto position = [&](int x) { return t0 + (((x >> 4) * KD_WARPS + warp) << 4) + (x & 15); };
        int scanned = 0, head = 0, tail = 0;
        int pg[4];                                             // pages of the next 128 keys
        uint32_t mk[4];                                        // and their masks
        auto fetch_pages = [&](int x0) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int x = x0 + 32 * k + lane, j = position(x);
                pg[k] = x < mine && j < t1 ? dep_load(table + (j >> lgP)) : -1;
            }
        };
        auto fetch_masks = [&](int x0) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int x = x0 + 32 * k + lane, j = position(x);
                mk[k] = 0u;
                if (x < mine && j < t1) {
                    if (pg[k] >= 0 && pg[k] < c.num_pages)
                        mk[k] = dep_load(reinterpret_cast<const uint32_t*>(masks + (size_t)pg[k] * c.page_bytes) + (j & pmask));
                    else
                        kv4_report(status, KV4_BAD_PAGE, b, j >> lgP, pg[k]);      // its keys are passed over
                }
            }
        };
        // list attended keys until a tile is full or the keys are through
        auto refill = [&] {
            while (tail - head < 16 && scanned < mine) {
                const int left = tail - head;
                if (head > 0) {
                    uint32_t kk = 0;
                    uint8_t bb = 0;
                    if (lane < left) { kk = key_s[warp][head + lane]; bb = bit_s[warp][head + lane]; }
                    __syncwarp();
                    if (lane < left) { key_s[warp][lane] = kk; bit_s[warp][lane] = bb; }
                    head = 0;
                    tail = left;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int x = scanned + 32 * k + lane, j = position(x);
                    uint32_t bits = 0;
                    if (x < mine && j < t1 && pg[k] >= 0 && pg[k] < c.num_pages) {
                        const bool local = last - j <= w;
#pragma unroll
                        for (int gg = 0; gg < KD_GMAX; ++gg)
                            if (gg < G && (local || (mq_all[gg] & mk[k]))) bits |= 1u << gg;
                    }
                    const uint32_t any = __ballot_sync(0xffffffffu, bits != 0u);
                    if (bits) {
                        const int at = tail + __popc(any & ((1u << lane) - 1u));
                        key_s[warp][at] = ((uint32_t)pg[k] << lgP) | (j & pmask);
                        bit_s[warp][at] = (uint8_t)bits;
                    }
                    tail += __popc(any);
                }
                scanned += 128;
                if (scanned < mine) { fetch_pages(scanned); fetch_masks(scanned); }
                __syncwarp();
            }
        };
        // the tile's rows: keys g and g + 8 of K, keys 2 qd, 2 qd + 1, 2 qd + 8, 2 qd + 9 of V (past the list's end: its last key, attended by no head)
        uint32_t kr[2][KW], vr[4][VW], ks[2], vs[4], bits[2];
        auto load_k = [&](int cnt) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int x = g + 8 * i, y = head + min(x, cnt - 1);
                const uint32_t key = key_s[warp][y];
                bits[i] = x < cnt ? bit_s[warp][y] : 0u;
                const size_t page = (size_t)(key >> lgP) * c.page_bytes;
                const uint32_t slot = key & pmask;
                kd_load<KW>(kr[i], codes + page + slot * D + qd * (D / 8));
                const unsigned char* sp = scales + page + slot * (D / 8) + qd * KSB;
                if constexpr (KSB == 1) ks[i] = *sp;
                else if constexpr (KSB == 2) ks[i] = *reinterpret_cast<const uint16_t*>(sp);
                else ks[i] = *reinterpret_cast<const uint32_t*>(sp);
            }
        };
        auto load_v = [&](int cnt) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int x = 2 * qd + (i & 1) + 8 * (i >> 1), y = head + min(x, cnt - 1);
                const uint32_t key = key_s[warp][y];
                const size_t page = (size_t)(key >> lgP) * c.page_bytes;
                const uint32_t slot = key & pmask;
                kd_load<VW>(vr[i], codes + page + slot * D + D / 2 + g * (D / 16));
                const unsigned char* sp = scales + page + slot * (D / 8) + D / 16;
                if constexpr (D == 64) vs[i] = sp[g >> 1];
                else if constexpr (D == 128) vs[i] = sp[g];
                else vs[i] = *reinterpret_cast<const uint16_t*>(sp + 2 * g);
            }
        };

        float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};    // of heads 2 qd, 2 qd + 1; l: this lane's keys alone
        float acc[MT][4];                                      // O: dimensions (D / 8) g + 2 i (elements 0, 1) and + 1 (2, 3), heads 2 qd, 2 qd + 1
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;

        if (mine > 0) { fetch_pages(0); fetch_masks(0); }
        refill();
        int cnt = min(16, tail - head);
        if (cnt > 0) { load_k(cnt); load_v(cnt); }
        while (cnt > 0) {
            // ---- S = K Q^T for 16 keys
            float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int wd = 0; wd < KW; ++wd) {
                uint32_t a[2][4];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    kv4_unpack8(kr[i][wd], a[i]);
                    const uint32_t two = kv4_scales(ks[i] >> (16 * (wd >> 2)));
                    const uint32_t sb = __byte_perm(two, two, (wd >> 1) & 1 ? 0x3232 : 0x1010);
#pragma unroll
                    for (int e = 0; e < 4; ++e) a[i][e] = kv4_mul2(a[i][e], sb);
                }
                mma_f16_16816(s0, a[0][0], a[1][0], a[0][1], a[1][1], qb[2 * wd][0], qb[2 * wd][1]);
                mma_f16_16816(s1, a[0][2], a[1][2], a[0][3], a[1][3], qb[2 * wd + 1][0], qb[2 * wd + 1][1]);
            }
            const uint32_t bt[2] = {bits[0] >> (2 * qd), bits[1] >> (2 * qd)};
            // the next tile's keys on their way
            head += cnt;
            __syncwarp();
            refill();
            const int nxt = min(16, tail - head);
            if (nxt > 0) load_k(nxt);
            // ---- scores of keys g (elements 0, 1) and g + 8 (2, 3) for heads 2 qd, 2 qd + 1, in log2 units
            float x[4];
            float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float t = (s0[e] + s1[e]) * mul[e & 1];
                if (softcap > 0.f) t = tanhf(t) * cap2;
                x[e] = (bt[e >> 1] >> (e & 1)) & 1u ? t : -INFINITY;
                top[e & 1] = fmaxf(top[e & 1], x[e]);
            }
#pragma unroll
            for (int off = 4; off <= 16; off <<= 1) {
                top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], off));
                top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], off));
            }
            if (__any_sync(0xffffffffu, top[0] > m_run[0] || top[1] > m_run[1])) {
                float fac[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float m_new = fmaxf(m_run[e], top[e]);
                    fac[e] = m_new == -INFINITY ? 1.f : kd_exp2(m_run[e] - m_new);
                    m_run[e] = m_new;
                    l_run[e] *= fac[e];
                }
#pragma unroll
                for (int i = 0; i < MT; ++i) { acc[i][0] *= fac[0]; acc[i][1] *= fac[1]; acc[i][2] *= fac[0]; acc[i][3] *= fac[1]; }
            }
            float p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // (a NaN score goes through; a maximum of minus infinity means that no key of the head has come yet)
                p[e] = x[e] == -INFINITY ? 0.f : kd_exp2(x[e] - m_run[e & 1] + KD_PSHIFT);
                l_run[e & 1] += p[e];
            }
            // probabilities as the column operand (key, head): two transposed 8 x 8 blocks
            const uint32_t pb0 = kd_transpose(kd_pack(p[0], p[1])), pb1 = kd_transpose(kd_pack(p[2], p[3]));
            // ---- O += V^T P
            uint32_t sab[D == 256 ? 2 : 1], scd[D == 256 ? 2 : 1];
#pragma unroll
            for (int i = 0; i < (D == 256 ? 2 : 1); ++i) {
                sab[i] = kd_no_nan(kv4_scales(__byte_perm(vs[0], vs[1], 0x0040 + 0x11 * i)));
                scd[i] = kd_no_nan(kv4_scales(__byte_perm(vs[2], vs[3], 0x0040 + 0x11 * i)));
            }
#pragma unroll
            for (int wd = 0; wd < VW; ++wd) {
                uint32_t a[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) kv4_unpack8(vr[i][wd], a[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    mma_f16_16816(acc[4 * wd + e], kv4_mul2(__byte_perm(a[0][e], a[1][e], 0x5410), sab[wd >> 1]),
                                  kv4_mul2(__byte_perm(a[0][e], a[1][e], 0x7632), sab[wd >> 1]), kv4_mul2(__byte_perm(a[2][e], a[3][e], 0x5410), scd[wd >> 1]),
                                  kv4_mul2(__byte_perm(a[2][e], a[3][e], 0x7632), scd[wd >> 1]), pb0, pb1);
            }
            if (nxt > 0) load_v(nxt);
            cnt = nxt;
        }

        // ---- join the warps
#pragma unroll
        for (int off = 4; off <= 16; off <<= 1) {
            l_run[0] += __shfl_xor_sync(0xffffffffu, l_run[0], off);
            l_run[1] += __shfl_xor_sync(0xffffffffu, l_run[1], off);
        }
        if (g == 0) {
#pragma unroll
            for (int e = 0; e < 2; ++e) { xw[warp][2 * qd + e][0] = m_run[e]; xw[warp][2 * qd + e][1] = l_run[e]; }
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<float2*>(&xw[warp][2 * qd + e][2 + (D / 8) * g + 2 * i]) = make_float2(acc[i][e], acc[i][2 + e]);
        }
        __syncthreads();
        const bool whole = u0 == 0 && u1 == units;             // the head's only range: its result, no partial one
        for (int idx = threadIdx.x; idx < G * D; idx += KD_WARPS * 32) {
            const int gg = idx / D, d = idx % D;
            float M = -INFINITY;
#pragma unroll
            for (int ww = 0; ww < KD_WARPS; ++ww) M = fmaxf(M, xw[ww][gg][0]);
            float L = 0.f, a = 0.f;
#pragma unroll
            for (int ww = 0; ww < KD_WARPS; ++ww) {
                const float wgt = xw[ww][gg][0] == -INFINITY ? 0.f : exp2f(xw[ww][gg][0] - M);
                L = fmaf(xw[ww][gg][1], wgt, L);
                a = fmaf(xw[ww][gg][2 + d], wgt, a);
            }
            if (whole) {
                o[(size_t)b * o_sb + (size_t)(hk * G + gg) * o_sh + d] = __float2bfloat16(L == 0.f ? 0.f : a / L * c.v_scale);
                if (d == 0) lse[(size_t)b * Hq + hk * G + gg] = L == 0.f ? -INFINITY : (M + log2f(L) - KD_PSHIFT) * KD_LN2;
            } else {
                float* dst = part + ((size_t)(bh + (int)blockIdx.x) * G + gg) * (D + 2);
                if (d == 0) { dst[0] = M; dst[1] = L; }
                dst[2 + d] = a;
            }
        }
        __syncthreads();                                       // the next head's results
    }
}

// One block per query head whose keys went to several CTAs: their partial results, joined by their maxima.  Partial result s of KV head bh
// is in place bh + s of the list: each step along the list of ranges moves to another head or to another CTA.
template <int D>
__global__ void __launch_bounds__(256)
kv4_merge_kernel(const Kv4View c, const float* part, const int2* ranges, int Hq, int G, int n, __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, float* lse) {
    constexpr int LANES = D / 2, ROWS = 256 / LANES, AHEAD = 8;
    __shared__ float wgt_s[KD_SMS * 4 + 1];
    __shared__ float red_s[2][8];
    __shared__ float2 acc_s[ROWS][LANES];
    const int b = blockIdx.x / Hq, hq = blockIdx.x - b * Hq, t = threadIdx.x, row = t / LANES, col = t % LANES;
    const int hk = hq / G, bh = b * c.Hkv + hk;
    dep_wait();
    dep_trigger();
    __nv_bfloat16* dst = o + (size_t)b * o_sb + (size_t)hq * o_sh + 2 * col;
    const int len = dep_load(c.lens + b);
    if (len <= 0 || len > n) {                                 // nothing to attend
        if (row == 0) dst[0] = dst[1] = __float2bfloat16(0.f);
        if (t == 0) lse[blockIdx.x] = -INFINITY;
        return;
    }
    const int2 rg = ranges[bh];
    const int cnt = rg.y - rg.x + 1;
    if (cnt == 1) return;                                      // written by its CTA
    const float* p = part + ((size_t)(bh + rg.x) * G + (hq - hk * G)) * (D + 2);
    const size_t step = (size_t)G * (D + 2);
    float2 v[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
        const int s = row + j * ROWS;
        v[j] = s < cnt ? *reinterpret_cast<const float2*>(p + s * step + 2 + 2 * col) : make_float2(0.f, 0.f);
    }
    float m = -INFINITY;
    for (int s = t; s < cnt; s += 256) m = fmaxf(m, p[s * step]);
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, off));
    if ((t & 31) == 0) red_s[0][t >> 5] = m;
    __syncthreads();
    float M = red_s[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) M = fmaxf(M, red_s[0][i]);
    float l = 0.f;
    for (int s = t; s < cnt; s += 256) {
        const float ms = p[s * step];
        const float wg = ms == -INFINITY ? 0.f : exp2f(ms - M);
        wgt_s[s] = wg;
        l = fmaf(p[s * step + 1], wg, l);
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
#pragma unroll 4
    for (int s = row + AHEAD * ROWS; s < cnt; s += ROWS) {
        const float2 x = *reinterpret_cast<const float2*>(p + s * step + 2 + 2 * col);
        const float wg = wgt_s[s];
        acc.x = fmaf(x.x, wg, acc.x);
        acc.y = fmaf(x.y, wg, acc.y);
    }
    acc_s[row][col] = acc;
    __syncthreads();
    float L = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) L += red_s[1][i];
    if (row == 0) {
#pragma unroll
        for (int r = 1; r < ROWS; ++r) { acc.x += acc_s[r][col].x; acc.y += acc_s[r][col].y; }
        const float f = L == 0.f ? 0.f : c.v_scale / L;
        dst[0] = __float2bfloat16(L == 0.f ? 0.f : acc.x * f);
        dst[1] = __float2bfloat16(L == 0.f ? 0.f : acc.y * f);
    }
    if (t == 0) lse[blockIdx.x] = L == 0.f ? -INFINITY : (M + log2f(L) - KD_PSHIFT) * KD_LN2;
}

// the partial results, one more than ranges per head, and the ranges of the heads; a function of the shape without its length
size_t kv4_decode_workspace_bytes(const focus_shape* s) {
    const size_t heads = (size_t)s->batch * s->Hkv;
    const int ctas = s->D == 256 ? KdCfg<256>::CTAS : KdCfg<128>::CTAS;
    return align_up(heads * sizeof(int2), 16) + (heads + ctas) * (s->Hq / s->Hkv) * (s->D + 2) * sizeof(float);
}

template <int D>
static int decode_d(const focus_shape* s, const Kv4View& c, const focus_tensor& q, const uint32_t* mq_new, const focus_tensor& o, float* lse, void* ws,
                    float scale, int32_t* status, cudaStream_t st) {
    const long long most = (long long)s->batch * s->Hkv * cdiv(s->n, KD_UNIT);
    const int grid = (int)(most < KdCfg<D>::CTAS ? most : KdCfg<D>::CTAS);
    const int G = s->Hq / s->Hkv;
    int2* ranges = reinterpret_cast<int2*>(ws);
    float* part = reinterpret_cast<float*>((char*)ws + align_up((size_t)s->batch * s->Hkv * sizeof(int2), 16));
    int rc = check_cuda(launch_dependent(kv4_decode_kernel<D>, dim3(grid), dim3(KD_WARPS * 32), 0, st, c, reinterpret_cast<const __nv_bfloat16*>(q.ptr),
                                         q.stride_b, q.stride_h, mq_new, s->batch, s->Hq, G, s->n, s->window, scale, s->softcap, part, ranges,
                                         reinterpret_cast<__nv_bfloat16*>(o.ptr), o.stride_b, o.stride_h, lse, status), "kv4 decode kernel launch");
    if (rc) return rc;
    return check_cuda(launch_dependent(kv4_merge_kernel<D>, dim3(s->batch * s->Hq), dim3(256), 0, st, c, part, ranges, s->Hq, G, s->n,
                                       reinterpret_cast<__nv_bfloat16*>(o.ptr), o.stride_b, o.stride_h, lse), "kv4 merge kernel launch");
}

int launch_kv4_decode(const focus_shape* s, const Kv4View& c, const focus_tensor& q, const uint32_t* mq_new, const focus_tensor& o, float* lse, void* ws,
                      float scale, int32_t* status, cudaStream_t st) {
    if (s->Hq / s->Hkv > KD_GMAX) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: more than %d query heads per KV head", KD_GMAX);
    if ((long long)s->batch * s->Hkv * cdiv(s->n, KD_UNIT) >= (1ll << 38)) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: batch * Hkv * n is too large");
    if (s->batch > KD_MAX_BATCH) return fail(FOCUS_ERR_UNSUPPORTED, "kv4 decode: more than %d sequences in one call", KD_MAX_BATCH);
    switch (s->D) {
        case 64: return decode_d<64>(s, c, q, mq_new, o, lse, ws, scale, status, st);
        case 128: return decode_d<128>(s, c, q, mq_new, o, lse, ws, scale, status, st);
        default: return decode_d<256>(s, c, q, mq_new, o, lse, ws, scale, status, st);
    }
}

}  // namespace focus
