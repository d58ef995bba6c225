// The passes of the attention's backward: one CTA per (head, 128 rows), its tiles of columns one after another.
//   warp 0        TMA: the two row tiles once, then both column tiles of every visited tile into a ring of slots (128-byte swizzle)
//   warp 2        number, head, lse, delta and assignments of the visited tiles, through a ring of their own
//   warp 1        MMA issuer: X = R1 C1^T, Y = R2 C2^T (operands in shared memory), then the sums with P or dS (bf16, tensor memory) as the
//                 first operand and C2 or C1 read along its other dimension as the second
//   warps 4-11    P = exp2(X - lse), dS = P (Y - delta): two threads a row, each half of the tile's columns
// The tensor pipe works in order, so a product may be issued into the place of an operand that an earlier one reads.
#pragma once

#include "attn_bwd.cuh"

namespace focus {

constexpr int BWD_THREADS = 384;

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int D, int MODE, int LD>
struct BwdCfg {
    static constexpr bool KEYS = MODE != BWD_Q;
    static constexpr bool HAS_V = MODE == BWD_KV || MODE == BWD_V, HAS_DS = MODE != BWD_V;
    static constexpr int NCOL = D == 256 ? 64 : 128;             // columns of a tile
    static constexpr int NC = NCOL / 2;                          // of a thread
    static constexpr int SUBT = D / 64;
    static constexpr uint32_t SUBR = 128 * 128, SUBC = NCOL * 128;
    static constexpr uint32_t R_BYTES = SUBR * SUBT, C_BYTES = SUBC * SUBT;
    static constexpr int NR = MODE == BWD_V ? 1 : 2;             // row tiles
    static constexpr int NX = MODE == BWD_KV ? 1 : 2;            // places of X
    static constexpr int NINFO = 2;                              // tiles handed on ahead
    static constexpr uint32_t STAT_BYTES = KEYS ? 2 * NCOL * 4 : 0;
    // The columns' assignments, copied beside the tile; at D = 256 there is no room, they are read from L1 (one address a warp)
    static constexpr bool GATE_SMEM = LD > 0 && D != 256;
    static constexpr uint32_t GATE_BYTES = GATE_SMEM ? NCOL * LD * 4 : 0;
    static constexpr uint32_t INFO_BYTES = STAT_BYTES + GATE_BYTES;
    static constexpr uint32_t CTL_BYTES = 512;
    static constexpr uint32_t ROOM = 227 * 1024 - CTL_BYTES - NR * R_BYTES - NINFO * INFO_BYTES;
    static constexpr int NSLOT = ROOM / C_BYTES > 8 ? 8 : ROOM / C_BYTES;
    static_assert(NSLOT >= 3, "two tiles of columns and one ahead");
    static constexpr uint32_t OFF_C = NR * R_BYTES, OFF_INFO = OFF_C + NSLOT * C_BYTES, OFF_CTL = OFF_INFO + NINFO * INFO_BYTES;
    static constexpr uint32_t SMEM = OFF_CTL + CTL_BYTES;
    static constexpr uint32_t COL_X = 0, COL_Y = NX * NCOL, COL_A = NCOL == 64 ? 256 : NX * NCOL + (MODE == BWD_V ? 0 : NCOL);
    static constexpr uint32_t COL_V = COL_A, COL_S = MODE == BWD_KV ? COL_A + D : COL_A;       // sums with P, with dS
    static_assert(COL_S + D <= 512, "tensor memory");
};

struct BwdCtl {
    uint64_t r_full, full[8], empty[8];
    uint64_t info_full[2], info_empty[2];
    uint64_t x_full[2], p_full[2], y_full, ds_full, acc_full, dg_full;
    uint32_t limit, tmem_base;
    int abort_flag;
    int more[8];                  // of a slot with C1: whether there is a tile at all
    int tile[2], head[2];         // column tile and its head; tile -1: no more
};
static_assert(sizeof(BwdCtl) <= 512, "CTL_BYTES");

// The visited tiles of an item, in order; run by the whole TMA warp
template <bool KEYS, int NCOL>
struct BwdWalk {
    const BwdParams& p;
    const int lane;
    int row_tile, b, h, hi, c, word;      // hi: query head of the group; c: next 128-tile; word: of 32 tiles, which are visited
    uint32_t bits;
    int part = NCOL == 64 ? 1 : 0;        // halves of a 128-tile
    int at = -1;
    __device__ __forceinline__ int first_col() const { return KEYS ? row_tile : 0; }
    __device__ __forceinline__ int end_col() const { return KEYS ? p.nt : row_tile + 1; }
    __device__ __forceinline__ BwdWalk(const BwdParams& p_, int lane_, int rt, int b_, int h_) : p(p_), lane(lane_), row_tile(rt), b(b_), h(h_), hi(0), bits(0) {
        c = first_col();
        word = c - 32;
    }
    __device__ __forceinline__ int query_head() const { return b * p.Hq + (KEYS ? h * p.G + hi : h); }
    // next tile in units of NCOL columns, or -1
    __device__ __forceinline__ int next() {
        if (NCOL == 64 && part == 0) {
            part = 1;
            return 2 * at + 1;
        }
        for (;;) {
            if (bits) {
                at = word + __ffs(bits) - 1;
                bits &= bits - 1;
                part = 0;
                return NCOL == 64 ? 2 * at : at;
            }
            word += 32;
            if (word >= end_col()) {
                if (!KEYS || ++hi >= p.G) return -1;
                word = first_col();
            }
            const int t = word + lane;
            bool use = t < end_col();
            if (use && p.live) {
                const int a = KEYS ? t : row_tile, k = KEYS ? row_tile : t;
                const int d = a * 128 - p.w;                       // key tiles before d / 128 are far
                if (d > 0 && k < (d >> 7)) use = dep_load(p.live + ((size_t)query_head() * p.nt + a) * p.nkw + (k >> 5)) >> (k & 31) & 1;
            }
            bits = __ballot_sync(0xffffffffu, use);
        }
    }
};

template <int D, int MODE, bool CAP, int LD>
__global__ void __launch_bounds__(BWD_THREADS, 1)
attn_bwd_kernel(const __grid_constant__ CUtensorMap tm_r1, const __grid_constant__ CUtensorMap tm_r2, const __grid_constant__ CUtensorMap tm_c1,
                const __grid_constant__ CUtensorMap tm_c2, const __grid_constant__ BwdParams p) {
    using C = BwdCfg<D, MODE, LD>;
    constexpr bool KEYS = C::KEYS;
    constexpr int NCOL = C::NCOL, NC = C::NC, NX = C::NX;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    BwdCtl& ctl = *reinterpret_cast<BwdCtl*>(smem_raw + C::OFF_CTL);
    const uint32_t base = smem_u32(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // the longest items first: key tile 0, or the last query tile
    const int q0 = p.by_heads.div((int)blockIdx.x), head = (int)blockIdx.x - q0 * p.heads;
    const int row_tile = KEYS ? q0 : p.nt - 1 - q0;
    const int b = p.by_rows_H.div(head), h = head - b * (KEYS ? p.Hkv : p.Hq);
    auto give_up = [&](int where) {
        *(volatile int*)&ctl.abort_flag = 1;
        if (p.status && atomicCAS(p.status, 0, 1) == 0) {
            p.status[1] = where; p.status[2] = row_tile; p.status[3] = (int)blockIdx.x;
        }
    };
    int bad = 0;                            // where a wait gave up
    // (bounded; few instructions: the try in front of the loop is what runs)
    auto wait = [&](uint64_t& bar, uint32_t parity, int where) -> bool {
        if (mbar_try_wait(smem_u32(&bar), parity)) return true;
        uint32_t t0 = 0;
#pragma unroll 1
        for (;;) {
            if (mbar_try_wait(smem_u32(&bar), parity)) return true;
            const uint32_t now = wait_ticks(globaltimer_ns()) | 1u;
            if (t0 == 0) t0 = now;
            if (*(volatile int*)&ctl.abort_flag || wait_over(t0, now, ctl.limit)) break;
        }
        bad = where;
        return false;
    };
    if (base & 1023u) {                     // the operands' swizzle is a function of the address
        if (threadIdx.x == 0 && p.status && atomicCAS(p.status, 0, 1) == 0) { p.status[1] = 2; p.status[2] = 0; p.status[3] = (int)blockIdx.x; }
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&ctl.r_full), 1);
        for (int s = 0; s < C::NSLOT; ++s) { mbar_init(smem_u32(&ctl.full[s]), 1); mbar_init(smem_u32(&ctl.empty[s]), 1); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&ctl.info_full[x]), 1);
            mbar_init(smem_u32(&ctl.info_empty[x]), 8);             // (warps 4 to 11)
            mbar_init(smem_u32(&ctl.x_full[x]), 1);
            mbar_init(smem_u32(&ctl.p_full[x]), 256);
        }
        mbar_init(smem_u32(&ctl.y_full), 1);
        mbar_init(smem_u32(&ctl.ds_full), 256);
        mbar_init(smem_u32(&ctl.acc_full), 1);
        mbar_init(smem_u32(&ctl.dg_full), 128);
        ctl.abort_flag = 0;
        ctl.limit = wait_limit(4000000000ull);
        fence_mbar_init();
    }
    if constexpr (C::GATE_SMEM) {           // (rows of assignments past the end of a sequence are not copied)
        for (int e = threadIdx.x; e < C::NINFO * (int)C::INFO_BYTES / 4; e += BWD_THREADS) reinterpret_cast<float*>(smem_raw + C::OFF_INFO)[e] = 0.f;
        fence_proxy_async_smem();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(&ctl.tmem_base), 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = ctl.tmem_base;
    dep_wait();
    dep_trigger();

    if (warp < 4) reg_dec<REGS_CONTROL>();
    if (warp == 0) {
        // ------------------------------------------------------------------ TMA: row tiles, column tiles
        const int hk = KEYS ? h : h / p.G;
        if (lane == 0) {
            mbar_arrive_expect_tx(smem_u32(&ctl.r_full), C::NR * C::R_BYTES);
#pragma unroll 1
            for (int c = 0; c < C::SUBT; ++c) {
                tma_load_4d(base + c * C::SUBR, &tm_r1, smem_u32(&ctl.r_full), c * 64, row_tile * 128, h, b);
                if (C::NR == 2) tma_load_4d(base + C::R_BYTES + c * C::SUBR, &tm_r2, smem_u32(&ctl.r_full), c * 64, row_tile * 128, h, b);
            }
        }
        BwdWalk<KEYS, NCOL> walk(p, lane, row_tile, b, h);
        RingAt<C::NSLOT> slot;
        for (;;) {
            const int t = walk.next();
            const int hc = KEYS ? h * p.G + walk.hi : hk;           // head of the columns
#pragma unroll
            for (int x = 0; x < 2; ++x, slot.next()) {
                if (!wait(ctl.empty[slot.slot], slot.phase ^ 1, 11)) break;
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&ctl.full[slot.slot]);
                    if (x == 0) ctl.more[slot.slot] = t >= 0;
                    if (t < 0) {
                        mbar_arrive(bar);
                    } else {
                        mbar_arrive_expect_tx(bar, C::C_BYTES);
#pragma unroll
                        for (int c = 0; c < C::SUBT; ++c)
                            tma_load_4d(base + C::OFF_C + slot.slot * C::C_BYTES + c * C::SUBC, x ? &tm_c2 : &tm_c1, bar, c * 64, t * NCOL, hc, b);
                    }
                }
                __syncwarp();
                if (t < 0) break;
            }
            if (bad || t < 0) break;
        }
        if (bad && lane == 0) give_up(bad);
        __syncwarp();
    } else if (warp == 2) {
        // ------------------------------------------------------------------ what the other warps need to know of a tile
        const int hk = KEYS ? h : h / p.G;
        BwdWalk<KEYS, NCOL> walk(p, lane, row_tile, b, h);
        RingAt<C::NINFO> handed;
        for (;;) {
            const int t = walk.next();
            const int hc = KEYS ? h * p.G + walk.hi : hk;
            if (!wait(ctl.info_empty[handed.slot], handed.phase ^ 1, 12)) break;
            if (lane == 0) {
                const uint32_t bar = smem_u32(&ctl.info_full[handed.slot]), at = base + C::OFF_INFO + handed.slot * C::INFO_BYTES;
                ctl.tile[handed.slot] = t;
                ctl.head[handed.slot] = hc;
                const int rows = min(NCOL, p.n - t * NCOL);           // (a half tile may lie past the end)
                const uint32_t gbytes = C::GATE_SMEM && t >= 0 && rows > 0 ? (uint32_t)rows * LD * 4 : 0u;
                if (t < 0 || C::STAT_BYTES + gbytes == 0) {
                    mbar_arrive(bar);
                } else {
                    mbar_arrive_expect_tx(bar, C::STAT_BYTES + gbytes);
                    if constexpr (KEYS) {
                        const float* st = p.stat + ((size_t)(b * p.Hq + hc) * p.nt + t * NCOL / 128) * 256 + t * NCOL % 128;
                        bulk_load(at, st, NCOL * 4, bar);
                        bulk_load(at + NCOL * 4, st + 128, NCOL * 4, bar);
                    }
                    if (gbytes) bulk_load(at + C::STAT_BYTES, p.g + ((size_t)b * p.n + (size_t)t * NCOL) * (LD > 0 ? LD : 1), gbytes, bar);
                }
            }
            __syncwarp();
            handed.next();
            if (t < 0) break;
        }
        if (bad && lane == 0) give_up(bad);
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer
        constexpr uint32_t IDESC_X = idesc_bf16(128, NCOL, 0, 0), IDESC_A = idesc_bf16(128, D, 0, 1);
        const uint32_t r1 = (uint32_t)smem_desc_sw128(base, 16, 1024), r2 = r1 + (C::R_BYTES >> 4);
        const uint32_t ck = (uint32_t)smem_desc_sw128(base + C::OFF_C, 16, 1024);                  // columns along D
        const uint32_t cm = (uint32_t)smem_desc_sw128(base + C::OFF_C, C::SUBC, 1024);             // along the tokens
        RingAt<C::NSLOT> slot;              // next slot to be taken, in the ring's order: C1 of a tile with its X, C2 with its Y (without Y, behind X)
        auto take = [&](uint32_t& at, int where) -> bool {
            at = slot.slot;
            if (!wait(ctl.full[at], slot.phase, where)) return false;
            slot.next();
            tc_fence_after();
            return true;
        };
        auto product = [&](uint32_t d, uint32_t r, uint32_t at) {
            const uint32_t c = ck + at * (C::C_BYTES >> 4);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) umma_ss_lo(d, r + (ks >> 2) * (C::SUBR >> 4) + (ks & 3) * 2, c + (ks >> 2) * (C::SUBC >> 4) + (ks & 3) * 2, IDESC_X, ks > 0);
        };
        // the two halves of the columns lie NC columns of tensor memory apart
        auto sum = [&](uint32_t d, uint32_t a, uint32_t at, bool more) {
            const uint32_t c = cm + at * (C::C_BYTES >> 4);
#pragma unroll
            for (int ks = 0; ks < NCOL / 16; ++ks) umma_ts_lo(d, a + (ks / (NC / 16)) * NC + (ks % (NC / 16)) * 8, c + ks * 128, IDESC_A, more || ks > 0);
        };
        // X of the next tile into place u; false: there is none (or `bad`)
        auto issue_x = [&](uint32_t u, uint32_t& c1) -> bool {
            if (!take(c1, 21)) return false;
            if (!*(volatile int*)&ctl.more[c1]) return false;
            if (elect_one()) {
                product(tmem + C::COL_X + u * NCOL, r1, c1);
                umma_commit(smem_u32(&ctl.x_full[u]));
                if (!C::HAS_DS) umma_commit(smem_u32(&ctl.empty[c1]));
            }
            __syncwarp();
            return true;
        };
        auto issue_y = [&](uint32_t& c2) -> bool {
            if (!take(c2, 22)) return false;
            if (elect_one()) {
                product(tmem + C::COL_Y, r2, c2);
                umma_commit(smem_u32(&ctl.y_full));
                if (!C::HAS_V) umma_commit(smem_u32(&ctl.empty[c2]));
            }
            __syncwarp();
            return true;
        };
        do {
            if (!wait(ctl.r_full, 0, 20)) break;
            tc_fence_after();
            uint32_t a1 = 0, a2 = 0, b1 = 0, b2 = 0;       // slots of tile t and of the next
            if (!issue_x(0, a1)) break;                    // (every item has its diagonal tile)
            if (C::HAS_DS ? !issue_y(a2) : !take(a2, 22)) break;
            bool next = false;                             // X of tile t + 1 has been issued
            if (NX == 2) {
                next = issue_x(1, b1);
                if (bad || (next && !C::HAS_DS && !take(b2, 22))) break;
            }
            for (uint32_t t = 0;; ++t) {
                const uint32_t i = NX == 2 ? t & 1 : 0;
                if (C::HAS_V) {
                    if (!wait(ctl.p_full[i], (NX == 2 ? t >> 1 : t) & 1, 24)) break;
                    tc_fence_after();
                    if (elect_one()) {
                        sum(tmem + C::COL_V, tmem + C::COL_X + i * NCOL, a2, t > 0);
                        umma_commit(smem_u32(&ctl.empty[a2]));
                    }
                    __syncwarp();
                    if (NX == 1) {
                        next = issue_x(0, b1);
                        if (bad) break;
                    }
                }
                if (C::HAS_DS) {
                    if (!wait(ctl.ds_full, t & 1, 25)) break;
                    tc_fence_after();
                    if (elect_one()) {
                        sum(tmem + C::COL_S, tmem + C::COL_Y, a1, t > 0);
                        umma_commit(smem_u32(&ctl.empty[a1]));
                    }
                    __syncwarp();
                    if (next && !issue_y(b2)) break;
                }
                if (!next) {
                    if (elect_one()) umma_commit(smem_u32(&ctl.acc_full));
                    __syncwarp();
                    break;
                }
                a1 = b1;
                a2 = b2;
                if (NX == 2) {
                    next = issue_x(i, b1);
                    if (bad || (next && !C::HAS_DS && !take(b2, 22))) break;
                }
            }
        } while (false);
        if (bad && lane == 0) give_up(bad);
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ P, dS, results
        reg_inc<REGS_SOFTMAX_2WG>();
        const int half = (warp - 4) >> 2;                  // of the tile's columns
        const int row_in_tile = ((warp & 3) << 5) | lane;
        const int row = row_tile * 128 + row_in_tile;      // position of this thread's token
        const bool valid = row < p.n;
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tm = tmem + lane_base;
        const float sl2 = CAP ? p.softcap * LOG2E : p.scale * LOG2E;
        const float cap_in = CAP ? p.scale / p.softcap : 0.f;
        float lrow = 0.f, drow = 0.f;                      // rows are queries: lse and delta of the row
        if constexpr (!KEYS) {
            const float* st = p.stat + ((size_t)head * p.nt + row_tile) * 256 + row_in_tile;
            lrow = dep_load(st);
            drow = dep_load(st + 128);
        }
        uint32_t mask = 0;
        if (p.bits) mask = valid ? dep_load(p.row_mask + (size_t)head * p.n + row) & (0xffffffffu >> (32 - p.K)) : 0u;
        constexpr int LDR = LD > 0 ? LD : 1;
        float gr[LDR], dg[LDR];                            // assignment of the row times -lambda log2(e), its gradient
        if constexpr (LD > 0) {
#pragma unroll
            for (int e = 0; e < LD; ++e) {
                gr[e] = valid ? dep_load(p.g + ((size_t)b * p.n + row) * LD + e) * (-p.lambda * LOG2E) : 0.f;
                dg[e] = 0.f;
            }
        }
        RingAt<C::NINFO> taken;
        uint32_t t = 0;
        for (;; ++t) {
            if (!wait(ctl.info_full[taken.slot], taken.phase, 39)) break;
            const int ct = *(volatile int*)&ctl.tile[taken.slot];
            if (ct < 0) break;
            const float* const info = reinterpret_cast<const float*>(smem_raw + C::OFF_INFO + taken.slot * C::INFO_BYTES) + half * NC;
            const float* const gcol = reinterpret_cast<const float*>(smem_raw + C::OFF_INFO + taken.slot * C::INFO_BYTES + C::STAT_BYTES) + half * NC * LDR;
            // ---- which columns count: bit c of word c / 32
            const int col0 = ct * NCOL + half * NC;
            auto gate_row = [&](int c) -> const float4* {
                return reinterpret_cast<const float4*>(C::GATE_SMEM ? gcol + c * LDR : p.g + ((size_t)b * p.n + min(col0 + c, p.n - 1)) * LDR);
            };
            uint32_t kw[NC / 32];
            bool masked;
            {
                const int lo_q = KEYS ? ct * NCOL : row_tile * 128, hi_q = KEYS ? ct * NCOL + NCOL - 1 : row_tile * 128 + 127;
                const int lo_k = KEYS ? row_tile * 128 : ct * NCOL, hi_k = KEYS ? row_tile * 128 + 127 : ct * NCOL + NCOL - 1;
                const bool causal = lo_q < hi_k, outside = hi_q - lo_k > p.w, far = lo_q - hi_k > p.w;
                masked = causal || (p.bits && outside);
                if (masked) {
#pragma unroll
                    for (int q = 0; q < NC / 32; ++q) kw[q] = 0xffffffffu;
                    if (p.bits && outside) {
#pragma unroll
                        for (int q = 0; q < NC / 32; ++q) kw[q] = 0u;
                        const uint32_t* gb = p.bits + ((size_t)(b * (KEYS ? p.Hq : p.Hkv) + ctl.head[taken.slot]) * p.nt + ct * NCOL / 128) * p.K * 4 + (col0 % 128) / 32;
#pragma unroll 1
                        for (uint32_t rem = mask; rem; rem &= rem - 1) {
                            const uint32_t* x = gb + (__ffs(rem) - 1) * 4;
#pragma unroll
                            for (int q = 0; q < NC / 32; ++q) kw[q] |= dep_load(x + q);
                        }
                        if (!far) {
#pragma unroll
                            for (int q = 0; q < NC / 32; ++q)        // inside the window: queries up to j + w, keys from i - w on
                                kw[q] |= KEYS ? low_bits(row - col0 - 32 * q + p.w + 1) : ~low_bits(row - p.w - col0 - 32 * q);
                        }
                    }
                    if (causal) {
#pragma unroll
                        for (int q = 0; q < NC / 32; ++q) kw[q] &= KEYS ? ~low_bits(row - col0 - 32 * q) : low_bits(row + 1 - col0 - 32 * q);
                    }
                }
            }
            // ---- P
            const uint32_t xb = NX == 2 ? t & 1 : 0;
            if (!wait(ctl.x_full[xb], NX == 2 ? (t >> 1) & 1 : t & 1, 30)) break;
            tc_fence_after();
            const uint32_t t_x = tm + C::COL_X + xb * NCOL + half * NC, t_y = tm + C::COL_Y + half * NC;
            float pr[NC];                                  // P times the slope of the logit
            float da[LD > 0 ? NC : 1];                     // gate: what turns ds into the gradient of g_i . g_j
#pragma unroll
            for (int c = 0; c < NC; c += 32) {
                uint32_t sr[32];
                tmem_ld32(t_x + c, sr);
                tmem_wait_ld();
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    float l[4];
                    if constexpr (KEYS) *reinterpret_cast<float4*>(l) = *reinterpret_cast<const float4*>(info + c + e);
                    else l[0] = l[1] = l[2] = l[3] = lrow;
                    float pv[4];
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const float x = __uint_as_float(sr[e + f]);
                        if constexpr (LD > 0) {
                            // sigmoid of a distant pair: 1 / (1 + z), z = exp(-lambda g_i . g_j); 1 - f = z f
                            const int col = col0 + c + e + f;
                            const bool distant = (KEYS ? col - row : row - col) > p.w;
                            const float4* gc = gate_row(c + e + f);
                            float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
                            for (int k = 0; k < LD / 4; ++k) {
                                const float4 v = gc[k];
                                s0 = __ffma2_rn(make_float2(gr[4 * k], gr[4 * k + 1]), make_float2(v.x, v.y), s0);
                                s1 = __ffma2_rn(make_float2(gr[4 * k + 2], gr[4 * k + 3]), make_float2(v.z, v.w), s1);
                            }
                            const float z = distant ? ex2_approx(fminf((s0.x + s0.y) + (s1.x + s1.y), 126.f)) : 0.f;
                            const float fac = rcp_approx(1.f + z);
                            const float y = ex2_approx(fmaf(x * fac, sl2, -l[f]));
                            pv[f] = !masked || (kw[(c + e + f) >> 5] >> ((c + e + f) & 31) & 1u) ? y : 0.f;
                            pr[c + e + f] = pv[f] * fac;
                            da[c + e + f] = x * p.scale * p.lambda * z * fac;
                        } else if constexpr (CAP) {
                            const float th = tanh_approx(x * cap_in);
                            const float y = ex2_approx(fmaf(th, sl2, -l[f]));
                            pv[f] = !masked || (kw[(c + e + f) >> 5] >> ((c + e + f) & 31) & 1u) ? y : 0.f;
                            pr[c + e + f] = pv[f] * fmaf(-th, th, 1.f);
                        } else {
                            const float y = ex2_approx(fmaf(x, sl2, -l[f]));
                            pv[f] = !masked || (kw[(c + e + f) >> 5] >> ((c + e + f) & 31) & 1u) ? y : 0.f;
                            pr[c + e + f] = pv[f];
                        }
                    }
                    if constexpr (C::HAS_V) {
                        sr[e / 2] = pack_bf16x2(pv[0], pv[1]);          // (words of this loop's earlier turns)
                        sr[e / 2 + 1] = pack_bf16x2(pv[2], pv[3]);
                    }
                }
                if constexpr (C::HAS_V) tmem_st16(t_x + c / 2, *reinterpret_cast<uint32_t(*)[16]>(&sr[0]));
            }
            if constexpr (C::HAS_V) tmem_wait_st();
            tc_fence_before();
            if constexpr (C::HAS_V) mbar_arrive(smem_u32(&ctl.p_full[xb]));
            // ---- dS
            if constexpr (C::HAS_DS) {
                if (!wait(ctl.y_full, t & 1, 31)) break;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < NC; c += 32) {
                    uint32_t sr[32];
                    tmem_ld32(t_y + c, sr);
                    tmem_wait_ld();
#pragma unroll
                    for (int e = 0; e < 32; e += 4) {
                        float d[4], ds[4];
                        if constexpr (KEYS) *reinterpret_cast<float4*>(d) = *reinterpret_cast<const float4*>(info + NCOL + c + e);
                        else d[0] = d[1] = d[2] = d[3] = drow;
#pragma unroll
                        for (int f = 0; f < 4; ++f) {
                            ds[f] = pr[c + e + f] * (__uint_as_float(sr[e + f]) - d[f]);
                            if constexpr (LD > 0) {
                                const float a = ds[f] * da[c + e + f];
                                const float4* gc = gate_row(c + e + f);
#pragma unroll
                                for (int k = 0; k < LD / 4; ++k) {
                                    const float4 v = gc[k];
                                    const float2 lo = __ffma2_rn(make_float2(a, a), make_float2(v.x, v.y), make_float2(dg[4 * k], dg[4 * k + 1]));
                                    const float2 hi = __ffma2_rn(make_float2(a, a), make_float2(v.z, v.w), make_float2(dg[4 * k + 2], dg[4 * k + 3]));
                                    dg[4 * k] = lo.x; dg[4 * k + 1] = lo.y; dg[4 * k + 2] = hi.x; dg[4 * k + 3] = hi.y;
                                }
                            }
                        }
                        sr[e / 2] = pack_bf16x2(ds[0], ds[1]);
                        sr[e / 2 + 1] = pack_bf16x2(ds[2], ds[3]);
                    }
                    tmem_st16(t_y + c / 2, *reinterpret_cast<uint32_t(*)[16]>(&sr[0]));
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&ctl.ds_full));
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl.info_empty[taken.slot]));
            taken.next();
        }
        if (!bad && t > 0) wait(ctl.acc_full, 0, 40);
        if (!bad) {
            tc_fence_after();
            // ---- results: BWD_KV: dV by the first four warps, dK by the others; one sum: half of its columns each
            constexpr int NOUT = MODE == BWD_KV ? D : D / 2;
            const bool v = MODE == BWD_V || (MODE == BWD_KV && half == 0);
            const float by = v ? 1.f : p.scale;
            const int col0 = MODE == BWD_KV ? 0 : half * NOUT;
            const uint32_t t_a = tm + (v ? C::COL_V : C::COL_S) + col0;
            __nv_bfloat16* out = v ? p.out1 + b * p.s1b + h * p.s1h + (int64_t)(valid ? row : 0) * p.s1n : p.out2 + b * p.s2b + h * p.s2h + (int64_t)(valid ? row : 0) * p.s2n;
            const bool wide = v ? p.wide1 : p.wide2;
            out += col0;
#pragma unroll 1
            for (int c = 0; c < NOUT; c += 16) {
                uint32_t ov[16];
                tmem_ld16(t_a + c, ov);
                tmem_wait_ld();
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = pack_bf16x2(__uint_as_float(ov[2 * e]) * by, __uint_as_float(ov[2 * e + 1]) * by);
                if (!valid) continue;
                if (wide) {
                    st_global_v8(out + c, w);
                } else {
                    *reinterpret_cast<uint4*>(out + c) = make_uint4(w[0], w[1], w[2], w[3]);
                    *reinterpret_cast<uint4*>(out + c + 8) = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
            tc_fence_before();
            if constexpr (LD > 0 && MODE != BWD_V) {
                // the two halves of a row's columns: the second hands its sums to the first (the slots are through)
                float* const x = reinterpret_cast<float*>(smem_raw + C::OFF_C) + row_in_tile;
                if (half == 1) {
#pragma unroll
                    for (int e = 0; e < LD; ++e) x[e * 128] = dg[e];
                }
                if (half == 1) mbar_arrive(smem_u32(&ctl.dg_full));
                if (half == 0 && wait(ctl.dg_full, 0, 41) && valid) {
#pragma unroll
                    for (int e = 0; e < LD; e += 4)
                        *reinterpret_cast<float4*>(p.dg_part + ((size_t)head * p.n + row) * LD + e) =
                            make_float4(dg[e] + x[e * 128], dg[e + 1] + x[(e + 1) * 128], dg[e + 2] + x[(e + 2) * 128], dg[e + 3] + x[(e + 3) * 128]);
                }
            }
        }
        if (bad && lane == 0) give_up(bad);
    }
    // ---------------------------------------------------------------------- end
    tc_fence_before();
    __syncthreads();
    if (*(volatile int*)&ctl.abort_flag) {
        // a role gave up: let copies that were already issued land before the CTA leaves
        const uint64_t t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 20000ull) { }
        __syncthreads();
    }
    if (warp == 1) tmem_dealloc(tmem, 512);
}

template <int D, int MODE, bool CAP, int LD>
static int launch_bwd_pass(const AttnBwdArgs& a, const BwdParams& p, cudaStream_t st) {
    using C = BwdCfg<D, MODE, LD>;
    const int B = a.s.batch, n = a.s.n;
    const focus_tensor &r1 = C::KEYS ? a.k : a.q, &r2 = C::KEYS ? a.v : a.dO, &c1 = C::KEYS ? a.q : a.k, &c2 = C::KEYS ? a.dO : a.v;
    const int HR = C::KEYS ? a.s.Hkv : a.s.Hq, HC = C::KEYS ? a.s.Hq : a.s.Hkv;
    CUtensorMap m1, m2, m3, m4;
    int rc;
    if ((rc = make_tmap_qkv(&m1, r1, B, HR, n, D)) || (rc = make_tmap_qkv(&m2, r2, B, HR, n, D)) || (rc = make_tmap_qkv(&m3, c1, B, HC, n, D, C::NCOL)) ||
        (rc = make_tmap_qkv(&m4, c2, B, HC, n, D, C::NCOL)))
        return rc;
    if ((rc = check_cuda(allow_smem<attn_bwd_kernel<D, MODE, CAP, LD>>(C::SMEM), "cudaFuncSetAttribute(attn_bwd)"))) return rc;
    auto kern = attn_bwd_kernel<D, MODE, CAP, LD>;
    return check_cuda(launch_dependent(kern, dim3((unsigned)(p.heads * p.nt)), dim3(BWD_THREADS), C::SMEM, st, m1, m2, m3, m4, p), "attention backward launch");
}

template <int D, bool CAP, int LD>
static int launch_bwd_passes(const AttnBwdArgs& a, const BwdParams& kv, const BwdParams& q, cudaStream_t st) {
    int rc;
    if constexpr (D == 256) {
        if ((rc = launch_bwd_pass<D, BWD_V, CAP, LD>(a, kv, st)) || (rc = launch_bwd_pass<D, BWD_K, CAP, LD>(a, kv, st))) return rc;
    } else {
        if ((rc = launch_bwd_pass<D, BWD_KV, CAP, LD>(a, kv, st))) return rc;
    }
    return launch_bwd_pass<D, BWD_Q, CAP, LD>(a, q, st);
}

template <int D>
int launch_bwd_d(const AttnBwdArgs& a, const BwdParams& kv, const BwdParams& q, cudaStream_t st) {
    if (a.g) {
        switch (focus_soft_ld(a.s.K)) {
            case 4: return launch_bwd_passes<D, false, 4>(a, kv, q, st);
            case 8: return launch_bwd_passes<D, false, 8>(a, kv, q, st);
            case 16: return launch_bwd_passes<D, false, 16>(a, kv, q, st);
        }
        if constexpr (D != 256) return launch_bwd_passes<D, false, 32>(a, kv, q, st);
        return fail(FOCUS_ERR_UNSUPPORTED, "the gated attention at D = 256 supports K <= 16");
    }
    return a.s.softcap > 0.f ? launch_bwd_passes<D, true, 0>(a, kv, q, st) : launch_bwd_passes<D, false, 0>(a, kv, q, st);
}

}  // namespace focus
