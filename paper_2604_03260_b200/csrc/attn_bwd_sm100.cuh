// The passes of the attention's backward: one CTA per (head, 128 rows), its tiles of columns one after another.
//   warp 0        TMA: the two row tiles once, then C1 of every visited tile into a ring of slots (128-byte swizzle); the tiles' numbers
//   warp 3        C2 of every tile into another ring; lse, delta and assignments of the columns
//   warps 1, 2    MMA issuers: X = R1 C1^T, Y = R2 C2^T (operands in shared memory), and the sums with P or dS (bf16, tensor memory) as the
//                 first operand and C2 or C1 read along its other dimension as the second.  Warp 1 what C2 is for, warp 2 what C1 is for.
//                 (One warp for both: 2360 cycles a tile of dQ at D = 128 with nothing else to wait for, where the products take 1630: a wait and
//                 what comes with it is some 150 cycles even where it need not wait, and what has been issued before lasts little longer.)
//   warps 4-7     P = exp2(X - lse), dS = P (Y - delta) of the even tiles, a thread a row
//   warps 8-11    of the odd ones
// The tensor pipe works in order, so a product may be issued into the place of an operand that an earlier one reads.  Two tiles are at work
// at a time: while one group of warps takes exponentials the other waits for, or works on, the other tile's products.  With both groups on
// the halves of one tile a tile took the sum of what both phases wait for (D = 128: 3300 and 2650 cycles for the two passes).
//
// Tensor memory: the sums, and two or three places for the tiles at work.  A tile has one place: X, P over it, Y when X (and the sum with P)
// is through, dS over that.  With three places the X of a group's next tile is there before it is done with the one before.
#pragma once

#include "attn_bwd.cuh"

namespace focus {

constexpr int BWD_THREADS = 384;

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The bits of 32 columns in the order in which they become masks of packed pairs: columns 0, 2, ... 14 in byte 0, 1, 3, ... 15 in byte 1,
// 16, 18, ... in byte 2, 17, 19, ... in byte 3; a shift brings a pair's two bits to the tops of two bytes, whose signs are then spread.
__device__ __forceinline__ uint32_t pair_bits(uint32_t x) {
    auto even = [](uint32_t v) {
        v &= 0x55555555u;
        v = (v | v >> 1) & 0x33333333u;
        v = (v | v >> 2) & 0x0f0f0f0fu;
        return (v | v >> 4) & 0x00ff00ffu;
    };
    return even(x) | even(x >> 1) << 8;
}

// bytes of a word, each the sign of one of its bytes eight times over (selectors 8 to 11: byte 0 to 3)
template <uint32_t SEL> __device__ __forceinline__ uint32_t byte_signs(uint32_t x) {
    uint32_t y;
    asm("prmt.b32 %0, %1, %1, %2;" : "=r"(y) : "r"(x), "n"(SEL));
    return y;
}

template <int D, int MODE, bool CAP, int LD>
struct BwdCfg {
    static constexpr bool KEYS = MODE != BWD_Q;
    static constexpr bool HAS_V = MODE == BWD_KV || MODE == BWD_V, HAS_DS = MODE != BWD_V;
    // Columns of a tile, all of them one thread's: 128 probabilities in registers; with the gate two numbers a pair are held, so 64, and at
    // D = 256 the row tiles leave no room for wider ones
    static constexpr int NCOL = D == 256 || LD > 0 ? 64 : 128;
    static constexpr int NPL = (MODE == BWD_KV && D == 128 && NCOL == 128) || (D == 256 && HAS_DS) ? 2 : 3;       // places (as many as fit; at D = 256 as many slots fit)
    static constexpr int SUBT = D / 64;
    static constexpr uint32_t SUBR = 128 * 128, SUBC = NCOL * 128;
    static constexpr uint32_t R_BYTES = SUBR * SUBT, C_BYTES = SUBC * SUBT;
    static constexpr int NR = MODE == BWD_V ? 1 : 2;             // row tiles
    // Rows are keys: lse and delta go by the column.  They come as six more numbers a column (-lse / scale and -delta in three bf16 terms
    // each, 24 bits), which one more 16-deep step of X and of Y, against rows of ones, adds to the products; a thread then needs nothing that
    // goes by the column.  Not where a cap or a gate comes between the product and lse, nor where shared memory has no room for it (D = 128,
    // dK at D = 256); there they are copied to shared memory and read.
    static constexpr bool AUG = KEYS && !CAP && LD == 0 && !(D == 128 && MODE == BWD_KV) && !(D == 256 && MODE == BWD_K);
    static constexpr uint32_t AUG_BYTES = AUG ? NCOL * 16 : 0, CONST_BYTES = AUG ? 4 * 2048 : 0;        // (ones for X, zeros, ones for Y, zeros)
    static constexpr uint32_t C1_BYTES = C_BYTES + AUG_BYTES;
    static constexpr uint32_t STAT_BYTES = KEYS && !AUG ? 2 * NCOL * 4 : 0;
    // The columns' assignments, copied beside the tile; at D = 256 there is no room, they are read from L1 (one address a warp)
    static constexpr bool GATE_SMEM = LD > 0 && D != 256;
    static constexpr uint32_t GATE_BYTES = GATE_SMEM ? NCOL * LD * 4 : 0;
    static constexpr uint32_t INFO_BYTES = STAT_BYTES + GATE_BYTES;               // one tile; two of them
    static constexpr uint32_t CTL_BYTES = 1024;
    static constexpr uint32_t ROOM = 227 * 1024 - CTL_BYTES - NR * R_BYTES - 2 * INFO_BYTES - CONST_BYTES;
    // C1 of a tile is held from its X to its sum with dS, NPL tiles later, C2 for a product or two: rings of their own
    static constexpr int NFIT = ROOM / C1_BYTES > 8 ? 8 : ROOM / C1_BYTES;
    static constexpr int NS1 = MODE == BWD_V ? NFIT - NFIT / 2 : NFIT > NPL + 1 ? (NFIT + 1 > 2 * (NPL + 1) ? (NFIT + 1) / 2 : NPL + 1) : NFIT - 1;
    static constexpr int NS2 = NFIT - NS1, NSLOT = NFIT;
    static constexpr bool EARLY = MODE == BWD_V || NS1 > NPL;    // C1 of the tile after next can be there before the sum with dS frees a slot
    static_assert(NS2 >= 1 && NS1 >= 2 && (EARLY || NS1 == NPL), "two tiles at work");
    static constexpr int P_PARTS = LD == 0 && KEYS ? 2 : 1;      // parts in which P and dS are handed over: most of a sum runs while the last are worked out
    static constexpr int PART0 = P_PARTS == 1 ? NCOL : NCOL == 128 ? 96 : 32;     // columns of the first
    static constexpr uint32_t OFF_C = NR * R_BYTES, OFF_CONST = OFF_C + NS1 * C1_BYTES + NS2 * C_BYTES, OFF_INFO = OFF_CONST + CONST_BYTES;
    static constexpr uint32_t OFF_CTL = OFF_INFO + 2 * INFO_BYTES, SMEM = OFF_CTL + CTL_BYTES;
    static __device__ __forceinline__ uint32_t slot_at(uint32_t s) { return s < NS1 ? s * C1_BYTES : NS1 * C1_BYTES + (s - NS1) * C_BYTES; }
    static constexpr uint32_t COL_V = NPL * NCOL > 256 ? 384 : 256, COL_S = MODE == BWD_KV ? COL_V + D : COL_V;
    static_assert(NPL * NCOL <= COL_V && COL_S + D <= 512, "tensor memory");
};

struct BwdCtl {
    uint64_t r_full, acc_full, dg_full, full[8], empty[8];      // slots of C1, then of C2
    uint64_t id_full[4], id_empty[4];             // numbers of the tiles
    uint64_t info_full[2], info_empty[2];         // what else there is of a tile
    uint64_t x_full[3], x_taken[3], p_full[3][2], y_full[3], ds_full[3][2];       // by the tile's place (and part)
    uint32_t limit, tmem_base;
    int abort_flag;
    int more[8];                  // of a slot: whether there is a tile at all
    int tile[4], head[4];         // column tile and its head; tile -1: no more
};
static_assert(sizeof(BwdCtl) <= 1024, "CTL_BYTES");

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
    using C = BwdCfg<D, MODE, CAP, LD>;
    constexpr bool KEYS = C::KEYS;
    constexpr int NCOL = C::NCOL;
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
        mbar_init(smem_u32(&ctl.acc_full), (C::HAS_V ? 1 : 0) + (C::HAS_DS ? 1 : 0));
        mbar_init(smem_u32(&ctl.dg_full), 128);
        for (int s = 0; s < C::NSLOT; ++s) { mbar_init(smem_u32(&ctl.full[s]), 1); mbar_init(smem_u32(&ctl.empty[s]), 1); }
        for (int x = 0; x < 4; ++x) { mbar_init(smem_u32(&ctl.id_full[x]), 1); mbar_init(smem_u32(&ctl.id_empty[x]), 4); }
        for (int x = 0; x < 2; ++x) {
            mbar_init(smem_u32(&ctl.info_full[x]), 1);
            mbar_init(smem_u32(&ctl.info_empty[x]), 4);             // (the four warps of a tile)
        }
        for (int x = 0; x < C::NPL; ++x) {
            mbar_init(smem_u32(&ctl.x_full[x]), 1);
            mbar_init(smem_u32(&ctl.x_taken[x]), 128);
            mbar_init(smem_u32(&ctl.y_full[x]), 1);
            for (int q = 0; q < 2; ++q) { mbar_init(smem_u32(&ctl.p_full[x][q]), 128); mbar_init(smem_u32(&ctl.ds_full[x][q]), 128); }
        }
        ctl.abort_flag = 0;
        ctl.limit = wait_limit(4000000000ull);
        fence_mbar_init();
    }
    if constexpr (C::AUG) {                 // rows of ones against the terms of lse, and of delta
        for (int e = threadIdx.x; e < 512; e += BWD_THREADS)
            *reinterpret_cast<uint4*>(smem_raw + C::OFF_CONST + e * 16) = e < 128 ? make_uint4(0x3f803f80u, 0x3f80u, 0u, 0u)
                                                                          : e >= 256 && e < 384 ? make_uint4(0u, 0x3f800000u, 0x3f803f80u, 0u) : make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
    }
    if constexpr (C::GATE_SMEM) {           // (rows of assignments past the end of a sequence are not copied)
        for (int e = threadIdx.x; e < 2 * (int)C::INFO_BYTES / 4; e += BWD_THREADS) reinterpret_cast<float*>(smem_raw + C::OFF_INFO)[e] = 0.f;
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
    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------ TMA: row tiles, C1 and the tiles' numbers; C2 and what goes by the column
        const bool one = warp == 0;
        const int hk = KEYS ? h : h / p.G;
        if (one && lane == 0) {
            mbar_arrive_expect_tx(smem_u32(&ctl.r_full), C::NR * C::R_BYTES);
#pragma unroll 1
            for (int c = 0; c < C::SUBT; ++c) {
                tma_load_4d(base + c * C::SUBR, &tm_r1, smem_u32(&ctl.r_full), c * 64, row_tile * 128, h, b);
                if (C::NR == 2) tma_load_4d(base + C::R_BYTES + c * C::SUBR, &tm_r2, smem_u32(&ctl.r_full), c * 64, row_tile * 128, h, b);
            }
        }
        BwdWalk<KEYS, NCOL> walk(p, lane, row_tile, b, h);
        const CUtensorMap* const map = one ? &tm_c1 : &tm_c2;
        const uint32_t slot0 = one ? 0 : C::NS1, slots = one ? C::NS1 : C::NS2;
        uint32_t slot = 0, phase = 0;
        RingAt<4> id;
        RingAt<2> info;
        // The numbers go ahead of the tiles: a group asks for its next one when it begins with a tile, and C1 of that may have to wait for it
        BwdWalk<KEYS, NCOL> ahead(p, lane, row_tile, b, h);
        int ends = one ? 0 : 2;
        auto hand_id = [&]() -> bool {
            if (ends == 2) return true;
            const int t = ends ? -1 : ahead.next();
            if (t < 0) ++ends;                                      // (a last one for each group of warps)
            if (!wait(ctl.id_empty[id.slot], id.phase ^ 1, 13)) return false;
            if (lane == 0) {
                ctl.tile[id.slot] = t;
                ctl.head[id.slot] = KEYS ? h * p.G + ahead.hi : hk;
                mbar_arrive(smem_u32(&ctl.id_full[id.slot]));
            }
            __syncwarp();
            id.next();
            return true;
        };
        for (int x = 0; x < 3; ++x) hand_id();
        for (;;) {
            const int t = walk.next();
            const int hc = KEYS ? h * p.G + walk.hi : hk;           // head of the columns
            if (!hand_id() || !wait(ctl.empty[slot0 + slot], phase ^ 1, 11)) break;
            if (lane == 0) {
                const uint32_t bar = smem_u32(&ctl.full[slot0 + slot]), at = base + C::OFF_C + C::slot_at(slot0 + slot);
                ctl.more[slot0 + slot] = t >= 0;
                if (t < 0) {
                    mbar_arrive(bar);
                } else {
                    mbar_arrive_expect_tx(bar, one ? C::C1_BYTES : C::C_BYTES);
#pragma unroll
                    for (int c = 0; c < C::SUBT; ++c) tma_load_4d(at + c * C::SUBC, map, bar, c * 64, t * NCOL, hc, b);
                    if (C::AUG && one)
                        bulk_load(at + C::C_BYTES, p.aug + (((size_t)(b * p.Hq + hc) * p.nt + t * NCOL / 128) * 128 + t * NCOL % 128) * 8, C::AUG_BYTES, bar);
                }
            }
            __syncwarp();
            if (!one && C::INFO_BYTES > 0 && t >= 0) {
                if (!wait(ctl.info_empty[info.slot], info.phase ^ 1, 12)) break;
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&ctl.info_full[info.slot]), at = base + C::OFF_INFO + info.slot * C::INFO_BYTES;
                    const int rows = min(NCOL, p.n - t * NCOL);       // (a half tile may lie past the end)
                    const uint32_t gbytes = C::GATE_SMEM && rows > 0 ? (uint32_t)rows * LD * 4 : 0u;
                    if (C::STAT_BYTES + gbytes == 0) mbar_arrive(bar); else mbar_arrive_expect_tx(bar, C::STAT_BYTES + gbytes);
                    if constexpr (C::STAT_BYTES > 0) {
                        const float* st = p.stat + ((size_t)(b * p.Hq + hc) * p.nt + t * NCOL / 128) * 256 + t * NCOL % 128;
                        bulk_load(at, st, NCOL * 4, bar);
                        bulk_load(at + NCOL * 4, st + 128, NCOL * 4, bar);
                    }
                    if (gbytes) bulk_load(at + C::STAT_BYTES, p.g + ((size_t)b * p.n + (size_t)t * NCOL) * (LD > 0 ? LD : 1), gbytes, bar);
                }
                __syncwarp();
                info.next();
            }
            if (t < 0) break;
            if (++slot == slots) { slot = 0; phase ^= 1; }
        }
        if (bad && lane == 0) give_up(bad);
        __syncwarp();
    } else if (warp < 4) {
        // ------------------------------------------------------------------ MMA issuers
        constexpr uint32_t IDESC_X = idesc_bf16(128, NCOL, 0, 0), IDESC_A = idesc_bf16(128, D, 0, 1);
        const uint32_t r1 = (uint32_t)smem_desc_sw128(base, 16, 1024), r2 = r1 + (C::R_BYTES >> 4);
        const uint32_t ck = (uint32_t)smem_desc_sw128(base + C::OFF_C, 16, 1024);                  // columns along D
        const uint32_t cm = (uint32_t)smem_desc_sw128(base + C::OFF_C, C::SUBC, 1024);             // along the tokens
        // d = rows (X: R1, Y: R2) times the columns in slot `at`; `aug`: slot of the tile's C1, behind which its lse and delta are
        auto product = [&](uint32_t d, bool y, uint32_t at, uint32_t aug) {
            const uint32_t r = y ? r2 : r1, c = ck + (C::slot_at(at) >> 4);
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) umma_ss_lo(d, r + (ks >> 2) * (C::SUBR >> 4) + (ks & 3) * 2, c + (ks >> 2) * (C::SUBC >> 4) + (ks & 3) * 2, IDESC_X, ks > 0);
            if constexpr (C::AUG) {
                const uint32_t ones = base + C::OFF_CONST + (y ? 4096 : 0), x = base + C::OFF_C + C::slot_at(aug) + C::C_BYTES;
                umma_ss(d, smem_desc_plain(ones, 2048, 128), smem_desc_plain(x, base + C::OFF_CONST + 2048 - x, 128), IDESC_X, 1);
            }
        };
        // a slot of either ring is waited for; false: there is no such tile (or `bad`)
        auto take = [&](uint32_t slot, uint32_t phase) -> bool { return wait(ctl.full[slot], phase, 21) && *(volatile int*)&ctl.more[slot]; };
        // (by the elected lane)
        auto put_x = [&](uint32_t place, uint32_t c1) {
            product(tmem + place * NCOL, false, c1, c1);
            umma_commit(smem_u32(&ctl.x_full[place]));
            if (!C::HAS_DS) umma_commit(smem_u32(&ctl.empty[c1]));
        };
        // a sum's steps, part by part as the first operand (at `a`) comes; then what `last` issues
        auto sum = [&](uint64_t (&bars)[2], uint32_t parity, int where, uint32_t d, uint32_t a, uint32_t at, bool more, auto last) -> bool {
            const uint32_t c = cm + (C::slot_at(at) >> 4);
#pragma unroll
            for (int q = 0; q < C::P_PARTS; ++q) {
                if (!wait(bars[q], parity, where + q)) return false;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int ks = q ? C::PART0 / 16 : 0; ks < (q == C::P_PARTS - 1 ? NCOL : C::PART0) / 16; ++ks)
                        umma_ts_lo(d, a + ks * 8, c + ks * 128, IDESC_A, more || ks > 0);
                    if (q == C::P_PARTS - 1) last();
                }
            }
            return true;
        };
        // The steps of a tile.  Warp 2: X; when dS is there, the sum with it, then X of the tile that has the place next.  Warp 1: when P is
        // there (with dS alone: when X has been read), the sum with it, then Y into the same place.  dV alone (no Y) is all warp 1's, since an
        // X has to come behind the sum whose place it takes.  Each sum is one warp's, and so in order.
        RingAt<C::NS1> at1, done1;                         // slots of C1: of the next X; of the next sum with dS, or the next Y (its lse and delta)
        RingAt<C::NS2> at2;                                // slots of C2
        RingAt<C::NPL> pl;                                 // place of the tile at work, parity of its use
        bool more = true;                                  // the last tile that X was asked for was there
        int left = 0;                                      // X's issued whose sum has not been
        auto first_x = [&]() -> bool {
#pragma unroll 1
            for (int x = 0; x < C::NPL; ++x) {             // (every item has its diagonal tile)
                more = take(at1.slot, at1.phase);
                if (!more) break;
                tc_fence_after();
                if (elect_one()) put_x(x, at1.slot);
                at1.next();
                ++left;
            }
            return !bad;
        };
        do {
            if (!wait(ctl.r_full, 0, 20)) break;
            tc_fence_after();
            if (warp == 2) {
                if (!C::HAS_DS || !first_x()) break;
                for (bool begun = false; left > 0; begun = true) {
                    if (C::EARLY && more) more = take(at1.slot, at1.phase);
                    if (bad) break;
                    if (!sum(ctl.ds_full[pl.slot], pl.phase, 26, tmem + C::COL_S, tmem + pl.slot * NCOL, done1.slot, begun, [&] {
                            umma_commit(smem_u32(&ctl.empty[done1.slot]));
                            if (C::EARLY && more) put_x(pl.slot, at1.slot);
                        })) break;
                    if (!C::EARLY && more) {
                        more = take(at1.slot, at1.phase);
                        if (bad) break;
                        tc_fence_after();
                        if (more && elect_one()) put_x(pl.slot, at1.slot);
                    }
                    if (more) at1.next(); else --left;
                    pl.next();
                    done1.next();
                }
                if (!bad && elect_one()) umma_commit(smem_u32(&ctl.acc_full));
            } else {
                if (!C::HAS_DS && !first_x()) break;
                for (bool begun = false;; begun = true) {
                    const uint32_t c2 = C::NS1 + at2.slot;
                    if (!take(c2, at2.phase)) break;
                    if (!C::HAS_DS && more) more = take(at1.slot, at1.phase);
                    if (bad) break;
                    auto put_y = [&] {
                        product(tmem + pl.slot * NCOL, true, c2, done1.slot);
                        umma_commit(smem_u32(&ctl.y_full[pl.slot]));
                    };
                    if constexpr (C::HAS_V) {
                        if (!sum(ctl.p_full[pl.slot], pl.phase, 24, tmem + C::COL_V, tmem + pl.slot * NCOL, c2, begun, [&] {
                                if (C::HAS_DS) put_y();
                                umma_commit(smem_u32(&ctl.empty[c2]));
                                if (!C::HAS_DS && more) put_x(pl.slot, at1.slot);
                            })) break;
                        if (!C::HAS_DS && more) at1.next();
                    } else {
                        if (!wait(ctl.x_taken[pl.slot], pl.phase, 23)) break;
                        tc_fence_after();
                        if (elect_one()) {
                            put_y();
                            umma_commit(smem_u32(&ctl.empty[c2]));
                        }
                    }
                    at2.next();
                    pl.next();
                    done1.next();
                }
                if (C::HAS_V && !bad && elect_one()) umma_commit(smem_u32(&ctl.acc_full));
            }
        } while (false);
        if (bad && lane == 0) give_up(bad);
        __syncwarp();
    } else if (warp >= 4) {
        // ------------------------------------------------------------------ P, dS, results
        reg_inc<REGS_SOFTMAX_2WG>();
        const int wg = (warp - 4) >> 2;                    // tiles of this parity
        const int row_in_tile = ((warp & 3) << 5) | lane;
        const int row = row_tile * 128 + row_in_tile;      // position of this thread's token
        const bool valid = row < p.n;
        const uint32_t tm = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float sl2 = CAP ? p.softcap * LOG2E : p.scale * LOG2E;
        const float cap_in = CAP ? p.scale / p.softcap : 0.f;
        float lrow = 0.f, drow = 0.f;                      // rows are queries: -lse log2(e) and -delta of the row
        if constexpr (!KEYS) {
            const float* st = p.stat + ((size_t)head * p.nt + row_tile) * 256 + row_in_tile;
            lrow = dep_load(st);
            drow = dep_load(st + 128);
        }
        uint32_t mask = 0;
        if (p.bits) mask = valid ? dep_load(p.row_mask + (size_t)head * p.n + row) & (0xffffffffu >> (32 - p.K)) : 0u;
        constexpr int LDR = LD > 0 ? LD : 1, NW = NCOL / 32;
        float gr[LDR], dg[LDR];                            // assignment of the row times -lambda log2(e), its gradient
        if constexpr (LD > 0) {
#pragma unroll
            for (int e = 0; e < LD; ++e) {
                gr[e] = valid ? dep_load(p.g + ((size_t)b * p.n + row) * LD + e) * (-p.lambda * LOG2E) : 0.f;
                dg[e] = 0.f;
            }
        }
        const float* const info = reinterpret_cast<const float*>(smem_raw + C::OFF_INFO + wg * C::INFO_BYTES);
        const float* const gcol = reinterpret_cast<const float*>(smem_raw + C::OFF_INFO + wg * C::INFO_BYTES + C::STAT_BYTES);
        // This group's next tile, and its columns' bitmaps of the row's groups, asked for while the tile before is at work.  (The words
        // of the first two groups are joined only when they are used.)
        int ct = -1;
        uint32_t w0[NW], w1[NW];
        auto peek = [&](uint32_t k) -> bool {              // k: the how manieth tile of this group
            const uint32_t slot = wg + 2 * (k & 1);
            if (!wait(ctl.id_full[slot], (k >> 1) & 1, 39)) return false;
            ct = *(volatile int*)&ctl.tile[slot];
            const int hc = *(volatile int*)&ctl.head[slot];
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl.id_empty[slot]));
#pragma unroll
            for (int q = 0; q < NW; ++q) w0[q] = w1[q] = 0u;
            const int lo_k = KEYS ? row_tile * 128 : ct * NCOL, hi_q = KEYS ? ct * NCOL + NCOL - 1 : row_tile * 128 + 127;
            if (!p.bits || ct < 0 || hi_q - lo_k <= p.w) return true;
            const uint32_t* gb = p.bits + ((size_t)(b * (KEYS ? p.Hq : p.Hkv) + hc) * p.nt + ct * NCOL / 128) * p.K * 4 + ct * NCOL % 128 / 32;
            uint32_t rem = mask;
            auto word = [&](uint32_t (&w)[NW], bool join) {
                const uint32_t* x = gb + (__ffs(rem) - 1) * 4;
                rem &= rem - 1;
                uint32_t v[NW];
                if constexpr (NW == 4) {
                    const uint4 y = dep_load(reinterpret_cast<const uint4*>(x));
                    v[0] = y.x; v[1] = y.y; v[2] = y.z; v[3] = y.w;
                } else {
                    const uint2 y = dep_load(reinterpret_cast<const uint2*>(x));
                    v[0] = y.x; v[1] = y.y;
                }
#pragma unroll
                for (int q = 0; q < NW; ++q) w[q] = join ? w[q] | v[q] : v[q];
            };
            if (rem) word(w0, false);
            if (rem) word(w1, false);
#pragma unroll 1
            while (rem) word(w1, true);
            return true;
        };
        uint32_t k = 0, place = wg, par = 0;               // the tile's place, the parity of its use
        if (peek(0)) {
#pragma unroll 1
            for (; ct >= 0; ++k) {
                const uint32_t t_x = tm + place * NCOL;
                const int now = ct;
                // ---- which columns count: bit c of word c / 32
                const int col0 = now * NCOL;
                auto gate_row = [&](int c) -> const float4* {
                    return reinterpret_cast<const float4*>(C::GATE_SMEM ? gcol + c * LDR : p.g + ((size_t)b * p.n + min(col0 + c, p.n - 1)) * LDR);
                };
                uint32_t kw[NW];
                bool masked;
                {
                    const int lo_q = KEYS ? col0 : row_tile * 128, hi_q = KEYS ? col0 + NCOL - 1 : row_tile * 128 + 127;
                    const int lo_k = KEYS ? row_tile * 128 : col0, hi_k = KEYS ? row_tile * 128 + 127 : col0 + NCOL - 1;
                    const bool causal = lo_q < hi_k, outside = p.bits && hi_q - lo_k > p.w;
                    masked = causal || outside;
#pragma unroll
                    for (int q = 0; q < NW; ++q) kw[q] = outside ? w0[q] | w1[q] : 0xffffffffu;
                    if (outside && lo_q - hi_k <= p.w) {
#pragma unroll
                        for (int q = 0; q < NW; ++q)             // inside the window: queries up to j + w, keys from i - w on
                            kw[q] |= KEYS ? low_bits(row - col0 - 32 * q + p.w + 1) : ~low_bits(row - p.w - col0 - 32 * q);
                    }
                    if (causal) {
#pragma unroll
                        for (int q = 0; q < NW; ++q) kw[q] &= KEYS ? ~low_bits(row - col0 - 32 * q) : low_bits(row + 1 - col0 - 32 * q);
                    }
                }
                if (LD == 0 && masked) {
#pragma unroll
                    for (int q = 0; q < NW; ++q) kw[q] = pair_bits(kw[q]);
                }
                // words of packed pairs, those that do not count set to zero
                auto strike = [&](uint32_t (&w)[16], uint32_t bits) {
                    if (LD == 0 && masked) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const uint32_t y = bits << (7 - e);
                            w[e] &= byte_signs<0x9988>(y);
                            w[e + 8] &= byte_signs<0xbbaa>(y);
                        }
                    }
                };
                // ---- what comes after this tile
                if (!peek(k + 1)) break;
                // ---- P
                if (C::INFO_BYTES > 0 && !wait(ctl.info_full[wg], k & 1, 38)) break;
                if (!wait(ctl.x_full[place], par, 30)) break;
                tc_fence_after();
                uint32_t pr[NCOL];                             // X, then P times the slope of the logit
                float da[LD > 0 ? NCOL : 1];                   // gate: what turns ds into the gradient of g_i . g_j
#pragma unroll
                for (int c = 0; c < NCOL; c += 32) tmem_ld32(t_x + c, *reinterpret_cast<uint32_t(*)[32]>(&pr[c]));
                tmem_wait_ld();
                if constexpr (!C::HAS_V) {
                    tc_fence_before();
                    mbar_arrive(smem_u32(&ctl.x_taken[place]));
                }
#pragma unroll
                for (int c = 0; c < NCOL; c += 32) {
                    uint32_t pk[16];
                    float4 lc[C::STAT_BYTES ? 8 : 1];          // (asked for together)
                    if constexpr (C::STAT_BYTES > 0) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) lc[e] = reinterpret_cast<const float4*>(info + c)[e];
                    }
#pragma unroll
                    for (int e = c; e < c + 32; e += 4) {
                        float2 l[2];
                        if constexpr (C::STAT_BYTES > 0) *reinterpret_cast<float4*>(l) = lc[(e - c) / 4];
                        else l[0] = l[1] = make_float2(lrow, lrow);
#pragma unroll
                        for (int f = 0; f < 2; ++f) {
                            uint32_t &u0 = pr[e + 2 * f], &u1 = pr[e + 2 * f + 1];
                            float2 x = make_float2(__uint_as_float(u0), __uint_as_float(u1)), y;
                            if constexpr (LD > 0) {
                                float2 fac;
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    // sigmoid of a distant pair: 1 / (1 + z), z = exp(-lambda g_i . g_j); 1 - f = z f
                                    const int at = e + 2 * f + i, col = col0 + at;
                                    const bool distant = (KEYS ? col - row : row - col) > p.w;
                                    const float4* gc = gate_row(at);
                                    float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
                                    for (int q = 0; q < LD / 4; ++q) {
                                        const float4 v = gc[q];
                                        s0 = __ffma2_rn(make_float2(gr[4 * q], gr[4 * q + 1]), make_float2(v.x, v.y), s0);
                                        s1 = __ffma2_rn(make_float2(gr[4 * q + 2], gr[4 * q + 3]), make_float2(v.z, v.w), s1);
                                    }
                                    s0 = __fadd2_rn(s0, s1);
                                    const float z = distant ? ex2_approx(fminf(s0.x + s0.y, 126.f)) : 0.f, r = rcp_approx(1.f + z);
                                    (i ? fac.y : fac.x) = r;
                                    da[at] = (i ? x.y : x.x) * p.scale * p.lambda * z * r;
                                }
                                y = __ffma2_rn(__fmul2_rn(x, fac), make_float2(sl2, sl2), l[f]);
                                y.x = ex2_approx(y.x);
                                y.y = ex2_approx(y.y);
                                if (masked) {
                                    y.x = kw[(e + 2 * f) >> 5] >> ((e + 2 * f) & 31) & 1u ? y.x : 0.f;
                                    y.y = kw[(e + 2 * f) >> 5] >> ((e + 2 * f + 1) & 31) & 1u ? y.y : 0.f;
                                }
                                x = __fmul2_rn(y, fac);
                            } else if constexpr (CAP) {
                                x = __fmul2_rn(x, make_float2(cap_in, cap_in));
                                x.x = tanh_approx(x.x);
                                x.y = tanh_approx(x.y);
                                y = __ffma2_rn(x, make_float2(sl2, sl2), l[f]);
                                y.x = ex2_approx(y.x);
                                y.y = ex2_approx(y.y);
                                x = __fmul2_rn(y, __ffma2_rn(make_float2(-x.x, -x.y), x, make_float2(1.f, 1.f)));
                            } else {
                                if constexpr (C::AUG) y = __fmul2_rn(x, make_float2(sl2, sl2));
                                else y = __ffma2_rn(x, make_float2(sl2, sl2), l[f]);
                                y.x = ex2_approx(y.x);
                                y.y = ex2_approx(y.y);
                                x = y;
                            }
                            u0 = __float_as_uint(x.x);
                            u1 = __float_as_uint(x.y);
                            if constexpr (C::HAS_V) pk[(e - c) / 2 + f] = pack_bf16x2(y.x, y.y);
                        }
                    }
                    if constexpr (C::HAS_V) {
                        strike(pk, kw[c / 32]);
                        tmem_st16(t_x + c / 2, pk);
                        if (c + 32 == C::PART0 || c + 32 == NCOL) {
                            tmem_wait_st();
                            tc_fence_before();
                            mbar_arrive(smem_u32(&ctl.p_full[place][c + 32 == C::PART0 ? 0 : 1]));
                        }
                    }
                }
                // ---- dS
                if constexpr (C::HAS_DS) {
                    if (!wait(ctl.y_full[place], par, 31)) break;
                    tc_fence_after();
                    uint32_t ya[16], yb[16];                   // two pieces of Y, the second on its way
                    tmem_ld16(t_x, ya);
#pragma unroll
                    for (int c = 0; c < NCOL; c += 32) {
                        uint32_t pk[16];
#pragma unroll
                        for (int hf = 0; hf < 2; ++hf) {
                            tmem_wait_ld();
                            if (hf == 0) {
                                tmem_ld16(t_x + c + 16, yb);
                            } else if (c + 32 < NCOL) {
                                tmem_ld16(t_x + c + 32, ya);
                            }
                            const uint32_t (&yr)[16] = hf ? yb : ya;
                            float4 dc[C::STAT_BYTES ? 4 : 1];
                            if constexpr (C::STAT_BYTES > 0) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) dc[e] = reinterpret_cast<const float4*>(info + NCOL + c + 16 * hf)[e];
                            }
#pragma unroll
                            for (int e = 0; e < 16; e += 4) {
                                const int at0 = c + 16 * hf + e;
                                float2 d[2];
                                if constexpr (C::STAT_BYTES > 0) *reinterpret_cast<float4*>(d) = dc[e / 4];
                                else d[0] = d[1] = make_float2(drow, drow);
#pragma unroll
                                for (int f = 0; f < 2; ++f) {
                                    const int at = at0 + 2 * f;
                                    const float2 u = make_float2(__uint_as_float(pr[at]), __uint_as_float(pr[at + 1]));
                                    float2 ds = make_float2(__uint_as_float(yr[e + 2 * f]), __uint_as_float(yr[e + 2 * f + 1]));
                                    ds = __fmul2_rn(u, C::AUG ? ds : __fadd2_rn(ds, d[f]));
                                    if constexpr (LD > 0) {
#pragma unroll
                                        for (int i = 0; i < 2; ++i) {
                                            const float a = (i ? ds.y : ds.x) * da[at + i];
                                            const float4* gc = gate_row(at + i);
#pragma unroll
                                            for (int q = 0; q < LD / 4; ++q) {
                                                const float4 v = gc[q];
                                                const float2 lo = __ffma2_rn(make_float2(a, a), make_float2(v.x, v.y), make_float2(dg[4 * q], dg[4 * q + 1]));
                                                const float2 hi = __ffma2_rn(make_float2(a, a), make_float2(v.z, v.w), make_float2(dg[4 * q + 2], dg[4 * q + 3]));
                                                dg[4 * q] = lo.x; dg[4 * q + 1] = lo.y; dg[4 * q + 2] = hi.x; dg[4 * q + 3] = hi.y;
                                            }
                                        }
                                    }
                                    pk[8 * hf + e / 2 + f] = pack_bf16x2(ds.x, ds.y);
                                }
                            }
                        }
                        strike(pk, kw[c / 32]);
                        // (in the place of Y itself only behind what has been read of it)
                        tmem_st16(t_x + c / 2, pk);
                        if (c + 32 == C::PART0 || c + 32 == NCOL) {
                            tmem_wait_st();
                            tc_fence_before();
                            mbar_arrive(smem_u32(&ctl.ds_full[place][c + 32 == C::PART0 ? 0 : 1]));
                        }
                    }
                }
                __syncwarp();
                if (C::INFO_BYTES > 0 && lane == 0) mbar_arrive(smem_u32(&ctl.info_empty[wg]));
                place += 2;
                if (place >= C::NPL) { place -= C::NPL; par ^= 1; }
            }
        }
        if (!bad) wait(ctl.acc_full, 0, 40);
        if (!bad) {
            tc_fence_after();
            // ---- results: BWD_KV: dV by the first four warps, dK by the others; one sum: half of its columns each
            constexpr int NOUT = MODE == BWD_KV ? D : D / 2;
            const bool v = MODE == BWD_V || (MODE == BWD_KV && wg == 0);
            const float by = v ? 1.f : p.scale;
            const int col0 = MODE == BWD_KV ? 0 : wg * NOUT;
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
                // the even and the odd tiles' sums: the second group hands its own to the first (the slots are through)
                float* const x = reinterpret_cast<float*>(smem_raw + C::OFF_C) + row_in_tile;
                if (wg == 1) {
#pragma unroll
                    for (int e = 0; e < LD; ++e) x[e * 128] = dg[e];
                    mbar_arrive(smem_u32(&ctl.dg_full));
                } else if (wait(ctl.dg_full, 0, 41) && valid) {
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
    using C = BwdCfg<D, MODE, CAP, LD>;
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
