// The passes of the attention's backward: one CTA per (head, 128 rows), its tiles of columns one after another.
//   warp 0        TMA: the two row tiles once, then C1 of every visited tile into a ring of slots (128-byte swizzle); the tiles' numbers
//   warp 3        C2 of every tile into another ring; lse, delta and assignments of the columns
//   warps 1, 2    MMA issuers: X = R1 C1^T, Y = R2 C2^T (operands in shared memory), and the sums with P or dS (bf16, tensor memory) as the
//                 first operand and C2 or C1 read along its other dimension as the second.  Warp 1 what C2 is for, warp 2 what C1 is for.
//                 (One warp for both, when it was so: 2360 cycles a tile of dQ at D = 128 with nothing else to wait for, where the products take
//                 1540: a wait and what comes with it is some 150 cycles even where it need not wait.)
//   warps 4-7     P = exp2(X - lse), dS = P (Y - delta) of the even tiles, a thread a row
//   warps 8-11    of the odd ones
// The tensor pipe works in order, so a product may be issued into the place of an operand that an earlier one reads.  Two tiles are at work
// at a time: while one group of warps takes exponentials the other waits for, or works on, the other tile's products.  (Both groups on the halves
// of one tile, when it was so: a tile took the sum of what both phases wait for, 8/2 heads x 16384 tokens 1751 us.)
//
// What bounds it: at D = 64 and 128 the chain of a tile, X - exponentials - Y - dS - sum, of which two are under way: 128 x 128 pairs of dK and dV take
// 3100 cycles at D = 128 (products alone 2048), of dQ 2200 (1536).  8/2 heads x 16384 tokens, D = 128, every causal pair: 1767 us, 778 TFLOP/s on the five
// products that the formulas need (seven are done); 32/8 x 8192, K = 4, top-2: 1860; D = 256 with a cap, 16/8 x 4096: 625 (each among others; on a cooler GPU up
// to 7 % less).  With the gate, the special functions: three a pair and pass, 16 a clock, and what each group's 64 columns wait for before and after; 32/8 x 4096, K = 8: 912 us.
//
// Tensor memory: the sums, and two or three places for the tiles at work.  A tile has one place: X, P over it, Y when X (and the sum with P)
// is through, dS over that.  With three places the X of a group's next tile is there before it is done with the one before.
#pragma once

#include "attn_bwd.cuh"

#include <type_traits>

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

// 16 lanes x 16 columns: thread t has of lane t/4 (words 4 j, 4 j + 1) and of lane t/4 + 8 (4 j + 2, 4 j + 3) columns 8 j + 2 (t % 4) and the next
__device__ __forceinline__ void tmem_ld_frag(uint32_t taddr, uint32_t (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_st_frag(uint32_t taddr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
// the same 16 columns as packed pairs, 8 columns: words 2 j of lane t/4, 2 j + 1 of lane t/4 + 8, column 4 j + t % 4
__device__ __forceinline__ void tmem_st_pairs(uint32_t taddr, const uint32_t (&r)[4]) {
    asm volatile("tcgen05.st.sync.aligned.16x128b.x2.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
}

template <int D, int MODE, bool CAP, int LD>
struct BwdCfg {
    static constexpr bool KEYS = MODE != BWD_Q;
    static constexpr bool HAS_V = MODE == BWD_KV || MODE == BWD_V, HAS_DS = MODE != BWD_V;
    // Columns of a tile, all of them one thread's: 128 probabilities in registers; with the gate two numbers a pair are held, so 64, and at
    // D = 256 the row tiles leave no room for wider ones
    static constexpr int NCOL = D == 256 || LD > 0 ? 64 : 128;
    static constexpr int NPL = LD > 0 || (MODE != BWD_V && D >= 128) ? 2 : 3;       // places (as many as fit)
    static constexpr uint32_t COL_U = NPL * NCOL;                // gate: a place for each group's g_i . g_j, then P times the factor
    static constexpr int SUBT = D / 64;
    static constexpr uint32_t SUBR = 128 * 128, SUBC = NCOL * 128;
    static constexpr uint32_t R_BYTES = SUBR * SUBT, C_BYTES = SUBC * SUBT;
    // Row tiles that go to tensor memory, where there is room for them, and are the first operand from there: more slots for columns, and
    // half the shared memory's traffic of a product
    static constexpr bool R1T = LD == 0 && MODE == BWD_Q && D <= 128, R2T = LD == 0 && (MODE == BWD_Q || (MODE == BWD_K && D == 256));
    static constexpr int NR = (R1T ? 0 : 1) + (R2T || MODE == BWD_V ? 0 : 1);     // those that stay in shared memory
    static constexpr int RU = ((R1T ? 1 : 0) + (R2T ? 1 : 0)) * SUBT;             // 64-column pieces of the others; they come through the last slots of both rings
    // Rows are keys: lse and delta go by the column.  They come as six more numbers a column (-lse / scale and -delta in three bf16 terms
    // each, 24 bits), which one more 16-deep step of X and of Y, against rows of ones, adds to the products; a thread then needs nothing that
    // goes by the column.  Not where a cap or a gate comes between the product and lse, nor where shared memory has no room for it (dK at
    // D = 256); there they are copied to shared memory and read.
    static constexpr bool AUG = KEYS && !CAP && LD == 0 && !(D == 256 && MODE == BWD_K);
    static constexpr uint32_t AUG_BYTES = AUG ? NCOL * 16 : 0, CONST_BYTES = AUG ? 4 * 2048 : 0;        // (ones for X, zeros, ones for Y, zeros)
    // The gate's g_i . g_j times -lambda log2(e), from the tensor cores too: both sides in three bf16 terms, the six products of terms above 2^-24 side
    // by side in GK numbers' depth.  The columns' come with C1, behind it.  (32/8 heads x 4096 tokens, K = 8, D = 128: 1241 us by instructions, 1037 so.
    // At D = 256 there is no room for them.)
    static constexpr bool GM = LD > 0 && D != 256;
    static constexpr int GK = GM ? gate_depth(LD) : 0;
    static constexpr uint32_t GC_BYTES = GK * NCOL * 2, GR_BYTES = GK * 256;
    static constexpr uint32_t C1_BYTES = C_BYTES + AUG_BYTES + GC_BYTES;
    static constexpr uint32_t STAT_BYTES = KEYS && !AUG ? 2 * NCOL * 4 : 0;
    // The columns' assignments, copied beside the tile; at D = 256 there is no room, they are read from L1 (one address a warp)
    static constexpr bool GATE_SMEM = LD > 0 && D != 256;
    static constexpr uint32_t GATE_BYTES = GATE_SMEM ? NCOL * LD * 4 : 0;
    // One tile's, and how many there are: a group's next one on its way while it works (32/8 heads x 4096 tokens, K = 8, the launch of the passes alone:
    // 938 us with two in all, for which alone 32 assignments leave room, 900 with four)
    static constexpr uint32_t INFO_BYTES = STAT_BYTES + GATE_BYTES;
    static constexpr int NI = D * LD >= 64 * 64 ? 2 : 4;
    static constexpr uint32_t CTL_BYTES = 1024;
    static constexpr uint32_t ROOM = 227 * 1024 - CTL_BYTES - NR * R_BYTES - NI * INFO_BYTES - CONST_BYTES - GR_BYTES;
    // C1 of a tile is held from its X to its sum with dS, NPL tiles later, C2 for a product or two: rings of their own
    static constexpr int NFIT = ROOM / C1_BYTES > 8 ? 8 : ROOM / C1_BYTES;
    // Registers of the warps that issue and of those that compute (12 heads x 4000 tokens, D = 64: K = 32 829 us with the usual ones, 709 so, 731 by now;
    // 8/2 heads x 4096, K = 16, where the others have what they need, 640 and 650)
    static constexpr int REGS_FEW = LD > 16 ? 40 : REGS_CONTROL, REGS_MANY = LD > 16 ? 232 : REGS_SOFTMAX_2WG;
    static_assert(REGS_FEW + 2 * REGS_MANY == 3 * 168, "the launch's registers");
    static constexpr int NG1 = 4 * C1_BYTES + 2 * C_BYTES <= ROOM ? 4 : 3 * C1_BYTES + C_BYTES <= ROOM ? 3 : 2, NG2 = (ROOM - NG1 * C1_BYTES) / C_BYTES;
    static constexpr int NS1 = GM ? NG1 : MODE == BWD_V ? NFIT - NFIT / 2 : NFIT > NPL + 1 ? (NFIT + 1 > 2 * (NPL + 1) ? (NFIT + 1) / 2 : NPL + 1) : NFIT - 1;
    static constexpr int NS2 = GM ? (NG2 > 8 - NG1 ? 8 - NG1 : NG2) : NFIT - NS1, NSLOT = NS1 + NS2;
    static constexpr bool EARLY = MODE == BWD_V || NS1 > NPL;    // C1 of the tile after next can be there before the sum with dS frees a slot
    static_assert(NS2 >= 1 && NS1 >= 2 && (EARLY || NS1 == NPL), "two tiles at work");
    static constexpr int P_PARTS = LD == 0 ? 2 : 1;      // parts in which P and dS are handed over: most of a sum runs while the last are worked out
    static constexpr int PART0 = P_PARTS == 1 ? NCOL : NCOL == 128 ? 96 : 32;     // columns of the first
    static constexpr uint32_t OFF_C = NR * R_BYTES, OFF_CONST = OFF_C + NS1 * C1_BYTES + NS2 * C_BYTES, OFF_GR = OFF_CONST + CONST_BYTES, OFF_INFO = OFF_GR + GR_BYTES;
    static constexpr uint32_t OFF_CTL = OFF_INFO + NI * INFO_BYTES, SMEM = OFF_CTL + CTL_BYTES;
    static_assert(SMEM <= 227 * 1024 && C1_BYTES % 1024 == 0, "shared memory");
    static __device__ __forceinline__ uint32_t slot_at(uint32_t s) { return s < NS1 ? s * C1_BYTES : NS1 * C1_BYTES + (s - NS1) * C_BYTES; }
    static constexpr uint32_t COL_R = NPL * NCOL;                // row tiles
    static constexpr uint32_t COL_V = RU > 0 ? COL_R + RU * 32 : NPL * NCOL > 256 ? 384 : 256, COL_S = MODE == BWD_KV ? COL_V + D : COL_V;
    static_assert(NPL * NCOL + (LD > 0 ? 2 * NCOL : 0) <= COL_V && COL_S + D <= 512, "tensor memory");
};

struct BwdCtl {
    uint64_t r_full, r_taken, acc_full, dg_full, full[8], empty[8];      // slots of C1, then of C2
    uint64_t id_full[4], id_empty[4];             // numbers of the tiles
    uint64_t info_full[4], info_empty[4];         // what else there is of a tile
    uint64_t x_full[3], x_taken[3], p_full[3][2], y_full[3], ds_full[3][2];       // by the tile's place (and part)
    uint32_t limit, tmem_base;
    int abort_flag;
    int more[8];                  // of a slot: whether there is a tile at all
    int tile[4], head[4];         // column tile and its head; tile -1: no more
    int none;                     // there is no tile at all
};
static_assert(sizeof(BwdCtl) <= 1024, "CTL_BYTES");

// The visited tiles of an item, in order; run by the whole TMA warp
template <bool KEYS, int NCOL>
struct BwdWalk {
    const BwdParams& p;
    const int lane;
    int row_tile, b, h, hi, hi_end, c, word;      // hi: query head of the group; c: next 128-tile; word: of 32 tiles, which are visited
    uint32_t bits;
    int part = NCOL == 64 ? 1 : 0;        // halves of a 128-tile
    int at = -1;
    __device__ __forceinline__ int first_col() const { return KEYS ? max(row_tile, p.col_lo) : p.col_lo; }
    __device__ __forceinline__ int end_col() const { return KEYS ? p.col_hi : min(row_tile + 1, p.col_hi); }
    __device__ __forceinline__ BwdWalk(const BwdParams& p_, int lane_, int rt, int b_, int h_, int part)
        : p(p_), lane(lane_), row_tile(rt), b(b_), h(h_), hi(part * p_.heads_each + p_.head_lo), hi_end(part * p_.heads_each + p_.head_hi), bits(0) {
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
                if (!KEYS || ++hi >= hi_end) return -1;
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

// One pass's item number `block`
template <int D, int MODE, bool CAP, int LD>
__device__ __forceinline__ void bwd_item(const CUtensorMap& tm_r1, const CUtensorMap& tm_r2, const CUtensorMap& tm_c1, const CUtensorMap& tm_c2, const BwdParams& p,
                                         const int block) {
    using C = BwdCfg<D, MODE, CAP, LD>;
    constexpr bool KEYS = C::KEYS;
    constexpr int NCOL = C::NCOL;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    BwdCtl& ctl = *reinterpret_cast<BwdCtl*>(smem_raw + C::OFF_CTL);
    const uint32_t base = smem_u32(smem_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    // the longest items first: key tile 0, or the last query tile
    const int q0 = p.by_heads.div(block), head = block - q0 * p.heads;
    const int row_tile = KEYS ? q0 : p.nt - 1 - q0;
    const int owner = KEYS ? p.by_split.div(head) : head, part = head - owner * (KEYS ? p.split : 1);       // part: of the query heads
    const int b = p.by_rows_H.div(owner), h = owner - b * (KEYS ? p.Hkv : p.Hq);
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
        mbar_init(smem_u32(&ctl.r_taken), 256);
        mbar_init(smem_u32(&ctl.acc_full), (C::HAS_V ? 1 : 0) + (C::HAS_DS ? 1 : 0));
        mbar_init(smem_u32(&ctl.dg_full), 128);
        for (int s = 0; s < C::NSLOT; ++s) { mbar_init(smem_u32(&ctl.full[s]), 1); mbar_init(smem_u32(&ctl.empty[s]), 1); }
        for (int x = 0; x < 4; ++x) { mbar_init(smem_u32(&ctl.id_full[x]), 1); mbar_init(smem_u32(&ctl.id_empty[x]), 4); }
        for (int x = 0; x < C::NI; ++x) {
            mbar_init(smem_u32(&ctl.info_full[x]), 1);
            mbar_init(smem_u32(&ctl.info_empty[x]), 4);             // (the four warps of a tile)
        }
        for (int x = 0; x < C::NPL; ++x) {
            mbar_init(smem_u32(&ctl.x_full[x]), 1);
            mbar_init(smem_u32(&ctl.x_taken[x]), 128);
            mbar_init(smem_u32(&ctl.y_full[x]), 1);
            for (int q = 0; q < 2; ++q) { mbar_init(smem_u32(&ctl.p_full[x][q]), 128); mbar_init(smem_u32(&ctl.ds_full[x][q]), 128); }
        }
        for (int x = 0; x < 8; ++x) ctl.more[x] = 1;
        ctl.abort_flag = 0;
        ctl.none = 0;
        ctl.limit = wait_limit(4000000000ull);
        fence_mbar_init();
    }
    if constexpr (C::AUG) {                 // rows of ones against the terms of lse, and of delta
        for (int e = threadIdx.x; e < 512; e += BWD_THREADS)
            *reinterpret_cast<uint4*>(smem_raw + C::OFF_CONST + e * 16) = e < 128 ? make_uint4(0x3f803f80u, 0x3f80u, 0u, 0u)
                                                                          : e >= 256 && e < 384 ? make_uint4(0u, 0x3f800000u, 0x3f803f80u, 0u) : make_uint4(0u, 0u, 0u, 0u);
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

    // 64-column piece u of the row tiles on their way to tensor memory
    auto unit_at = [&](int u) -> uint32_t {
        constexpr int H = C::RU > 0 ? C::RU / 2 : 1;
        return base + C::OFF_C + C::slot_at(u < H ? C::NS1 - 1 : C::NSLOT - 1) + (uint32_t)(u % H) * C::SUBR;
    };
    if (warp < 4) reg_dec<C::REGS_FEW>();
    if (warp == 0 || warp == 3) {
        // ------------------------------------------------------------------ TMA: row tiles, C1 and the tiles' numbers; C2 and what goes by the column
        const bool one = warp == 0;
        const int hk = KEYS ? h : h / p.G;
        if (one && lane == 0) {
            mbar_arrive_expect_tx(smem_u32(&ctl.r_full), C::NR * C::R_BYTES + C::RU * C::SUBR + C::GR_BYTES);
            if constexpr (C::GM) bulk_load(base + C::OFF_GR, p.g_rows + ((size_t)b * p.nt + row_tile) * 128 * C::GK, C::GR_BYTES, smem_u32(&ctl.r_full));
#pragma unroll 1
            for (int c = 0; c < C::SUBT; ++c) {
                tma_load_4d(C::R1T ? unit_at(c) : base + c * C::SUBR, &tm_r1, smem_u32(&ctl.r_full), c * 64, row_tile * 128, h, b);
                if (MODE != BWD_V)
                    tma_load_4d(C::R2T ? unit_at((C::R1T ? C::SUBT : 0) + c) : base + C::R_BYTES + c * C::SUBR, &tm_r2, smem_u32(&ctl.r_full), c * 64, row_tile * 128, h, b);
            }
        }
        BwdWalk<KEYS, NCOL> walk(p, lane, row_tile, b, h, part);
        const CUtensorMap* const map = one ? &tm_c1 : &tm_c2;
        const uint32_t slot0 = one ? 0 : C::NS1, slots = one ? C::NS1 : C::NS2;
        uint32_t slot = 0, phase = 0;
        RingAt<4> id;
        RingAt<C::NI> info;
        // The numbers go ahead of the tiles: a group asks for its next one when it begins with a tile, and C1 of that may have to wait for it
        BwdWalk<KEYS, NCOL> ahead(p, lane, row_tile, b, h, part);
        int ends = one ? 0 : 2;
        auto hand_id = [&]() -> bool {
            if (ends == 2) return true;
            const int t = ends ? -1 : ahead.next();
            if (t < 0) ++ends;                                      // (a last one for each group of warps)
            if (!wait(ctl.id_empty[id.slot], id.phase ^ 1, 13)) return false;
            if (lane == 0) {
                if (t < 0 && ahead.at < 0) ctl.none = 1;
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
            if (!hand_id()) break;
            // (what can be is done before the slot is free: what comes after is in the way of the tile.  The bytes are announced behind the
            // wait: before it the slot's last copy may be under way, and its phase with it.)
            const uint32_t bar = smem_u32(&ctl.full[slot0 + slot]), at = base + C::OFF_C + C::slot_at(slot0 + slot);
            const int row0 = t * NCOL;
            const __nv_bfloat16* const aug = p.aug + (((size_t)(b * p.Hq + hc) * p.nt + row0 / 128) * 128 + row0 % 128) * 8;
            if (!wait(ctl.empty[slot0 + slot], phase ^ 1, 11)) break;
            if (C::RU > 0 && phase == 0 && slot == slots - 1 && !wait(ctl.r_taken, 0, 14)) break;
            if (lane == 0) {
                if (t >= 0) {
                    mbar_arrive_expect_tx(bar, one ? C::C1_BYTES : C::C_BYTES);
#pragma unroll
                    for (int c = 0; c < C::SUBT; ++c) tma_load_4d(at + c * C::SUBC, map, bar, c * 64, row0, hc, b);
                    if (C::AUG && one) bulk_load(at + C::C_BYTES, aug, C::AUG_BYTES, bar);
                    if (C::GM && one) bulk_load(at + C::C_BYTES, p.g_cols + ((size_t)b * p.nt * 2 + t) * 64 * C::GK, C::GC_BYTES, bar);
                } else {
                    ctl.more[slot0 + slot] = 0;
                    mbar_arrive(bar);
                }
            }
            __syncwarp();
            if (!one && C::INFO_BYTES > 0 && t >= 0) {
                if (!wait(ctl.info_empty[info.slot], info.phase ^ 1, 12)) break;
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&ctl.info_full[info.slot]), at = base + C::OFF_INFO + info.slot * C::INFO_BYTES;
                    mbar_arrive_expect_tx(bar, C::INFO_BYTES);
                    if constexpr (C::STAT_BYTES > 0) {
                        const float* st = p.stat + ((size_t)(b * p.Hq + hc) * p.nt + t * NCOL / 128) * 256 + t * NCOL % 128;
                        bulk_load(at, st, NCOL * 4, bar);
                        bulk_load(at + NCOL * 4, st + 128, NCOL * 4, bar);
                    }
                    if constexpr (C::GATE_SMEM) bulk_load(at + C::STAT_BYTES, p.g_flat + ((size_t)b * p.nt * 2 + t) * 64 * LD, C::GATE_BYTES, bar);
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
            const uint32_t c = ck + (C::slot_at(at) >> 4);
            auto step = [&](int ks) { return c + (ks >> 2) * (C::SUBC >> 4) + (ks & 3) * 2; };
            if (y ? C::R2T : C::R1T) {
                const uint32_t r = tmem + C::COL_R + (y && C::R1T ? D / 2 : 0);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) umma_ts_lo(d, r + ks * 8, step(ks), IDESC_X, ks > 0);
            } else {
                const uint32_t r = y ? r2 : r1;
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) umma_ss_lo(d, r + (ks >> 2) * (C::SUBR >> 4) + (ks & 3) * 2, step(ks), IDESC_X, ks > 0);
            }
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
            if constexpr (C::GM) {
                const uint64_t r = smem_desc_plain(base + C::OFF_GR, 2048, 128), c = smem_desc_plain(base + C::OFF_C + C::slot_at(c1) + C::C_BYTES, NCOL * 16, 128);
#pragma unroll
                for (int ks = 0; ks < C::GK / 16; ++ks) umma_ss(tmem + C::COL_U + place * NCOL, r + ks * (4096 >> 4), c + ks * (NCOL * 32 >> 4), IDESC_X, ks > 0);
            }
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
            for (int x = 0; x < C::NPL; ++x) {
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
            if (!wait(ctl.r_full, 0, 20) || (C::RU > 0 && !wait(ctl.r_taken, 0, 28))) break;
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
        reg_inc<C::REGS_MANY>();
        const int wg = (warp - 4) >> 2;                    // tiles of this parity
        const int row_in_tile = ((warp & 3) << 5) | lane;
        const int row = row_tile * 128 + row_in_tile;      // position of this thread's token
        const bool valid = row < p.n;
        const uint32_t tm = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const float sl2 = CAP ? p.softcap * LOG2E : p.scale * LOG2E;
        const float cap_in = CAP ? p.scale / p.softcap : 0.f;
        // A thread has a row.  With the gate, which needs a column's assignment for every pair, it has four rows, 8 apart, and of every 8 columns
        // two, so that what goes by the column is read once for four rows.  (Without the gate: tensor memory gives a row a thread faster, 3130 cycles a
        // tile of dK and dV at D = 128 where four rows a thread took 3390.)
        const int l4 = lane >> 2, c2 = 2 * (lane & 3);     // row (of each 8) and first column (of each 8)
        const int rowq = row_tile * 128 + (warp & 3) * 32 + l4;        // its rows: rowq + 8 q
        constexpr int ROWS = LD > 0 ? 4 : 1;
        float lrow[ROWS] = {}, drow[ROWS] = {};            // rows are queries: -lse log2(e) and -delta
        if constexpr (!KEYS) {
            const float* st = p.stat + ((size_t)head * p.nt + row_tile) * 256 + (LD > 0 ? (warp & 3) * 32 + l4 : row_in_tile);
#pragma unroll
            for (int q = 0; q < ROWS; ++q) {
                lrow[q] = dep_load(st + 8 * q);
                drow[q] = dep_load(st + 128 + 8 * q);
            }
        }
        uint32_t mask = 0;
        if (p.bits) mask = valid ? dep_load(p.row_mask + (size_t)owner * p.n + row) & (0xffffffffu >> (32 - p.K)) : 0u;
        constexpr int LDR = LD > 0 ? LD : 1, LQ = LD > 0 ? 4 : 1, NW = NCOL / 32;
        float gr[C::GM ? 1 : LQ][C::GM ? 1 : LDR], dg[LQ][LDR];        // assignments of the rows times -lambda log2(e), their gradients over scale lambda
        if constexpr (LD > 0) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int e = 0; e < LD; ++e) {
                    if constexpr (!C::GM) gr[q][e] = rowq + 8 * q < p.n ? dep_load(p.g + ((size_t)b * p.n + rowq + 8 * q) * LD + e) * (-p.lambda * LOG2E) : 0.f;
                    dg[q][e] = 0.f;
                }
            }
        }
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
            if (lane == 0 && (ct | hc) >= -1) mbar_arrive(smem_u32(&ctl.id_empty[slot]));      // (always so: but not known before the two are there)
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
        if constexpr (C::RU > 0) {
            // the row tiles to tensor memory: a thread its row, each group half of the pieces
            if (wait(ctl.r_full, 0, 29)) {
#pragma unroll 1
                for (int u = wg * (C::RU / 2); u < (wg + 1) * (C::RU / 2); ++u) {
                    const unsigned char* const at = smem_raw + (unit_at(u) - base) + row_in_tile * 128;
                    uint32_t w[32];
#pragma unroll
                    for (int e = 0; e < 8; ++e) *reinterpret_cast<uint4*>(&w[4 * e]) = *reinterpret_cast<const uint4*>(at + ((e ^ (row_in_tile & 7)) << 4));
                    tmem_st32(tm + C::COL_R + u * 32, w);
                }
                tmem_wait_st();
                fence_proxy_async_smem();          // (read here, copied over by the tiles)
                tc_fence_before();
                mbar_arrive(smem_u32(&ctl.r_taken));
            }
        }
        uint32_t k = 0, place = wg, par = 0;               // the tile's place, the parity of its use
        if (!bad && peek(0)) {
#pragma unroll 1
            for (; ct >= 0; ++k) {
                const uint32_t t_x = tm + place * NCOL;
                const uint32_t at_info = C::NI == 2 ? wg : wg + 2 * (k & 1);
                const float* const info = reinterpret_cast<const float*>(smem_raw + C::OFF_INFO + at_info * C::INFO_BYTES);
                const float* const gcol = info + C::STAT_BYTES / 4;
                const int now = ct;
                // ---- which columns count: bit c of word c / 32
                const int col0 = now * NCOL;
                // a quarter of column c + c2's assignments (in shared memory side by side for the four lanes that read at once)
                auto gate_at = [&](int c, int e) -> float4 {
                    if constexpr (C::GATE_SMEM) return reinterpret_cast<const float4*>(gcol)[((c / 8 * 2 + c % 2) * (LDR / 4) + e) * 4 + (lane & 3)];
                    else return reinterpret_cast<const float4*>(p.g + ((size_t)b * p.n + min(col0 + c + c2, p.n - 1)) * LDR)[e];
                };
                uint32_t kw[NW];
                bool masked, near;                             // near: some pairs of the tile are not distant
                {
                    const int lo_q = KEYS ? col0 : row_tile * 128, hi_q = KEYS ? col0 + NCOL - 1 : row_tile * 128 + 127;
                    const int lo_k = KEYS ? row_tile * 128 : col0, hi_k = KEYS ? row_tile * 128 + 127 : col0 + NCOL - 1;
                    const bool causal = lo_q < hi_k, outside = p.bits && hi_q - lo_k > p.w;
                    masked = causal || outside;
                    near = lo_q - hi_k <= p.w;
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
                if (LD == 0 && !peek(k + 1)) break;
                // ---- P
                if (C::INFO_BYTES > 0 && !wait(ctl.info_full[at_info], (C::NI == 2 ? k : k >> 1) & 1, 38)) break;
                if (!wait(ctl.x_full[place], par, 30)) break;
                tc_fence_after();
                if constexpr (LD == 0) {
                    uint32_t pr[NCOL];                             // X, then P times the slope of the logit
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
                        auto piece = [&](auto far) {
#pragma unroll
                            for (int e = c; e < c + 32; e += 4) {
                                float2 l[2];
                                if constexpr (C::STAT_BYTES > 0) *reinterpret_cast<float4*>(l) = lc[(e - c) / 4];
                                else l[0] = l[1] = make_float2(lrow[0], lrow[0]);
#pragma unroll
                                for (int f = 0; f < 2; ++f) {
                                    uint32_t &u0 = pr[e + 2 * f], &u1 = pr[e + 2 * f + 1];
                                    float2 x = make_float2(__uint_as_float(u0), __uint_as_float(u1)), y;
                                    if constexpr (CAP) {
                                        x = __fmul2_rn(x, make_float2(cap_in, cap_in));
                                        const float2 z = x;
                                        x.x = tanh_approx(x.x);
                                        x.y = tanh_approx(x.y);
                                        y = __ffma2_rn(x, make_float2(sl2, sl2), l[f]);
                                        y.x = ex2_approx(y.x);
                                        y.y = ex2_approx(y.y);
                                        if constexpr (decltype(far)::value) {
                                            const float2 w = make_float2(ex2_approx(fabsf(z.x) * (-2.f * LOG2E)), ex2_approx(fabsf(z.y) * (-2.f * LOG2E)));
                                            x = make_float2(1.f + fabsf(x.x), 1.f + fabsf(x.y));
                                            x = __fmul2_rn(__fmul2_rn(y, w), __fmul2_rn(x, x));
                                        } else {
                                            x = __fmul2_rn(y, __ffma2_rn(make_float2(-x.x, -x.y), x, make_float2(1.f, 1.f)));
                                        }
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
                        };
                        // The cap's slope 1 - t^2: where t is next to 1 the difference has nothing left (with the hardware's t: right to 2^-12
                        // up to 3.5 caps, 1 % off from 4 on, a quarter at 7, all of it from 8).  Beyond 3.5 it is e (1 + |t|)^2, e = exp(-2 |x|):
                        // t = (1 - e) / (1 + e), so that 1 + t = 2 / (1 + e).  That is an exponential more a pair, which a warp takes where one of its
                        // 32 x 32 scores needs it (32/8 heads x 4096, D = 128: 669 us with the difference alone, 847 with the other alone, 691 so, and
                        // 920 for scores most of which are beyond).  At D = 256, whose passes wait for copies, to look at the scores costs more
                        // than the exponential (16/8 x 4096: 518, 550 and 561 us): always.
                        bool far = D == 256;
                        if constexpr (CAP && C::HAS_DS && D != 256) {
                            float m = 0.f;
#pragma unroll
                            for (int e = c; e < c + 32; ++e) m = fmaxf(m, fabsf(__uint_as_float(pr[e])));
                            far = __any_sync(0xffffffffu, m * cap_in > 3.5f);
                        }
                        if (CAP && C::HAS_DS && far) piece(std::true_type());
                        else piece(std::false_type());
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
                                    else d[0] = d[1] = make_float2(drow[0], drow[0]);
#pragma unroll
                                    for (int f = 0; f < 2; ++f) {
                                        const int at = at0 + 2 * f;
                                        const float2 u = make_float2(__uint_as_float(pr[at]), __uint_as_float(pr[at + 1]));
                                        float2 ds = make_float2(__uint_as_float(yr[e + 2 * f]), __uint_as_float(yr[e + 2 * f + 1]));
                                        ds = __fmul2_rn(u, C::AUG ? ds : __fadd2_rn(ds, d[f]));
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
                } else {
                    // The gate.  P times the factor waits for Y in tensor memory, what turns dS into the gradient of g_i . g_j in registers.
                    constexpr uint32_t HALF = 16u << 16;       // 16 lanes on
                    const uint32_t t_u = tm + C::COL_U + wg * NCOL;
                    float2 da[4][NCOL / 8];                    // [row][two columns of every 8]
                    int bound[4], last[4];                     // columns beyond which a pair is distant; the diagonal
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        last[q] = rowq + 8 * q - col0 - c2;
                        bound[q] = KEYS ? last[q] + p.w : last[q] - p.w;
                    }
#pragma unroll
                    for (int c = 0; c < NCOL; c += 16) {
                        uint32_t xr[2][8];
                        tmem_ld_frag(t_x + c, xr[0]);
                        tmem_ld_frag(t_x + HALF + c, xr[1]);
                        uint32_t gx[2][C::GM ? 8 : 1];
                        if constexpr (C::GM) {
                            tmem_ld_frag(t_u + c, gx[0]);
                            tmem_ld_frag(t_u + HALF + c, gx[1]);
                        }
                        tmem_wait_ld();
                        if (C::GM && near) {                   // pairs that are not distant: f = 1, z = 0
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const int cj = c + 8 * (e / 2) + e % 2;
                                    uint32_t& u = gx[q / 2][C::GM ? 4 * (e / 2) + 2 * (q % 2) + e % 2 : 0];
                                    u = (KEYS ? cj > bound[q] : cj < bound[q]) ? u : 0xff800000u;
                                }
                            }
                        }
                        if (!C::HAS_V && c + 16 == NCOL) {
                            tc_fence_before();
                            mbar_arrive(smem_u32(&ctl.x_taken[place]));
                        }
                        uint32_t pk[2][4];
                        // (step by step for all 16 columns)
                        float2 s[8], f[8], lc[2] = {};             // [j][row]; s: both columns' g_i . g_j times -lambda log2(e), then z
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const int cj = c + 8 * j;
                            if constexpr (KEYS) lc[j] = *reinterpret_cast<const float2*>(info + cj + c2);
                            if constexpr (C::GM) {
#pragma unroll
                                for (int q = 0; q < 4; ++q)
                                    s[4 * j + q] = make_float2(__uint_as_float(gx[q / 2][4 * j + 2 * (q % 2)]), __uint_as_float(gx[q / 2][4 * j + 2 * (q % 2) + 1]));
                            } else {
                                float2 part[2][4];
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
#pragma unroll
                                    for (int q = 0; q < 4; ++q) part[i][q] = make_float2(0.f, 0.f);
#pragma unroll
                                    for (int e = 0; e < LD / 4; ++e) {
                                        const float4 v = gate_at(cj + i, e);
#pragma unroll
                                        for (int q = 0; q < 4; ++q) {
                                            part[i][q] = __ffma2_rn(make_float2(gr[q][4 * e], gr[q][4 * e + 1]), make_float2(v.x, v.y), part[i][q]);
                                            part[i][q] = __ffma2_rn(make_float2(gr[q][4 * e + 2], gr[q][4 * e + 3]), make_float2(v.z, v.w), part[i][q]);
                                        }
                                    }
                                }
#pragma unroll
                                for (int q = 0; q < 4; ++q) {
                                    s[4 * j + q] = make_float2(part[0][q].x + part[0][q].y, part[1][q].x + part[1][q].y);
                                    if (!(KEYS ? cj > bound[q] : cj < bound[q])) s[4 * j + q].x = -INFINITY;
                                    if (!(KEYS ? cj + 1 > bound[q] : cj + 1 < bound[q])) s[4 * j + q].y = -INFINITY;
                                }
                            }
                        }
                        // sigmoid of a distant pair: 1 / (1 + z), z = exp(-lambda g_i . g_j); 1 - f = z f
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            s[e].x = ex2_approx(fminf(s[e].x, 126.f));
                            s[e].y = ex2_approx(fminf(s[e].y, 126.f));
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            f[e] = __fadd2_rn(s[e], make_float2(1.f, 1.f));
                            f[e].x = rcp_approx(f[e].x);
                            f[e].y = rcp_approx(f[e].y);
                        }
                        float2 y[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int j = e / 4, q = e % 4;
                            const uint32_t* const u = &xr[q / 2][4 * j + 2 * (q % 2)];
                            const float2 xf = __fmul2_rn(make_float2(__uint_as_float(u[0]), __uint_as_float(u[1])), f[e]);
                            da[q][c / 8 + j] = __fmul2_rn(s[e], xf);            // (dS, by which it is multiplied, has the other f)
                            y[e] = __ffma2_rn(xf, make_float2(sl2, sl2), KEYS ? lc[j] : make_float2(lrow[q], lrow[q]));
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            y[e].x = ex2_approx(y[e].x);
                            y[e].y = ex2_approx(y[e].y);
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int j = e / 4, q = e % 4, hf = q / 2, r = q % 2;
                            if constexpr (C::HAS_V) pk[hf][2 * j + r] = pack_bf16x2(y[e].x, y[e].y);
                            const float2 u = __fmul2_rn(y[e], f[e]);
                            xr[hf][4 * j + 2 * r] = __float_as_uint(u.x);
                            xr[hf][4 * j + 2 * r + 1] = __float_as_uint(u.y);
                        }
                        if (masked) {                          // (causality alone)
#pragma unroll
                            for (int q = 0; q < 4; ++q) {
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const int cj = c + 8 * j, hf = q / 2, w = 2 * j + q % 2;
                                    const bool k0 = KEYS ? cj >= last[q] : cj <= last[q], k1 = KEYS ? cj + 1 >= last[q] : cj + 1 <= last[q];
                                    xr[hf][2 * w] = k0 ? xr[hf][2 * w] : 0u;
                                    xr[hf][2 * w + 1] = k1 ? xr[hf][2 * w + 1] : 0u;
                                    if constexpr (C::HAS_V) pk[hf][w] &= (k0 ? 0xffffu : 0u) | (k1 ? 0xffff0000u : 0u);
                                }
                            }
                        }
                        if constexpr (C::HAS_DS) {
                            tmem_st_frag(t_u + c, xr[0]);
                            tmem_st_frag(t_u + HALF + c, xr[1]);
                        }
                        if constexpr (C::HAS_V) {
                            tmem_st_pairs(t_x + c / 2, pk[0]);
                            tmem_st_pairs(t_x + HALF + c / 2, pk[1]);
                        }
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    if constexpr (C::HAS_V) mbar_arrive(smem_u32(&ctl.p_full[place][0]));
                    if (!peek(k + 1)) break;                   // (a number alone: while Y is on its way)
                    // ---- dS
                    if constexpr (C::HAS_DS) {
                        if (!wait(ctl.y_full[place], par, 31)) break;
                        tc_fence_after();
#pragma unroll
                        for (int c = 0; c < NCOL; c += 16) {
                            uint32_t pk[2][4];
#pragma unroll
                            for (int hf = 0; hf < 2; ++hf) {
                                uint32_t yr[8], ur[8];
                                tmem_ld_frag(t_x + hf * HALF + c, yr);
                                tmem_ld_frag(t_u + hf * HALF + c, ur);
                                tmem_wait_ld();
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const int cj = c + 8 * j;
                                    float2 dc = make_float2(0.f, 0.f);
                                    if constexpr (KEYS) dc = *reinterpret_cast<const float2*>(info + NCOL + cj + c2);
#pragma unroll
                                    for (int r = 0; r < 2; ++r) {
                                        const int q = 2 * hf + r;
                                        const float2 d = KEYS ? dc : make_float2(drow[q], drow[q]);
                                        const float2 y = __fadd2_rn(make_float2(__uint_as_float(yr[4 * j + 2 * r]), __uint_as_float(yr[4 * j + 2 * r + 1])), d);
                                        const float2 ds = __fmul2_rn(make_float2(__uint_as_float(ur[4 * j + 2 * r]), __uint_as_float(ur[4 * j + 2 * r + 1])), y);
                                        da[q][cj / 8] = __fmul2_rn(da[q][cj / 8], ds);
                                        pk[hf][2 * j + r] = pack_bf16x2(ds.x, ds.y);
                                    }
                                }
                            }
                            tmem_st_pairs(t_x + c / 2, pk[0]);
                            tmem_st_pairs(t_x + HALF + c / 2, pk[1]);
                        }
                        tmem_wait_st();
                        tc_fence_before();
                        mbar_arrive(smem_u32(&ctl.ds_full[place][0]));
#pragma unroll
                        for (int cj = 0; cj < NCOL; cj += 8) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
#pragma unroll
                                for (int e = 0; e < LD / 4; ++e) {
                                    const float4 v = gate_at(cj + i, e);
#pragma unroll
                                    for (int q = 0; q < 4; ++q) {
                                        const float a = i ? da[q][cj / 8].y : da[q][cj / 8].x;
                                        const float2 lo = __ffma2_rn(make_float2(a, a), make_float2(v.x, v.y), make_float2(dg[q][4 * e], dg[q][4 * e + 1]));
                                        const float2 hi = __ffma2_rn(make_float2(a, a), make_float2(v.z, v.w), make_float2(dg[q][4 * e + 2], dg[q][4 * e + 3]));
                                        dg[q][4 * e] = lo.x; dg[q][4 * e + 1] = lo.y; dg[q][4 * e + 2] = hi.x; dg[q][4 * e + 3] = hi.y;
                                    }
                                }
                            }
                        }
                    }
                }
                // Every read of what goes by the column has to be through before the next copy over it.  Reads go by the generic proxy, the copy writes by the
                // async one, and a barrier's arrival orders the first with what comes after it only within its own proxy: so the fence between the two, by every
                // thread that read.  (Without it, D = 64 and K = 4: dg of some rows with the numbers of the tile after next.  lse and delta had gone into what
                // was handed over before, and were right all the same.)
                if constexpr (C::INFO_BYTES > 0) fence_proxy_async_smem();
                __syncwarp();
                if (C::INFO_BYTES > 0 && lane == 0) mbar_arrive(smem_u32(&ctl.info_empty[at_info]));
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
            // sums of the launches before, and whether this is the last for these rows
            const bool add = KEYS ? p.later || row_tile < p.col_lo : p.col_lo > 0, done = KEYS ? p.last && p.split == 1 : row_tile < p.col_hi;
            float* const sums = (v ? p.part1 : p.part2) + ((size_t)head * p.n + (valid ? row : 0)) * D + col0;
            const bool none = *(volatile int*)&ctl.none;
#pragma unroll 1
            for (int c = 0; c < NOUT; c += 16) {
                uint32_t ov[16];
                tmem_ld16(t_a + c, ov);
                tmem_wait_ld();
                if (none) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) ov[e] = 0u;
                }
                if (add && valid) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        const float4 x = *reinterpret_cast<const float4*>(sums + c + e);
                        ov[e] = __float_as_uint(x.x + __uint_as_float(ov[e]));
                        ov[e + 1] = __float_as_uint(x.y + __uint_as_float(ov[e + 1]));
                        ov[e + 2] = __float_as_uint(x.z + __uint_as_float(ov[e + 2]));
                        ov[e + 3] = __float_as_uint(x.w + __uint_as_float(ov[e + 3]));
                    }
                }
                if (!done) {
                    if (valid) {
#pragma unroll
                        for (int e = 0; e < 16; e += 4) *reinterpret_cast<uint4*>(sums + c + e) = make_uint4(ov[e], ov[e + 1], ov[e + 2], ov[e + 3]);
                    }
                    continue;
                }
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
                // a row's sums are those of four lanes, and of the even and the odd tiles: the second group hands its own to the first (the
                // slots are through)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int e = 0; e < LD; ++e) {
                        dg[q][e] += __shfl_xor_sync(0xffffffffu, dg[q][e], 1);
                        dg[q][e] += __shfl_xor_sync(0xffffffffu, dg[q][e], 2);
                        dg[q][e] *= p.scale * p.lambda;
                    }
                }
                float* const x = reinterpret_cast<float*>(smem_raw + C::OFF_C) + (threadIdx.x & 127);       // [e][thread]: lane t has row t / 4 + 8 (t % 4)
                const bool other = wg == 0 && wait(ctl.dg_full, 0, 41);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    if ((lane & 3) != q) continue;
                    if (wg == 1) {
#pragma unroll
                        for (int e = 0; e < LD; ++e) x[e * 128] = dg[q][e];
                    } else if (other && rowq + 8 * q < p.n) {
                        float4* const to = reinterpret_cast<float4*>(p.dg_part + ((size_t)head * p.n + rowq + 8 * q) * LD);
#pragma unroll
                        for (int e = 0; e < LD; e += 4) {
                            const float4 old = add ? to[e / 4] : make_float4(0.f, 0.f, 0.f, 0.f);
                            to[e / 4] = make_float4(old.x + (dg[q][e] + x[e * 128]), old.y + (dg[q][e + 1] + x[(e + 1) * 128]), old.z + (dg[q][e + 2] + x[(e + 2) * 128]),
                                                    old.w + (dg[q][e + 3] + x[(e + 3) * 128]));
                        }
                    }
                }
                if (wg == 1) mbar_arrive(smem_u32(&ctl.dg_full));
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

// All passes in one launch: they need nothing of one another, and the blocks of one fill the places that the other's last ones leave
// (32 query on 8 KV heads x 8192 tokens 1801 -> 1753 us, 12 heads x 1024 34 -> 21).  Tensor maps of q, k, v and do, first for row tiles, then for column tiles.
struct BwdMaps {
    CUtensorMap r[4], c[4];
};

template <int D, bool CAP, int LD>
__global__ void __launch_bounds__(BWD_THREADS, 1)
attn_bwd_kernel(const __grid_constant__ BwdMaps m, const __grid_constant__ BwdParams kv, const __grid_constant__ BwdParams q) {
    const int nkv = kv.heads * kv.row_tiles, block = (int)blockIdx.x;
    if constexpr (D == 256) {
        if (block < nkv) bwd_item<D, BWD_K, CAP, LD>(m.r[1], m.r[2], m.c[0], m.c[3], kv, block);
        else if (block < 2 * nkv) bwd_item<D, BWD_V, CAP, LD>(m.r[1], m.r[2], m.c[0], m.c[3], kv, block - nkv);
        else bwd_item<D, BWD_Q, CAP, LD>(m.r[0], m.r[3], m.c[1], m.c[2], q, block - 2 * nkv);
    } else {
        if (block < nkv) bwd_item<D, BWD_KV, CAP, LD>(m.r[1], m.r[2], m.c[0], m.c[3], kv, block);
        else bwd_item<D, BWD_Q, CAP, LD>(m.r[0], m.r[3], m.c[1], m.c[2], q, block - nkv);
    }
}

template <int D, bool CAP, int LD>
static int launch_bwd_passes(const AttnBwdArgs& a, const BwdParams& kv, const BwdParams& q, cudaStream_t st) {
    using KV = BwdCfg<D, D == 256 ? BWD_K : BWD_KV, CAP, LD>;
    using V = BwdCfg<D, D == 256 ? BWD_V : BWD_KV, CAP, LD>;
    using Q = BwdCfg<D, BWD_Q, CAP, LD>;
    constexpr uint32_t smem = KV::SMEM > Q::SMEM ? (KV::SMEM > V::SMEM ? KV::SMEM : V::SMEM) : (Q::SMEM > V::SMEM ? Q::SMEM : V::SMEM);
    const focus_tensor* const t[4] = {&a.q, &a.k, &a.v, &a.dO};
    const int heads[4] = {a.s.Hq, a.s.Hkv, a.s.Hkv, a.s.Hq};
    BwdMaps m;
    int rc;
    for (int i = 0; i < 4; ++i)
        if ((rc = make_tmap_qkv(&m.r[i], *t[i], a.s.batch, heads[i], a.s.n, D)) || (rc = make_tmap_qkv(&m.c[i], *t[i], a.s.batch, heads[i], a.s.n, D, Q::NCOL))) return rc;
    const long long most = (long long)kv.heads * kv.nt * (D == 256 ? 2 : 1) + (long long)q.heads * q.nt;
    if (most > 0x7fffffffll) return fail(FOCUS_ERR_UNSUPPORTED, "attention backward: %lld tiles exceed 2^31 - 1", most);
    if ((rc = check_cuda(allow_smem<attn_bwd_kernel<D, CAP, LD>>(smem), "cudaFuncSetAttribute(attn_bwd)"))) return rc;
    // The longest way first: a pass over keys takes its heads together as far as they go, or each in pieces; one over queries its keys in pieces
    auto kern = attn_bwd_kernel<D, CAP, LD>;
    const int step = kv.nt < BWD_LAUNCH_TILES ? kv.nt : BWD_LAUNCH_TILES, pieces = cdiv(kv.nt, step), together = bwd_heads_together(kv.nt, kv.heads_each);
    const int runs = cdiv(kv.heads_each, together) * pieces;
    for (int x = 0; x < runs; ++x) {
        BwdParams k = kv, r = q;
        k.head_lo = x / pieces * together;
        k.head_hi = k.head_lo + together < kv.heads_each ? k.head_lo + together : kv.heads_each;
        k.col_lo = x % pieces * step;
        k.col_hi = k.col_lo + step < kv.nt ? k.col_lo + step : kv.nt;
        k.later = k.head_lo > 0;
        k.last = x == runs - 1;
        k.row_tiles = k.col_hi;
        r.col_lo = x < pieces ? k.col_lo : kv.nt;
        r.col_hi = x < pieces ? k.col_hi : kv.nt;
        r.head_hi = 1;
        r.row_tiles = kv.nt - r.col_lo;
        const long long blocks = (long long)k.heads * k.row_tiles * (D == 256 ? 2 : 1) + (long long)r.heads * r.row_tiles;
        if ((rc = check_cuda(launch_dependent(kern, dim3((unsigned)blocks), dim3(BWD_THREADS), smem, st, m, k, r), "attention backward launch"))) return rc;
    }
    return FOCUS_OK;
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
