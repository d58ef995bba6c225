// focus_qk_norm_rope and its derivative: the query and key heads of a layer normalised head by head and rotated by their positions, as
// focus_assign and the attention read them; focus_rope_frequencies (host): what a position is multiplied by.
//
//   y = x * r * w,  r = (mean x^2 + eps)^(-1/2);   (a, b) -> (a cos t - b sin t, a sin t + b cos t) * amplitude,  t = position * freq_i
// and back: with g the rotated-back gradient of y, xhat = x r and u = g w:
//   dx = r (u - xhat mean(u xhat)),   dw = sum over rows of g xhat.
// HBM-bound: every vector read once and written once (backward: vectors and gradients read, gradients written).  One pass over them, rows
// under way in shared memory; what is left to the bound is the start of a CTA, before which its angles and weights have to be there (8192
// tokens, 32 + 8 heads of 128, bf16: forward 28.9 us, 5.8 TB/s, 88 % of what a copy reaches; backward with the weights' gradients 46.4 us,
// 5.4 TB/s, 82 %).  Few rows are bound by latency: the forward pass over 16 sequences of one token takes 2.9 us, the backward pass over
// 3 sequences of 1021 tokens of 12 + 12 heads of 64 takes 9.3 to 9.7 with the sums of the weights' gradients.
#include "common.cuh"
#include "f32x2.cuh"

#include <math.h>

namespace focus {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_SMS = 148;
constexpr int ROPE_GRID = ROPE_SMS * 4;           // CTAs that sum weight gradients, at most
constexpr int ROPE_TOKENS = 16;                   // per tile at most

struct RopeArgs {
    const __nv_bfloat16 *x[2], *g[2];             // [0] queries, [1] keys: vectors, and the gradients of the results
    __nv_bfloat16* out[2];
    int64_t x_b[2], x_h[2], x_n[2], g_b[2], g_h[2], g_n[2], o_b[2], o_h[2], o_n[2];
    const float* w[2];
    const double* freq;
    const int32_t* positions;
    float* partial;                               // backward with a norm: [CTAs of a side][D] sums of g xhat, queries' CTAs first
    int heads[2], batch, n, rot;
    float eps, amplitude;
    int lgT[2], per_seq[2];                       // tokens per tile (log), tiles per sequence (forward: [0] for both sides)
    FixedDiv by_seq[2];                           // division by per_seq
    uint32_t parts;                               // forward: parts that a tile's heads are cut into
    FixedDiv by_parts;
    int ctas[2], passes[2];                       // backward: CTAs of a side, passes of a tile;
    int whole[2], rest[2], over[2];               // whole tiles of each CTA, passes behind those, CTAs that share them
    FixedDiv by_passes[2];
};

// cos and sin (times the amplitude) of position * freq: the angle is reduced in 64 bits, since positions reach a million and fp32 would
// leave an error of 0.06 there
__device__ __forceinline__ float2 rope_cos_sin(const RopeArgs& a, int pos, int f) {
    double turns = (double)pos * (dep_load(a.freq + f) * 0.15915494309189533577);
    turns -= rint(turns);
    float sn, cn;
    sincospif((float)(2.0 * turns), &sn, &cn);
    return make_float2(cn * a.amplitude, sn * a.amplitude);
}

// A row is cut into units of 16 dimensions, one per lane: two 16-byte pieces, whose eight pairs are turned.  Rotating halves, unit
// u < rot / 16 has the pieces at 8 u and rot / 2 + 8 u, and behind the rotated part the pieces likewise lie half of the rest apart; interleaved, every
// piece is four whole pairs, and they lie D / 2 apart: so neighbouring lanes have neighbouring pieces (interleaved with both pieces of a lane side by
// side, whose every 32 bytes are then asked for twice: 8192 tokens forward 40.8 us, not 28.3, backward 70.5, not 46.8).  In registers a unit is
// the pairs' first numbers and their second ones: in halves the first piece and the second, interleaved the low and the high numbers of the
// words (INTER, a flag of the template: a branch on it in every row costs 5 %).
template <int D> struct RopeCfg {
    static constexpr int LPR = D / 16;                        // lanes per row
    static constexpr int RPP = ROPE_THREADS / LPR;            // rows per pass of a CTA
};

struct RopeUnit {
    F2 p[4], r[4];                                            // firsts and seconds of pairs (0, 1), (2, 3), (4, 5), (6, 7)
};
__device__ __forceinline__ float bf_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
template <bool INTER>
__device__ __forceinline__ RopeUnit rope_unpack(const uint4 (&raw)[2]) {
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    RopeUnit u;
    if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u.p[i] = f2(bf_lo(w[2 * i]), bf_lo(w[2 * i + 1]));
            u.r[i] = f2(bf_hi(w[2 * i]), bf_hi(w[2 * i + 1]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            u.p[i] = f2(bf_lo(w[i]), bf_hi(w[i]));
            u.r[i] = f2(bf_lo(w[4 + i]), bf_hi(w[4 + i]));
        }
    }
    return u;
}
__device__ __forceinline__ uint32_t bf_pack(float lo, float hi) {
    const __nv_bfloat162 t = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&t);
}
template <bool INTER>
__device__ __forceinline__ void rope_pack(const RopeUnit& u, uint4 (&raw)[2]) {
    uint32_t w[8];
    if constexpr (INTER) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = f2_get(u.p[i]), r = f2_get(u.r[i]);
            w[2 * i] = bf_pack(p.x, r.x);
            w[2 * i + 1] = bf_pack(p.y, r.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 p = f2_get(u.p[i]), r = f2_get(u.r[i]);
            w[i] = bf_pack(p.x, p.y);
            w[4 + i] = bf_pack(r.x, r.y);
        }
    }
    raw[0] = make_uint4(w[0], w[1], w[2], w[3]);
    raw[1] = make_uint4(w[4], w[5], w[6], w[7]);
}
// cosines, sines and negative sines of a unit's pairs; (p, r) -> (p c - r s, p s + r c)
struct RopeAngles {
    F2 c[4], s[4], ns[4];
};
__device__ __forceinline__ void rope_turn(RopeUnit& u, const RopeAngles& a) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const F2 p = u.p[i], r = u.r[i];
        u.p[i] = f2_fma(p, a.c[i], f2_mul(r, a.ns[i]));
        u.r[i] = f2_fma(p, a.s[i], f2_mul(r, a.c[i]));
    }
}
__device__ __forceinline__ float rope_dot(const RopeUnit& a, const RopeUnit& b) {
    F2 t = f2_mul(a.p[0], b.p[0]), v = f2_mul(a.r[0], b.r[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) { t = f2_fma(a.p[i], b.p[i], t); v = f2_fma(a.r[i], b.r[i], v); }
    const float2 x = f2_get(t), y = f2_get(v);
    return (x.x + x.y) + (y.x + y.y);
}
template <int LPR>
__device__ __forceinline__ float rope_row_sum(float x) {
#pragma unroll
    for (int off = LPR / 2; off >= 1; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// where a lane's unit lies in a row
struct RopePlace {
    int d0, d1;
};
template <int D, bool INTER>
__device__ __forceinline__ RopePlace rope_place(const RopeArgs& a, int u) {
    RopePlace x;
    const bool rest = !INTER && 16 * u >= a.rot;
    x.d0 = 8 * u + (rest ? a.rot / 2 : 0);         // (rot + 8 (u - rot / 16))
    x.d1 = x.d0 + (INTER ? D : rest ? D - a.rot : a.rot) / 2;
    return x;
}
// Weights and angles wait in shared memory as the units want them, 16 numbers each (firsts then seconds; cosines then sines), 4 numbers
// apart: eight lanes read eight units' 16 bytes without asking a bank twice.
constexpr int ROPE_UROW = 20;
template <int D, bool INTER>
__device__ __forceinline__ void rope_put_weights(float (*w)[ROPE_UROW], const RopeArgs& a, int side) {
    for (int i = threadIdx.x; i < D; i += ROPE_THREADS) {
        const int u = i / 16, e = i % 16;
        const RopePlace x = rope_place<D, INTER>(a, u);
        // e-th number of the unit: pair e % 8, its first (e < 8) or second
        const int pr = e % 8, d = INTER ? (pr < 4 ? x.d0 : x.d1) + 2 * (pr % 4) + e / 8 : (e < 8 ? x.d0 : x.d1) + pr;
        w[u][e] = a.w[side] ? dep_load(a.w[side] + d) : 1.f;
    }
}
template <int D, bool INTER>
__device__ __forceinline__ void rope_put_angles(float (*t)[D / 16][ROPE_UROW], const RopeArgs& a, int b, int t0, int T, float sign) {
    for (int i = threadIdx.x; i < T * (D / 2); i += ROPE_THREADS) {
        const int k = i / (D / 2), f = i % (D / 2);
        float2 x = make_float2(1.f, 0.f);                     // (behind the rotated part, and where there is no token)
        if (2 * f < a.rot && t0 + k < a.n) x = rope_cos_sin(a, a.positions ? dep_load(a.positions + (size_t)b * a.n + t0 + k) : t0 + k, f);
        const int u = INTER ? f % (D / 4) / 4 : f / 8, pr = INTER ? f / (D / 4) * 4 + f % 4 : f % 8;
        t[k][u][pr] = x.x;
        t[k][u][8 + pr] = sign * x.y;
    }
}
__device__ __forceinline__ RopeUnit rope_get(const float* row) {
    RopeUnit u;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 t = *reinterpret_cast<const float4*>(row + 4 * i);
        F2(&to)[4] = i < 2 ? u.p : u.r;
        to[2 * (i & 1)] = f2(t.x, t.y);
        to[2 * (i & 1) + 1] = f2(t.z, t.w);
    }
    return u;
}
__device__ __forceinline__ RopeAngles rope_get_angles(const float* row) {
    const RopeUnit u = rope_get(row);
    RopeAngles x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x.c[i] = u.p[i];
        x.s[i] = u.r[i];
        const float2 t = f2_get(u.r[i]);
        x.ns[i] = f2(-t.x, -t.y);
    }
    return x;
}

// A thread's pieces wait in places of its own in shared memory, `STAGES` rows of them: copied there asynchronously, so that rows under way cost no
// registers, and read by nobody else, so that no barrier is needed.  Place of piece i of a stage: 16 bytes per thread, thread by thread.
__device__ __forceinline__ uint32_t rope_place_of(int stage, int pieces, int i) { return (uint32_t)(((stage * pieces + i) * ROPE_THREADS + threadIdx.x) * 16); }
// (zeros where it is not `on`: a copy of no bytes reads nothing, wherever src points)
__device__ __forceinline__ void rope_copy(uint32_t dst, const __nv_bfloat16* src, bool on) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(on ? 16 : 0) : "memory");
}
template <bool INTER>
__device__ __forceinline__ void rope_store(__nv_bfloat16* p, int apart, const RopeUnit& u) {
    uint4 out[2];
    rope_pack<INTER>(u, out);
    *reinterpret_cast<uint4*>(p) = out[0];
    *reinterpret_cast<uint4*>(p + apart) = out[1];
}

// Forward: a CTA takes 2^lgT tokens and all their heads, queries then keys (a part of them where there are few tokens).  A thread's token
// and place in the row are the same in every pass, and so what a pair is multiplied by, cosine and sine (worked out once per token) times
// the side's weights, stays in registers; the row's own scale comes last.
constexpr int ROPE_FWD_STAGES = 4;
template <int D, bool INTER>
__global__ void __launch_bounds__(ROPE_THREADS, 3)
qk_norm_rope_kernel(const RopeArgs a) {
    using C = RopeCfg<D>;
    constexpr int STAGES = ROPE_FWD_STAGES;
    extern __shared__ __align__(16) unsigned char smem[];     // the stages
    __shared__ __align__(16) float cs_s[ROPE_TOKENS][D / 16][ROPE_UROW];
    __shared__ __align__(16) float w_s[2][D / 16][ROPE_UROW];
    const int unit = threadIdx.x % C::LPR, rs = threadIdx.x / C::LPR;
    const int lgT = a.lgT[0], T = 1 << lgT, tok = rs & (T - 1), hofs = rs >> lgT, hstep = C::RPP >> lgT;
    const RopePlace at = rope_place<D, INTER>(a, unit);
    const int apart = at.d1 - at.d0;
    const uint32_t tile = a.by_parts(blockIdx.x), part = blockIdx.x - tile * a.parts;
    const int b = a.by_seq[0](tile), t0 = (int)(tile - b * a.per_seq[0]) << lgT, t = min(t0 + tok, a.n - 1);
    const bool live = t0 + tok < a.n;
    // heads of the part, of either side, in whole passes; passes are counted over both
    int h_lo[2], h_hi[2], passes[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int whole = (a.heads[s] + hstep - 1) / hstep, lo = (int)a.by_parts(whole * part), hi = (int)a.by_parts(whole * (part + 1));
        h_lo[s] = lo * hstep + hofs;
        h_hi[s] = min(hi * hstep, a.heads[s]);
        passes[s] = hi - lo;
    }
    dep_wait();
    dep_trigger();
    const uint32_t stages = (uint32_t)__cvta_generic_to_shared(smem);
    // the copies' walk over the rows, ahead of the work's: pointers that move on (addresses worked out row by row: 31.0 us, not 29.3)
    const __nv_bfloat16* src[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) src[s] = a.x[s] + b * a.x_b[s] + t * a.x_n[s] + h_lo[s] * a.x_h[s] + at.d0;
    const __nv_bfloat16* c_at = src[0];
    int64_t c_step = hstep * a.x_h[0];
    int c_left = passes[0], c_h = h_lo[0], c_end = h_hi[0], c_side = 0, into = 0, from = 0;
    auto issue = [&] {
        if (c_left == 0 && c_side == 0) {
            c_side = 1;
            c_at = src[1];
            c_step = hstep * a.x_h[1];
            c_left = passes[1];
            c_h = h_lo[1];
            c_end = h_hi[1];
        }
        if (c_left > 0) {
            const bool on = c_h < c_end;
            rope_copy(stages + rope_place_of(into, 2, 0), c_at, on);
            rope_copy(stages + rope_place_of(into, 2, 1), c_at + apart, on);
            c_at += c_step;
            c_h += hstep;
            --c_left;
            into = (into + 1) % STAGES;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue();
    rope_put_weights<D, INTER>(w_s[0], a, 0);
    rope_put_weights<D, INTER>(w_s[1], a, 1);
    rope_put_angles<D, INTER>(cs_s, a, b, t0, T, 1.f);
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const bool norm = a.w[s] != nullptr;
        // (p, r) -> (p A + r B, p E + r F)
        F2 A[4], B[4], E[4], F[4];
        {
            const RopeUnit w = rope_get(w_s[s][unit]), cs = rope_get(cs_s[tok][unit]);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 sn = f2_get(cs.r[e]);
                A[e] = f2_mul(cs.p[e], w.p[e]);
                B[e] = f2_mul(f2(-sn.x, -sn.y), w.r[e]);
                E[e] = f2_mul(cs.r[e], w.p[e]);
                F[e] = f2_mul(cs.p[e], w.r[e]);
            }
        }
        const int64_t o_step = hstep * a.o_h[s];
        __nv_bfloat16* z = a.out[s] + b * a.o_b[s] + t * a.o_n[s] + h_lo[s] * a.o_h[s] + at.d0;
        for (int k = 0; k < passes[s]; ++k) {
            issue();                                           // into the stage that the pass before has left
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            uint4 raw[2];
            raw[0] = *reinterpret_cast<const uint4*>(smem + rope_place_of(from, 2, 0));
            raw[1] = *reinterpret_cast<const uint4*>(smem + rope_place_of(from, 2, 1));
            RopeUnit x = rope_unpack<INTER>(raw);
            const float r = norm ? rsqrtf(rope_row_sum<C::LPR>(rope_dot(x, x)) * (1.f / D) + a.eps) : 1.f;
            const F2 r2 = f2(r, r);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const F2 p = x.p[e], q = x.r[e];
                x.p[e] = f2_mul(f2_fma(q, B[e], f2_mul(p, A[e])), r2);
                x.r[e] = f2_mul(f2_fma(q, F[e], f2_mul(p, E[e])), r2);
            }
            if (live && h_lo[s] + k * hstep < h_hi[s]) rope_store<INTER>(z, apart, x);
            z += o_step;
            from = (from + 1) % STAGES;
        }
    }
}

// Backward: the CTAs of a side walk its tiles of tokens, all heads of a tile, side by side; the tiles behind
// the last round, too few for all CTAs, are dealt out pass by pass (12 heads of 64, 3 sequences of 1021 tokens: 14.3 -> 12.1 us, when interleaved rows cost 2.4 more).  Behind four
// rounds and more it is a tile per CTA, as the memory is busy without the others (32 + 8 heads of 128, 8192 tokens: 47.5 us, and 48.6 pass by
// pass; dealt out in one piece per CTA 49.5).  The copies go two rows ahead.  The sums over rows of g xhat stay in registers to the end, then go to
// `partial`.
constexpr int ROPE_BWD_STAGES = 3;
template <int D>
struct RopeBwd {
    static constexpr size_t TABLES = sizeof(float) * 2 * ROPE_TOKENS * (D / 16) * ROPE_UROW, SUMS = sizeof(float) * RopeCfg<D>::RPP * (D + 4);
    static constexpr size_t COPIES = (size_t)ROPE_BWD_STAGES * 4 * ROPE_THREADS * 16;
    static constexpr size_t SMEM = COPIES + (TABLES > SUMS ? TABLES : SUMS);
};
template <int D, bool INTER>
__global__ void __launch_bounds__(ROPE_THREADS, 2)
qk_norm_rope_bwd_kernel(const RopeArgs a) {
    using C = RopeCfg<D>;
    constexpr int STAGES = ROPE_BWD_STAGES;
    extern __shared__ __align__(16) unsigned char smem[];
    auto cs_s = reinterpret_cast<float(*)[ROPE_TOKENS][D / 16][ROPE_UROW]>(smem + RopeBwd<D>::COPIES);     // two tables in turn
    auto red_s = reinterpret_cast<float(*)[D + 4]>(smem + RopeBwd<D>::COPIES);             // when the tables are through
    __shared__ __align__(16) float w_s[D / 16][ROPE_UROW];
    const int unit = threadIdx.x % C::LPR, rs = threadIdx.x / C::LPR;
    const int side = (int)blockIdx.x >= a.ctas[0];
    const int id = blockIdx.x - (side ? a.ctas[0] : 0);
    const int lgT = a.lgT[side], T = 1 << lgT;
    const int tok = rs & (T - 1), hofs = rs >> lgT, hstep = C::RPP >> lgT, H = a.heads[side];
    const RopePlace at = rope_place<D, INTER>(a, unit);
    const int apart = at.d1 - at.d0;
    const bool norm = a.w[side] != nullptr;
    const int64_t o_step = hstep * a.o_h[side];
    dep_wait();
    dep_trigger();
    rope_put_weights<D, INTER>(w_s, a, side);
    RopeUnit dw;
#pragma unroll
    for (int e = 0; e < 4; ++e) dw.p[e] = dw.r[e] = f2(0.f, 0.f);
    const int passes = a.passes[side];
    const int whole = a.whole[side], over = a.over[side], rest_lo = (int)((long long)a.rest[side] * min(id, over) / over);
    int left = whole * passes + (int)((long long)a.rest[side] * min(id + 1, over) / over) - rest_lo;
    // the CTA's i-th tile, after `tile`, and its first pass there
    auto enter = [&](int i, int& tile, int& k) {
        tile = i < whole ? id + i * a.ctas[side] : i > whole ? tile + 1 : whole * a.ctas[side] + (int)a.by_passes[side](rest_lo);
        k = i == whole ? rest_lo - (tile - whole * a.ctas[side]) * passes : 0;
    };
    // the copies' own walk over the rows, ahead of the work's
    const uint32_t stages = (uint32_t)__cvta_generic_to_shared(smem);
    int c_left = left, c_i = 0, c_tile = 0, c_k = 0, c_h = 0, into = 0;
    const __nv_bfloat16 *xp = nullptr, *gp = nullptr;
    bool c_live = false;
    auto aim = [&] {                                           // at the rows of the next tile
        enter(c_i++, c_tile, c_k);
        const int b = a.by_seq[side](c_tile), t0 = (int)(c_tile - b * a.per_seq[side]) << lgT, t = min(t0 + tok, a.n - 1);
        c_live = t0 + tok < a.n;
        xp = a.x[side] + b * a.x_b[side] + t * a.x_n[side] + at.d0;
        gp = a.g[side] + b * a.g_b[side] + t * a.g_n[side] + at.d0;
        c_h = c_k * hstep + hofs;
    };
    auto issue = [&] {
        if (c_left > 0) {
            const bool on = c_live && c_h < H;
            const __nv_bfloat16* p = gp + (on ? c_h : 0) * a.g_h[side];
            rope_copy(stages + rope_place_of(into, 4, 0), p, on);
            rope_copy(stages + rope_place_of(into, 4, 1), p + apart, on);
            if (norm) {
                p = xp + (on ? c_h : 0) * a.x_h[side];
                rope_copy(stages + rope_place_of(into, 4, 2), p, on);
                rope_copy(stages + rope_place_of(into, 4, 3), p + apart, on);
            }
            c_h += hstep;
            --c_left;
            if (++c_k == passes && c_left > 0) aim();
        }
        into = into == STAGES - 1 ? 0 : into + 1;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (c_left > 0) aim();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue();
    int buf = 0, from = 0;
    for (int i = 0, tile = 0, k0; left > 0; ++i, buf ^= 1) {
        enter(i, tile, k0);
        const int b = a.by_seq[side](tile), t0 = (int)(tile - b * a.per_seq[side]) << lgT, t = min(t0 + tok, a.n - 1);
        const bool live = t0 + tok < a.n;
        const int count = min(passes - k0, left);
        left -= count;
        int h = k0 * hstep + hofs;
        __nv_bfloat16* z = a.out[side] + b * a.o_b[side] + t * a.o_n[side] + h * a.o_h[side] + at.d0;
        rope_put_angles<D, INTER>(cs_s[buf], a, b, t0, T, -1.f);      // (worked out a tile ahead instead: 47.6 -> 49.0 us)
        __syncthreads();                                       // (the other table is free: its readers have passed this barrier)
        const RopeAngles ang = rope_get_angles(cs_s[buf][tok][unit]);
        for (int k = 0; k < count; ++k, h += hstep) {
            const bool on = live && h < H;
            issue();                                           // into the stage that the row before has left
            asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
            uint4 raw[2];
            raw[0] = *reinterpret_cast<const uint4*>(smem + rope_place_of(from, 4, 0));
            raw[1] = *reinterpret_cast<const uint4*>(smem + rope_place_of(from, 4, 1));
            RopeUnit g = rope_unpack<INTER>(raw);
            rope_turn(g, ang);
            if (norm) {
                raw[0] = *reinterpret_cast<const uint4*>(smem + rope_place_of(from, 4, 2));
                raw[1] = *reinterpret_cast<const uint4*>(smem + rope_place_of(from, 4, 3));
                const RopeUnit x = rope_unpack<INTER>(raw);
                RopeUnit u;
                {
                    const RopeUnit w = rope_get(w_s[unit]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) { u.p[e] = f2_mul(g.p[e], w.p[e]); u.r[e] = f2_mul(g.r[e], w.r[e]); }
                }
                float ss = rope_dot(x, x), dot = rope_dot(x, u);
#pragma unroll
                for (int off = C::LPR / 2; off >= 1; off >>= 1) {
                    ss += __shfl_xor_sync(0xffffffffu, ss, off);
                    dot += __shfl_xor_sync(0xffffffffu, dot, off);
                }
                // (a row that is not there has x = 0 and g = 0, and without eps an infinite r)
                const float r = on ? rsqrtf(ss * (1.f / D) + a.eps) : 0.f, m = dot * r * (1.f / D);        // m = mean(u xhat)
                const F2 r2 = f2(r, r), mr2 = f2(-m * r, -m * r);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const F2 xp2 = f2_mul(x.p[e], r2), xq2 = f2_mul(x.r[e], r2);
                    dw.p[e] = f2_fma(g.p[e], xp2, dw.p[e]);
                    dw.r[e] = f2_fma(g.r[e], xq2, dw.r[e]);
                    g.p[e] = f2_fma(xp2, mr2, f2_mul(u.p[e], r2));
                    g.r[e] = f2_fma(xq2, mr2, f2_mul(u.r[e], r2));
                }
            }
            if (on) rope_store<INTER>(z, apart, g);
            z += o_step;
            from = from == STAGES - 1 ? 0 : from + 1;
        }
    }
    if (!a.partial) return;
    // the CTA's sums: rows of threads in a fixed order
    __syncthreads();
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float2 p = f2_get(dw.p[e]), r = f2_get(dw.r[e]);
        float* row = red_s[rs];
        if constexpr (INTER) {
            float* z = row + (e < 2 ? at.d0 : at.d1) + 4 * (e % 2);
            z[0] = p.x; z[1] = r.x; z[2] = p.y; z[3] = r.y;
        } else {
            row[at.d0 + 2 * e] = p.x; row[at.d0 + 2 * e + 1] = p.y; row[at.d1 + 2 * e] = r.x; row[at.d1 + 2 * e + 1] = r.y;
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < D; d += ROPE_THREADS) {
        float t = 0.f;
#pragma unroll 8
        for (int r = 0; r < C::RPP; ++r) t += red_s[r][d];
        a.partial[(size_t)blockIdx.x * D + d] = t;
    }
}

// Rotating halves that are not whole 16-byte pieces (rot % 16 != 0): a warp per row, lane l has the pairs l, l + 32, ... of it, number by
// number.  Rows of a side over the warps of its CTAs, which in the backward pass sum their g xhat as above.
template <int D, bool BWD>
__global__ void __launch_bounds__(ROPE_THREADS)
qk_norm_rope_odd_kernel(const RopeArgs a) {
    constexpr int UPL = D / 64, WARPS = ROPE_THREADS / 32;     // pairs per lane
    __shared__ float red_s[BWD ? WARPS : 1][BWD ? D : 1];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int side = (int)blockIdx.x >= a.ctas[0];
    const int id = blockIdx.x - (side ? a.ctas[0] : 0);
    const int half = a.rot >> 1, H = a.heads[side];
    const bool norm = a.w[side] != nullptr;
    dep_wait();
    dep_trigger();
    int d0[UPL], d1[UPL];
    float w0[UPL], w1[UPL], dw0[UPL], dw1[UPL];
#pragma unroll
    for (int i = 0; i < UPL; ++i) {
        const int u = lane + 32 * i;
        d0[i] = u < half ? u : 2 * u;
        d1[i] = u < half ? half + u : 2 * u + 1;
        w0[i] = norm ? dep_load(a.w[side] + d0[i]) : 1.f;
        w1[i] = norm ? dep_load(a.w[side] + d1[i]) : 1.f;
        dw0[i] = dw1[i] = 0.f;
    }
    const int tokens = a.batch * a.n;
    for (int t = id * WARPS + warp; t < tokens; t += a.ctas[side] * WARPS) {
        const int b = t / a.n, i0 = t - b * a.n;
        const int pos = a.positions ? dep_load(a.positions + t) : i0;
        float cn[UPL], sn[UPL];
#pragma unroll
        for (int i = 0; i < UPL; ++i) {
            const float2 x = lane + 32 * i < half ? rope_cos_sin(a, pos, lane + 32 * i) : make_float2(1.f, 0.f);
            cn[i] = x.x;
            sn[i] = BWD ? -x.y : x.y;
        }
        for (int h = 0; h < H; ++h) {
            const __nv_bfloat16* xp = a.x[side] + (size_t)b * a.x_b[side] + (size_t)h * a.x_h[side] + (size_t)i0 * a.x_n[side];
            const __nv_bfloat16* gp = a.g[side] + (BWD ? (size_t)b * a.g_b[side] + (size_t)h * a.g_h[side] + (size_t)i0 * a.g_n[side] : 0);
            __nv_bfloat16* op = a.out[side] + (size_t)b * a.o_b[side] + (size_t)h * a.o_h[side] + (size_t)i0 * a.o_n[side];
            float x0[UPL], x1[UPL], g0[UPL], g1[UPL];
            float ss = 0.f, dot = 0.f;
#pragma unroll
            for (int i = 0; i < UPL; ++i) {
                x0[i] = x1[i] = g0[i] = g1[i] = 0.f;
                if (!BWD || norm) { x0[i] = __bfloat162float(xp[d0[i]]); x1[i] = __bfloat162float(xp[d1[i]]); }
                if (BWD) {
                    const float p = __bfloat162float(gp[d0[i]]), r = __bfloat162float(gp[d1[i]]);
                    g0[i] = p * cn[i] - r * sn[i];
                    g1[i] = p * sn[i] + r * cn[i];
                }
                ss = fmaf(x0[i], x0[i], fmaf(x1[i], x1[i], ss));
                dot = fmaf(x0[i], g0[i] * w0[i], fmaf(x1[i], g1[i] * w1[i], dot));
            }
            if (norm) {
                ss = rope_row_sum<32>(ss);
                if (BWD) dot = rope_row_sum<32>(dot);
                const float r = rsqrtf(ss * (1.f / D) + a.eps), m = dot * r * (1.f / D);
#pragma unroll
                for (int i = 0; i < UPL; ++i) {
                    x0[i] *= r;
                    x1[i] *= r;
                    if (BWD) {
                        dw0[i] = fmaf(g0[i], x0[i], dw0[i]);
                        dw1[i] = fmaf(g1[i], x1[i], dw1[i]);
                        g0[i] = r * (g0[i] * w0[i] - x0[i] * m);
                        g1[i] = r * (g1[i] * w1[i] - x1[i] * m);
                    } else {
                        x0[i] *= w0[i];
                        x1[i] *= w1[i];
                    }
                }
            }
            __syncwarp();                                      // (the result may lie over the input: all of the row has been read)
#pragma unroll
            for (int i = 0; i < UPL; ++i) {
                op[d0[i]] = __float2bfloat16(BWD ? g0[i] : x0[i] * cn[i] - x1[i] * sn[i]);
                op[d1[i]] = __float2bfloat16(BWD ? g1[i] : x0[i] * sn[i] + x1[i] * cn[i]);
            }
        }
    }
    if constexpr (BWD) {
        if (!a.partial) return;
#pragma unroll
        for (int i = 0; i < UPL; ++i) { red_s[warp][d0[i]] = dw0[i]; red_s[warp][d1[i]] = dw1[i]; }
        __syncthreads();
        for (int d = threadIdx.x; d < D; d += ROPE_THREADS) {
            float t = 0.f;
#pragma unroll
            for (int r = 0; r < WARPS; ++r) t += red_s[r][d];
            a.partial[(size_t)blockIdx.x * D + d] = t;
        }
    }
}

// dw[d] of a side = sum over its CTAs of partial[cta][d]; a block per 32 dimensions, 32 rows of threads, eight loads of each under way, all sums in
// a fixed order
__global__ void __launch_bounds__(1024)
norm_weight_grad_kernel(const float* partial, int ctas_q, int ctas_k, int D, float* dwq, float* dwk) {
    __shared__ float red[32][33];
    const int side = blockIdx.x * 32 >= D, col0 = blockIdx.x * 32 - (side ? D : 0), col = col0 + threadIdx.x;
    const int first = side ? ctas_q : 0, last = first + (side ? ctas_k : ctas_q);
    dep_wait();
    dep_trigger();
    float t = 0.f;
    for (int r = first + threadIdx.y; r < last; r += 32 * 8) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = r + 32 * i < last ? dep_load(partial + (size_t)(r + 32 * i) * D + col) : 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) t += x[i];
    }
    red[threadIdx.y][threadIdx.x] = t;
    __syncthreads();
    // a warp per column
    t = red[threadIdx.x][threadIdx.y];
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) t += __shfl_xor_sync(0xffffffffu, t, off);
    float* dst = side ? dwk : dwq;
    if (threadIdx.x == 0 && dst) dst[col0 + threadIdx.y] = t;
}

size_t qk_norm_rope_bwd_workspace_bytes(const focus_shape* s) { return (size_t)ROPE_GRID * s->D * sizeof(float); }

// Tokens per tile of the forward pass: as many as `rows` rows of a CTA have room for all their heads (16 rows of a token block are 4 KB in one piece
// when the layout is head by head), fewer where that leaves more than half of the multiprocessors without a tile; where it leaves some, the
// heads are cut too (1024 tokens of 12 + 12 heads of 64: 3.7 us; fewer tokens from two tiles per multiprocessor on 5.6, from a quarter on 3.8).
static int rope_tile(int rows, int heads, int batch, int n) {
    int lg = 0;
    while ((2 << lg) <= ROPE_TOKENS && (long long)(2 << lg) * heads <= rows && (long long)batch * cdiv(n, 2 << lg) >= ROPE_SMS / 2) ++lg;
    return lg;
}

constexpr int ROPE_PASSES = 8;                    // of a CTA over a tile's heads
constexpr int ROPE_EVEN = 4;                      // rounds of whole tiles up to which the tiles behind them are dealt out pass by pass, see above

template <int D, bool INTER>
static int launch_rope_d(const focus_shape* s, RopeArgs& a, bool bwd, float* dwq, float* dwk, cudaStream_t st) {
    using C = RopeCfg<D>;
    const bool odd = !INTER && a.rot % 16 != 0;
    const long long tokens = (long long)s->batch * s->n;
    if (tokens >= (1ll << 30)) return fail(FOCUS_ERR_UNSUPPORTED, "norm and rotation: batch * n (%lld) is too large for one call", tokens);
    if (!bwd && !odd) {
        int rc = require_sm100();                              // (when the sizes have been looked at: they are refused without a device too)
        if (rc) return rc;
        const int all = s->Hq + s->Hkv;
        a.lgT[0] = rope_tile(ROPE_PASSES * C::RPP, all, s->batch, s->n);
        a.per_seq[0] = cdiv(s->n, 1 << a.lgT[0]);
        a.by_seq[0] = fixed_div(a.per_seq[0]);
        const long long tiles = (long long)s->batch * a.per_seq[0];
        const int passes = cdiv(s->Hq, C::RPP >> a.lgT[0]) + cdiv(s->Hkv, C::RPP >> a.lgT[0]);
        // few tiles: a tile's passes over several CTAs
        long long parts = tiles >= ROPE_SMS ? 1 : ROPE_SMS / tiles;
        if (parts > passes) parts = passes;
        a.parts = (uint32_t)parts;
        a.by_parts = fixed_div(a.parts);
        constexpr size_t smem = (size_t)ROPE_FWD_STAGES * 2 * ROPE_THREADS * 16;
        rc = check_cuda(allow_smem<qk_norm_rope_kernel<D, INTER>>(smem), "cudaFuncSetAttribute(norm and rotation)");
        if (rc) return rc;
        return check_cuda(launch_dependent(qk_norm_rope_kernel<D, INTER>, dim3((unsigned)(tiles * parts)), dim3(ROPE_THREADS), smem, st, a),
                          "norm and rotation kernel launch");
    }
    // CTAs of the two sides: in proportion to their heads, no more than they have work
    const int places = bwd && !odd ? 2 * ROPE_SMS : ROPE_GRID;
    int share[2] = {0, (int)((long long)places * a.heads[1] / (a.heads[0] + a.heads[1]))};
    if (share[1] < 1) share[1] = 1;
    share[0] = places - share[1];
    for (int i = 0; i < 2; ++i) {
        // tokens per tile: those with the fewest passes and tiles (a tile's angles and barrier take about as long as a pass) one after another
        // (as many as leave every CTA a pass: 8 sequences of 68 tokens of 12 + 12 heads 9.6 us, not 5.6, 400 tokens of 32 + 8 heads 12.3, not 7.3)
        const int H = a.heads[i];
        long long best = 0, work = (tokens + 7) / 8;            // (of the kernel for odd halves: eight rows at a time)
        for (int lg = 0; !odd && (1 << lg) <= ROPE_TOKENS && (lg == 0 || (long long)(1 << lg) * H <= ROPE_PASSES * C::RPP); ++lg) {
            const int per_seq = cdiv(s->n, 1 << lg), passes = cdiv(H, C::RPP >> lg);
            const long long tiles = (long long)s->batch * per_seq, all = tiles * passes;
            const long long cost = (all + share[i] - 1) / share[i] + (tiles + share[i] - 1) / share[i];
            if (lg > 0 && cost >= best) continue;
            best = cost;
            work = all;
            a.lgT[i] = lg;
            a.per_seq[i] = per_seq;
            a.passes[i] = passes;
        }
        if (work >= (1ll << 31)) return fail(FOCUS_ERR_UNSUPPORTED, "norm and rotation: batch * n * heads (%lld rows) is too large for one call", tokens * H);
        a.ctas[i] = (int)(work < share[i] ? work : share[i]);
        if (odd) continue;
        a.by_seq[i] = fixed_div(a.per_seq[i]);
        a.by_passes[i] = fixed_div(a.passes[i]);
        a.whole[i] = s->batch * a.per_seq[i] / a.ctas[i];
        const int tiles = s->batch * a.per_seq[i] - a.whole[i] * a.ctas[i];
        a.rest[i] = tiles * a.passes[i];
        a.over[i] = a.whole[i] < ROPE_EVEN || tiles == 0 ? a.ctas[i] : tiles;
    }
    const dim3 g(a.ctas[0] + a.ctas[1]), t(ROPE_THREADS);
    int rc = require_sm100();
    if (rc) return rc;
    rc = odd ? FOCUS_OK : check_cuda(allow_smem<qk_norm_rope_bwd_kernel<D, INTER>>(RopeBwd<D>::SMEM), "cudaFuncSetAttribute(norm and rotation backward)");
    if (rc) return rc;
    rc = odd ? check_cuda(bwd ? launch_dependent(qk_norm_rope_odd_kernel<D, true>, g, t, 0, st, a) : launch_dependent(qk_norm_rope_odd_kernel<D, false>, g, t, 0, st, a),
                              "norm and rotation kernel launch")
                 : check_cuda(launch_dependent(qk_norm_rope_bwd_kernel<D, INTER>, g, t, RopeBwd<D>::SMEM, st, a), "norm and rotation backward kernel launch");
    if (rc || !bwd || !a.partial) return rc;
    return check_cuda(launch_dependent(norm_weight_grad_kernel, dim3(2 * D / 32), dim3(32, 32), 0, st, a.partial, a.ctas[0], a.ctas[1], D, dwq, dwk),
                      "norm weight gradient kernel launch");
}

static void put(RopeArgs& a, int s, const focus_tensor& x, const focus_tensor& out) {
    a.x[s] = reinterpret_cast<const __nv_bfloat16*>(x.ptr);
    a.x_b[s] = x.stride_b; a.x_h[s] = x.stride_h; a.x_n[s] = x.stride_n;
    a.out[s] = reinterpret_cast<__nv_bfloat16*>(out.ptr);
    a.o_b[s] = out.stride_b; a.o_h[s] = out.stride_h; a.o_n[s] = out.stride_n;
}

int launch_qk_norm_rope(const focus_shape* s, const focus_rope* rope, const focus_tensor (&x)[2], const float* const (&w)[2], const double* freq,
                        const int32_t* positions, const focus_tensor* grads, const focus_tensor (&out)[2], float* dwq, float* dwk, float* partial,
                        cudaStream_t st) {
    RopeArgs a = {};
    for (int i = 0; i < 2; ++i) {
        put(a, i, x[i], out[i]);
        a.w[i] = w[i];
        if (grads) {
            a.g[i] = reinterpret_cast<const __nv_bfloat16*>(grads[i].ptr);
            a.g_b[i] = grads[i].stride_b; a.g_h[i] = grads[i].stride_h; a.g_n[i] = grads[i].stride_n;
        }
    }
    a.heads[0] = s->Hq;
    a.heads[1] = s->Hkv;
    a.batch = s->batch;
    a.n = s->n;
    a.rot = rope->rotary;
    a.eps = rope->eps;
    a.amplitude = rope->amplitude == 0.f ? 1.f : rope->amplitude;
    a.freq = freq;
    a.positions = positions;
    a.partial = w[0] || w[1] ? partial : nullptr;
    const bool bwd = grads != nullptr;
    switch (s->D * 2 + (rope->interleaved ? 1 : 0)) {
        case 128: return launch_rope_d<64, false>(s, a, bwd, dwq, dwk, st);
        case 129: return launch_rope_d<64, true>(s, a, bwd, dwq, dwk, st);
        case 256: return launch_rope_d<128, false>(s, a, bwd, dwq, dwk, st);
        case 257: return launch_rope_d<128, true>(s, a, bwd, dwq, dwk, st);
        case 512: return launch_rope_d<256, false>(s, a, bwd, dwq, dwk, st);
        default: return launch_rope_d<256, true>(s, a, bwd, dwq, dwk, st);
    }
}

int rope_frequencies(int rotary, double base, int scaling, double factor, double low, double high, double trained, double* out, float* amplitude) {
    const double tau = 6.283185307179586476925;
    if (scaling == FOCUS_ROPE_BASE && rotary > 2) base *= pow(factor, (double)rotary / (rotary - 2));
    for (int i = 0; i < rotary / 2; ++i) {
        double f = pow(base, -2.0 * i / rotary);
        if (scaling == FOCUS_ROPE_LINEAR) f /= factor;
        if (scaling == FOCUS_ROPE_PARTS) {
            double keep = (trained * f / tau - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = keep * f + (1.0 - keep) * f / factor;
        }
        out[i] = f;
    }
    if (amplitude) *amplitude = scaling == FOCUS_ROPE_PARTS ? (float)(0.1 * log(factor) + 1.0) : 1.f;
    return FOCUS_OK;
}

}  // namespace focus
