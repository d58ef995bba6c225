// focus_attn_bwd / focus_gate_attn_bwd: the derivative of the attention forward pass.  With x = scale q.k (times the gate's factor f of a
// distant pair, or capped), over the attended pairs
//     p = exp(x - lse)     delta_i = do_i . o_i     ds = p (do.v - delta)   (times the cap's slope 1 - tanh^2)
//     dv_j = sum_i p do_i      dq_i = scale sum_j ds f k_j      dk_j = scale sum_i ds f q_i
//     distant pairs, gate: da = ds scale (q.k) lambda f (1 - f);   dg_i += da g_j,  dg_j += da g_i   (sigmoid' = f (1 - f))
// The probabilities are worked out again from lse; nothing of size n x n is kept.  A pass over key rows gives dk and dv, all query heads of
// a KV head in one block (or in a few, whose sums are joined), one over query rows dq: seven products of tiles where five would do, but every sum has one owner and one order.
// Here: what comes before and after those passes.
#include "attn_bwd.cuh"

namespace focus {

// -lse log2(e) and -delta, 128 of each per tile: rows past the end, and rows without any pair (lse = -inf), get -inf in the place of the
// first, so that every probability is 0.  The same as six bf16 numbers a row (the first divided by scale log2(e), in place of -inf a number
// beyond every score): what the passes over keys add to their products.  With masks, which queries of the tile are members of each group.
// A block per (head, tile):
// D / 8 threads a row, every 16-byte piece of the tile asked for at once.  Before those, with the gate, a block per tile of a sequence: terms of
// its assignments, of the rows times `by` and of the columns: in the order of the products lo hi, hi lo, mid mid, mid hi, hi mid,
// hi hi (the smallest first); and the columns' assignments as they are, in the order in which they are read.
template <int D>
__global__ void __launch_bounds__(256)
bwd_rows_kernel(const __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, int64_t o_sn, const __nv_bfloat16* dO, int64_t d_sb, int64_t d_sh, int64_t d_sn,
                const float* lse, int Hq, int n, int nt, const uint32_t* mq, int K, float sl2, float* stat, __nv_bfloat16* aug, uint32_t* qbits, int lead, const float* g, float by,
                int log_ld, int depth, __nv_bfloat16* g_rows, __nv_bfloat16* g_cols, float* g_flat) {
    __shared__ float sl[128], sd[128];
    constexpr int TPR = D / 8, RPP = 256 / TPR, U = D == 256 ? 8 : 128 / RPP;       // threads a row, rows a turn, turns at once
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int block = (int)blockIdx.x - lead, hq = block / nt, tile = block % nt, b = hq / Hq, h = hq % Hq, i0 = tile * 128;
    dep_wait();
    dep_trigger();
    if (block < 0) {
        const int bt = blockIdx.x, r = threadIdx.x & 127, i = bt % nt * 128 + r;
        const bool col = threadIdx.x >= 128;
        const int ld = 1 << log_ld;
        const float* const gp = g + ((size_t)(bt / nt) * n + i) * ld;
        for (int ch = 0; ch < depth / 8; ++ch) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int at = ch * 8 + e, product = at >> log_ld;
                float v = i < n && product < 6 ? gp[at & (ld - 1)] * (col ? 1.f : by) : 0.f;
                const int term = (col ? 0x010120 : 0x001102) >> (4 * product) & 3;
                __nv_bfloat16 y = __float2bfloat16_rn(v);
                for (int x = 0; x < term; ++x) {
                    v -= __bfloat162float(y);
                    y = __float2bfloat16_rn(v);
                }
                w[e / 2] = e & 1 ? w[e / 2] | (uint32_t)__bfloat16_as_ushort(y) << 16 : (uint32_t)__bfloat16_as_ushort(y);
            }
            uint4* const to = col ? reinterpret_cast<uint4*>(g_cols) + ((size_t)(2 * bt + (r >> 6)) * (depth / 8) + ch) * 64 + (r & 63)
                                  : reinterpret_cast<uint4*>(g_rows) + ((size_t)bt * (depth / 8) + ch) * 128 + r;
            *to = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (col)
            for (int e = 0; e < ld / 4; ++e)
                reinterpret_cast<float4*>(g_flat)[(((size_t)bt * 16 + r / 8) * 2 + r % 2) * ld + e * 4 + r % 8 / 2] =
                    i < n ? reinterpret_cast<const float4*>(gp)[e] : make_float4(0.f, 0.f, 0.f, 0.f);
        return;
    }
    float* const t = stat + (size_t)block * 256;
    const int r0 = threadIdx.x / TPR, c = threadIdx.x % TPR * 8;
    const __nv_bfloat16* const ob = o + b * o_sb + h * o_sh + (int64_t)i0 * o_sn + c;
    const __nv_bfloat16* const db = dO + b * d_sb + h * d_sh + (int64_t)i0 * d_sn + c;
    if (threadIdx.x < 128) {
        const int i = i0 + threadIdx.x;
        const float l = i < n ? lse[(size_t)hq * n + i] : -INFINITY;
        t[threadIdx.x] = sl[threadIdx.x] = l == -INFINITY ? -INFINITY : -l * LOG2E;
    }
#pragma unroll 1
    for (int v = 0; v < 128 / RPP; v += U) {
        uint4 x[U], y[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int r = r0 + (v + u) * RPP;
            x[u] = y[u] = make_uint4(0u, 0u, 0u, 0u);
            if (i0 + r < n) {
                x[u] = *reinterpret_cast<const uint4*>(ob + r * o_sn);
                y[u] = *reinterpret_cast<const uint4*>(db + r * d_sn);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t xs[4] = {x[u].x, x[u].y, x[u].z, x[u].w}, ys[4] = {y[u].x, y[u].y, y[u].z, y[u].w};
            float s = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                s = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(ys[e] << 16), s);
                s = fmaf(__uint_as_float(xs[e] & 0xffff0000u), __uint_as_float(ys[e] & 0xffff0000u), s);
            }
#pragma unroll
            for (int off = TPR / 2; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            if (threadIdx.x % TPR == 0) t[128 + r0 + (v + u) * RPP] = sd[r0 + (v + u) * RPP] = -s;
        }
    }
    __syncthreads();
    if (threadIdx.x < 128) {
        const float x = sl[threadIdx.x] / sl2;
        float v[2] = {isnan(x) ? x : fminf(fmaxf(x, -3e38f), 3e38f), sd[threadIdx.x]};
        uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 6; ++e) {
            const __nv_bfloat16 y = __float2bfloat16_rn(v[e / 3]);
            v[e / 3] -= __bfloat162float(y);
            w[e / 2] |= (uint32_t)__bfloat16_as_ushort(y) << (16 * (e & 1));
        }
        reinterpret_cast<uint4*>(aug)[(size_t)block * 128 + threadIdx.x] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    if (mq && warp < 4) {
        const int i = i0 + warp * 32 + lane;
        const uint32_t m = i < n ? mq[(size_t)hq * n + i] : 0u;
        for (int g = 0; g < K; ++g) {
            const uint32_t w = __ballot_sync(0xffffffffu, (m >> g) & 1u);
            if (lane == 0) qbits[((size_t)block * K + g) * 4 + warp] = w;
        }
    }
}

template <int D>
static int launch_bwd_rows(const AttnBwdArgs& a, int nt, float* stat, __nv_bfloat16* aug, uint32_t* qbits, __nv_bfloat16* g_rows, __nv_bfloat16* g_cols, float* g_flat,
                           cudaStream_t st) {
    auto kern = bwd_rows_kernel<D>;
    const int lead = g_rows ? a.s.batch * nt : 0, ld = focus_soft_ld(a.s.K);
    return check_cuda(launch_dependent(kern, dim3((unsigned)(lead + a.s.batch * a.s.Hq * nt)), dim3(256), 0, st, (const __nv_bfloat16*)a.o.ptr, a.o.stride_b, a.o.stride_h,
                                       a.o.stride_n, (const __nv_bfloat16*)a.dO.ptr, a.dO.stride_b, a.dO.stride_h, a.dO.stride_n, a.lse, a.s.Hq, a.s.n, nt,
                                       a.tiles ? a.mq : nullptr, a.s.K, a.scale * LOG2E, stat, aug, qbits, lead, a.g, -a.lambda * LOG2E, ld == 4 ? 2 : ld == 8 ? 3 : ld == 16 ? 4 : 5,
                      g_rows ? gate_depth(ld) : 0, g_rows, g_cols, g_flat),
                      "attention backward rows launch");
}

// dg[b][i][:] = sum over the heads of both sides' partial sums, in their order; columns from K on are written as 0
__global__ void __launch_bounds__(256)
bwd_gate_sum_kernel(const float* gq, const float* gk, int Hq, int Hkv, long long row, int ld, int K, long long count, float* dg) {
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    dep_wait();
    dep_trigger();
    if (e >= count) return;
    const long long b = e / row, at = e % row;
    float s = 0.f;
#pragma unroll 16
    for (int h = 0; h < Hq; ++h) s += gq[(b * Hq + h) * row + at];
#pragma unroll 16
    for (int h = 0; h < Hkv; ++h) s += gk[(b * Hkv + h) * row + at];
    dg[e] = (int)(at % ld) < K ? s : 0.f;
}

// dk, dv: the parts' sums of a row, in their order.  Eight columns a thread.
__global__ void __launch_bounds__(256)
bwd_join_kernel(const float* part1, const float* part2, int split, int Hkv, int n, int D, long long count, float scale, focus_tensor dv, focus_tensor dk) {
    const long long e = (long long)blockIdx.x * 256 + threadIdx.x;
    dep_wait();
    dep_trigger();
    if (e >= count) return;
    const int each = D / 8, c = (int)(e % each) * 8;
    const long long at = e / each, owner = at / n, row = at % n;
    const long long b = owner / Hkv, h = owner % Hkv;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const float* p = (x ? part2 : part1) + ((size_t)owner * split * n + row) * D + c;
        float s[8] = {};
#pragma unroll 4
        for (int i = 0; i < split; ++i, p += (size_t)n * D) {
            const float4 u = reinterpret_cast<const float4*>(p)[0], w = reinterpret_cast<const float4*>(p)[1];
            s[0] += u.x; s[1] += u.y; s[2] += u.z; s[3] += u.w; s[4] += w.x; s[5] += w.y; s[6] += w.z; s[7] += w.w;
        }
        const float by = x ? scale : 1.f;
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 y = __floats2bfloat162_rn(s[2 * i] * by, s[2 * i + 1] * by);
            w[i] = *reinterpret_cast<const uint32_t*>(&y);
        }
        const focus_tensor& t = x ? dk : dv;
        *reinterpret_cast<uint4*>((__nv_bfloat16*)t.ptr + b * t.stride_b + h * t.stride_h + row * t.stride_n + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// Parts into which a KV head's query heads are cut, so that the first key tile, which has every query tile of all G heads one after another, is not
// what the launch takes: 8/2 heads x 4000 tokens, D = 128, 258 us with one part and 136 with four, with the gate (K = 16, 4096) 634 and 347; 32/8 x 1024
// 74 and, with two, 58.  More
// items cost what is around an item's tiles, and a launch that joins the parts' sums (16/8 heads x 1000, D = 256: 60 with one, 81 with two).  So the
// longest item is weighed against an SM's share, in thousands of cycles: a tile of dK and dV 3 (D = 256: 4 and 3 in two items), of dQ 2 (4), with the gate
// 6 more, 12 (24) around an item, 6 (12) for the join.  (With every causal pair: what the masks leave out is not known here.)
static int bwd_split(const focus_shape* s, bool gate) {
    const double nt = cdiv(s->n, 128), tiles = nt * (nt + 1) / 2 * s->batch * s->Hq, more = gate ? 6 : 0;
    const bool two = s->D == 256;
    const double kv = (two ? 4 : 3) + more, q = (two ? 4 : 2) + more, second = two ? 3 + more : 0, around = two ? 24 : 12, join = two ? 12 : 6;
    const int G = s->Hq / s->Hkv;
    int best = 1;
    double least = 0;
    for (int S = 1; S <= G; ++S) {
        if (G % S) continue;
        const double items = nt * s->batch * ((double)s->Hkv * S * (two ? 2 : 1) + s->Hq), longest = G / S * nt * kv + around;
        const double share = (tiles * (kv + second + q) + items * around) / 148, t = (1.15 * longest > share ? 1.15 * longest : share) + (S > 1 ? join : 0);
        if (S == 1 || t < least) { best = S; least = t; }
    }
    return best;
}

struct BwdWorkspace {
    size_t part1, part2, part_q;
    size_t stat, aug, qbits, gq, gk, g_rows, g_cols, g_flat, bytes;
};
static BwdWorkspace bwd_workspace(const focus_shape* s, bool gate) {
    const size_t HQ = (size_t)s->batch * s->Hq, HK = (size_t)s->batch * s->Hkv, nt = cdiv(s->n, 128), row = (size_t)s->n * focus_soft_ld(s->K) * 4;
    BwdWorkspace w;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    w.stat = take(HQ * nt * 256 * 4);
    w.aug = take(HQ * nt * 128 * 16);
    w.qbits = gate ? 0 : take(HQ * nt * s->K * 16);
    w.gq = gate ? take(HQ * row) : 0;
    const size_t split = bwd_split(s, gate), each = s->Hq / s->Hkv / split;
    const bool parts = split > 1 || (int)nt > BWD_LAUNCH_TILES || bwd_heads_together((int)nt, (int)each) < (int)each;       // of a row's sums
    const size_t sums = parts ? HK * split * s->n * s->D * 4 : 0;
    w.gk = gate ? take(HK * split * row) : 0;
    w.part1 = take(sums);
    w.part2 = take(sums);
    w.part_q = take((int)nt > BWD_LAUNCH_TILES ? HQ * s->n * s->D * 4 : 0);
    const size_t terms = gate && s->D != 256 ? (size_t)s->batch * nt * 128 * gate_depth(focus_soft_ld(s->K)) * 2 : 0;
    w.g_rows = take(terms);
    w.g_cols = take(terms);
    w.g_flat = take(terms ? (size_t)s->batch * nt * 128 * focus_soft_ld(s->K) * 4 : 0);
    w.bytes = off;
    return w;
}

size_t attn_bwd_workspace_bytes(const focus_shape* s, bool gate) { return bwd_workspace(s, gate).bytes; }

int launch_attn_bwd(const AttnBwdArgs& a, cudaStream_t st) {
    const focus_shape& s = a.s;
    const BwdWorkspace w = bwd_workspace(&s, a.g != nullptr);
    const int nt = cdiv(s.n, 128), HQ = s.batch * s.Hq, HK = s.batch * s.Hkv;
    if ((long long)(HQ + s.batch) * nt > 0x7fffffffll) return fail(FOCUS_ERR_UNSUPPORTED, "attention backward: %lld tiles exceed 2^31 - 1", (long long)HQ * nt);
    float* const stat = reinterpret_cast<float*>(a.ws + w.stat);
    __nv_bfloat16* const aug = reinterpret_cast<__nv_bfloat16*>(a.ws + w.aug);
    uint32_t* const qbits = reinterpret_cast<uint32_t*>(a.ws + w.qbits);
    const bool terms = a.g && s.D != 256;
    __nv_bfloat16* const g_rows = terms ? reinterpret_cast<__nv_bfloat16*>(a.ws + w.g_rows) : nullptr;
    __nv_bfloat16* const g_cols = terms ? reinterpret_cast<__nv_bfloat16*>(a.ws + w.g_cols) : nullptr;
    float* const g_flat = reinterpret_cast<float*>(a.ws + w.g_flat);
    int rc = s.D == 64    ? launch_bwd_rows<64>(a, nt, stat, aug, qbits, g_rows, g_cols, g_flat, st)
             : s.D == 128 ? launch_bwd_rows<128>(a, nt, stat, aug, qbits, g_rows, g_cols, g_flat, st)
                          : launch_bwd_rows<256>(a, nt, stat, aug, qbits, g_rows, g_cols, g_flat, st);
    if (rc) return rc;
    BwdParams p = {};
    p.Hq = s.Hq; p.Hkv = s.Hkv; p.G = s.Hq / s.Hkv; p.n = s.n; p.nt = nt; p.K = s.K; p.w = s.window < s.n ? s.window : s.n;
    p.scale = a.scale; p.softcap = s.softcap; p.lambda = a.lambda;
    p.stat = stat;
    p.aug = aug;
    p.g = a.g;
    p.g_rows = g_rows;
    p.g_cols = g_cols;
    p.g_flat = g_flat;
    p.nkw = cdiv(nt, 32);
    p.live = a.tiles ? reinterpret_cast<const uint32_t*>(a.tiles + a.L.live) : nullptr;
    p.status = a.dev_status;
    auto wide = [](const focus_tensor& t) { return (uintptr_t)t.ptr % 32 == 0 && (t.stride_b | t.stride_h | t.stride_n) % 16 == 0; };
    BwdParams kv = p, q = p;
    kv.split = bwd_split(&s, a.g != nullptr); kv.heads_each = p.G / kv.split; kv.by_split = Divisor(kv.split);
    kv.heads = HK * kv.split; kv.by_heads = Divisor(kv.heads); kv.by_rows_H = Divisor(s.Hkv);
    kv.part1 = reinterpret_cast<float*>(a.ws + w.part1); kv.part2 = reinterpret_cast<float*>(a.ws + w.part2);
    kv.row_mask = a.mk; kv.bits = a.tiles ? qbits : nullptr;
    kv.dg_part = reinterpret_cast<float*>(a.ws + w.gk);
    kv.out1 = (__nv_bfloat16*)a.dv.ptr; kv.s1b = a.dv.stride_b; kv.s1h = a.dv.stride_h; kv.s1n = a.dv.stride_n; kv.wide1 = wide(a.dv);
    kv.out2 = (__nv_bfloat16*)a.dk.ptr; kv.s2b = a.dk.stride_b; kv.s2h = a.dk.stride_h; kv.s2n = a.dk.stride_n; kv.wide2 = wide(a.dk);
    q.heads = HQ; q.by_heads = Divisor(HQ); q.by_rows_H = Divisor(s.Hq);
    q.part2 = reinterpret_cast<float*>(a.ws + w.part_q);
    q.row_mask = a.mq; q.bits = a.tiles ? reinterpret_cast<const uint32_t*>(a.tiles + a.L.gbits) : nullptr;
    q.dg_part = reinterpret_cast<float*>(a.ws + w.gq);
    q.out2 = (__nv_bfloat16*)a.dq.ptr; q.s2b = a.dq.stride_b; q.s2h = a.dq.stride_h; q.s2n = a.dq.stride_n; q.wide2 = wide(a.dq);
    rc = s.D == 64 ? launch_bwd_d<64>(a, kv, q, st) : s.D == 128 ? launch_bwd_d<128>(a, kv, q, st) : launch_bwd_d<256>(a, kv, q, st);
    if (rc) return rc;
    if (kv.split > 1) {
        const long long count = (long long)HK * s.n * (s.D / 8);
        if (count > 0x7fffffffll * 256) return fail(FOCUS_ERR_UNSUPPORTED, "attention backward: too many keys");
        rc = check_cuda(launch_dependent(bwd_join_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, (const float*)kv.part1, (const float*)kv.part2, kv.split, s.Hkv, s.n,
                                         s.D, count, a.scale, a.dv, a.dk), "attention backward join launch");
    }
    if (rc || !a.g) return rc;
    const int ld = focus_soft_ld(s.K);
    const long long row = (long long)s.n * ld, count = row * s.batch;
    if (count > 0x7fffffffll * 256) return fail(FOCUS_ERR_UNSUPPORTED, "attention backward: too many assignments");
    return check_cuda(launch_dependent(bwd_gate_sum_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, (const float*)q.dg_part, (const float*)kv.dg_part, s.Hq, s.Hkv * kv.split,
                                       row, ld, s.K, count, a.dg), "attention backward sum launch");
}

}  // namespace focus
