// focus_attn_bwd / focus_gate_attn_bwd: the derivative of the attention forward pass.  With x = scale q.k (times the gate's factor f of a
// distant pair, or capped), over the attended pairs
//     p = exp(x - lse)     delta_i = do_i . o_i     ds = p (do.v - delta)   (times the cap's slope 1 - tanh^2)
//     dv_j = sum_i p do_i      dq_i = scale sum_j ds f k_j      dk_j = scale sum_i ds f q_i
//     distant pairs, gate: da = ds scale (q.k) lambda f (1 - f);   dg_i += da g_j,  dg_j += da g_i   (sigmoid' = f (1 - f))
// The probabilities are worked out again from lse; nothing of size n x n is kept.  A pass over key rows gives dk and dv, all query heads of
// a KV head in one block, one over query rows dq: seven products of tiles where five would do, but every sum has one owner and one order.
// Here: what comes before and after those passes.
#include "attn_bwd.cuh"

namespace focus {

// delta and lse log2(e), 128 of each per tile: rows past the end, and rows without any pair (lse = -inf), get lse = +inf, so that every
// probability is 0.  With masks, which queries of the tile are members of each group.  A block per (head, tile), a warp per row.
__global__ void __launch_bounds__(256)
bwd_rows_kernel(const __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, int64_t o_sn, const __nv_bfloat16* dO, int64_t d_sb, int64_t d_sh, int64_t d_sn,
                const float* lse, int Hq, int n, int nt, int D, const uint32_t* mq, int K, float* stat, uint32_t* qbits) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int hq = blockIdx.x / nt, tile = blockIdx.x % nt, b = hq / Hq, h = hq % Hq;
    dep_wait();
    dep_trigger();
    float* const t = stat + (size_t)blockIdx.x * 256;
    for (int r = warp; r < 128; r += 8) {
        const int i = tile * 128 + r;
        float s = 0.f, l = INFINITY;
        if (i < n) {
            const __nv_bfloat162* orow = reinterpret_cast<const __nv_bfloat162*>(o + b * o_sb + h * o_sh + (int64_t)i * o_sn);
            const __nv_bfloat162* drow = reinterpret_cast<const __nv_bfloat162*>(dO + b * d_sb + h * d_sh + (int64_t)i * d_sn);
            for (int d = lane; d < D / 2; d += 32) {
                const float2 x = __bfloat1622float2(orow[d]), y = __bfloat1622float2(drow[d]);
                s = fmaf(x.x, y.x, fmaf(x.y, y.y, s));
            }
            for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            l = lse[(size_t)hq * n + i];
            l = l == -INFINITY ? INFINITY : l * LOG2E;
        }
        if (lane == 0) {
            t[r] = l;
            t[128 + r] = s;
        }
    }
    if (mq && warp < 4) {
        const int i = tile * 128 + warp * 32 + lane;
        const uint32_t m = i < n ? mq[(size_t)hq * n + i] : 0u;
        for (int g = 0; g < K; ++g) {
            const uint32_t w = __ballot_sync(0xffffffffu, (m >> g) & 1u);
            if (lane == 0) qbits[((size_t)blockIdx.x * K + g) * 4 + warp] = w;
        }
    }
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
    for (int h = 0; h < Hq; ++h) s += gq[(b * Hq + h) * row + at];
    for (int h = 0; h < Hkv; ++h) s += gk[(b * Hkv + h) * row + at];
    dg[e] = (int)(at % ld) < K ? s : 0.f;
}

struct BwdWorkspace {
    size_t stat, qbits, gq, gk, bytes;
};
static BwdWorkspace bwd_workspace(const focus_shape* s, bool gate) {
    const size_t HQ = (size_t)s->batch * s->Hq, HK = (size_t)s->batch * s->Hkv, nt = cdiv(s->n, 128), row = (size_t)s->n * focus_soft_ld(s->K) * 4;
    BwdWorkspace w;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    w.stat = take(HQ * nt * 256 * 4);
    w.qbits = gate ? 0 : take(HQ * nt * s->K * 16);
    w.gq = gate ? take(HQ * row) : 0;
    w.gk = gate ? take(HK * row) : 0;
    w.bytes = off;
    return w;
}

size_t attn_bwd_workspace_bytes(const focus_shape* s, bool gate) { return bwd_workspace(s, gate).bytes; }

int launch_attn_bwd(const AttnBwdArgs& a, cudaStream_t st) {
    const focus_shape& s = a.s;
    const BwdWorkspace w = bwd_workspace(&s, a.g != nullptr);
    const int nt = cdiv(s.n, 128), HQ = s.batch * s.Hq, HK = s.batch * s.Hkv;
    if ((long long)HQ * nt > 0x7fffffffll) return fail(FOCUS_ERR_UNSUPPORTED, "attention backward: %lld tiles exceed 2^31 - 1", (long long)HQ * nt);
    float* const stat = reinterpret_cast<float*>(a.ws + w.stat);
    uint32_t* const qbits = reinterpret_cast<uint32_t*>(a.ws + w.qbits);
    int rc = check_cuda(launch_dependent(bwd_rows_kernel, dim3((unsigned)(HQ * nt)), dim3(256), 0, st, (const __nv_bfloat16*)a.o.ptr, a.o.stride_b, a.o.stride_h,
                                         a.o.stride_n, (const __nv_bfloat16*)a.dO.ptr, a.dO.stride_b, a.dO.stride_h, a.dO.stride_n, a.lse, s.Hq, s.n, nt, s.D,
                                         a.tiles ? a.mq : nullptr, s.K, stat, qbits), "attention backward rows launch");
    if (rc) return rc;
    BwdParams p = {};
    p.Hq = s.Hq; p.Hkv = s.Hkv; p.G = s.Hq / s.Hkv; p.n = s.n; p.nt = nt; p.K = s.K; p.w = s.window < s.n ? s.window : s.n;
    p.scale = a.scale; p.softcap = s.softcap; p.lambda = a.lambda;
    p.stat = stat;
    p.g = a.g;
    p.nkw = cdiv(nt, 32);
    p.live = a.tiles ? reinterpret_cast<const uint32_t*>(a.tiles + a.L.live) : nullptr;
    p.status = a.dev_status;
    auto wide = [](const focus_tensor& t) { return (uintptr_t)t.ptr % 32 == 0 && (t.stride_b | t.stride_h | t.stride_n) % 16 == 0; };
    BwdParams kv = p, q = p;
    kv.heads = HK; kv.by_heads = Divisor(HK); kv.by_rows_H = Divisor(s.Hkv);
    kv.row_mask = a.mk; kv.bits = a.tiles ? qbits : nullptr;
    kv.dg_part = reinterpret_cast<float*>(a.ws + w.gk);
    kv.out1 = (__nv_bfloat16*)a.dv.ptr; kv.s1b = a.dv.stride_b; kv.s1h = a.dv.stride_h; kv.s1n = a.dv.stride_n; kv.wide1 = wide(a.dv);
    kv.out2 = (__nv_bfloat16*)a.dk.ptr; kv.s2b = a.dk.stride_b; kv.s2h = a.dk.stride_h; kv.s2n = a.dk.stride_n; kv.wide2 = wide(a.dk);
    q.heads = HQ; q.by_heads = Divisor(HQ); q.by_rows_H = Divisor(s.Hq);
    q.row_mask = a.mq; q.bits = a.tiles ? reinterpret_cast<const uint32_t*>(a.tiles + a.L.gbits) : nullptr;
    q.dg_part = reinterpret_cast<float*>(a.ws + w.gq);
    q.out2 = (__nv_bfloat16*)a.dq.ptr; q.s2b = a.dq.stride_b; q.s2h = a.dq.stride_h; q.s2n = a.dq.stride_n; q.wide2 = wide(a.dq);
    rc = s.D == 64 ? launch_bwd_d<64>(a, kv, q, st) : s.D == 128 ? launch_bwd_d<128>(a, kv, q, st) : launch_bwd_d<256>(a, kv, q, st);
    if (rc || !a.g) return rc;
    const int ld = focus_soft_ld(s.K);
    const long long row = (long long)s.n * ld, count = row * s.batch;
    if (count > 0x7fffffffll * 256) return fail(FOCUS_ERR_UNSUPPORTED, "attention backward: too many assignments");
    return check_cuda(launch_dependent(bwd_gate_sum_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, (const float*)q.dg_part, (const float*)kv.dg_part, s.Hq, s.Hkv,
                                       row, ld, s.K, count, a.dg), "attention backward sum launch");
}

}  // namespace focus
