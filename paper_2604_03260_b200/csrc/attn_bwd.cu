// focus_attn_bwd / focus_gate_attn_bwd: the derivative of the attention forward pass.  With x = scale q.k (times the gate's factor f of a
// distant pair, or capped), over the attended pairs
//     p = exp(x - lse)     delta_i = do_i . o_i     ds = p (do.v - delta)   (times the cap's slope 1 - tanh^2)
//     dv_j = sum_i p do_i      dq_i = scale sum_j ds f k_j      dk_j = scale sum_i ds f q_i
//     distant pairs, gate: da = ds scale (q.k) lambda f (1 - f);   dg_i += da g_j,  dg_j += da g_i   (sigmoid' = f (1 - f))
// The probabilities are worked out again from lse; nothing of size n x n is kept.  Two passes, one over key rows (dk, dv, all query heads of
// a KV head in one block, so that nothing is added up by atomics) and one over query rows (dq).
#include "attn_bwd.cuh"

namespace focus {

constexpr int BT = 32;          // rows and columns of a tile

// delta and lse log2(e), 128 of each per tile: rows past the end, and rows without any pair (lse = -inf), get lse = +inf, so that every
// probability is 0.  A warp per row.
__global__ void __launch_bounds__(256)
bwd_rows_kernel(const __nv_bfloat16* o, int64_t o_sb, int64_t o_sh, int64_t o_sn, const __nv_bfloat16* dO, int64_t d_sb, int64_t d_sh, int64_t d_sn,
                const float* lse, int Hq, int n, int nt, int D, float* stat) {
    const int lane = threadIdx.x & 31;
    const int i = blockIdx.x * 8 + (threadIdx.x >> 5), hq = blockIdx.y, b = hq / Hq, h = hq % Hq;
    dep_wait();
    dep_trigger();
    float s = 0.f, l = INFINITY;
    if (i < n) {
        const __nv_bfloat16* orow = o + b * o_sb + h * o_sh + (int64_t)i * o_sn;
        const __nv_bfloat16* drow = dO + b * d_sb + h * d_sh + (int64_t)i * d_sn;
        for (int d = lane; d < D; d += 32) s = fmaf(__bfloat162float(orow[d]), __bfloat162float(drow[d]), s);
        for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        l = lse[(size_t)hq * n + i];
        l = l == -INFINITY ? INFINITY : l * LOG2E;
    }
    if (lane == 0) {
        float* t = stat + ((size_t)hq * nt + (i >> 7)) * 256 + (i & 127);
        t[0] = l;
        t[128] = s;
    }
}

struct SimpleBwd {
    const __nv_bfloat16 *q, *k, *v, *dO;
    focus_tensor tq, tk, tv, td, tdq, tdk, tdv;
    const uint32_t *mq, *mk;
    const float* stat;
    const float* g;
    float *gq, *gk;          // partial gradients of the assignments, [B Hq][n][ld] and [B Hkv][n][ld]
    int B, Hq, Hkv, n, nt, w, ld;
    float scale, softcap, lambda;
};

// KEYS: rows are 32 keys, columns the queries of all heads; otherwise rows are 32 queries of one head
template <int D, bool KEYS, bool GATE>
__global__ void __launch_bounds__(256) bwd_simple_kernel(const SimpleBwd p) {
    extern __shared__ float4 sm4[];
    __nv_bfloat16* const r1 = reinterpret_cast<__nv_bfloat16*>(sm4);       // K / Q rows, then V / dO rows, then those of the columns
    __nv_bfloat16 *const r2 = r1 + BT * (D + 2), *const c1 = r2 + BT * (D + 2), *const c2 = c1 + BT * (D + 2);
    float* const P = reinterpret_cast<float*>(c2 + BT * (D + 2));
    float *const S = P + BT * (BT + 1), *const A = S + BT * (BT + 1);
    float *const gr = A + BT * (BT + 1), *const gc = gr + BT * 32;
    const int t = threadIdx.x, G = p.Hq / p.Hkv;
    const int row0 = blockIdx.x * BT, head = blockIdx.y;
    const int b = head / (KEYS ? p.Hkv : p.Hq), hr = head % (KEYS ? p.Hkv : p.Hq);
    dep_wait();
    dep_trigger();
    auto load = [&](__nv_bfloat16* dst, const focus_tensor& x, int h, int first) {
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(x.ptr) + b * x.stride_b + h * x.stride_h;
        for (int e = t; e < BT * D; e += 256) {
            const int r = e / D, d = e % D;
            dst[r * (D + 2) + d] = first + r < p.n ? src[(int64_t)(first + r) * x.stride_n + d] : __float2bfloat16(0.f);
        }
    };
    auto load_g = [&](float* dst, int first) {
        for (int e = t; e < BT * p.ld; e += 256) {
            const int r = e / p.ld;
            dst[r * 32 + e % p.ld] = first + r < p.n ? p.g[((size_t)b * p.n + first + r) * p.ld + e % p.ld] : 0.f;
        }
    };
    load(r1, KEYS ? p.tk : p.tq, hr, row0);
    load(r2, KEYS ? p.tv : p.td, hr, row0);
    if (GATE) load_g(gr, row0);
    float acc1[BT * D / 256], acc2[BT * D / 256], accg[4] = {0.f, 0.f, 0.f, 0.f};
    for (int e = 0; e < BT * D / 256; ++e) acc1[e] = acc2[e] = 0.f;
    const int heads = KEYS ? G : 1;
    for (int hh = 0; hh < heads; ++hh) {
        const int hq = KEYS ? hr * G + hh : hr, hk = KEYS ? hr : hr / G;
        const int first = KEYS ? row0 : 0, end = KEYS ? p.n : min(p.n, row0 + BT);
        for (int col0 = first; col0 < end; col0 += BT) {
            __syncthreads();
            load(c1, KEYS ? p.tq : p.tk, KEYS ? hq : hk, col0);
            load(c2, KEYS ? p.td : p.tv, KEYS ? hq : hk, col0);
            if (GATE) load_g(gc, col0);
            __syncthreads();
            for (int e = t; e < BT * BT; e += 256) {
                const int r = e / BT, c = e % BT;
                const int i = KEYS ? col0 + c : row0 + r, j = KEYS ? row0 + r : col0 + c;
                float x = 0.f, y = 0.f, aff = 0.f;
                for (int d = 0; d < D; ++d) {
                    x = fmaf(__bfloat162float(r1[r * (D + 2) + d]), __bfloat162float(c1[c * (D + 2) + d]), x);
                    y = fmaf(__bfloat162float(r2[r * (D + 2) + d]), __bfloat162float(c2[c * (D + 2) + d]), y);
                }
                const bool in = i < p.n && j <= i, near = i - j <= p.w;
                bool keep = in;
                if (!GATE && p.mq && in && !near)
                    keep = (p.mq[((size_t)b * p.Hq + hq) * p.n + i] & p.mk[((size_t)b * p.Hkv + hk) * p.n + j]) != 0;
                x *= p.scale;
                float logit = x, slope = 1.f, a = 0.f;
                if (GATE && !near) {
                    for (int q = 0; q < p.ld; ++q) aff = fmaf(gr[r * 32 + q], gc[c * 32 + q], aff);
                    slope = 1.f / (1.f + expf(-p.lambda * aff));
                    logit = x * slope;
                } else if (!GATE && p.softcap > 0.f) {
                    const float th = tanhf(x / p.softcap);
                    logit = p.softcap * th;
                    slope = 1.f - th * th;
                }
                float pr = 0.f, ds = 0.f;
                if (keep) {
                    const float* st = p.stat + (((size_t)b * p.Hq + hq) * p.nt + (i >> 7)) * 256 + (i & 127);
                    pr = exp2f(logit * LOG2E - st[0]);
                    ds = pr * (y - st[128]);
                    if (GATE && !near) a = ds * x * p.lambda * slope * (1.f - slope);
                    ds *= slope;
                }
                P[r * (BT + 1) + c] = pr;
                S[r * (BT + 1) + c] = ds;
                if (GATE) A[r * (BT + 1) + c] = a;
            }
            __syncthreads();
            for (int e = 0; e < BT * D / 256; ++e) {
                const int r = (e * 256 + t) / D, d = (e * 256 + t) % D;
                float u = acc1[e], v = acc2[e];
                for (int c = 0; c < BT; ++c) {
                    u = fmaf(S[r * (BT + 1) + c], __bfloat162float(c1[c * (D + 2) + d]), u);
                    if (KEYS) v = fmaf(P[r * (BT + 1) + c], __bfloat162float(c2[c * (D + 2) + d]), v);
                }
                acc1[e] = u;
                acc2[e] = v;
            }
            if (GATE) {
                for (int e = 0; e < 4; ++e) {
                    const int r = (e * 256 + t) / 32, q = (e * 256 + t) % 32;
                    if (q < p.ld)
                        for (int c = 0; c < BT; ++c) accg[e] = fmaf(A[r * (BT + 1) + c], gc[c * 32 + q], accg[e]);
                }
            }
        }
    }
    const focus_tensor& o1 = KEYS ? p.tdk : p.tdq;
    for (int e = 0; e < BT * D / 256; ++e) {
        const int r = (e * 256 + t) / D, d = (e * 256 + t) % D;
        if (row0 + r >= p.n) continue;
        reinterpret_cast<__nv_bfloat16*>(o1.ptr)[b * o1.stride_b + hr * o1.stride_h + (int64_t)(row0 + r) * o1.stride_n + d] = __float2bfloat16(acc1[e] * p.scale);
        if (KEYS) reinterpret_cast<__nv_bfloat16*>(p.tdv.ptr)[b * p.tdv.stride_b + hr * p.tdv.stride_h + (int64_t)(row0 + r) * p.tdv.stride_n + d] = __float2bfloat16(acc2[e]);
    }
    if (GATE) {
        for (int e = 0; e < 4; ++e) {
            const int r = (e * 256 + t) / 32, q = (e * 256 + t) % 32;
            if (q < p.ld && row0 + r < p.n) (KEYS ? p.gk : p.gq)[((size_t)head * p.n + row0 + r) * p.ld + q] = accg[e];
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

size_t attn_bwd_workspace_bytes(const focus_shape* s, bool gate) {
    const size_t HQ = (size_t)s->batch * s->Hq, HK = (size_t)s->batch * s->Hkv, nt = cdiv(s->n, 128);
    size_t bytes = align_up(HQ * nt * 256 * 4, 256);
    if (gate) bytes += align_up((HQ + HK) * (size_t)s->n * focus_soft_ld(s->K) * 4, 256);
    return bytes;
}

template <int D, bool GATE>
static int launch_simple(const AttnBwdArgs& a, const SimpleBwd& p, cudaStream_t st) {
    constexpr size_t smem = 4 * BT * (D + 2) * 2 + 3 * BT * (BT + 1) * 4 + 2 * BT * 32 * 4;
    int rc;
    if ((rc = check_cuda(allow_smem<bwd_simple_kernel<D, true, GATE>>(smem), "cudaFuncSetAttribute(attn_bwd)"))) return rc;
    if ((rc = check_cuda(allow_smem<bwd_simple_kernel<D, false, GATE>>(smem), "cudaFuncSetAttribute(attn_bwd)"))) return rc;
    const unsigned tiles = (unsigned)cdiv(p.n, BT);
    if ((rc = check_cuda(launch_dependent(bwd_simple_kernel<D, true, GATE>, dim3(tiles, p.B * p.Hkv), dim3(256), smem, st, p), "attention backward launch"))) return rc;
    return check_cuda(launch_dependent(bwd_simple_kernel<D, false, GATE>, dim3(tiles, p.B * p.Hq), dim3(256), smem, st, p), "attention backward launch");
}

int launch_attn_bwd(const AttnBwdArgs& a, cudaStream_t st) {
    const focus_shape& s = a.s;
    SimpleBwd p = {};
    p.tq = a.q; p.tk = a.k; p.tv = a.v; p.td = a.dO; p.tdq = a.dq; p.tdk = a.dk; p.tdv = a.dv;
    p.mq = a.tiles ? a.mq : nullptr; p.mk = a.mk;
    p.B = s.batch; p.Hq = s.Hq; p.Hkv = s.Hkv; p.n = s.n; p.nt = cdiv(s.n, 128); p.w = s.window;
    p.scale = a.scale; p.softcap = s.softcap;
    p.g = a.g; p.lambda = a.lambda; p.ld = a.g ? focus_soft_ld(s.K) : 0;
    float* stat = reinterpret_cast<float*>(a.ws);
    p.stat = stat;
    const size_t HQ = (size_t)s.batch * s.Hq;
    p.gq = reinterpret_cast<float*>(a.ws + align_up(HQ * p.nt * 256 * 4, 256));
    p.gk = p.gq + HQ * s.n * p.ld;
    int rc = check_cuda(launch_dependent(bwd_rows_kernel, dim3((unsigned)p.nt * 16, (unsigned)HQ), dim3(256), 0, st, (const __nv_bfloat16*)a.o.ptr, a.o.stride_b,
                                         a.o.stride_h, a.o.stride_n, (const __nv_bfloat16*)a.dO.ptr, a.dO.stride_b, a.dO.stride_h, a.dO.stride_n, a.lse, s.Hq, s.n,
                                         p.nt, s.D, stat), "attention backward rows launch");
    if (rc) return rc;
    switch (s.D) {
        case 64: rc = a.g ? launch_simple<64, true>(a, p, st) : launch_simple<64, false>(a, p, st); break;
        case 128: rc = a.g ? launch_simple<128, true>(a, p, st) : launch_simple<128, false>(a, p, st); break;
        default: rc = a.g ? launch_simple<256, true>(a, p, st) : launch_simple<256, false>(a, p, st);
    }
    if (rc || !a.g) return rc;
    const long long row = (long long)s.n * p.ld, count = row * s.batch;
    return check_cuda(launch_dependent(bwd_gate_sum_kernel, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, st, p.gq, p.gk, s.Hq, s.Hkv, row, p.ld, s.K, count, a.dg),
                      "attention backward sum launch");
}

}  // namespace focus
