// focus_router_scores_bwd: the derivative of S = (h W_g) C^T.  With T = dS^T h (K vectors of d, summed over all tokens)
//     dC = T W_g      dW_g = T^T C      dh = dS F,  F = C W_g^T
// so the hidden states are read once and their gradient written once, and everything else is of size K d: bound by the memory.
// A block has a strip of columns and a run of tokens and goes down its rows: a thread holds 4 columns (2 from K = 9 on) of F and of its part
// of T, both with K numbers a column, and a row costs it K/2 reads of the row's dS (pairs (w, w), one address a warp) and 4 K (2 K) packed
// multiply-adds.
#include "common.cuh"

namespace focus {

constexpr int RB_THREADS = 128;
constexpr int RB_ROWS = 32;                 // tokens whose dS is in shared memory at a time
constexpr int RB_TOTAL_COLS = 64;           // columns of a block that adds the parts up

// F[g][e] = sum_j W_g[e][j] C[g][j]
__global__ void __launch_bounds__(256) router_fold_kernel(const float* Wg, const float* C, int d, int dg, float* F) {
    const int e = blockIdx.x * 256 + threadIdx.x, g = blockIdx.y;
    dep_wait();
    dep_trigger();
    if (e >= d) return;
    float s = 0.f;
    for (int j = 0; j < dg; ++j) s = fmaf(Wg[(size_t)e * dg + j], C[(size_t)g * dg + j], s);
    F[(size_t)g * d + e] = s;
}

// Pairs of columns of a thread: two, or one where K is so large that F and T would not fit the registers
constexpr int rb_pairs(int LD) { return LD <= 8 ? 2 : 1; }

template <int LD>
__global__ void __launch_bounds__(RB_THREADS)
router_bwd_kernel(const __nv_bfloat16* h, int64_t h_sb, int64_t h_sn, const float* dS, const float* F, int n, int runs, int run, int d, int K, __nv_bfloat16* dh,
                  int64_t d_sb, int64_t d_sn, float* part, unsigned* done) {
    constexpr int P = rb_pairs(LD);
    __shared__ float2 s[RB_ROWS * LD];
    const int t = threadIdx.x, b = blockIdx.y / runs, tok0 = blockIdx.y % runs * run, e = (blockIdx.x * RB_THREADS + t) * 2 * P;
    const bool in = e < d;                                   // (d is a multiple of 8)
    dep_wait();
    dep_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && t == 0) *done = 0u;
    const int rows = min(run, n - tok0);
    float2 f[LD][P], acc[LD][P];
#pragma unroll
    for (int g = 0; g < LD; ++g) {
#pragma unroll
        for (int c = 0; c < P; ++c) {
            f[g][c] = in && dh && g < K ? *reinterpret_cast<const float2*>(F + (size_t)g * d + e + 2 * c) : make_float2(0.f, 0.f);
            acc[g][c] = make_float2(0.f, 0.f);
        }
    }
    const __nv_bfloat16* hp = h + b * h_sb + (int64_t)tok0 * h_sn + e;
    __nv_bfloat16* dp = dh ? dh + b * d_sb + (int64_t)tok0 * d_sn + e : nullptr;
    const float* sp = dS + ((size_t)b * n + tok0) * LD;
    struct __align__(4 * P) Words { uint32_t w[P]; };
    for (int r0 = 0; r0 < rows; r0 += RB_ROWS) {
        const int m = min(RB_ROWS, rows - r0);
        __syncthreads();
        for (int q = t; q < RB_ROWS * LD; q += RB_THREADS) {
            const float w = q < m * LD && q % LD < K ? sp[(size_t)r0 * LD + q] : 0.f;        // (columns from K on may hold anything)
            s[q] = make_float2(w, w);
        }
        __syncthreads();
        if (!in) continue;
        constexpr int AHEAD = 8;
        for (int r = 0; r < m; r += AHEAD) {
            Words x[AHEAD] = {};
#pragma unroll
            for (int u = 0; u < AHEAD; ++u)
                if (r + u < m) x[u] = *reinterpret_cast<const Words*>(hp + (int64_t)(r0 + r + u) * h_sn);
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) {
                float2 v[P], y[P];
#pragma unroll
                for (int c = 0; c < P; ++c) {
                    v[c] = make_float2(__uint_as_float(x[u].w[c] << 16), __uint_as_float(x[u].w[c] & 0xffff0000u));
                    y[c] = make_float2(0.f, 0.f);
                }
#pragma unroll
                for (int g = 0; g < LD; g += 2) {
                    const float4 w2 = *reinterpret_cast<const float4*>(&s[(r + u) * LD + g]);
                    const float2 w[2] = {make_float2(w2.x, w2.y), make_float2(w2.z, w2.w)};
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
#pragma unroll
                        for (int c = 0; c < P; ++c) {
                            acc[g + k][c] = __ffma2_rn(w[k], v[c], acc[g + k][c]);
                            y[c] = __ffma2_rn(w[k], f[g + k][c], y[c]);
                        }
                    }
                }
                if (dp && r + u < m) {
                    Words z;
#pragma unroll
                    for (int c = 0; c < P; ++c) {
                        const __nv_bfloat162 a = __float22bfloat162_rn(y[c]);
                        z.w[c] = *reinterpret_cast<const uint32_t*>(&a);
                    }
                    *reinterpret_cast<Words*>(dp + (int64_t)(r0 + r + u) * d_sn) = z;
                }
            }
        }
    }
    if (!in) return;
#pragma unroll
    for (int g = 0; g < LD; ++g) {
        if (g >= K) break;
#pragma unroll
        for (int c = 0; c < P; ++c) *reinterpret_cast<float2*>(part + ((size_t)blockIdx.y * K + g) * d + e + 2 * c) = acc[g][c];
    }
}

// T = sum of the parts, dW_g = T^T C and this block's part of dC = T W_g; the last block to be through adds those up, in their order.
__global__ void __launch_bounds__(256)
router_total_kernel(const float* part, const float* C, const float* Wg, int parts, int d, int dg, int K, float* dWg, float* dC_part, float* dC, unsigned* done) {
    __shared__ float T[32][RB_TOTAL_COLS];
    __shared__ float quarter[4][RB_TOTAL_COLS];
    __shared__ bool last;
    const int t = threadIdx.x, e0 = blockIdx.x * RB_TOTAL_COLS, c = t % RB_TOTAL_COLS, q = t / RB_TOTAL_COLS, cols = min(RB_TOTAL_COLS, d - e0);
    dep_wait();
    dep_trigger();
    for (int g = 0; g < K; ++g) {
        float x = 0.f;
        if (c < cols) {
#pragma unroll 4
            for (int r = q; r < parts; r += 4) x += part[((size_t)r * K + g) * d + e0 + c];
        }
        quarter[q][c] = x;
        __syncthreads();
        if (q == 0) T[g][c] = (quarter[0][c] + quarter[1][c]) + (quarter[2][c] + quarter[3][c]);
        __syncthreads();
    }
    for (int i = t; i < cols * dg; i += 256) {
        const int x = i / dg, j = i % dg;
        float y = 0.f;
        for (int g = 0; g < K; ++g) y = fmaf(T[g][x], C[(size_t)g * dg + j], y);
        dWg[(size_t)(e0 + x) * dg + j] = y;
    }
    for (int i = t; i < K * dg; i += 256) {
        const int g = i / dg, j = i % dg;
        float y = 0.f;
        for (int x = 0; x < cols; ++x) y = fmaf(T[g][x], Wg[(size_t)(e0 + x) * dg + j], y);
        dC_part[(size_t)blockIdx.x * K * dg + i] = y;
    }
    __threadfence();
    __syncthreads();
    if (t == 0) last = atomicAdd(done, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    for (int i = t; i < K * dg; i += 256) {
        float y = 0.f;
        for (int x = 0; x < (int)gridDim.x; ++x) y += __ldcg(dC_part + (size_t)x * K * dg + i);
        dC[i] = y;
    }
}

// How the tokens are cut: runs of `run` tokens of a sequence, `runs` a sequence.  Enough blocks for the SMs' places (four blocks each at
// K <= 8) and no run shorter than 16 tokens, whose part of T would cost more than its rows
struct RouterCut {
    int run, runs;
};
static int router_strips(const focus_shape* s, int d) { return cdiv(d, 2 * rb_pairs(focus_soft_ld(s->K)) * RB_THREADS); }
static RouterCut router_cut(const focus_shape* s, int d) {
    const int strips = router_strips(s, d), want = cdiv(592, strips * s->batch);
    RouterCut c;
    c.run = cdiv(s->n, want < 1 ? 1 : want);
    if (c.run < 16) c.run = 16;
    c.runs = cdiv(s->n, c.run);
    return c;
}

struct RouterWorkspace {
    size_t F, part, dC, done, bytes;
};
static RouterWorkspace router_workspace(const focus_shape* s, int d, int dg) {
    RouterWorkspace w;
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t o = off; off = align_up(off + bytes, 256); return o; };
    w.done = take(4);
    w.F = take((size_t)s->K * d * 4);
    w.part = take((size_t)s->batch * router_cut(s, d).runs * s->K * d * 4);
    w.dC = take((size_t)cdiv(d, RB_TOTAL_COLS) * s->K * dg * 4);
    w.bytes = off;
    return w;
}

size_t router_bwd_workspace_bytes(const focus_shape* s, int d, int dg) { return router_workspace(s, d, dg).bytes; }

template <int LD>
static int launch_tokens(const focus_shape* s, const RouterBwdArgs& a, const RouterCut& c, const float* F, float* part, unsigned* done, cudaStream_t st) {
    auto kern = router_bwd_kernel<LD>;
    return check_cuda(launch_dependent(kern, dim3((unsigned)router_strips(s, a.d_model), (unsigned)(s->batch * c.runs)), dim3(RB_THREADS), 0, st, a.h, a.h_sb, a.h_sn, a.ds, F,
                                       s->n, c.runs, c.run, a.d_model, s->K, a.dh, a.dh_sb, a.dh_sn, part, done), "router backward launch");
}

int launch_router_bwd(const focus_shape* s, const RouterBwdArgs& a, cudaStream_t st) {
    const int d = a.d_model, K = s->K;
    const RouterCut c = router_cut(s, d);
    const RouterWorkspace w = router_workspace(s, d, a.d_g);
    if ((long long)s->batch * c.runs > 65535) return fail(FOCUS_ERR_UNSUPPORTED, "router backward: %lld runs of tokens exceed 65535", (long long)s->batch * c.runs);
    float *F = reinterpret_cast<float*>(a.ws + w.F), *part = reinterpret_cast<float*>(a.ws + w.part), *dC_part = reinterpret_cast<float*>(a.ws + w.dC);
    unsigned* done = reinterpret_cast<unsigned*>(a.ws + w.done);
    int rc = FOCUS_OK;
    if (a.dh) rc = check_cuda(launch_dependent(router_fold_kernel, dim3((unsigned)cdiv(d, 256), (unsigned)K), dim3(256), 0, st, a.Wg, a.C, d, a.d_g, F), "router fold launch");
    if (rc) return rc;
    switch (focus_soft_ld(K)) {
        case 4: rc = launch_tokens<4>(s, a, c, F, part, done, st); break;
        case 8: rc = launch_tokens<8>(s, a, c, F, part, done, st); break;
        case 16: rc = launch_tokens<16>(s, a, c, F, part, done, st); break;
        default: rc = launch_tokens<32>(s, a, c, F, part, done, st);
    }
    if (rc) return rc;
    return check_cuda(launch_dependent(router_total_kernel, dim3((unsigned)cdiv(d, RB_TOTAL_COLS)), dim3(256), 0, st, (const float*)part, a.C, a.Wg, s->batch * c.runs, d, a.d_g,
                                       K, a.dWg, dC_part, a.dC, done), "router totals launch");
}

}  // namespace focus
