// focus_router_scores_bwd: the derivative of S = (h W_g) C^T.  With T = dS^T h (K vectors of d, summed over all tokens)
//     dC = T W_g      dW_g = T^T C      dh = dS F,  F = C W_g^T
// so the hidden states are read once and their gradient written once, and everything else is of size K d: bound by the memory.
// A block has a strip of columns and a run of tokens and goes down its rows: a thread holds 4 columns (2 from K = 9 on) of F and of its part
// of T, both with K numbers a column.  A row costs it K/2 reads of the row's dS (pairs (w, w), one address a warp) and 4 K (2 K) packed
// multiply-adds.  Its pieces of the rows come by asynchronous copies through a ring of its own in shared memory, 24 to 32 rows ahead, which
// needs no barrier.
#include "common.cuh"

namespace focus {

constexpr int RB_THREADS = 128;
constexpr int RB_ROWS = 32;                 // rows of the ring; tokens whose dS is in shared memory at a time (two such pieces)
constexpr int RB_GROUP = 8;                 // rows copied, and worked on, at a time
constexpr int RB_TOTAL_COLS = 32;           // columns of a block that adds the parts up
constexpr int RB_FOLD = 512;                // up to K d_g of this, a block works out its columns of F itself

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

template <int BYTES> __device__ __forceinline__ void rb_copy(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}

// F: the folded projection, or nullptr: worked out here
template <int LD>
__global__ void __launch_bounds__(RB_THREADS)
router_bwd_kernel(const __nv_bfloat16* h, int64_t h_sb, int64_t h_sn, const float* dS, const float* F, const float* Wg, const float* C, int dg, int n, int runs, int run,
                  int d, int K, __nv_bfloat16* dh, int64_t d_sb, int64_t d_sn, float* part, unsigned* done) {
    constexpr int P = rb_pairs(LD), PER = RB_ROWS * LD / RB_THREADS;
    static_assert(PER >= 1, "a number of dS at least for every thread");
    struct __align__(4 * P) Words { uint32_t w[P]; };
    __shared__ float2 s[2][RB_ROWS * LD];
    __shared__ Words ring[RB_ROWS][RB_THREADS];
    __shared__ float cs[RB_FOLD];
    const int t = threadIdx.x, b = blockIdx.y / runs, tok0 = blockIdx.y % runs * run, e = (blockIdx.x * RB_THREADS + t) * 2 * P;
    const bool in = e < d;                                   // (d is a multiple of 8)
    dep_wait();
    dep_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && t == 0) *done = 0u;
    const int rows = min(run, n - tok0);
    const __nv_bfloat16* hp = h + b * h_sb + (int64_t)tok0 * h_sn + e;
    __nv_bfloat16* dp = dh ? dh + b * d_sb + (int64_t)tok0 * d_sn + e : nullptr;
    const float* sp = dS + ((size_t)b * n + tok0) * LD;
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&ring[0][t]);
    // group `g` of rows on its way (an empty one past the end)
    auto copy = [&](int g) {
#pragma unroll
        for (int u = 0; u < RB_GROUP; ++u) {
            const int r = g * RB_GROUP + u;
            if (in && r < rows) rb_copy<4 * P>(mine + (r % RB_ROWS) * (uint32_t)sizeof(ring[0]), hp + (int64_t)r * h_sn);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    constexpr int GROUPS = RB_ROWS / RB_GROUP;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) copy(g);
    float w[PER];
    auto load = [&](int r0) {                                // dS of the next RB_ROWS rows; columns from K on may hold anything
#pragma unroll
        for (int x = 0; x < PER; ++x) {
            const int q = x * RB_THREADS + t;
            w[x] = r0 + q / LD < rows && q % LD < K ? sp[(size_t)r0 * LD + q] : 0.f;
        }
    };
    load(0);
    float2 f[LD][P], acc[LD][P];
#pragma unroll
    for (int g = 0; g < LD; ++g) {
#pragma unroll
        for (int c = 0; c < P; ++c) {
            acc[g][c] = make_float2(0.f, 0.f);
            f[g][c] = F && in && dh && g < K ? *reinterpret_cast<const float2*>(F + (size_t)g * d + e + 2 * c) : make_float2(0.f, 0.f);
        }
    }
    if (!F && dh) {
        for (int i = t; i < K * dg; i += RB_THREADS) cs[i] = C[i];
        __syncthreads();
    }
    if (!F && in && dh) {
#pragma unroll 8
        for (int j = 0; j < dg; ++j) {
            float2 x[P];
#pragma unroll
            for (int c = 0; c < P; ++c) x[c] = make_float2(Wg[(size_t)(e + 2 * c) * dg + j], Wg[(size_t)(e + 2 * c + 1) * dg + j]);
#pragma unroll
            for (int g = 0; g < LD; ++g) {
                const float y = g < K ? cs[g * dg + j] : 0.f;
#pragma unroll
                for (int c = 0; c < P; ++c) f[g][c] = __ffma2_rn(make_float2(y, y), x[c], f[g][c]);
            }
        }
    }
    int buf = 0;
    for (int r0 = 0; r0 < rows; r0 += RB_ROWS, buf ^= 1) {
#pragma unroll
        for (int x = 0; x < PER; ++x) s[buf][x * RB_THREADS + t] = make_float2(w[x], w[x]);
        __syncthreads();                                     // (who still reads the other piece is no more than this one ahead)
        load(r0 + RB_ROWS);
#pragma unroll 1
        for (int g = 0; g < GROUPS; ++g) {
            if (r0 + g * RB_GROUP >= rows) break;
            asm volatile("cp.async.wait_group %0;" ::"n"(GROUPS - 1) : "memory");
            Words x[RB_GROUP];
#pragma unroll
            for (int u = 0; u < RB_GROUP; ++u) x[u] = ring[g * RB_GROUP + u][t];
#pragma unroll
            for (int u = 0; u < RB_GROUP; ++u) {
                const int r = r0 + g * RB_GROUP + u;
                float2 v[P], y[P];
#pragma unroll
                for (int c = 0; c < P; ++c) {
                    if (r >= rows) x[u].w[c] = 0u;
                    v[c] = make_float2(__uint_as_float(x[u].w[c] << 16), __uint_as_float(x[u].w[c] & 0xffff0000u));
                    y[c] = make_float2(0.f, 0.f);
                }
#pragma unroll
                for (int q = 0; q < LD; q += 2) {
                    const float4 w2 = *reinterpret_cast<const float4*>(&s[buf][(g * RB_GROUP + u) * LD + q]);
                    const float2 ww[2] = {make_float2(w2.x, w2.y), make_float2(w2.z, w2.w)};
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
#pragma unroll
                        for (int c = 0; c < P; ++c) {
                            acc[q + i][c] = __ffma2_rn(ww[i], v[c], acc[q + i][c]);
                            y[c] = __ffma2_rn(ww[i], f[q + i][c], y[c]);
                        }
                    }
                }
                if (dp && in && r < rows) {
                    Words z;
#pragma unroll
                    for (int c = 0; c < P; ++c) {
                        const __nv_bfloat162 a = __float22bfloat162_rn(y[c]);
                        z.w[c] = *reinterpret_cast<const uint32_t*>(&a);
                    }
                    *reinterpret_cast<Words*>(dp + (int64_t)r * d_sn) = z;
                }
            }
            copy(r0 / RB_GROUP + g + GROUPS);
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
// A thread adds up an eighth of the parts of a column.
template <int LD>
__global__ void __launch_bounds__(256)
router_total_kernel(const float* part, const float* C, const float* Wg, int parts, int d, int dg, int K, float* dWg, float* dC_part, float* dC, unsigned* done) {
    __shared__ float eighth[8][LD][RB_TOTAL_COLS + 1];
    __shared__ float T[LD][RB_TOTAL_COLS + 1];
    __shared__ bool last;
    const int t = threadIdx.x, e0 = blockIdx.x * RB_TOTAL_COLS, c = t % RB_TOTAL_COLS, q = t / RB_TOTAL_COLS, cols = min(RB_TOTAL_COLS, d - e0);
    dep_wait();
    dep_trigger();
    float x[LD];
#pragma unroll
    for (int g = 0; g < LD; ++g) x[g] = 0.f;
    if (c < cols) {
#pragma unroll 2
        for (int r = q; r < parts; r += 8) {
            const float* p = part + (size_t)r * K * d + e0 + c;
#pragma unroll
            for (int g = 0; g < LD; ++g)
                if (g < K) x[g] += p[(size_t)g * d];
        }
    }
#pragma unroll
    for (int g = 0; g < LD; ++g) eighth[q][g][c] = x[g];
    __syncthreads();
    for (int i = t; i < LD * RB_TOTAL_COLS; i += 256) {
        const int g = i / RB_TOTAL_COLS, k = i % RB_TOTAL_COLS;
        float y = 0.f;
#pragma unroll
        for (int z = 0; z < 8; ++z) y += eighth[z][g][k];
        T[g][k] = y;
    }
    __syncthreads();
    for (int i = t; i < cols * dg; i += 256) {
        const int k = i / dg, j = i % dg;
        float y = 0.f;
#pragma unroll
        for (int g = 0; g < LD; ++g)
            if (g < K) y = fmaf(T[g][k], C[(size_t)g * dg + j], y);
        dWg[(size_t)(e0 + k) * dg + j] = y;
    }
    for (int i = t; i < K * dg; i += 256) {
        const int g = i / dg, j = i % dg;
        float y = 0.f;
#pragma unroll 8
        for (int k = 0; k < cols; ++k) y = fmaf(T[g][k], Wg[(size_t)(e0 + k) * dg + j], y);
        dC_part[(size_t)blockIdx.x * K * dg + i] = y;
    }
    __threadfence();
    __syncthreads();
    if (t == 0) last = atomicAdd(done, 1u) == gridDim.x - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // eight lanes a number
    for (int i0 = 0; i0 < K * dg; i0 += 32) {
        const int i = i0 + t / 8;
        float y = 0.f;
        if (i < K * dg) {
#pragma unroll 4
            for (int z = t % 8; z < (int)gridDim.x; z += 8) y += __ldcg(dC_part + (size_t)z * K * dg + i);
        }
        for (int off = 4; off; off >>= 1) y += __shfl_xor_sync(0xffffffffu, y, off);
        if (i < K * dg && t % 8 == 0) dC[i] = y;
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
static int launch_router(const focus_shape* s, const RouterBwdArgs& a, const RouterCut& c, const float* F, float* part, float* dC_part, unsigned* done, cudaStream_t st) {
    auto kern = router_bwd_kernel<LD>;
    int rc = check_cuda(launch_dependent(kern, dim3((unsigned)router_strips(s, a.d_model), (unsigned)(s->batch * c.runs)), dim3(RB_THREADS), 0, st, a.h, a.h_sb, a.h_sn, a.ds,
                                         F, a.Wg, a.C, a.d_g, s->n, c.runs, c.run, a.d_model, s->K, a.dh, a.dh_sb, a.dh_sn, part, done), "router backward launch");
    if (rc) return rc;
    return check_cuda(launch_dependent(router_total_kernel<LD>, dim3((unsigned)cdiv(a.d_model, RB_TOTAL_COLS)), dim3(256), 0, st, (const float*)part, a.C, a.Wg,
                                       s->batch * c.runs, a.d_model, a.d_g, s->K, a.dWg, dC_part, a.dC, done), "router totals launch");
}

int launch_router_bwd(const focus_shape* s, const RouterBwdArgs& a, cudaStream_t st) {
    const int d = a.d_model, K = s->K;
    const RouterCut c = router_cut(s, d);
    const RouterWorkspace w = router_workspace(s, d, a.d_g);
    if ((long long)s->batch * c.runs > 65535) return fail(FOCUS_ERR_UNSUPPORTED, "router backward: %lld runs of tokens exceed 65535", (long long)s->batch * c.runs);
    float *F = reinterpret_cast<float*>(a.ws + w.F), *part = reinterpret_cast<float*>(a.ws + w.part), *dC_part = reinterpret_cast<float*>(a.ws + w.dC);
    unsigned* done = reinterpret_cast<unsigned*>(a.ws + w.done);
    const bool fold = a.dh && (long long)K * a.d_g > RB_FOLD;
    int rc = FOCUS_OK;
    if (fold) rc = check_cuda(launch_dependent(router_fold_kernel, dim3((unsigned)cdiv(d, 256), (unsigned)K), dim3(256), 0, st, a.Wg, a.C, d, a.d_g, F), "router fold launch");
    if (rc) return rc;
    if (!fold) F = nullptr;
    switch (focus_soft_ld(K)) {
        case 4: return launch_router<4>(s, a, c, F, part, dC_part, done, st);
        case 8: return launch_router<8>(s, a, c, F, part, dC_part, done, st);
        case 16: return launch_router<16>(s, a, c, F, part, dC_part, done, st);
    }
    return launch_router<32>(s, a, c, F, part, dC_part, done, st);
}

}  // namespace focus
