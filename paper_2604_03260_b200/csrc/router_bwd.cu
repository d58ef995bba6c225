// focus_router_scores_bwd: the derivative of S = (h W_g) C^T.  With T = dS^T h (K vectors of d, summed over all tokens)
//     dC = T W_g      dW_g = T^T C      dh = dS (C W_g^T)
// so the hidden states are read once and their gradient written once, and everything else is of size K d.
#include "common.cuh"

namespace focus {

constexpr int RB_TOKENS = 128;      // tokens of a block
constexpr int RB_COLS = 512;        // columns of a block: two a thread

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

template <int LD>
__global__ void __launch_bounds__(256)
router_bwd_kernel(const __nv_bfloat16* h, int64_t h_sb, int64_t h_sn, const float* dS, const float* F, int n, int nt, int d, int K, __nv_bfloat16* dh,
                  int64_t d_sb, int64_t d_sn, float* part) {
    __shared__ float s[RB_TOKENS * LD];
    const int t = threadIdx.x, tile = blockIdx.y, b = tile / nt, tok0 = (tile % nt) * RB_TOKENS, e = blockIdx.x * RB_COLS + 2 * t;
    dep_wait();
    dep_trigger();
    const int rows = min(RB_TOKENS, n - tok0);
    for (int q = t; q < rows * LD; q += 256) s[q] = q % LD < K ? dS[((size_t)b * n + tok0) * LD + q] : 0.f;
    __syncthreads();
    if (e >= d) return;
    float2 f[LD], acc[LD];
#pragma unroll
    for (int g = 0; g < LD; ++g) {
        f[g] = g < K ? *reinterpret_cast<const float2*>(F + (size_t)g * d + e) : make_float2(0.f, 0.f);
        acc[g] = make_float2(0.f, 0.f);
    }
    const __nv_bfloat16* hp = h + b * h_sb + (int64_t)tok0 * h_sn + e;
    __nv_bfloat16* dp = dh ? dh + b * d_sb + (int64_t)tok0 * d_sn + e : nullptr;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
        const float2 x = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(hp + r * h_sn));
        float2 y = make_float2(0.f, 0.f);
#pragma unroll
        for (int g = 0; g < LD; ++g) {
            const float w = s[r * LD + g];
            acc[g].x = fmaf(w, x.x, acc[g].x); acc[g].y = fmaf(w, x.y, acc[g].y);
            y.x = fmaf(w, f[g].x, y.x); y.y = fmaf(w, f[g].y, y.y);
        }
        if (dp) *reinterpret_cast<__nv_bfloat162*>(dp + r * d_sn) = __float22bfloat162_rn(y);
    }
#pragma unroll
    for (int g = 0; g < LD; ++g)
        if (g < K) *reinterpret_cast<float2*>(part + ((size_t)tile * K + g) * d + e) = acc[g];
}

// T = sum of the partial sums, dW_g = T^T C.  A block per 8 columns, a warp per column.
__global__ void __launch_bounds__(256)
router_bwd_weights_kernel(const float* part, const float* C, int tiles, int d, int dg, int K, float* T, float* dWg) {
    __shared__ float tk[8][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, e = blockIdx.x * 8 + warp;
    dep_wait();
    dep_trigger();
    if (e >= d) return;
    for (int g = 0; g < K; ++g) {
        double s = 0.0;
        for (int x = lane; x < tiles; x += 32) s += part[((size_t)x * K + g) * d + e];
        for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        if (lane == 0) T[(size_t)g * d + e] = tk[warp][g] = (float)s;
    }
    __syncwarp();
    for (int j = lane; j < dg; j += 32) {
        float s = 0.f;
        for (int g = 0; g < K; ++g) s = fmaf(tk[warp][g], C[(size_t)g * dg + j], s);
        dWg[(size_t)e * dg + j] = s;
    }
}

// dC = T W_g: a block per (group, column of the projection)
__global__ void __launch_bounds__(256) router_bwd_centroids_kernel(const float* T, const float* Wg, int d, int dg, float* dC) {
    __shared__ double s[8];
    const int g = blockIdx.y, j = blockIdx.x;
    dep_wait();
    dep_trigger();
    double x = 0.0;
    for (int e = threadIdx.x; e < d; e += 256) x += (double)T[(size_t)g * d + e] * Wg[(size_t)e * dg + j];
    for (int off = 16; off; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) x += s[w];
        dC[(size_t)g * dg + j] = (float)x;
    }
}

static int router_tiles(const focus_shape* s) { return s->batch * cdiv(s->n, RB_TOKENS); }

size_t router_bwd_workspace_bytes(const focus_shape* s, int d) {
    return align_up((size_t)s->K * d * 4, 256) * 2 + align_up((size_t)router_tiles(s) * s->K * d * 4, 256);
}

template <int LD>
static int launch_tokens(const focus_shape* s, const RouterBwdArgs& a, const float* F, float* part, cudaStream_t st) {
    auto kern = router_bwd_kernel<LD>;
    return check_cuda(launch_dependent(kern, dim3((unsigned)cdiv(a.d_model, RB_COLS), (unsigned)router_tiles(s)), dim3(256), 0, st, a.h, a.h_sb, a.h_sn, a.ds, F, s->n,
                                       cdiv(s->n, RB_TOKENS), a.d_model, s->K, a.dh, a.dh_sb, a.dh_sn, part), "router backward launch");
}

int launch_router_bwd(const focus_shape* s, const RouterBwdArgs& a, cudaStream_t st) {
    const int d = a.d_model, tiles = router_tiles(s), K = s->K;
    float* F = reinterpret_cast<float*>(a.ws);
    float* T = F + align_up((size_t)K * d * 4, 256) / 4;
    float* part = T + align_up((size_t)K * d * 4, 256) / 4;
    int rc = check_cuda(launch_dependent(router_fold_kernel, dim3((unsigned)cdiv(d, 256), (unsigned)K), dim3(256), 0, st, a.Wg, a.C, d, a.d_g, F), "router fold launch");
    if (rc) return rc;
    switch (focus_soft_ld(K)) {
        case 4: rc = launch_tokens<4>(s, a, F, part, st); break;
        case 8: rc = launch_tokens<8>(s, a, F, part, st); break;
        case 16: rc = launch_tokens<16>(s, a, F, part, st); break;
        default: rc = launch_tokens<32>(s, a, F, part, st);
    }
    if (rc) return rc;
    if ((rc = check_cuda(launch_dependent(router_bwd_weights_kernel, dim3((unsigned)cdiv(d, 8)), dim3(256), 0, st, part, a.C, tiles, d, a.d_g, K, T, a.dWg), "router weights launch"))) return rc;
    return check_cuda(launch_dependent(router_bwd_centroids_kernel, dim3((unsigned)a.d_g, (unsigned)K), dim3(256), 0, st, T, a.Wg, d, a.d_g, a.dC), "router centroids launch");
}

}  // namespace focus
