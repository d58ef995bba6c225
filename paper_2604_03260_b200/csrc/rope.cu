// focus_qk_norm_rope and its derivative: the query and key heads of a layer normalised head by head and rotated by their positions, as
// focus_assign and the attention read them; focus_rope_frequencies (host): what a position is multiplied by.
//
//   y = x * r * w,  r = (mean x^2 + eps)^(-1/2);   (a, b) -> (a cos t - b sin t, a sin t + b cos t) * amplitude,  t = position * freq_i
// and back: with g the rotated-back gradient of y, xhat = x r and u = g w:
//   dx = r (u - xhat mean(u xhat)),   dw = sum over rows of g xhat.
// HBM-bound: every vector read once and written once (backward: vectors and gradients read, gradients written).
#include "common.cuh"

#include <math.h>

namespace focus {

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_GRID = 148 * 4;
constexpr int ROPE_TOKENS = 16;                   // per tile at most

struct RopeArgs {
    const __nv_bfloat16 *x[2], *g[2];             // [0] queries, [1] keys: vectors, and the gradients of the results
    __nv_bfloat16* out[2];
    int64_t x_b[2], x_h[2], x_n[2], g_b[2], g_h[2], g_n[2], o_b[2], o_h[2], o_n[2];
    const float* w[2];
    const double* freq;
    const int32_t* positions;
    float* partial;                               // backward with a norm: [blocks][2][D] sums of g xhat
    int heads[2], n, rot, interleaved;
    float eps, amplitude;
    int T, lgT, hsplit;                           // tokens per tile (a power of two), parts that the heads of a tile are cut into
    long long tiles;                              // batch * ceil(n / T) * hsplit
};

// A row is cut into units of 2 * V dimensions: V pairs that are turned together.  Rotating halves, unit u < rot / (2 V) holds dimensions
// V u .. and rot / 2 + V u ..; interleaved, and behind the rotated part, 2 V consecutive ones.  V = 8 (16-byte pieces) unless halves are
// not whole pieces (rot % 16 != 0), where V = 1.
template <int D, int V> struct RopeCfg {
    static constexpr int UNITS = D / (2 * V);
    static constexpr int LPR = UNITS < 32 ? UNITS : 32;       // lanes per row
    static constexpr int UPL = UNITS / LPR;                   // units per lane
    static constexpr int RPP = ROPE_THREADS / LPR;            // rows per pass of a CTA
};

template <int V>
__device__ __forceinline__ void rope_load(float (&f)[V], const __nv_bfloat16* p) {
    if constexpr (V == 8) {
        const uint4 r = *reinterpret_cast<const uint4*>(p);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) f[i] = __bfloat162float(p[i]);
    }
}
template <int V>
__device__ __forceinline__ void rope_store(__nv_bfloat16* p, const float (&f)[V]) {
    if constexpr (V == 8) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = __float2bfloat16(f[i]);
    }
}

__device__ __forceinline__ void rope_turn(float& p, float& r, float cs, float sn) {
    const float p0 = p;
    p = p0 * cs - r * sn;
    r = p0 * sn + r * cs;
}

// A CTA takes T tokens and (a part of) all their heads.  The thread's token and its place in the row are the same in every pass, so the
// sines and cosines of its pairs, which cost a reduction of the angle in 64 bits (positions reach a million, and fp32 would leave an
// error of 0.06 there), are worked out once per token and stay in registers; the weights do too.
template <int D, int V, bool BWD>
__global__ void __launch_bounds__(ROPE_THREADS)
qk_norm_rope_kernel(const RopeArgs a) {
    using C = RopeCfg<D, V>;
    __shared__ float2 cs_s[ROPE_TOKENS][D / 2 + 1];           // [token][pair]
    __shared__ float red_s[BWD ? C::RPP : 1][BWD ? D : 1];
    const int lane_r = threadIdx.x % C::LPR, rs = threadIdx.x / C::LPR;
    const int tok = rs & (a.T - 1), hofs = rs >> a.lgT, hstep = C::RPP >> a.lgT;
    const int half = a.rot >> 1;
    const int turned = a.interleaved ? (a.rot + 2 * V - 1) / (2 * V) : a.rot / (2 * V);    // units with a rotation
    // a unit's two pieces
    int d0[C::UPL], d1[C::UPL];
#pragma unroll
    for (int i = 0; i < C::UPL; ++i) {
        const int u = lane_r + i * C::LPR;
        const bool halves = !a.interleaved && u < turned;
        d0[i] = halves ? V * u : 2 * V * u;
        d1[i] = halves ? half + V * u : 2 * V * u + V;
    }
    dep_wait();
    dep_trigger();
    float dw[2][C::UPL][2 * V];
    if constexpr (BWD) {
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int i = 0; i < C::UPL; ++i)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) dw[s][i][e] = 0.f;
    }
    const int per_seq = (a.n + a.T - 1) >> a.lgT;
    const int all = a.heads[0] + a.heads[1];
    for (long long tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int part = (int)(tile % a.hsplit);
        const long long tt = tile / a.hsplit;
        const int b = (int)(tt / per_seq), t0 = (int)(tt - (long long)b * per_seq) << a.lgT;
        // sines and cosines of the tile
        if (half > 0) {
            __syncthreads();
            for (int i = threadIdx.x; i < half << a.lgT; i += ROPE_THREADS) {
                const int t = i / half, f = i - t * half;
                if (t0 + t < a.n) {
                    const int pos = a.positions ? dep_load(a.positions + (size_t)b * a.n + t0 + t) : t0 + t;
                    double turns = (double)pos * (dep_load(a.freq + f) * 0.15915494309189533577);
                    turns -= rint(turns);
                    float sn, cn;
                    sincospif((float)(2.0 * turns), &sn, &cn);
                    cs_s[t][f] = make_float2(cn * a.amplitude, sn * a.amplitude);
                }
            }
            __syncthreads();
        }
        const bool live = t0 + tok < a.n;
        float cn[C::UPL][V], sn[C::UPL][V];
#pragma unroll
        for (int i = 0; i < C::UPL; ++i) {
            const int u = lane_r + i * C::LPR;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                cn[i][e] = 1.f;
                sn[i][e] = 0.f;
                if (live && u < turned && V * u + e < half) {
                    const float2 x = cs_s[tok][V * u + e];
                    cn[i][e] = x.x;
                    sn[i][e] = x.y;
                }
            }
        }
        const int h0 = (int)((long long)all * part / a.hsplit), h1 = (int)((long long)all * (part + 1) / a.hsplit);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int lo = s ? max(h0 - a.heads[0], 0) : h0, hi = s ? h1 - a.heads[0] : min(h1, a.heads[0]);
            const bool norm = a.w[s] != nullptr;
            float w[C::UPL][2 * V];
#pragma unroll
            for (int i = 0; i < C::UPL; ++i)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) w[i][e] = norm ? dep_load(a.w[s] + (e < V ? d0[i] + e : d1[i] + e - V)) : 1.f;
            const size_t xo = (size_t)b * a.x_b[s] + (size_t)(t0 + tok) * a.x_n[s];
            const size_t go = BWD ? (size_t)b * a.g_b[s] + (size_t)(t0 + tok) * a.g_n[s] : 0;
            const size_t oo = (size_t)b * a.o_b[s] + (size_t)(t0 + tok) * a.o_n[s];
            // (all lanes of a row take part in its sums; the bound is the same for the whole warp)
#pragma unroll 2
            for (int hb = lo; hb < hi; hb += hstep) {
                const int h = hb + hofs;
                const bool on = live && h < hi;
                float x[C::UPL][2 * V], y[C::UPL][2 * V];
                float ss = 0.f, dot = 0.f;
#pragma unroll
                for (int i = 0; i < C::UPL; ++i) {
#pragma unroll
                    for (int e = 0; e < 2 * V; ++e) x[i][e] = y[i][e] = 0.f;
                    if (on && (!BWD || norm)) {
                        const __nv_bfloat16* p = a.x[s] + xo + (size_t)h * a.x_h[s];
                        rope_load<V>(*reinterpret_cast<float(*)[V]>(&x[i][0]), p + d0[i]);
                        rope_load<V>(*reinterpret_cast<float(*)[V]>(&x[i][V]), p + d1[i]);
                    }
                    if (BWD && on) {
                        const __nv_bfloat16* p = a.g[s] + go + (size_t)h * a.g_h[s];
                        rope_load<V>(*reinterpret_cast<float(*)[V]>(&y[i][0]), p + d0[i]);
                        rope_load<V>(*reinterpret_cast<float(*)[V]>(&y[i][V]), p + d1[i]);
                    }
                }
                // element (first, second) of pair e of a unit: (e, V + e) where halves turn, (2 e, 2 e + 1) where pairs are interleaved
                auto turn = [&](float (&f)[2 * V], int i, float sign) {
                    if (a.interleaved) {
#pragma unroll
                        for (int e = 0; e < V; ++e) rope_turn(f[2 * e], f[2 * e + 1], cn[i][e], sign * sn[i][e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < V; ++e) rope_turn(f[e], f[V + e], cn[i][e], sign * sn[i][e]);
                    }
                };
                if constexpr (BWD) {
#pragma unroll
                    for (int i = 0; i < C::UPL; ++i) turn(y[i], i, -1.f);
                }
                if (norm) {
#pragma unroll
                    for (int i = 0; i < C::UPL; ++i)
#pragma unroll
                        for (int e = 0; e < 2 * V; ++e) {
                            ss = fmaf(x[i][e], x[i][e], ss);
                            if (BWD) dot = fmaf(x[i][e], y[i][e] * w[i][e], dot);
                        }
#pragma unroll
                    for (int off = C::LPR / 2; off >= 1; off >>= 1) {
                        ss += __shfl_xor_sync(0xffffffffu, ss, off);
                        if (BWD) dot += __shfl_xor_sync(0xffffffffu, dot, off);
                    }
                    const float r = 1.f / sqrtf(ss * (1.f / D) + a.eps);
                    if constexpr (!BWD) {
#pragma unroll
                        for (int i = 0; i < C::UPL; ++i)
#pragma unroll
                            for (int e = 0; e < 2 * V; ++e) x[i][e] *= r * w[i][e];
                    } else {
                        const float m = dot * r * (1.f / D);                   // mean(u xhat)
#pragma unroll
                        for (int i = 0; i < C::UPL; ++i)
#pragma unroll
                            for (int e = 0; e < 2 * V; ++e) {
                                const float xhat = x[i][e] * r;
                                dw[s][i][e] = fmaf(y[i][e], on ? xhat : 0.f, dw[s][i][e]);
                                y[i][e] = r * (y[i][e] * w[i][e] - xhat * m);
                            }
                    }
                }
                if (on) {
                    __nv_bfloat16* p = a.out[s] + oo + (size_t)h * a.o_h[s];
#pragma unroll
                    for (int i = 0; i < C::UPL; ++i) {
                        if constexpr (!BWD) turn(x[i], i, 1.f);
                        float(&f)[2 * V] = BWD ? y[i] : x[i];
                        rope_store<V>(p + d0[i], *reinterpret_cast<float(*)[V]>(&f[0]));
                        rope_store<V>(p + d1[i], *reinterpret_cast<float(*)[V]>(&f[V]));
                    }
                }
            }
        }
    }
    if constexpr (BWD) {
        if (!a.partial) return;
        // the CTA's sums: rows of threads in a fixed order
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < C::UPL; ++i)
#pragma unroll
                for (int e = 0; e < 2 * V; ++e) red_s[rs][e < V ? d0[i] + e : d1[i] + e - V] = dw[s][i][e];
            __syncthreads();
            for (int d = threadIdx.x; d < D; d += ROPE_THREADS) {
                float t = 0.f;
                for (int r = 0; r < C::RPP; ++r) t += red_s[r][d];
                a.partial[((size_t)blockIdx.x * 2 + s) * D + d] = t;
            }
        }
    }
}

// dw[s][d] = sum over the CTAs of partial[cta][s][d]; a block per 32 dimensions, 32 rows of threads in a fixed order
__global__ void __launch_bounds__(1024)
norm_weight_grad_kernel(const float* partial, int ctas, int D, float* dwq, float* dwk) {
    __shared__ float red[32][33];
    const int col = blockIdx.x * 32 + threadIdx.x;            // 0 .. 2 D - 1
    dep_wait();
    dep_trigger();
    float t = 0.f;
#pragma unroll 4
    for (int r = threadIdx.y; r < ctas; r += 32) t += dep_load(partial + (size_t)r * 2 * D + col);
    red[threadIdx.y][threadIdx.x] = t;
    __syncthreads();
    if (threadIdx.y == 0) {
        t = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) t += red[r][threadIdx.x];
        float* dst = col < D ? dwq : dwk;
        if (dst) dst[col < D ? col : col - D] = t;
    }
}

size_t qk_norm_rope_bwd_workspace_bytes(const focus_shape* s) { return (size_t)ROPE_GRID * 2 * s->D * sizeof(float); }

template <int D, int V, bool BWD>
static int launch_rope_dv(const focus_shape* s, RopeArgs& a, float* dwq, float* dwk, cudaStream_t st) {
    using C = RopeCfg<D, V>;
    const int all = s->Hq + s->Hkv;
    // tokens per tile: as many as leave every multiprocessor two tiles, 16 at most (16 head-major rows of a token block are 4 KB in one piece)
    const int most = C::RPP < ROPE_TOKENS ? C::RPP : ROPE_TOKENS;
    a.T = 1;
    a.lgT = 0;
    while (a.T < most && (long long)s->batch * cdiv(s->n, 2 * a.T) >= 2 * 148) { a.T *= 2; ++a.lgT; }
    const long long tok_tiles = (long long)s->batch * cdiv(s->n, a.T);
    // few tiles: the heads of a tile over several CTAs, a pass each at the least
    const int passes = cdiv(all * a.T, C::RPP);
    long long split = tok_tiles >= ROPE_GRID ? 1 : ROPE_GRID / tok_tiles;
    if (split > passes) split = passes;
    if (split > all) split = all;
    a.hsplit = (int)split;
    a.tiles = tok_tiles * split;
    const int grid = (int)(a.tiles < ROPE_GRID ? a.tiles : ROPE_GRID);
    int rc = check_cuda(launch_dependent(qk_norm_rope_kernel<D, V, BWD>, dim3(grid), dim3(ROPE_THREADS), 0, st, a), "norm and rotation kernel launch");
    if (rc || !BWD || !a.partial) return rc;
    return check_cuda(launch_dependent(norm_weight_grad_kernel, dim3(2 * D / 32), dim3(32, 32), 0, st, a.partial, grid, D, dwq, dwk),
                      "norm weight gradient kernel launch");
}

template <int D, bool BWD>
static int launch_rope_d(const focus_shape* s, RopeArgs& a, float* dwq, float* dwk, cudaStream_t st) {
    return a.interleaved || a.rot % 16 == 0 ? launch_rope_dv<D, 8, BWD>(s, a, dwq, dwk, st) : launch_rope_dv<D, 1, BWD>(s, a, dwq, dwk, st);
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
    a.n = s->n;
    a.rot = rope->rotary;
    a.interleaved = rope->interleaved;
    a.eps = rope->eps;
    a.amplitude = rope->amplitude == 0.f ? 1.f : rope->amplitude;
    a.freq = freq;
    a.positions = positions;
    a.partial = w[0] || w[1] ? partial : nullptr;
    if (grads) {
        switch (s->D) {
            case 64: return launch_rope_d<64, true>(s, a, dwq, dwk, st);
            case 128: return launch_rope_d<128, true>(s, a, dwq, dwk, st);
            default: return launch_rope_d<256, true>(s, a, dwq, dwk, st);
        }
    }
    switch (s->D) {
        case 64: return launch_rope_d<64, false>(s, a, nullptr, nullptr, st);
        case 128: return launch_rope_d<128, false>(s, a, nullptr, nullptr, st);
        default: return launch_rope_d<256, false>(s, a, nullptr, nullptr, st);
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
