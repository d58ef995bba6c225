// focus_grad_clip: the norm over many tensors, and the tensors scaled where it is above a bound.  Two passes, each a few launches (one per
// CLIP_TENSORS tensors, whose addresses travel as kernel arguments): sums of squares, one per block, and the scaled copies, in which every
// block adds those sums up for itself, in the same order.  Bound by the memory: read, read again and written; the second pass goes backwards,
// so that it meets what the first one left in L2.
//
// Squares: 8 numbers' squares are added in fp32 and those sums in fp64 (a conversion per number would be as slow as the memory:
// 16 a clock and SM).  Where such a sum is beyond the range in which fp32 loses nothing (overflow, or so small that squares may have
// vanished) the 8 are taken again in fp64; 8 zeros too, so that 1 GB of fp32 zeros takes 1 % longer than of other numbers, 0.5 GB of bf16 zeros 10 % (304 us for 276).
#include "common.cuh"

#include <string.h>

namespace focus {

constexpr int CLIP_TENSORS = 100;       // of a launch: 4 KB of arguments hold them
constexpr int CLIP_BLOCKS = 592;        // at most, of a launch: four per SM
constexpr int CLIP_BYTES = 32768;       // of a tensor that a block takes at a time

struct ClipTable {
    const void* src[CLIP_TENSORS];
    void* dst[CLIP_TENSORS];
    long long count[CLIP_TENSORS];
    int first[CLIP_TENSORS + 1];        // first chunk of each tensor
    uint32_t half[(CLIP_TENSORS + 31) / 32];      // which are bf16
    int tensors;
    bool add;                           // sums are added to those of the launch before
};

// chunk -> its tensor and the numbers [from, to) of it; chunks begin at multiples of CLIP_BYTES of the address, so that all but a
// tensor's first begin on a 16-byte boundary
struct ClipChunk {
    const char* src;
    char* dst;
    long long count;         // numbers
    bool half;
};
__device__ __forceinline__ ClipChunk clip_chunk(const ClipTable& t, int chunk) {
    int lo = 0, hi = t.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    ClipChunk c;
    c.half = t.half[lo >> 5] >> (lo & 31) & 1;
    const int size = c.half ? 2 : 4;
    const char* const src = (const char*)t.src[lo];
    const long long head = (long long)((uintptr_t)src & 15), end = t.count[lo] * size;
    const long long k = chunk - t.first[lo];
    const long long from = k == 0 ? 0 : k * CLIP_BYTES - head, to = min(end, (k + 1) * CLIP_BYTES - head);
    c.src = src + from;
    c.dst = (char*)t.dst[lo] + from;
    c.count = (to - from) / size;
    return c;
}
inline long long clip_chunks(const void* src, long long bytes) { return bytes == 0 ? 0 : ((long long)((uintptr_t)src & 15) + bytes + CLIP_BYTES - 1) / CLIP_BYTES; }

__device__ __forceinline__ double block_sum(double x, double* s) {
    for (int off = 16; off; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < 8; ++w) x += s[w];
    return x;
}

__device__ __forceinline__ float2 clip_pair(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float clip_number(const char* p, long long e, bool half) {
    return half ? __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[e]) : reinterpret_cast<const float*>(p)[e];
}

// the squares of 8 numbers
__device__ __forceinline__ double clip_eight(const float (&v)[8]) {
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int e = 0; e < 8; e += 2) s = __ffma2_rn(make_float2(v[e], v[e + 1]), make_float2(v[e], v[e + 1]), s);
    const float f = s.x + s.y;
    if (f > 1e-22f && f < 3e38f) return (double)f;
    double x = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) x += (double)v[e] * (double)v[e];
    return x;
}

__global__ void __launch_bounds__(256, 4) clip_squares_kernel(const __grid_constant__ ClipTable t, double* sums) {
    __shared__ double s[8];
    double x = 0.0;
    dep_wait();
    dep_trigger();
    for (int chunk = blockIdx.x; chunk < t.first[t.tensors]; chunk += gridDim.x) {
        const ClipChunk c = clip_chunk(t, chunk);
        const int size = c.half ? 2 : 4;
        // to the first 16-byte boundary, whole pieces of 32 bytes (bf16: 16), and what is left
        const int lead = (int)min(c.count, (long long)((16 - ((uintptr_t)c.src & 15)) & 15) / size);
        const int pieces = (int)((c.count - lead) / 8);
        const char* const body = c.src + lead * size;
        if (c.half) {
            const uint4* const p = reinterpret_cast<const uint4*>(body);
            for (int i = threadIdx.x; i < pieces; i += 1024) {
                uint4 w[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) w[u] = i + 256 * u < pieces ? p[i + 256 * u] : make_uint4(0, 0, 0, 0);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const float2 a = clip_pair(w[u].x), b = clip_pair(w[u].y), d = clip_pair(w[u].z), e = clip_pair(w[u].w);
                    const float v[8] = {a.x, a.y, b.x, b.y, d.x, d.y, e.x, e.y};
                    if (i + 256 * u < pieces) x += clip_eight(v);
                }
            }
        } else {
            const float4* const p = reinterpret_cast<const float4*>(body);
            for (int i = threadIdx.x; i < pieces; i += 512) {
                float4 w[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) w[u] = i + 256 * (u / 2) < pieces ? p[2 * (i + 256 * (u / 2)) + u % 2] : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int u = 0; u < 4; u += 2) {
                    const float v[8] = {w[u].x, w[u].y, w[u].z, w[u].w, w[u + 1].x, w[u + 1].y, w[u + 1].z, w[u + 1].w};
                    if (i + 256 * (u / 2) < pieces) x += clip_eight(v);
                }
            }
        }
        const int rest = (int)c.count - lead - 8 * pieces;           // at most 7 before and 7 behind
        if ((int)threadIdx.x < lead + rest) {
            const double v = clip_number(c.src, (int)threadIdx.x < lead ? (long long)threadIdx.x : 8ll * pieces + threadIdx.x, c.half);
            x += v * v;
        }
    }
    x = block_sum(x, s);
    if (threadIdx.x == 0) sums[blockIdx.x] = t.add ? sums[blockIdx.x] + x : x;
}

__global__ void __launch_bounds__(256, 4) clip_scale_kernel(const __grid_constant__ ClipTable t, const double* sums, int blocks, double bound, float* norm_out) {
    __shared__ double s[8];
    dep_wait();
    dep_trigger();
    double x = 0.0;
    for (int e = threadIdx.x; e < blocks; e += 256) x += sums[e];
    const double norm = sqrt(block_sum(x, s));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const double by = norm > bound && isfinite((float)norm) ? bound / norm : 1.0;       // (what is reported as not finite is left to the caller)
    // A factor below fp32's normal numbers would have lost bits (below 2^-149: all of them, though what a large number becomes may be a normal one):
    // then every product is taken in fp64, one number at a time
    const bool tiny = by < 0x1p-126;
    const float f = (float)by;
    const int total = t.first[t.tensors];
    for (int chunk = total - 1 - (int)blockIdx.x; chunk >= 0; chunk -= gridDim.x) {
        const ClipChunk c = clip_chunk(t, chunk);
        if (by == 1.0 && c.src == c.dst) continue;
        const int size = c.half ? 2 : 4;
        auto one = [&](long long e) {
            const float x = clip_number(c.src, e, c.half), v = tiny ? (float)((double)x * by) : x * f;
            if (c.half) reinterpret_cast<__nv_bfloat16*>(c.dst)[e] = __float2bfloat16_rn(v);
            else reinterpret_cast<float*>(c.dst)[e] = v;
        };
        if (tiny || ((uintptr_t)c.src ^ (uintptr_t)c.dst) & 15) {      // (or no boundary in common)
            for (long long e = threadIdx.x; e < c.count; e += 256) one(e);
            continue;
        }
        const int lead = (int)min(c.count, (long long)((16 - ((uintptr_t)c.src & 15)) & 15) / size), per = 16 / size;
        const int pieces = (int)((c.count - lead) / per);
        const uint4* const p = reinterpret_cast<const uint4*>(c.src + lead * size);
        uint4* const q = reinterpret_cast<uint4*>(c.dst + lead * size);
        for (int i = threadIdx.x; i < pieces; i += 1024) {
            uint4 w[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + 256 * u < pieces) w[u] = p[i + 256 * u];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t* const v = reinterpret_cast<uint32_t*>(&w[u]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (c.half) {
                        const float2 y = clip_pair(v[e]);
                        const __nv_bfloat162 z = __floats2bfloat162_rn(y.x * f, y.y * f);
                        v[e] = *reinterpret_cast<const uint32_t*>(&z);
                    } else {
                        v[e] = __float_as_uint(__uint_as_float(v[e]) * f);
                    }
                }
                if (i + 256 * u < pieces) q[i + 256 * u] = w[u];
            }
        }
        const int rest = (int)c.count - lead - per * pieces;
        if ((int)threadIdx.x < lead + rest) one((int)threadIdx.x < lead ? (long long)threadIdx.x : (long long)per * pieces + threadIdx.x);
    }
}

size_t grad_clip_workspace_bytes() { return CLIP_BLOCKS * sizeof(double); }

int launch_grad_clip(const focus_grad* grads, int count, double bound, float* norm_out, double* sums, cudaStream_t st) {
    int blocks = 0;                     // sums that the first pass writes: as many as the largest launch has blocks
    for (int pass = 0; pass < 3; ++pass) {
        bool first = true;
        for (int at = 0; at < count || first; at += CLIP_TENSORS) {
            ClipTable t;
            t.tensors = count - at < CLIP_TENSORS ? count - at : CLIP_TENSORS;
            t.first[0] = 0;
            memset(t.half, 0, sizeof t.half);
            for (int i = 0; i < t.tensors; ++i) {
                const focus_grad& g = grads[at + i];
                const bool half = g.dtype == FOCUS_GRAD_BF16;
                t.src[i] = g.src;
                t.dst[i] = g.dst;
                t.count[i] = g.count;
                const long long next = t.first[i] + clip_chunks(g.src, g.count * (half ? 2 : 4));
                if (next > 0x7fffffffll) return fail(FOCUS_ERR_UNSUPPORTED, "grad_clip: too many numbers");
                t.first[i + 1] = (int)next;
                if (half) t.half[i >> 5] |= 1u << (i & 31);
            }
            t.add = !first;
            const int chunks = t.first[t.tensors], own = chunks < CLIP_BLOCKS ? (chunks > 0 ? chunks : 1) : CLIP_BLOCKS;
            int rc = FOCUS_OK;
            if (pass == 0) {
                if (own > blocks) blocks = own;
                if (count <= CLIP_TENSORS) break;           // (one launch)
            } else if (pass == 1) {
                rc = check_cuda(launch_dependent(clip_squares_kernel, dim3((unsigned)blocks), dim3(256), 0, st, t, sums), "squares launch");
            } else {
                rc = check_cuda(launch_dependent(clip_scale_kernel, dim3((unsigned)own), dim3(256), 0, st, t, (const double*)sums, blocks, bound,
                                                 first ? norm_out : nullptr), "scale launch");
            }
            if (rc) return rc;
            first = false;
        }
    }
    return FOCUS_OK;
}

}  // namespace focus
