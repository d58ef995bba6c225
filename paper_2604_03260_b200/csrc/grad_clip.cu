// focus_grad_clip: the norm over many tensors, and the tensors scaled where it is above a bound.  Two passes, each a few launches (one per
// CLIP_TENSORS tensors, whose addresses travel as kernel arguments): sums of squares, one per block, and the scaled copies, in which every
// block adds those sums up for itself, in the same order.
#include "common.cuh"

namespace focus {

constexpr int CLIP_TENSORS = 100;       // of a launch: 4 KB of arguments hold them
constexpr int CLIP_BLOCKS = 592;        // at most, of a launch: four per SM
constexpr int CLIP_CHUNK = 8192;        // numbers of a tensor that a block takes at a time

struct ClipTable {
    const void* src[CLIP_TENSORS];
    void* dst[CLIP_TENSORS];
    long long count[CLIP_TENSORS];
    int first[CLIP_TENSORS + 1];        // first chunk of each tensor
    uint32_t half[(CLIP_TENSORS + 31) / 32];      // which are bf16
    int tensors;
    bool add;                           // sums are added to those of the launch before
};

// the tensor of a chunk
__device__ __forceinline__ int clip_find(const ClipTable& t, int chunk) {
    int lo = 0, hi = t.tensors - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= chunk) lo = mid; else hi = mid - 1;
    }
    return lo;
}

__device__ __forceinline__ double block_sum(double x, double* s) {
    for (int off = 16; off; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0.0;
    for (int w = 0; w < 8; ++w) x += s[w];
    return x;
}

__global__ void __launch_bounds__(256) clip_squares_kernel(const __grid_constant__ ClipTable t, double* sums) {
    __shared__ double s[8];
    double x = 0.0;
    dep_wait();
    dep_trigger();
    for (int chunk = blockIdx.x; chunk < t.first[t.tensors]; chunk += gridDim.x) {
        const int at = clip_find(t, chunk);
        const long long from = (long long)(chunk - t.first[at]) * CLIP_CHUNK, to = min(t.count[at], from + CLIP_CHUNK);
        const bool half = t.half[at >> 5] >> (at & 31) & 1;
        for (long long e = from + threadIdx.x; e < to; e += 256) {
            const double v = half ? (double)__bfloat162float(((const __nv_bfloat16*)t.src[at])[e]) : (double)((const float*)t.src[at])[e];
            x += v * v;
        }
    }
    x = block_sum(x, s);
    if (threadIdx.x == 0) sums[blockIdx.x] = t.add ? sums[blockIdx.x] + x : x;
}

__global__ void __launch_bounds__(256) clip_scale_kernel(const __grid_constant__ ClipTable t, const double* sums, int blocks, double bound, float* norm_out) {
    __shared__ double s[8];
    dep_wait();
    dep_trigger();
    double x = 0.0;
    for (int e = threadIdx.x; e < blocks; e += 256) x += sums[e];
    const double norm = sqrt(block_sum(x, s));
    if (norm_out && blockIdx.x == 0 && threadIdx.x == 0) *norm_out = (float)norm;
    const float f = norm > bound && isfinite(norm) ? (float)(bound / norm) : 1.f;       // (what is not finite is left to the caller)
    for (int chunk = blockIdx.x; chunk < t.first[t.tensors]; chunk += gridDim.x) {
        const int at = clip_find(t, chunk);
        if (f == 1.f && t.src[at] == t.dst[at]) continue;
        const long long from = (long long)(chunk - t.first[at]) * CLIP_CHUNK, to = min(t.count[at], from + CLIP_CHUNK);
        const bool half = t.half[at >> 5] >> (at & 31) & 1;
        for (long long e = from + threadIdx.x; e < to; e += 256) {
            if (half) ((__nv_bfloat16*)t.dst[at])[e] = __float2bfloat16_rn(__bfloat162float(((const __nv_bfloat16*)t.src[at])[e]) * f);
            else ((float*)t.dst[at])[e] = ((const float*)t.src[at])[e] * f;
        }
    }
}

size_t grad_clip_workspace_bytes() { return CLIP_BLOCKS * sizeof(double); }

int launch_grad_clip(const focus_grad* grads, int count, double bound, float* norm_out, double* sums, cudaStream_t st) {
    int blocks = 1;
    for (int pass = 0; pass < 2; ++pass) {
        bool first = true;
        for (int at = 0; at < count || first; at += CLIP_TENSORS) {
            ClipTable t = {};
            t.tensors = count - at < CLIP_TENSORS ? count - at : CLIP_TENSORS;
            for (int i = 0; i < t.tensors; ++i) {
                const focus_grad& g = grads[at + i];
                t.src[i] = g.src;
                t.dst[i] = g.dst;
                t.count[i] = g.count;
                const long long next = t.first[i] + (g.count + CLIP_CHUNK - 1) / CLIP_CHUNK;
                if (next > 0x7fffffffll) return fail(FOCUS_ERR_UNSUPPORTED, "grad_clip: too many numbers");
                t.first[i + 1] = (int)next;
                if (g.dtype == FOCUS_GRAD_BF16) t.half[i >> 5] |= 1u << (i & 31);
            }
            t.add = !first;
            // (the first launch writes all the sums that there are)
            if (pass == 0 && first) blocks = CLIP_BLOCKS;
            const int own = pass == 0 ? blocks : (t.first[t.tensors] < CLIP_BLOCKS ? (t.first[t.tensors] > 0 ? t.first[t.tensors] : 1) : CLIP_BLOCKS);
            int rc = pass == 0 ? check_cuda(launch_dependent(clip_squares_kernel, dim3((unsigned)own), dim3(256), 0, st, t, sums), "squares launch")
                               : check_cuda(launch_dependent(clip_scale_kernel, dim3((unsigned)own), dim3(256), 0, st, t, (const double*)sums, blocks, bound,
                                                             first ? norm_out : nullptr), "scale launch");
            if (rc) return rc;
            first = false;
        }
    }
    return FOCUS_OK;
}

}  // namespace focus
