// The 4-bit cache: layout of a page, and the conversions between its codes and 16-bit numbers.
//
// A page holds P tokens (a power of two, 16 to 256) of all KV heads of a layer, in three parts:
//   [Hkv][P] rows of D bytes    the codes of the key (D / 2 bytes), then of the value; two dimensions a byte, the even one in the low bits
//   [Hkv][P] rows of D / 8 bytes  the scales of the key's blocks of 16 dimensions, then of the value's
//   [Hkv][P] uint32             the key's group mask
// so that a token that some query attends costs one aligned row of codes and one of scales, and one that none attends costs its mask.
// A code is a sign and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (e2m1); a scale is an e4m3 number.  Their product has at most six significant
// bits: exact in fp16 and in bf16.
#pragma once

#include "common.cuh"

#include <cuda_fp16.h>

namespace focus {

struct Kv4View {
    unsigned char* pages;
    const int32_t* table;
    const int32_t* lens;
    size_t page_bytes;
    uint32_t scale_off, mask_off;        // of the second and third part of a page
    int num_pages, max_pages, lgP, Hkv;
    float k_scale, v_scale;
};

inline size_t kv4_page_bytes(int Hkv, int D, int P) { return (size_t)Hkv * P * (D + D / 8 + 4); }

// error word of a call (dev_status of the entry points): the first thread that finds something wrong says what
constexpr int KV4_BAD_PAGE = 1, KV4_BAD_LENGTH = 2, KV4_BAD_PAIR = 3;

#ifdef __CUDACC__
__device__ __forceinline__ void kv4_report(int32_t* status, int code, int a, int b, int c) {
    if (status && atomicCAS(status, 0, code) == 0) { status[1] = a; status[2] = b; status[3] = c; }
}

// eight codes of a word as four pairs of fp16: dimensions (0, 1), (2, 3), (4, 5), (6, 7)
__device__ __forceinline__ void kv4_unpack8(uint32_t w, uint32_t (&r)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tmov.b32 {b0, b1, b2, b3}, %4;\n\tcvt.rn.f16x2.e2m1x2 %0, b0;\n\tcvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\tcvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(w));
}
// two scales (the first in the low byte) as a pair of fp16
__device__ __forceinline__ uint32_t kv4_scales(uint32_t two) {
    uint32_t r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
    return r;
}
__device__ __forceinline__ uint32_t kv4_mul2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// eight numbers as codes of a word, the first in the low bits; to nearest, a tie to the even code, beyond 6 to 6
__device__ __forceinline__ uint32_t kv4_code8(const float2 (&y)[4]) {
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\tcvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\tmov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r) : "f"(y[0].x), "f"(y[0].y), "f"(y[1].x), "f"(y[1].y), "f"(y[2].x), "f"(y[2].y), "f"(y[3].x), "f"(y[3].y));
    return r;
}
__device__ __forceinline__ uint32_t kv4_scale_code(float s) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.f), "f"(s));
    return r;
}
#endif

// what the kernels of kv4.cu and kv4_decode.cu take, beyond the checks of a shape and a cache; their launchers
int kv4_rows_check(const focus_shape* s);
int kv4_copy_check(const Kv4View& c, int count);
int kv4_decode_check(const focus_shape* s, const Kv4View& c);
int launch_kv4_append(const focus_shape* s, const Kv4View& c, const focus_tensor& k, const focus_tensor& v, const uint32_t* mk,
                      const int32_t* counts, int32_t* status, cudaStream_t st);
int launch_kv4_read(const focus_shape* s, const Kv4View& c, const int32_t* first, const focus_tensor& k, const focus_tensor& v,
                    uint32_t* mk, int32_t* status, cudaStream_t st);
int launch_kv4_copy(const Kv4View& c, const int32_t* src, const int32_t* dst, int count, int32_t* status, cudaStream_t st);
size_t kv4_decode_workspace_bytes(const focus_shape* s);
int launch_kv4_decode(const focus_shape* s, const Kv4View& c, const focus_tensor& q, const uint32_t* mq_new, const focus_tensor& o,
                      float* lse, void* ws, float scale, int32_t* status, cudaStream_t st);

}  // namespace focus
