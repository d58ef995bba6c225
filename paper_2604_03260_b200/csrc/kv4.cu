// focus_kv4_append, focus_kv4_read, focus_kv4_copy_pages: what goes into the pages of the 4-bit cache, comes out of them, and moves
// between them.  HBM-bound by their bytes; the quantisation's instructions take as long as its reads, and the way back is two waves of
// dependent loads (8192 tokens of 8 KV heads of 128 in and out again: 19.8 us, 4.4 TB/s over both; 1024 pages of 76 KB moved: 25.9 us, 6.0 TB/s;
// one token of 32 sequences in and out: 3.9 us).
#include "kv4_common.cuh"
#include "f32x2.cuh"

namespace focus {

constexpr int KV4_THREADS = 256;

// D / 16 threads per (sequence, KV head, token), one per block of 16 dimensions: that block of the key and that of the value, so that
// what is looked up and worked out about the token (some 70 instructions) is for 32 numbers.
template <int D> struct Kv4Row {
    static constexpr int TPR = D / 16;                       // threads per row
    static constexpr int ROWS = KV4_THREADS / TPR;           // rows of a CTA
};

// sequence, head and token of a row
struct Kv4At {
    uint32_t b, h, t;
};
struct Kv4Rows {
    uint32_t rows;
    int n, Hkv;
    FixedDiv by_n, by_heads;
};
__device__ __forceinline__ Kv4At kv4_at(uint32_t row, const Kv4Rows& r) {
    Kv4At x;
    const uint32_t bh = r.by_n(row);
    x.t = row - bh * r.n;
    x.b = r.by_heads(bh);
    x.h = bh - x.b * r.Hkv;
    return x;
}

__device__ __forceinline__ uint32_t kv4_max2(uint32_t a, uint32_t b) { return __vmaxu2(a, b); }

// a / s, to the nearest: r is about 1 / s.  The residual of the first product is exact in a fused multiply-add, so a quotient that is an
// fp32 number comes out as itself.
__device__ __forceinline__ float kv4_quotient(float a, float s, float r) {
    const float y = a * r;
    return fmaf(fmaf(-y, s, a), r, y);
}
// two of them at once; `ns` is -s twice
__device__ __forceinline__ float2 kv4_quotient2(F2 a, F2 ns, F2 r) {
    const F2 y = f2_mul(a, r);
    return f2_get(f2_fma(f2_fma(y, ns, a), r, y));
}

// x (16 numbers of a block) -> codes and scale, with `gs` the power of two on top and `inv_gs` its inverse.  s = amax / 6 rounded to e4m3, code =
// x / s rounded to e2m1, both to nearest with ties to even.  A bf16 number has 8 significant bits and a scale 4, so a quotient that is
// not a tie is at least 1 / (60 * 256) of it away from one and no rounding of an fp32 quotient can push it across; a tie comes out exact.
// 150 instructions for a block, where IEEE divisions, limits and tests number by number took 384 (20.7 us for 8192 tokens of 8 heads
// of 128): the maximum and the test for infinities and NaN go over the bits, two numbers at once.
__device__ __forceinline__ uint2 kv4_quantise(const uint4 (&raw)[2], float gs, float inv_gs, uint32_t& scale_code, bool& bad) {
    uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    uint32_t m = w[0] & 0x7fff7fffu;
#pragma unroll
    for (int i = 1; i < 8; ++i) m = kv4_max2(m, w[i] & 0x7fff7fffu);
    m = max(m & 0xffffu, m >> 16);                           // the largest magnitude, as bf16 bits
    bad = m >= 0x7f80u;
    const float amax = __uint_as_float(m << 16) * inv_gs;
    scale_code = kv4_scale_code(kv4_quotient(fminf(amax, 4096.f), 6.f, 1.f / 6.f));        // (beyond 6 * 448 it is 448)
    const float s = __half2float(__ushort_as_half((unsigned short)(kv4_scales(scale_code) & 0xffffu))) * gs;
    const float r = s > 0.f ? __fdividef(1.f, s) : 0.f;      // a block whose scale is 0 has codes 0
    if (amax > 4096.f) {                                     // far beyond the largest code: limited, so that the quotients stay finite
        const float top = 4096.f * gs;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = fminf(fmaxf(__uint_as_float(w[i] << 16), -top), top), b = fminf(fmaxf(__uint_as_float(w[i] & 0xffff0000u), -top), top);
            w[i] = __float_as_uint(a) >> 16 | (__float_as_uint(b) & 0xffff0000u);
        }
    }
    const F2 ns2 = f2(-s, -s), r2 = f2(r, r);
    uint32_t c[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float2 y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            y[i] = kv4_quotient2(f2(__uint_as_float(w[4 * h + i] << 16), __uint_as_float(w[4 * h + i] & 0xffff0000u)), ns2, r2);
        c[h] = kv4_code8(y);
    }
    return make_uint2(c[0], c[1]);
}

// A token whose key or value holds an infinity or a NaN is stored with NaN scales throughout: it reads back as NaN, and a query that
// attends it becomes NaN as it would with the numbers themselves; one that does not is untouched.
// A row's numbers are on their way while its length and page are looked up (one that turns out not to be written, of a padded batch, has
// been read in vain).
template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_append_kernel(const Kv4View c, const __nv_bfloat16* k, int64_t k_sb, int64_t k_sh, int64_t k_sn, const __nv_bfloat16* v, int64_t v_sb,
                  int64_t v_sh, int64_t v_sn, const uint32_t* mk, const int32_t* counts, const Kv4Rows all, int32_t* status) {
    using R = Kv4Row<D>;
    const int j = threadIdx.x % R::TPR, P = 1 << c.lgP;
    const uint32_t row = blockIdx.x * R::ROWS + threadIdx.x / R::TPR;
    const bool there = row < all.rows;
    const Kv4At at = kv4_at(there ? row : 0u, all);
    dep_wait();
    dep_trigger();
    const uint4* ks = reinterpret_cast<const uint4*>(k + at.b * k_sb + at.h * k_sh + at.t * k_sn + j * 16);
    const uint4* vs = reinterpret_cast<const uint4*>(v + at.b * v_sb + at.h * v_sh + at.t * v_sn + j * 16);
    const uint4 kr[2] = {ks[0], ks[1]}, vr[2] = {vs[0], vs[1]};
    const int len = dep_load(c.lens + at.b), cnt = counts ? dep_load(counts + at.b) : all.n;
    const uint32_t mask = j == 0 ? dep_load(mk + (there ? row : 0u)) : 0u;
    const bool fits = cnt >= 0 && cnt <= all.n && len >= cnt && len <= c.max_pages * (long long)P;
    if (!fits && there && j == 0) kv4_report(status, KV4_BAD_LENGTH, at.b, len, cnt);
    const int pos = len - cnt + (int)at.t;
    unsigned char* page = nullptr;
    if (there && fits && (int)at.t < cnt) {
        const int pg = dep_load(c.table + (size_t)at.b * c.max_pages + (pos >> c.lgP));
        if (pg >= 0 && pg < c.num_pages) page = c.pages + (size_t)pg * c.page_bytes;
        else if (j == 0) kv4_report(status, KV4_BAD_PAGE, at.b, pos >> c.lgP, pg);
    }
    uint32_t sk, sv;
    bool bad_k, bad_v;
    uint2 ck = kv4_quantise(kr, c.k_scale, 1.f / c.k_scale, sk, bad_k), cv = kv4_quantise(vr, c.v_scale, 1.f / c.v_scale, sv, bad_v);
    const uint32_t group = ((1u << R::TPR) - 1u) << ((threadIdx.x & 31) / R::TPR * R::TPR);
    if (__ballot_sync(0xffffffffu, bad_k || bad_v) & group) { ck = cv = make_uint2(0, 0); sk = sv = 0x7f; }
    if (!page) return;
    const uint32_t slot = (at.h << c.lgP) + (pos & (P - 1));
    unsigned char* codes = page + (size_t)slot * D + j * 8;
    *reinterpret_cast<uint2*>(codes) = ck;
    *reinterpret_cast<uint2*>(codes + D / 2) = cv;
    unsigned char* scales = page + c.scale_off + (size_t)slot * (D / 8) + j;
    scales[0] = (unsigned char)sk;
    scales[D / 16] = (unsigned char)sv;
    if (j == 0) *reinterpret_cast<uint32_t*>(page + c.mask_off + (size_t)slot * 4) = mask;
}

// a block's codes and scale as 16 bf16 numbers (exact)
__device__ __forceinline__ void kv4_expand(uint2 code, uint32_t sc, float gs, uint4* dst) {
    const float s = __half2float(__ushort_as_half((unsigned short)(kv4_scales(sc) & 0xffffu))) * gs;
    const F2 s2 = f2(s, s);
    uint32_t out[8];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t f[4];
        kv4_unpack8(w ? code.y : code.x, f);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&f[e]));
            const float2 z = f2_get(f2_mul(f2(y.x, y.y), s2));
            const __nv_bfloat162 b2 = __floats2bfloat162_rn(z.x, z.y);
            out[4 * w + e] = *reinterpret_cast<const uint32_t*>(&b2);
        }
    }
    dst[0] = make_uint4(out[0], out[1], out[2], out[3]);
    dst[1] = make_uint4(out[4], out[5], out[6], out[7]);
}

template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_read_kernel(const Kv4View c, const int32_t* first, __nv_bfloat16* k, int64_t k_sb, int64_t k_sh, int64_t k_sn, __nv_bfloat16* v,
                int64_t v_sb, int64_t v_sh, int64_t v_sn, uint32_t* mk, const Kv4Rows all, int32_t* status) {
    using R = Kv4Row<D>;
    const int j = threadIdx.x % R::TPR, P = 1 << c.lgP;
    const uint32_t row = blockIdx.x * R::ROWS + threadIdx.x / R::TPR;
    dep_wait();
    dep_trigger();
    if (row >= all.rows) return;
    const Kv4At at = kv4_at(row, all);
    // length and page at once
    const int from = first ? dep_load(first + at.b) : 0, len = dep_load(c.lens + at.b);
    const long long pos = (long long)from + at.t, most = c.max_pages * (long long)P;
    const int pg = from >= 0 && pos < most ? dep_load(c.table + (size_t)at.b * c.max_pages + (int)(pos >> c.lgP)) : -1;
    if (from < 0 || len < 0 || len > most) {
        if (j == 0) kv4_report(status, KV4_BAD_LENGTH, at.b, len, from);
        return;
    }
    if (pos >= len) return;                                  // rows behind the last token stay as they are
    if (pg < 0 || pg >= c.num_pages) {
        if (j == 0) kv4_report(status, KV4_BAD_PAGE, at.b, (int)(pos >> c.lgP), pg);
        return;
    }
    const unsigned char* page = c.pages + (size_t)pg * c.page_bytes;
    const uint32_t slot = (at.h << c.lgP) + ((uint32_t)pos & (P - 1));
    const unsigned char *codes = page + (size_t)slot * D + j * 8, *scales = page + c.scale_off + (size_t)slot * (D / 8) + j;
    const uint2 ck = *reinterpret_cast<const uint2*>(codes), cv = *reinterpret_cast<const uint2*>(codes + D / 2);
    const uint32_t sk = scales[0], sv = scales[D / 16];
    if (j == 0 && mk) mk[row] = *reinterpret_cast<const uint32_t*>(page + c.mask_off + (size_t)slot * 4);
    kv4_expand(ck, sk, c.k_scale, reinterpret_cast<uint4*>(k + at.b * k_sb + at.h * k_sh + at.t * k_sn + j * 16));
    kv4_expand(cv, sv, c.v_scale, reinterpret_cast<uint4*>(v + at.b * v_sb + at.h * v_sh + at.t * v_sn + j * 16));
}

// Pages src[i] -> dst[i], 16 KB of a page per CTA, four 16-byte pieces per thread under way.
constexpr int KV4_COPY_UNROLL = 4;
constexpr int KV4_COPY_CHUNK = KV4_THREADS * KV4_COPY_UNROLL;        // 16-byte pieces per CTA
__global__ void __launch_bounds__(KV4_THREADS)
kv4_copy_kernel(unsigned char* pages, size_t page_bytes, int num_pages, const int32_t* src, const int32_t* dst, uint32_t chunks, int32_t* status) {
    const uint32_t pair = blockIdx.x / chunks, chunk = blockIdx.x - pair * chunks;
    dep_wait();
    dep_trigger();
    const int from = dep_load(src + pair), to = dep_load(dst + pair);
    if (from < 0 || from >= num_pages || to < 0 || to >= num_pages) {
        if (chunk == 0 && threadIdx.x == 0) kv4_report(status, KV4_BAD_PAIR, pair, from, to);
        return;
    }
    if (from == to) return;
    const uint4* a = reinterpret_cast<const uint4*>(pages + (size_t)from * page_bytes);
    uint4* z = reinterpret_cast<uint4*>(pages + (size_t)to * page_bytes);
    const size_t count = page_bytes / 16, at = (size_t)chunk * KV4_COPY_CHUNK + threadIdx.x;
    uint4 x[KV4_COPY_UNROLL];
#pragma unroll
    for (int i = 0; i < KV4_COPY_UNROLL; ++i)
        if (at + i * KV4_THREADS < count) x[i] = a[at + i * KV4_THREADS];
#pragma unroll
    for (int i = 0; i < KV4_COPY_UNROLL; ++i)
        if (at + i * KV4_THREADS < count) z[at + i * KV4_THREADS] = x[i];
}

int kv4_rows_check(const focus_shape* s) {
    const long long r = (long long)s->batch * s->Hkv * s->n;
    return r >= (1ll << 31) ? fail(FOCUS_ERR_UNSUPPORTED, "kv4: batch * Hkv * n (%lld) is too large for one call", r) : FOCUS_OK;
}

static long long copy_chunks(const Kv4View& c) { return ((long long)(c.page_bytes / 16) + KV4_COPY_CHUNK - 1) / KV4_COPY_CHUNK; }
int kv4_copy_check(const Kv4View& c, int count) {
    return copy_chunks(c) * count >= (1ll << 31) ? fail(FOCUS_ERR_UNSUPPORTED, "kv4: %d pages of %zu bytes are too much for one call", count, c.page_bytes) : FOCUS_OK;
}

static Kv4Rows rows_of(const focus_shape* s) {
    Kv4Rows rows;
    rows.rows = (uint32_t)((long long)s->batch * s->Hkv * s->n);
    rows.n = s->n;
    rows.Hkv = s->Hkv;
    rows.by_n = fixed_div((uint32_t)s->n);
    rows.by_heads = fixed_div((uint32_t)s->Hkv);
    return rows;
}

template <int D>
static int append_d(const focus_shape* s, const Kv4View& c, const focus_tensor& k, const focus_tensor& v, const uint32_t* mk, const int32_t* counts,
                    int32_t* status, cudaStream_t st) {
    const Kv4Rows rows = rows_of(s);
    const uint32_t per = Kv4Row<D>::ROWS;
    return check_cuda(launch_dependent(kv4_append_kernel<D>, dim3((rows.rows + per - 1) / per), dim3(KV4_THREADS), 0, st, c,
                                       reinterpret_cast<const __nv_bfloat16*>(k.ptr), k.stride_b, k.stride_h, k.stride_n,
                                       reinterpret_cast<const __nv_bfloat16*>(v.ptr), v.stride_b, v.stride_h, v.stride_n, mk, counts, rows, status),
                      "kv4 append kernel launch");
}

template <int D>
static int read_d(const focus_shape* s, const Kv4View& c, const int32_t* first, const focus_tensor& k, const focus_tensor& v, uint32_t* mk,
                  int32_t* status, cudaStream_t st) {
    const Kv4Rows rows = rows_of(s);
    const uint32_t per = Kv4Row<D>::ROWS;
    return check_cuda(launch_dependent(kv4_read_kernel<D>, dim3((rows.rows + per - 1) / per), dim3(KV4_THREADS), 0, st, c, first,
                                       reinterpret_cast<__nv_bfloat16*>(k.ptr), k.stride_b, k.stride_h, k.stride_n,
                                       reinterpret_cast<__nv_bfloat16*>(v.ptr), v.stride_b, v.stride_h, v.stride_n, mk, rows, status),
                      "kv4 read kernel launch");
}

int launch_kv4_append(const focus_shape* s, const Kv4View& c, const focus_tensor& k, const focus_tensor& v, const uint32_t* mk, const int32_t* counts,
                      int32_t* status, cudaStream_t st) {
    switch (s->D) {
        case 64: return append_d<64>(s, c, k, v, mk, counts, status, st);
        case 128: return append_d<128>(s, c, k, v, mk, counts, status, st);
        default: return append_d<256>(s, c, k, v, mk, counts, status, st);
    }
}

int launch_kv4_read(const focus_shape* s, const Kv4View& c, const int32_t* first, const focus_tensor& k, const focus_tensor& v, uint32_t* mk,
                    int32_t* status, cudaStream_t st) {
    switch (s->D) {
        case 64: return read_d<64>(s, c, first, k, v, mk, status, st);
        case 128: return read_d<128>(s, c, first, k, v, mk, status, st);
        default: return read_d<256>(s, c, first, k, v, mk, status, st);
    }
}

int launch_kv4_copy(const Kv4View& c, const int32_t* src, const int32_t* dst, int count, int32_t* status, cudaStream_t st) {
    const long long chunks = copy_chunks(c);
    return check_cuda(launch_dependent(kv4_copy_kernel, dim3((unsigned)(chunks * count)), dim3(KV4_THREADS), 0, st, c.pages, c.page_bytes, c.num_pages,
                                       src, dst, (uint32_t)chunks, status), "kv4 copy kernel launch");
}

}  // namespace focus
