// focus_kv4_append, focus_kv4_read, focus_kv4_copy_pages: what goes into the pages of the 4-bit cache, comes out of them, and moves
// between them.  All three are HBM-bound.
#include "kv4_common.cuh"

namespace focus {

constexpr int KV4_THREADS = 256;

// D / 8 threads per (sequence, KV head, token): one per block of 16 dimensions, the key's blocks first, then the value's.
template <int D> struct Kv4Row {
    static constexpr int TPR = D / 8;                        // threads per row
    static constexpr int BLOCKS = D / 16;                    // blocks of the key (and of the value)
    static constexpr int ROWS = KV4_THREADS / TPR;           // rows per pass of a CTA
};

// sequence, head and token of a row
struct Kv4At {
    uint32_t b, h, t;
};
__device__ __forceinline__ Kv4At kv4_at(uint32_t row, int n, int Hkv) {
    Kv4At x;
    const uint32_t bh = row / (uint32_t)n;
    x.t = row - bh * n;
    x.b = bh / (uint32_t)Hkv;
    x.h = bh - x.b * Hkv;
    return x;
}

// x (16 numbers of a block) -> codes and scale.  s = amax / 6 rounded to e4m3, code = x / s rounded to e2m1, both to nearest with ties to
// even.  A bf16 number has 8 significant bits and a scale 4, so a quotient that is not a tie is at least 1 / (60 * 256) of it away from
// one and no rounding of an fp32 division can push it across; a tie has to come out exact, which y + (x - y s) r does (the residual is
// exact in a fused multiply-add).
__device__ __forceinline__ uint2 kv4_quantise(const uint4 (&raw)[2], float inv_scale, uint32_t& scale_code, bool& bad) {
    float x[16];
    const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    float amax = 0.f;
    bad = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        bad |= (w[i] & 0x7f80u) == 0x7f80u || (w[i] & 0x7f800000u) == 0x7f800000u;
        // beyond 6 * 448 everything has the largest code and scale; the limit keeps the quotients finite
        x[2 * i] = fminf(fmaxf(__uint_as_float(w[i] << 16) * inv_scale, -4096.f), 4096.f);
        x[2 * i + 1] = fminf(fmaxf(__uint_as_float(w[i] & 0xffff0000u) * inv_scale, -4096.f), 4096.f);
        amax = fmaxf(amax, fmaxf(fabsf(x[2 * i]), fabsf(x[2 * i + 1])));
    }
    scale_code = kv4_scale_code(__fdiv_rn(amax, 6.f));
    const float s = __half2float(__ushort_as_half((unsigned short)(kv4_scales(scale_code) & 0xffffu)));
    const float r = s > 0.f ? __fdiv_rn(1.f, s) : 0.f;       // a block whose scale is 0 has codes 0
    uint32_t c[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float y[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float a = x[2 * i + e], y0 = a * r;
            y[e] = fmaf(fmaf(-y0, s, a), r, y0);
        }
        c[i >> 2] |= kv4_code2(y[0], y[1]) << (8 * (i & 3));
    }
    return make_uint2(c[0], c[1]);
}

// A token whose key or value holds an infinity or a NaN is stored with NaN scales throughout: it reads back as NaN, and a query that
// attends it becomes NaN as it would with the numbers themselves; one that does not is untouched.
// AHEAD rows a thread; their numbers are on their way while length and page are looked up (a row that turns out not to be written, of a
// padded batch, has been read in vain).
template <int D, int AHEAD>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_append_kernel(const Kv4View c, const __nv_bfloat16* k, int64_t k_sb, int64_t k_sh, int64_t k_sn, const __nv_bfloat16* v, int64_t v_sb,
                  int64_t v_sh, int64_t v_sn, const uint32_t* mk, const int32_t* counts, int n, uint32_t rows, int32_t* status) {
    using R = Kv4Row<D>;
    const int j = threadIdx.x % R::TPR, sub = threadIdx.x / R::TPR;
    const bool isv = j >= R::BLOCKS;
    const int blk = isv ? j - R::BLOCKS : j, P = 1 << c.lgP;
    const __nv_bfloat16* x = (isv ? v : k) + blk * 16;
    const int64_t sb = isv ? v_sb : k_sb, sh = isv ? v_sh : k_sh, sn = isv ? v_sn : k_sn;
    dep_wait();
    dep_trigger();
    uint4 raw[AHEAD][2];
    Kv4At at[AHEAD];
    int len[AHEAD], cnt[AHEAD];
    uint32_t mask[AHEAD];
    const uint32_t first = blockIdx.x * (AHEAD * R::ROWS) + sub;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const uint32_t row = first + i * R::ROWS;
        raw[i][0] = raw[i][1] = make_uint4(0, 0, 0, 0);
        cnt[i] = len[i] = 0;
        mask[i] = 0;
        if (row < rows) {
            at[i] = kv4_at(row, n, c.Hkv);
            const __nv_bfloat16* src = x + (size_t)at[i].b * sb + (size_t)at[i].h * sh + (size_t)at[i].t * sn;
            raw[i][0] = reinterpret_cast<const uint4*>(src)[0];
            raw[i][1] = reinterpret_cast<const uint4*>(src)[1];
            len[i] = dep_load(c.lens + at[i].b);
            cnt[i] = counts ? dep_load(counts + at[i].b) : n;
            if (j == 0) mask[i] = dep_load(mk + row);
        }
    }
    unsigned char* page[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        page[i] = nullptr;
        if (first + i * R::ROWS < rows) {
            const bool fits = cnt[i] >= 0 && cnt[i] <= n && len[i] >= cnt[i] && len[i] <= c.max_pages * (long long)P;
            if (!fits && j == 0) kv4_report(status, KV4_BAD_LENGTH, at[i].b, len[i], cnt[i]);
            if (fits && (int)at[i].t < cnt[i]) {
                const int pos = len[i] - cnt[i] + (int)at[i].t;
                const int pg = dep_load(c.table + (size_t)at[i].b * c.max_pages + (pos >> c.lgP));
                if (pg >= 0 && pg < c.num_pages) page[i] = c.pages + (size_t)pg * c.page_bytes;
                else if (j == 0) kv4_report(status, KV4_BAD_PAGE, at[i].b, pos >> c.lgP, pg);
            }
        }
    }
    const float inv_scale = 1.f / (isv ? c.v_scale : c.k_scale);       // a power of two: exact
    const int lane = threadIdx.x & 31;
    const uint32_t group = (R::TPR == 32 ? 0xffffffffu : ((1u << R::TPR) - 1u)) << (lane / R::TPR * R::TPR);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        uint32_t sc;
        bool bad;
        uint2 code = kv4_quantise(raw[i], inv_scale, sc, bad);
        if (__ballot_sync(0xffffffffu, bad) & group) { code = make_uint2(0, 0); sc = 0x7f; }
        if (!page[i]) continue;
        const uint32_t slot = (at[i].h << c.lgP) + ((len[i] - cnt[i] + (int)at[i].t) & (P - 1));
        *reinterpret_cast<uint2*>(page[i] + (size_t)slot * D + j * 8) = code;      // (the value's codes follow the key's)
        page[i][c.scale_off + (size_t)slot * (D / 8) + j] = (unsigned char)sc;
        if (j == 0) *reinterpret_cast<uint32_t*>(page[i] + c.mask_off + (size_t)slot * 4) = mask[i];
    }
}

template <int D, int AHEAD>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_read_kernel(const Kv4View c, const int32_t* first, __nv_bfloat16* k, int64_t k_sb, int64_t k_sh, int64_t k_sn, __nv_bfloat16* v,
                int64_t v_sb, int64_t v_sh, int64_t v_sn, uint32_t* mk, int n, uint32_t rows, int32_t* status) {
    using R = Kv4Row<D>;
    const int j = threadIdx.x % R::TPR, sub = threadIdx.x / R::TPR;
    const bool isv = j >= R::BLOCKS;
    const int blk = isv ? j - R::BLOCKS : j, P = 1 << c.lgP;
    __nv_bfloat16* x = (isv ? v : k) + blk * 16;
    const int64_t sb = isv ? v_sb : k_sb, sh = isv ? v_sh : k_sh, sn = isv ? v_sn : k_sn;
    dep_wait();
    dep_trigger();
    Kv4At at[AHEAD];
    int len[AHEAD], pg[AHEAD];
    long long pos[AHEAD];
    const uint32_t row0 = blockIdx.x * (AHEAD * R::ROWS) + sub;
    // lengths and pages at once
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        const uint32_t row = row0 + i * R::ROWS;
        len[i] = -1;
        pg[i] = -1;
        pos[i] = 0;
        if (row < rows) {
            at[i] = kv4_at(row, n, c.Hkv);
            const int from = first ? dep_load(first + at[i].b) : 0;
            len[i] = dep_load(c.lens + at[i].b);
            pos[i] = (long long)from + at[i].t;
            if (from >= 0 && pos[i] < c.max_pages * (long long)P) pg[i] = dep_load(c.table + (size_t)at[i].b * c.max_pages + (pos[i] >> c.lgP));
            if ((from < 0 || len[i] < 0 || len[i] > c.max_pages * (long long)P) && j == 0) kv4_report(status, KV4_BAD_LENGTH, at[i].b, len[i], from);
            if (from < 0 || len[i] > c.max_pages * (long long)P) len[i] = -1;
        }
    }
    uint2 code[AHEAD];
    uint32_t sc[AHEAD], mask[AHEAD];
    bool live[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        live[i] = pos[i] < len[i];                           // rows behind the last token stay as they are
        if (live[i] && (pg[i] < 0 || pg[i] >= c.num_pages)) {
            if (j == 0) kv4_report(status, KV4_BAD_PAGE, at[i].b, (int)(pos[i] >> c.lgP), pg[i]);
            live[i] = false;
        }
        if (live[i]) {
            const unsigned char* page = c.pages + (size_t)pg[i] * c.page_bytes;
            const uint32_t slot = (at[i].h << c.lgP) + (uint32_t)(pos[i] & (P - 1));
            code[i] = *reinterpret_cast<const uint2*>(page + (size_t)slot * D + j * 8);
            sc[i] = page[c.scale_off + (size_t)slot * (D / 8) + j];
            if (j == 0 && mk) mask[i] = *reinterpret_cast<const uint32_t*>(page + c.mask_off + (size_t)slot * 4);
        }
    }
    const float scale = isv ? c.v_scale : c.k_scale;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
        if (!live[i]) continue;
        const float s = __half2float(__ushort_as_half((unsigned short)(kv4_scales(sc[i]) & 0xffffu))) * scale;
        uint32_t out[8];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t f[4];
            kv4_unpack8(w ? code[i].y : code[i].x, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 y = __half22float2(*reinterpret_cast<const __half2*>(&f[e]));
                const __nv_bfloat162 z = __floats2bfloat162_rn(y.x * s, y.y * s);          // exact
                out[4 * w + e] = *reinterpret_cast<const uint32_t*>(&z);
            }
        }
        __nv_bfloat16* dst = x + (size_t)at[i].b * sb + (size_t)at[i].h * sh + (size_t)at[i].t * sn;
        reinterpret_cast<uint4*>(dst)[0] = make_uint4(out[0], out[1], out[2], out[3]);
        reinterpret_cast<uint4*>(dst)[1] = make_uint4(out[4], out[5], out[6], out[7]);
        if (j == 0 && mk) mk[row0 + i * R::ROWS] = mask[i];
    }
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

// two rows a thread where that leaves a CTA for every multiprocessor
constexpr int KV4_SMS = 148;
static int rows_of(const focus_shape* s, uint32_t& rows, bool& two) {
    const long long r = (long long)s->batch * s->Hkv * s->n;
    if (r >= (1ll << 31)) return fail(FOCUS_ERR_UNSUPPORTED, "kv4: batch * Hkv * n (%lld) is too large for one call", r);
    rows = (uint32_t)r;
    two = r >= 2ll * KV4_SMS * (KV4_THREADS / (s->D / 8));
    return FOCUS_OK;
}

template <int D>
static int append_d(const focus_shape* s, const Kv4View& c, const focus_tensor& k, const focus_tensor& v, const uint32_t* mk, const int32_t* counts,
                    int32_t* status, cudaStream_t st) {
    uint32_t rows;
    bool two;
    int rc = rows_of(s, rows, two);
    if (rc) return rc;
    const uint32_t per = Kv4Row<D>::ROWS * (two ? 2 : 1);
    return check_cuda(launch_dependent(two ? kv4_append_kernel<D, 2> : kv4_append_kernel<D, 1>, dim3((rows + per - 1) / per), dim3(KV4_THREADS), 0, st, c,
                                       reinterpret_cast<const __nv_bfloat16*>(k.ptr), k.stride_b, k.stride_h, k.stride_n,
                                       reinterpret_cast<const __nv_bfloat16*>(v.ptr), v.stride_b, v.stride_h, v.stride_n, mk, counts, s->n, rows, status),
                      "kv4 append kernel launch");
}

template <int D>
static int read_d(const focus_shape* s, const Kv4View& c, const int32_t* first, const focus_tensor& k, const focus_tensor& v, uint32_t* mk,
                  int32_t* status, cudaStream_t st) {
    uint32_t rows;
    bool two;
    int rc = rows_of(s, rows, two);
    if (rc) return rc;
    const uint32_t per = Kv4Row<D>::ROWS * (two ? 2 : 1);
    return check_cuda(launch_dependent(two ? kv4_read_kernel<D, 2> : kv4_read_kernel<D, 1>, dim3((rows + per - 1) / per), dim3(KV4_THREADS), 0, st, c,
                                       first, reinterpret_cast<__nv_bfloat16*>(k.ptr), k.stride_b, k.stride_h, k.stride_n,
                                       reinterpret_cast<__nv_bfloat16*>(v.ptr), v.stride_b, v.stride_h, v.stride_n, mk, s->n, rows, status),
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
    const long long chunks = ((long long)(c.page_bytes / 16) + KV4_COPY_CHUNK - 1) / KV4_COPY_CHUNK;
    if (chunks * count >= (1ll << 31)) return fail(FOCUS_ERR_UNSUPPORTED, "kv4: %d pages of %zu bytes are too much for one call", count, c.page_bytes);
    return check_cuda(launch_dependent(kv4_copy_kernel, dim3((unsigned)(chunks * count)), dim3(KV4_THREADS), 0, st, c.pages, c.page_bytes, c.num_pages,
                                       src, dst, (uint32_t)chunks, status), "kv4 copy kernel launch");
}

}  // namespace focus
