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
    static constexpr int AHEAD = 2;                          // rows per thread whose loads are under way together
};

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
// 8192 tokens of 8 heads of 128: 33.5 MB read, 9.7 MB written.
template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_append_kernel(const Kv4View c, const __nv_bfloat16* k, int64_t k_sb, int64_t k_sh, int64_t k_sn, const __nv_bfloat16* v, int64_t v_sb,
                  int64_t v_sh, int64_t v_sn, const uint32_t* mk, const int32_t* counts, int n, uint32_t rows, int32_t* status) {
    using R = Kv4Row<D>;
    const int j = threadIdx.x % R::TPR, sub = threadIdx.x / R::TPR;
    const bool isv = j >= R::BLOCKS;
    const int blk = isv ? j - R::BLOCKS : j;
    const int P = 1 << c.lgP;
    dep_wait();
    dep_trigger();
    uint4 raw[R::AHEAD][2];
    unsigned char* page[R::AHEAD];
    int slot[R::AHEAD];
    uint32_t head[R::AHEAD], row[R::AHEAD];
#pragma unroll
    for (int i = 0; i < R::AHEAD; ++i) {
        row[i] = (blockIdx.x * R::AHEAD + i) * R::ROWS + sub;
        page[i] = nullptr;
        slot[i] = 0;
        head[i] = 0;
        raw[i][0] = raw[i][1] = make_uint4(0, 0, 0, 0);
        if (row[i] < rows) {
            const uint32_t bh = row[i] / (uint32_t)n, t = row[i] - bh * n;
            const uint32_t b = bh / (uint32_t)c.Hkv, h = bh - b * c.Hkv;
            const int len = dep_load(c.lens + b), cnt = counts ? dep_load(counts + b) : n;
            const bool fits = cnt >= 0 && cnt <= n && len >= cnt && len <= c.max_pages * (long long)P;
            if (!fits && j == 0) kv4_report(status, KV4_BAD_LENGTH, b, len, cnt);
            if (fits && (int)t < cnt) {
                const int pos = len - cnt + (int)t;
                const int pg = dep_load(c.table + (size_t)b * c.max_pages + (pos >> c.lgP));
                if (pg >= 0 && pg < c.num_pages) {
                    page[i] = c.pages + (size_t)pg * c.page_bytes;
                    slot[i] = pos & (P - 1);
                    head[i] = h;
                    const __nv_bfloat16* src = isv ? v + (size_t)b * v_sb + (size_t)h * v_sh + (size_t)t * v_sn
                                                   : k + (size_t)b * k_sb + (size_t)h * k_sh + (size_t)t * k_sn;
                    raw[i][0] = reinterpret_cast<const uint4*>(src + blk * 16)[0];
                    raw[i][1] = reinterpret_cast<const uint4*>(src + blk * 16)[1];
                } else if (j == 0) {
                    kv4_report(status, KV4_BAD_PAGE, b, pos >> c.lgP, pg);
                }
            }
        }
    }
    const float inv_scale = 1.f / (isv ? c.v_scale : c.k_scale);       // a power of two: exact
    const int lane = threadIdx.x & 31;
    const uint32_t group = (R::TPR == 32 ? 0xffffffffu : ((1u << R::TPR) - 1u)) << (lane / R::TPR * R::TPR);
#pragma unroll
    for (int i = 0; i < R::AHEAD; ++i) {
        uint32_t sc;
        bool bad;
        uint2 code = kv4_quantise(raw[i], inv_scale, sc, bad);
        if (__ballot_sync(0xffffffffu, bad) & group) { code = make_uint2(0, 0); sc = 0x7f; }
        if (!page[i]) continue;
        const uint32_t at = (head[i] << c.lgP) + slot[i];
        *reinterpret_cast<uint2*>(page[i] + (size_t)at * D + j * 8) = code;        // (the value's codes follow the key's)
        page[i][c.scale_off + (size_t)at * (D / 8) + j] = (unsigned char)sc;
        if (j == 0) *reinterpret_cast<uint32_t*>(page[i] + c.mask_off + (size_t)at * 4) = dep_load(mk + row[i]);
    }
}

template <int D>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_read_kernel(const Kv4View c, const int32_t* first, __nv_bfloat16* k, int64_t k_sb, int64_t k_sh, int64_t k_sn, __nv_bfloat16* v,
                int64_t v_sb, int64_t v_sh, int64_t v_sn, uint32_t* mk, int n, uint32_t rows, int32_t* status) {
    using R = Kv4Row<D>;
    const int j = threadIdx.x % R::TPR, sub = threadIdx.x / R::TPR;
    const bool isv = j >= R::BLOCKS;
    const int blk = isv ? j - R::BLOCKS : j;
    const int P = 1 << c.lgP;
    dep_wait();
    dep_trigger();
    uint2 code[R::AHEAD];
    uint32_t sc[R::AHEAD], mask[R::AHEAD];
    bool live[R::AHEAD];
#pragma unroll
    for (int i = 0; i < R::AHEAD; ++i) {
        const uint32_t row = (blockIdx.x * R::AHEAD + i) * R::ROWS + sub;
        live[i] = false;
        if (row >= rows) continue;
        const uint32_t bh = row / (uint32_t)n, t = row - bh * n;
        const uint32_t b = bh / (uint32_t)c.Hkv, h = bh - b * c.Hkv;
        const int len = dep_load(c.lens + b), from = first ? dep_load(first + b) : 0;
        const bool fits = from >= 0 && len >= 0 && len <= c.max_pages * (long long)P;
        if (!fits && j == 0) kv4_report(status, KV4_BAD_LENGTH, b, len, from);
        const long long pos = (long long)from + t;
        if (!fits || pos >= len) continue;                   // rows behind the last token stay as they are
        const int pg = dep_load(c.table + (size_t)b * c.max_pages + (pos >> c.lgP));
        if (pg < 0 || pg >= c.num_pages) {
            if (j == 0) kv4_report(status, KV4_BAD_PAGE, b, (int)(pos >> c.lgP), pg);
            continue;
        }
        const unsigned char* page = c.pages + (size_t)pg * c.page_bytes;
        const uint32_t at = (h << c.lgP) + (uint32_t)(pos & (P - 1));
        live[i] = true;
        code[i] = *reinterpret_cast<const uint2*>(page + (size_t)at * D + j * 8);
        sc[i] = page[c.scale_off + (size_t)at * (D / 8) + j];
        if (j == 0 && mk) mask[i] = *reinterpret_cast<const uint32_t*>(page + c.mask_off + (size_t)at * 4);
    }
    const float scale = isv ? c.v_scale : c.k_scale;
#pragma unroll
    for (int i = 0; i < R::AHEAD; ++i) {
        if (!live[i]) continue;
        const uint32_t row = (blockIdx.x * R::AHEAD + i) * R::ROWS + sub;
        const uint32_t bh = row / (uint32_t)n, t = row - bh * n;
        const uint32_t b = bh / (uint32_t)c.Hkv, h = bh - b * c.Hkv;
        const float s = __half2float(__ushort_as_half((unsigned short)(kv4_scales(sc[i]) & 0xffffu))) * scale;
        uint32_t out[8];
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            uint32_t f[4];
            kv4_unpack8(w ? code[i].y : code[i].x, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&f[e]));
                const __nv_bfloat162 y = __floats2bfloat162_rn(x.x * s, x.y * s);          // exact
                out[4 * w + e] = *reinterpret_cast<const uint32_t*>(&y);
            }
        }
        __nv_bfloat16* dst = isv ? v + (size_t)b * v_sb + (size_t)h * v_sh + (size_t)t * v_sn
                                 : k + (size_t)b * k_sb + (size_t)h * k_sh + (size_t)t * k_sn;
        reinterpret_cast<uint4*>(dst + blk * 16)[0] = make_uint4(out[0], out[1], out[2], out[3]);
        reinterpret_cast<uint4*>(dst + blk * 16)[1] = make_uint4(out[4], out[5], out[6], out[7]);
        if (j == 0 && mk) mk[row] = mask[i];
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

static int rows_of(const focus_shape* s, int D, uint32_t& rows, uint32_t& blocks) {
    const long long r = (long long)s->batch * s->Hkv * s->n;
    if (r >= (1ll << 31)) return fail(FOCUS_ERR_UNSUPPORTED, "kv4: batch * Hkv * n (%lld) is too large for one call", r);
    const long long per = KV4_THREADS / (D / 8) * 2;
    rows = (uint32_t)r;
    blocks = (uint32_t)((r + per - 1) / per);
    return FOCUS_OK;
}

template <int D>
static int append_d(const focus_shape* s, const Kv4View& c, const focus_tensor& k, const focus_tensor& v, const uint32_t* mk, const int32_t* counts,
                    int32_t* status, cudaStream_t st) {
    uint32_t rows, blocks;
    int rc = rows_of(s, D, rows, blocks);
    if (rc) return rc;
    return check_cuda(launch_dependent(kv4_append_kernel<D>, dim3(blocks), dim3(KV4_THREADS), 0, st, c, reinterpret_cast<const __nv_bfloat16*>(k.ptr),
                                       k.stride_b, k.stride_h, k.stride_n, reinterpret_cast<const __nv_bfloat16*>(v.ptr), v.stride_b, v.stride_h,
                                       v.stride_n, mk, counts, s->n, rows, status), "kv4 append kernel launch");
}

template <int D>
static int read_d(const focus_shape* s, const Kv4View& c, const int32_t* first, const focus_tensor& k, const focus_tensor& v, uint32_t* mk,
                  int32_t* status, cudaStream_t st) {
    uint32_t rows, blocks;
    int rc = rows_of(s, D, rows, blocks);
    if (rc) return rc;
    return check_cuda(launch_dependent(kv4_read_kernel<D>, dim3(blocks), dim3(KV4_THREADS), 0, st, c, first, reinterpret_cast<__nv_bfloat16*>(k.ptr),
                                       k.stride_b, k.stride_h, k.stride_n, reinterpret_cast<__nv_bfloat16*>(v.ptr), v.stride_b, v.stride_h, v.stride_n,
                                       mk, s->n, rows, status), "kv4 read kernel launch");
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
