// focus_router_scores_bwd: the derivative of S = (h W_g) C^T.  With T = dS^T h (K vectors of d, summed over all tokens)
//     dC = T W_g      dW_g = T^T C      dh = dS F,  F = C W_g^T
// so the hidden states are read once and their gradient written once, and everything else is of size K d: bound by the memory, if the two
// products with K columns cost less.  On the fp32 pipe they do not (K = 8: as long as the memory, 166 us for 32768 x 4096 where that takes 83); on
// the tensor cores dS and F go in bf16 terms: T takes dS in three (24 bits, exact products with the hidden states), dh, which is rounded to bf16, dS
// and F in two each.  The tiles are too thin for a tcgen05 instruction's 128 rows and its tensor memory (K rows, or K deep), so mma.sync does.
//
// A block has a strip of columns and a run of tokens, a warp 64 columns of it (32 and 16 at K > 8 and > 16), and goes down its rows 32 at a time; the
// rows come by asynchronous copies through a ring of three to four such pieces in shared memory.  Measured with dh (device time, graph replay): 32768 x 4096,
// K = 8, d_g = 32: 108 us, of which some 96 for the pass over the tokens (5.6 TB/s) and the rest for adding the parts up; 1024 x 768, K = 4: 10.9 us, two
// launches and the chain of loads of each.  The same on the fp32 pipe, rows through a private ring: 175 and 16.4 us.
#include "common.cuh"

namespace focus {

constexpr int RB_THREADS = 128;
constexpr int RB_ROWS = 32;                 // tokens at a time
constexpr int RB_TOTAL_COLS = 32;           // columns of a block that adds the parts up
constexpr int RB_TOTAL_DG = 32;             // and of those of W_g and C
constexpr int RB_LAST = 256;                // up to K d_g of this, the last block of the totals adds dC's parts up
constexpr int RB_FOLD = 512;                // up to K d_g of this, a block works out its columns of F itself

// F[g][e] = sum_j W_g[e][j] C[g][j]: a block 32 rows of W_g, 64 of their numbers at a time, a thread a row and every eighth group
// (a thread a row and group, rows read from global memory: 8000 x 4096 with K = 32, d_g = 128 took 426 us in all)
__global__ void __launch_bounds__(256) router_fold_kernel(const float* Wg, const float* C, int d, int dg, int K, float* F) {
    __shared__ float ws[32][65], cs[32][64];
    const int t = threadIdx.x, e0 = blockIdx.x * 32, e = t % 32, q = t / 32;
    dep_wait();
    dep_trigger();
    float s[4] = {};
    for (int j0 = 0; j0 < dg; j0 += 64) {
        const int w = min(64, dg - j0);
        for (int i = t; i < 32 * 64; i += 256) {
            const int r = i / 64, j = i % 64;
            ws[r][j] = e0 + r < d && j < w ? Wg[(size_t)(e0 + r) * dg + j0 + j] : 0.f;
            cs[r][j] = r < K && j < w ? C[(size_t)r * dg + j0 + j] : 0.f;
        }
        __syncthreads();
#pragma unroll 16
        for (int j = 0; j < 64; ++j) {
#pragma unroll
            for (int v = 0; v < 4; ++v) s[v] = fmaf(ws[e][j], cs[q + 8 * v][j], s[v]);
        }
        __syncthreads();
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
        if (q + 8 * v < K && e0 + e < d) F[(size_t)(q + 8 * v) * d + e0 + e] = s[v];
}

// dC = sum of the blocks' parts, where they are too many numbers for the last block to add up: a block 32 of them, a thread every eighth part
__global__ void __launch_bounds__(256) router_dc_kernel(const float* dC_part, int parts, int count, float* dC) {
    __shared__ float eighth[8][32];
    const int c = threadIdx.x % 32, q = threadIdx.x / 32, i = blockIdx.x * 32 + c;
    dep_wait();
    dep_trigger();
    float s = 0.f;
    if (i < count) {
#pragma unroll 16
        for (int z = q; z < parts; z += 8) s += dC_part[(size_t)z * count + i];
    }
    eighth[q][c] = s;
    __syncthreads();
    if (q || i >= count) return;
    for (int x = 1; x < 8; ++x) s += eighth[x][c];
    dC[i] = s;
}

template <int LD> struct RouterCfg {
    static constexpr int G8 = LD <= 8 ? 1 : LD / 8;              // blocks of 8 groups
    static constexpr int CW = 64 / G8, COLS = 4 * CW;            // columns of a warp, of a block
    static constexpr int NT = CW >= 32 ? 4 : 2;                  // 8-column tiles of dh whose columns are dealt out so that a lane has 2 NT in a row
    static constexpr int STAGES = G8 == 1 ? 3 : 4;
    static constexpr int CHUNKS = COLS / 8;                      // 16-byte pieces of a row
    static constexpr int PER = RB_ROWS * LD / RB_THREADS;        // numbers of dS of a thread and piece
    static constexpr uint32_t STAGE_BYTES = RB_ROWS * COLS * 2;
    static constexpr int TPITCH = 40, APITCH = 24;               // bf16 numbers between rows of the two layouts of dS: no bank conflicts
    static constexpr uint32_t T_BYTES = 3 * 8 * G8 * TPITCH * 2, A_BYTES = RB_ROWS * APITCH * 2 * G8;
    static constexpr uint32_t OFF_T = STAGES * STAGE_BYTES, OFF_A = OFF_T + 2 * T_BYTES, OFF_F = OFF_A + 2 * A_BYTES, OFF_C = OFF_F + 8 * G8 * COLS * 4;
    static constexpr uint32_t SMEM = OFF_C + RB_FOLD * 4;
};
constexpr int rb_cols(int LD) { return LD <= 8 ? 256 : 2048 / LD; }
static_assert(rb_cols(8) == RouterCfg<8>::COLS && rb_cols(16) == RouterCfg<16>::COLS && rb_cols(32) == RouterCfg<32>::COLS, "columns of a block");

__device__ __forceinline__ void rb_copy(uint32_t dst, const void* src, bool in) {        // zeros where not `in`
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void rb_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// F: the folded projection, or nullptr: worked out here
template <int LD>
__global__ void __launch_bounds__(RB_THREADS)
router_bwd_kernel(const __nv_bfloat16* h, int64_t h_sb, int64_t h_sn, const float* dS, const float* F, const float* Wg, const float* C, int dg, int n, int runs, int run,
                  int d, int K, __nv_bfloat16* dh, int64_t d_sb, int64_t d_sn, float* part, unsigned* done) {
    using R = RouterCfg<LD>;
    constexpr int G8 = R::G8, CW = R::CW, NT = R::NT;
    extern __shared__ __align__(128) unsigned char sm[];
    const uint32_t base = (uint32_t)__cvta_generic_to_shared(sm);
    __nv_bfloat16* const dsT = reinterpret_cast<__nv_bfloat16*>(sm + R::OFF_T);       // [buffer][term][group][token]
    __nv_bfloat16* const dsA = reinterpret_cast<__nv_bfloat16*>(sm + R::OFF_A);       // [buffer][block of groups][token][term][group]
    float* const fs = reinterpret_cast<float*>(sm + R::OFF_F);                        // [group][column]
    float* const cs = reinterpret_cast<float*>(sm + R::OFF_C);
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, q = lane & 3, l4 = lane >> 2;
    const int b = blockIdx.y / runs, tok0 = blockIdx.y % runs * run, e0 = blockIdx.x * R::COLS;
    for (uint32_t i = t; i < (R::OFF_F - R::OFF_T) / 4; i += RB_THREADS) reinterpret_cast<uint32_t*>(sm + R::OFF_T)[i] = 0u;       // (groups from LD on stay zero)
    dep_wait();
    dep_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0 && t == 0) *done = 0u;
    const int rows = min(run, n - tok0), pieces = (rows + RB_ROWS - 1) / RB_ROWS;
    const __nv_bfloat16* const hp = h + b * h_sb + (int64_t)tok0 * h_sn + e0;
    __nv_bfloat16* const dp = dh ? dh + b * d_sb + (int64_t)tok0 * d_sn + e0 : nullptr;
    const float* const sp = dS + ((size_t)b * n + tok0) * LD;
    // piece `x` of the rows on its way (an empty group past the end): 16-byte pieces of a row in an order that goes by the row, so that the
    // eight rows of an 8 x 8 tile lie in different banks
    auto copy = [&](int x) {
        if (x < pieces) {
            const uint32_t st = base + (x % R::STAGES) * R::STAGE_BYTES;
#pragma unroll
            for (int i = 0; i < RB_ROWS * R::CHUNKS / RB_THREADS; ++i) {
                const int k = i * RB_THREADS + t, r = k / R::CHUNKS, c = k % R::CHUNKS, row = x * RB_ROWS + r;
                const bool in = row < rows && e0 + 8 * c < d;                       // (d is a multiple of 8)
                rb_copy(st + r * (R::COLS * 2) + ((c ^ (r & 7)) << 4), in ? hp + (int64_t)row * h_sn + 8 * c : hp, in);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int x = 0; x < R::STAGES - 1; ++x) copy(x);
    float w[R::PER];
    auto load = [&](int r0) {                                // dS of the next rows; columns from K on may hold anything
#pragma unroll
        for (int x = 0; x < R::PER; ++x) {
            const int k = x * RB_THREADS + t;
            w[x] = r0 + k / LD < rows && k % LD < K ? sp[(size_t)r0 * LD + k] : 0.f;
        }
    };
    load(0);
    // F of the strip, and of it this lane's part: groups 2 q and 2 q + 1 of each block, a column of every tile, in two terms
    uint32_t fr[G8][CW / 8][2];
    if (dh) {
        if (!F) {
            for (int i = t; i < K * dg; i += RB_THREADS) cs[i] = C[i];
            __syncthreads();
            for (int c = t; c < R::COLS; c += RB_THREADS) {
                float y[LD];
#pragma unroll
                for (int g = 0; g < LD; ++g) y[g] = 0.f;
                if (e0 + c < d) {
#pragma unroll 8
                    for (int j = 0; j < dg; ++j) {
                        const float x = Wg[(size_t)(e0 + c) * dg + j];
#pragma unroll
                        for (int g = 0; g < LD; ++g)
                            if (g < K) y[g] = fmaf(x, cs[g * dg + j], y[g]);
                    }
                }
#pragma unroll
                for (int g = 0; g < 8 * G8; ++g) fs[g * R::COLS + c] = g < LD ? y[g < LD ? g : 0] : 0.f;
            }
        } else {
            for (int i = t; i < 8 * G8 * R::COLS; i += RB_THREADS) {
                const int g = i / R::COLS, c = i % R::COLS;
                fs[i] = g < K && e0 + c < d ? F[(size_t)g * d + e0 + c] : 0.f;
            }
        }
    }
    __syncthreads();
    if (dh) {
#pragma unroll
        for (int v = 0; v < G8; ++v) {
#pragma unroll
            for (int x = 0; x < CW / 8; ++x) {
                const int col = warp * CW + x / NT * (8 * NT) + 2 * NT * (l4 / 2) + 2 * (x % NT) + l4 % 2;
                const float f0 = fs[(8 * v + 2 * q) * R::COLS + col], f1 = fs[(8 * v + 2 * q + 1) * R::COLS + col];
                const __nv_bfloat162 hi = __floats2bfloat162_rn(f0, f1);
                const __nv_bfloat162 mid = __floats2bfloat162_rn(f0 - __low2float(hi), f1 - __high2float(hi));
                fr[v][x][0] = *reinterpret_cast<const uint32_t*>(&hi);
                fr[v][x][1] = *reinterpret_cast<const uint32_t*>(&mid);
            }
        }
    }
    float T[CW / 16][G8][4];
#pragma unroll
    for (int m = 0; m < CW / 16; ++m) {
#pragma unroll
        for (int v = 0; v < G8; ++v) T[m][v][0] = T[m][v][1] = T[m][v][2] = T[m][v][3] = 0.f;
    }
    for (int x = 0; x < pieces; ++x) {
        __nv_bfloat16* const tp = dsT + (x & 1) * (R::T_BYTES / 2);
        __nv_bfloat16* const ap = dsA + (x & 1) * (R::A_BYTES / 2);
#pragma unroll
        for (int i = 0; i < R::PER; ++i) {
            const int k = i * RB_THREADS + t, r = k / LD, g = k % LD;
            float v = w[i];
#pragma unroll
            for (int m = 0; m < 3; ++m) {
                const __nv_bfloat16 y = __float2bfloat16_rn(v);
                v -= __bfloat162float(y);
                tp[(m * 8 * G8 + g) * R::TPITCH + r] = y;
                if (m < 2) ap[((g >> 3) * RB_ROWS + r) * R::APITCH + 8 * m + (g & 7)] = y;
            }
        }
        asm volatile("cp.async.wait_group %0;" ::"n"(R::STAGES - 2) : "memory");
        __syncthreads();                                     // (what is copied to next was read before this barrier, dS's other buffer too)
        copy(x + R::STAGES - 1);
        load((x + 1) * RB_ROWS);
        const uint32_t st = base + (x % R::STAGES) * R::STAGE_BYTES;
        // (sums of the tensor cores are cut off, not rounded: one of 32 rows at a time, and those are added here)
        float P[CW / 16][G8][4];
#pragma unroll
        for (int m = 0; m < CW / 16; ++m) {
#pragma unroll
            for (int v = 0; v < G8; ++v) P[m][v][0] = P[m][v][1] = P[m][v][2] = P[m][v][3] = 0.f;
        }
#pragma unroll
        for (int k16 = 0; k16 < RB_ROWS / 16; ++k16) {
            const int r0 = 16 * k16;
            uint32_t bt[3][G8][2], aa[G8][4];
#pragma unroll
            for (int v = 0; v < G8; ++v) {
#pragma unroll
                for (int m = 0; m < 3; ++m) {
                    const __nv_bfloat16* const y = tp + (m * 8 * G8 + 8 * v + l4) * R::TPITCH + r0 + 2 * q;
                    bt[m][v][0] = *reinterpret_cast<const uint32_t*>(y);
                    bt[m][v][1] = *reinterpret_cast<const uint32_t*>(y + 8);
                }
                const __nv_bfloat16* const y = ap + (v * RB_ROWS + r0 + l4) * R::APITCH + 2 * q;
                aa[v][0] = *reinterpret_cast<const uint32_t*>(y);
                aa[v][1] = *reinterpret_cast<const uint32_t*>(y + 8 * R::APITCH);
                aa[v][2] = *reinterpret_cast<const uint32_t*>(y + 8);
                aa[v][3] = *reinterpret_cast<const uint32_t*>(y + 8 * R::APITCH + 8);
            }
            // P += h^T dS: rows of the product are columns of h
#pragma unroll
            for (int m = 0; m < CW / 16; ++m) {
                const int r = r0 + (lane & 7) + (lane >= 16 ? 8 : 0), c = warp * (CW / 8) + 2 * m + ((lane >> 3) & 1);
                uint32_t a[4];
                asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3])
                             : "r"(st + r * (R::COLS * 2) + ((c ^ (r & 7)) << 4)) : "memory");
#pragma unroll
                for (int v = 0; v < G8; ++v) {
#pragma unroll
                    for (int z = 2; z >= 0; --z) rb_mma(P[m][v], a, bt[z][v][0], bt[z][v][1]);
                }
            }
            // dh = dS F
            if (dp) {
#pragma unroll
                for (int y = 0; y < CW / 8; y += NT) {
                    uint32_t o[2][NT];
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int v = 0; v < G8; ++v) {
                            rb_mma(s, aa[v], fr[v][y + j][1], fr[v][y + j][1]);
                            rb_mma(s, aa[v], fr[v][y + j][0], fr[v][y + j][0]);
                        }
                        const __nv_bfloat162 u = __floats2bfloat162_rn(s[0], s[1]), z = __floats2bfloat162_rn(s[2], s[3]);
                        o[0][j] = *reinterpret_cast<const uint32_t*>(&u);
                        o[1][j] = *reinterpret_cast<const uint32_t*>(&z);
                    }
                    const int col = warp * CW + 8 * y + 2 * NT * q, row = x * RB_ROWS + r0 + l4;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        if (row + 8 * u >= rows || e0 + col >= d) continue;
                        __nv_bfloat16* const to = dp + (int64_t)(row + 8 * u) * d_sn + col;
                        if constexpr (NT == 4) *reinterpret_cast<uint4*>(to) = make_uint4(o[u][0], o[u][1], o[u][2], o[u][3]);
                        else *reinterpret_cast<uint2*>(to) = make_uint2(o[u][0], o[u][1]);
                    }
                }
            }
        }
#pragma unroll
        for (int m = 0; m < CW / 16; ++m) {
#pragma unroll
            for (int v = 0; v < G8; ++v) {
#pragma unroll
                for (int i = 0; i < 4; ++i) T[m][v][i] += P[m][v][i];
            }
        }
    }
#pragma unroll
    for (int m = 0; m < CW / 16; ++m) {
#pragma unroll
        for (int v = 0; v < G8; ++v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int g = 8 * v + 2 * q + (i & 1), col = e0 + warp * CW + 16 * m + l4 + (i >= 2 ? 8 : 0);
                if (g < K && col < d) part[((size_t)blockIdx.y * K + g) * d + col] = T[m][v][i];
            }
        }
    }
}

// T = sum of the parts, and for 32 of the d_g numbers dW_g = T^T C and this block's part of dC = T W_g; up to K d_g = RB_LAST the last block to be
// through adds those up, in their order.  (All of d_g in a block: 1000 x 1024, K = 32, d_g = 128 48 us, so 29.)
// A thread adds up an eighth of the parts of a column.
template <int LD>
__global__ void __launch_bounds__(256)
router_total_kernel(const float* part, const float* C, const float* Wg, int parts, int d, int dg, int K, float* dWg, float* dC_part, float* dC, unsigned* done) {
    __shared__ float eighth[8][LD][RB_TOTAL_COLS + 1];
    __shared__ float T[LD][RB_TOTAL_COLS + 1];
    __shared__ bool last;
    __shared__ float cs[LD * RB_TOTAL_DG], ws[RB_TOTAL_COLS * RB_TOTAL_DG];
    const int t = threadIdx.x, e0 = blockIdx.x * RB_TOTAL_COLS, c = t % RB_TOTAL_COLS, q = t / RB_TOTAL_COLS, cols = min(RB_TOTAL_COLS, d - e0);
    // The weights while the kernel before runs (what wrote them is older than that one, and complete)
    const int j0 = blockIdx.y * RB_TOTAL_DG, w = min(RB_TOTAL_DG, dg - j0);
    for (int i = t; i < K * RB_TOTAL_DG; i += 256) cs[i] = i % RB_TOTAL_DG < w ? C[(size_t)(i / RB_TOTAL_DG) * dg + j0 + i % RB_TOTAL_DG] : 0.f;
    for (int i = t; i < cols * RB_TOTAL_DG; i += 256) ws[i] = i % RB_TOTAL_DG < w ? Wg[(size_t)(e0 + i / RB_TOTAL_DG) * dg + j0 + i % RB_TOTAL_DG] : 0.f;
    dep_wait();
    dep_trigger();
    float x[LD];
#pragma unroll
    for (int g = 0; g < LD; ++g) x[g] = 0.f;
    if (c < cols) {
#pragma unroll 4
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
    for (int i = t; i < cols * RB_TOTAL_DG; i += 256) {
        const int k = i / RB_TOTAL_DG, j = i % RB_TOTAL_DG;
        float y = 0.f;
#pragma unroll
        for (int g = 0; g < LD; ++g)
            if (g < K) y = fmaf(T[g][k], cs[g * RB_TOTAL_DG + j], y);
        if (j < w) dWg[(size_t)(e0 + k) * dg + j0 + j] = y;
    }
    for (int i = t; i < K * RB_TOTAL_DG; i += 256) {
        const int g = i / RB_TOTAL_DG, j = i % RB_TOTAL_DG;
        float y = 0.f;
#pragma unroll 8
        for (int k = 0; k < cols; ++k) y = fmaf(T[g][k], ws[k * RB_TOTAL_DG + j], y);
        if (j < w) dC_part[(size_t)blockIdx.x * K * dg + (size_t)g * dg + j0 + j] = y;
    }
    if (K * dg > RB_LAST) return;
    __threadfence();
    __syncthreads();
    if (t == 0) last = atomicAdd(done, 1u) == gridDim.x * gridDim.y - 1;
    __syncthreads();
    if (!last) return;
    __threadfence();
    // as many lanes a number as there are threads for
    int lanes = 1;
    while (lanes < 32 && 2 * lanes * K * dg <= 256) lanes *= 2;
    for (int i0 = 0; i0 < K * dg; i0 += 256 / lanes) {
        const int i = i0 + t / lanes;
        float y = 0.f;
        if (i < K * dg) {
#pragma unroll 32
            for (int z = t % lanes; z < (int)gridDim.x; z += lanes) y += __ldcg(dC_part + (size_t)z * K * dg + i);
        }
        for (int off = lanes / 2; off; off >>= 1) y += __shfl_xor_sync(0xffffffffu, y, off);
        if (i < K * dg && t % lanes == 0) dC[i] = y;
    }
}

// How the tokens are cut: runs of `run` tokens of a sequence, a multiple of 32, `runs` a sequence: enough blocks for three on an SM
struct RouterCut {
    int run, runs;
};
static int router_strips(const focus_shape* s, int d) { return cdiv(d, rb_cols(focus_soft_ld(s->K))); }
static RouterCut router_cut(const focus_shape* s, int d) {
    const int want = 444 / (router_strips(s, d) * s->batch);            // (one more block than there are places for takes as long again)
    RouterCut c;
    c.run = cdiv(cdiv(s->n, want < 1 ? 1 : want), RB_ROWS) * RB_ROWS;
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
    int rc = check_cuda(allow_smem<router_bwd_kernel<LD>>(RouterCfg<LD>::SMEM), "cudaFuncSetAttribute(router_bwd)");
    if (rc) return rc;
    rc = check_cuda(launch_dependent(kern, dim3((unsigned)router_strips(s, a.d_model), (unsigned)(s->batch * c.runs)), dim3(RB_THREADS), RouterCfg<LD>::SMEM, st, a.h, a.h_sb, a.h_sn, a.ds,
                                         F, a.Wg, a.C, a.d_g, s->n, c.runs, c.run, a.d_model, s->K, a.dh, a.dh_sb, a.dh_sn, part, done), "router backward launch");
    if (rc) return rc;
    rc = check_cuda(launch_dependent(router_total_kernel<LD>, dim3((unsigned)cdiv(a.d_model, RB_TOTAL_COLS), (unsigned)cdiv(a.d_g, RB_TOTAL_DG)), dim3(256), 0, st, (const float*)part, a.C, a.Wg,
                                     s->batch * c.runs, a.d_model, a.d_g, s->K, a.dWg, dC_part, a.dC, done), "router totals launch");
    const long long count = (long long)s->K * a.d_g;
    if (rc || count <= RB_LAST) return rc;
    return check_cuda(launch_dependent(router_dc_kernel, dim3((unsigned)((count + 31) / 32)), dim3(256), 0, st, (const float*)dC_part, cdiv(a.d_model, RB_TOTAL_COLS), (int)count, a.dC),
                      "router centroids launch");
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
    if (fold) rc = check_cuda(launch_dependent(router_fold_kernel, dim3((unsigned)cdiv(d, 32)), dim3(256), 0, st, a.Wg, a.C, d, a.d_g, K, F), "router fold launch");
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
