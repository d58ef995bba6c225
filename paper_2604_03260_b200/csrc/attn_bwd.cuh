// What the entry points hand to the attention's backward pass, and what its kernels share.
#pragma once

#include "attn_common.cuh"
#include "tma_host.cuh"

namespace focus {

struct AttnBwdArgs {
    focus_shape s;
    focus_tensor q, k, v, o, dO, dq, dk, dv;
    const uint32_t* mq;
    const uint32_t* mk;
    const char* tiles;        // nullptr = every causal pair
    focus_tiles_layout L;     // valid when tiles != nullptr
    const float* lse;
    float scale;              // resolved logit scale
    const float* g;           // training-time soft gate: assignments [batch, n, ld]; nullptr = no gate
    float lambda;
    float* dg;
    char* ws;
    int32_t* dev_status;
};

size_t attn_bwd_workspace_bytes(const focus_shape* s, bool gate);
int launch_attn_bwd(const AttnBwdArgs& a, cudaStream_t st);

// A pass: rows R1, R2 stay in shared memory, columns C1, C2 stream by.  X = R1 C1^T, Y = R2 C2^T, P and dS of the tile; then
// BWD_KV   rows are keys: dV += P^T C2 and dK += dS^T C1 (R1 = K, R2 = V, C1 = Q, C2 = dO)
// BWD_V    rows are keys: dV alone (where the two sums do not fit tensor memory)
// BWD_K    rows are keys: dK alone
// BWD_Q    rows are queries: dQ += dS C1 (R1 = Q, R2 = dO, C1 = K, C2 = V)
enum : int { BWD_KV = 0, BWD_V = 1, BWD_K = 2, BWD_Q = 3 };

// Columns of an item in one launch at most: what is longer is walked by several launches, each of which adds its sums in fp32 to those of the one
// before.  The tensor cores add 16 products at a time to a sum and cut off, where all terms have one sign by 2^-23.5 of the result a step: of these 2048
// steps 2^-12.5, where without an end to it 16 query heads x 131072 tokens lost 2^-6.5 of dV (a half step of bf16 is 2^-9 to 2^-8).  Half as long: 32/8
// heads x 8192 tokens, which have just as many, would need two.  (Sums taken out within a launch instead: what that adds around
// the loop over the tiles cost 4 to 12 % where no sum is that long.)
constexpr int BWD_LAUNCH_TILES = 32768 / 128;
inline int bwd_heads_together(int nt, int heads) { return nt >= BWD_LAUNCH_TILES ? 1 : heads < BWD_LAUNCH_TILES / nt ? heads : BWD_LAUNCH_TILES / nt; }

// Depth of the product that gives the gate's g_i . g_j: six products of bf16 terms, in steps of 16
constexpr int gate_depth(int ld) { return (6 * ld + 15) / 16 * 16; }

struct BwdParams {
    int Hq, Hkv, G, n, nt, K, w;
    int heads;                // batch * heads of the rows (keys: times split)
    Divisor by_heads, by_rows_H, by_split;          // by that; by heads per sequence of the rows; by split
    int split, heads_each;    // keys: parts of a KV head's query heads, each an item with sums of its own; query heads of a part
    float *part1, *part2;     // sums in fp32: of keys [batch Hkv split][n][D], dV and dK over scale, of queries [batch Hq][n][D], part2 alone; or nullptr
    // What this launch walks of an item: query heads [head_lo, head_hi) of the part, columns in 128-tiles [col_lo, col_hi)
    int head_lo, head_hi, col_lo, col_hi;
    bool later, last;         // keys: other heads of the part were walked before; this launch is the last
    int row_tiles;            // that have such columns: the first of keys, the last of queries
    float scale, softcap, lambda;
    const float* stat;        // [batch Hq][nt][2][128]: -lse log2(e), -delta
    const __nv_bfloat16* aug; // [batch Hq][nt][128][8]: -lse / scale, -delta in three terms each
    const uint32_t* row_mask; // masks of the rows' tokens
    const uint32_t* bits;     // columns' bitmaps per group [heads of the columns][nt][K][4]; nullptr = every causal pair
    const uint32_t* live;     // live far tiles [batch Hq][nt][nkw]
    int nkw;
    const float* g;
    const __nv_bfloat16 *g_rows, *g_cols; // its terms: of the rows [batch][nt][depth / 8][128][8], of the columns [batch][2 nt][depth / 8][64][8]
    const float* g_flat;      // and as it is [batch][2 nt][8 columns at a time][even, odd][ld / 4][4 of them][4]
    float* dg_part;           // [heads][n][ld]
    __nv_bfloat16 *out1, *out2;           // dV (BWD_KV, BWD_V); dK / dQ
    int64_t s1b, s1h, s1n, s2b, s2h, s2n;
    bool wide1, wide2;        // 32-byte stores
    int32_t* status;
};

template <int D> int launch_bwd_d(const AttnBwdArgs& a, const BwdParams& kv, const BwdParams& q, cudaStream_t st);

}  // namespace focus
