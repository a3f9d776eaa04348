// Products with 4-bit weights and group scales (layout: skim_group.h), for one token to many:
//   y = x W^T,   a = silu(x Wg^T) * (x Wu^T),   dx = dy W,   and the backward pass of a.
// All of them run on the matrix cores with exact operands: a code is a whole number, a code times its scale a bfloat16, and x comes in
// bfloat16 or e4m3.  Sums are float32; the one rounding is that of a result to its type.
#include "skim_group.h"
#include "skim_tiles.h"

#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace {

typedef uint32_t gq_word2 __attribute__((ext_vector_type(2)));
typedef short gq_short4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) gq_short4 lds_short4;

// What one launch works on.  Two matrices where gate and up are read together.
struct MmArgs {
    const gq_word4 *codes[2];
    const uint16_t *scales[2];
    long long n, m;              // rows and columns of the matrices
    const void *x;               // [T][ldx]: the input, or the gradient that dx is made of
    const void *x2;              // ... that of the second matrix
    long long ldx;
    const float *x_scales;       // e4m3: one a token
    long long T;
    void *y;                     // result, [T][columns]
    int y_f32;
    const uint16_t *da;          // backward pass of the gated block
    long long ldda;
    uint16_t *dgate, *dup;
    // Gradients in two pieces, 16 bits of them.  Written: rows 2 t and 2 t + 1 of dgate and, 2 T rows on, of dup, ldp values each (a multiple of 16, zeros past n).
    // Read (dx): x and x2 are such rows, T counts them, and a token's result is the sum of its two.
    uint16_t *pieces;
    long long ldp;
    bool paired;
    bool quads;                  // results (and da) can be taken in fours
};

enum { MM_PLAIN, MM_GLU, MM_GLU_BACK };

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float from_bf16(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
// What v has beyond its bfloat16 (0 where that is no number to take it from).
__device__ __forceinline__ uint16_t second_piece(float v, uint16_t first) { return (first & 0x7F80) == 0x7F80 ? (uint16_t)0 : to_bf16(v - from_bf16(first)); }
__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + expf(-g)); }

// Four neighbouring results of a token, of rows `row` .. row + 3 of `rows`; the token is inside.  Sums come times `by`.
template <int MODE>
__device__ __forceinline__ void finish4(const MmArgs &A, long long t, long long row, long long rows, gq_float4 g, gq_float4 u, float by) {
    if (row >= rows) {
        if constexpr (MODE == MM_GLU_BACK) {
            if (A.pieces && row < A.ldp) {
#pragma unroll
                for (int i = 0; i < 4; ++i) *(gq_short4 *)(A.pieces + ((i >> 1) * 2 * A.T + 2 * t + (i & 1)) * A.ldp + row) = gq_short4{};
            }
        }
        return;
    }
    const long long at = t * rows + row;
    const bool quad = A.quads;                    // rows come in fours, everything on borders of fours
    if constexpr (MODE == MM_GLU_BACK) {
        gq_short4 d = {}, dg, du, dg2, du2;
        const uint16_t *p = A.da + t * A.ldda + row;
        if (quad) d = *(const gq_short4 *)p;
        else
            for (int i = 0; i < 4; ++i)
                if (row + i < rows) d[i] = (short)p[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool in = row + i < rows;                                // (past the last row the sums are zeros, but for a token with an infinity or a NaN)
            const float gi = g[i] * by, ui = u[i] * by, di = from_bf16((uint16_t)d[i]), s = sigmoid(gi);
            const float vg = in ? di * ui * s * fmaf(gi, 1.f - s, 1.f) : 0.f, vu = in ? di * gi * s : 0.f;
            dg[i] = (short)to_bf16(vg);
            du[i] = (short)to_bf16(vu);
            dg2[i] = (short)second_piece(vg, (uint16_t)dg[i]);
            du2[i] = (short)second_piece(vu, (uint16_t)du[i]);
        }
        if (A.pieces) {
            uint16_t *q = A.pieces + 2 * t * A.ldp + row;
            *(gq_short4 *)q = dg;
            *(gq_short4 *)(q + A.ldp) = dg2;
            q += 2 * A.T * A.ldp;
            *(gq_short4 *)q = du;
            *(gq_short4 *)(q + A.ldp) = du2;
        }
        if (quad) {
            *(gq_short4 *)(A.dgate + at) = dg;
            *(gq_short4 *)(A.dup + at) = du;
        } else {
            for (int i = 0; i < 4; ++i)
                if (row + i < rows) A.dgate[at + i] = (uint16_t)dg[i], A.dup[at + i] = (uint16_t)du[i];
        }
        return;
    }
    gq_float4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float gi = g[i] * by;
        v[i] = MODE == MM_GLU ? gi * sigmoid(gi) * (u[i] * by) : gi;
    }
    if (A.y_f32) {
        float *p = (float *)A.y + at;
        if (quad) *(gq_float4 *)p = v;
        else
            for (int i = 0; i < 4; ++i)
                if (row + i < rows) p[i] = v[i];
    } else {
        uint16_t *p = (uint16_t *)A.y + at;
        gq_short4 o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = (short)to_bf16(v[i]);
        if (quad) *(gq_short4 *)p = o;
        else
            for (int i = 0; i < 4; ++i)
                if (row + i < rows) p[i] = (uint16_t)o[i];
    }
}

// ---- operands ------------------------------------------------------------------------------------------------------------

// Scaled weights of a word, exact in bfloat16.
__device__ __forceinline__ gq_word4 weight_operand(uint32_t w, float s) {
    gq_word4 v;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t bytes = h ? gq_high(w) : gq_low(w);
        const gq_float2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bytes, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bytes, 512.f, true);
        v[2 * h] = __builtin_amdgcn_perm(__float_as_uint(s * a.y), __float_as_uint(s * a.x), 0x07060302u);
        v[2 * h + 1] = __builtin_amdgcn_perm(__float_as_uint(s * b.y), __float_as_uint(s * b.x), 0x07060302u);
    }
    return v;
}

// The codes of a word times 2^-9 of a power of two, in bfloat16.
__device__ __forceinline__ gq_bf16x8 code_operand(uint32_t w, float power) {
    const uint32_t lo = gq_low(w), hi = gq_high(w);
    const gq_word4 u{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, power, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, power, true))};
    return __builtin_bit_cast(gq_bf16x8, u);
}

// Eight e4m3 values in bfloat16, exactly.  (The 8-bit matrix instructions would take them as they are, but drop what lies 2^-10 below the largest
// of the products that they add up.)
__device__ __forceinline__ gq_bf16x8 widen(gq_word2 v) {
    const gq_word4 u{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[0], 1.f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[0], 1.f, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[1], 1.f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(v[1], 1.f, true))};
    return __builtin_bit_cast(gq_bf16x8, u);
}

__device__ __forceinline__ gq_float4 mfma(gq_bf16x8 a, gq_bf16x8 b, gq_float4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// 8 values of a row of x, as they come from memory, from column col on; zeros past column m.  VEC: rows start on borders of the octet's size and m
// is a multiple of 8.
template <int XT>
struct XOctet {
    typedef std::conditional_t<XT == SKIM_BF16, uint16_t, uint8_t> E;
    std::conditional_t<XT == SKIM_BF16, gq_word4, gq_word2> v;
    __device__ __forceinline__ void load_whole(const void *x, long long at) { __builtin_memcpy(&v, (const E *)x + at, sizeof(v)); }      // (one load, of any alignment)
    template <bool VEC>
    __device__ __forceinline__ void load(const void *x, long long row0, long long col, long long m) {
        const E *p = (const E *)x + row0 + col;
        if constexpr (VEC) {
            if (col < m) v = *(const decltype(v) *)p;
            else v = decltype(v){};
        } else if (col + 8 <= m) {
            load_whole(p, 0);
        } else {
            E e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = col + i < m ? p[i] : (E)0;
            __builtin_memcpy(&v, e, sizeof(v));
        }
    }
    __device__ __forceinline__ gq_bf16x8 operand() const {
        if constexpr (XT == SKIM_BF16) return __builtin_bit_cast(gq_bf16x8, v);
        else return widen(v);
    }
};

// ---- few tokens ----------------------------------------------------------------------------------------------------------

// A workgroup makes 16 rows of the result for 16 tokens, or (NT = 2) 32 for 32; its wavefronts share the columns block by block, and their sums are added up in
// LDS in the order of the wavefronts.  Bound by the codes' way from memory: with up to 16 tokens a wavefront asks for U blocks at once, with their scales and
// their columns of x, before it takes the first apart.  One token on 4096 x 11008 7.8 us (3.0 TB/s; 13.5 with a block at a time), gated on 11008 x 4096 12.6
// (3.7 TB/s); in the 128 registers of its wavefronts is room for no more.
// A scale s is a power of two times its significand, 1 to 2.  Up to 16 tokens (LATE) codes enter the matrix cores times that power, which their conversion brings along
// for nothing, and a group's sum is multiplied by the significand once: no sum overflows that the formula's does not (sums of q x alone do, for x above 2^118), and
// none is smaller than a half of it.  (Powers are at most 2^118, where the conversion's own, 2^9 times that, ends; the rest of a larger scale goes with its significand.)
// x is the first operand there: a lane's four sums are of one row then, and take one significand.  More tokens take weights times scales, as the tiles do.  us the one way
// / the other: one token on 4096 x 11008 7.8 / 8.6, gated on 11008 x 4096 12.6 / 14.4; 32 tokens on 4096 x 11008 with groups of 32 29 / 25.5, gated 64 36 / 33.
constexpr int FEW_POWER = 118;
constexpr int FEW_TOKEN = 20;         // floats of a token's 16 rows in LDS: so that 64 lanes' of one access lie in different banks
template <int XT, int NT, int G, int MODE, bool VEC>
__global__ void __launch_bounds__(NT == 1 ? 1024 : 512) group_few_kernel(MmArgs A, int chunks) {
    constexpr int RT = NT, MATS = MODE == MM_PLAIN ? 1 : 2, U = NT > 1 ? 1 : MATS * (GQ_COLS / G) * (XT == SKIM_BF16 ? 2 : 1) <= 2 ? 4 : 2, GS = GQ_COLS / G;
    constexpr bool LATE = NT == 1;
    extern __shared__ __align__(16) unsigned char few_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), nw = blockDim.x >> 6;
    const int c = lane >> 4, l16 = lane & 15;
    const long long rt0 = (long long)(blockIdx.x / chunks) * RT, t0 = (long long)(blockIdx.x % chunks) * (16 * NT);
    const int kbs = (int)gq_col_blocks(A.m);
    const long long rbs = gq_row_blocks(A.n), n16 = rbs * GQ_ROWS;
    // (lanes without a token keep zeros and load nothing)
    XOctet<XT> x[U][4][NT] = {};
    gq_float4 acc[MATS][RT][NT] = {};
    for (int first = wave; first < kbs; first += nw * U) {
        gq_word4 w[U][MATS][RT];
        uint32_t s[U][MATS][RT][GS];                                               // of the lane's row
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int kb = first + u * nw;
            if (kb >= kbs) continue;
#pragma unroll
            for (int a = 0; a < MATS; ++a)
#pragma unroll
                for (int r = 0; r < RT; ++r) {
                    const long long rt = min(rt0 + r, rbs - 1);
                    w[u][a][r] = A.codes[a][(rt * kbs + kb) * 64 + lane];
#pragma unroll
                    for (int g = 0; g < GS; ++g) s[u][a][r][g] = A.scales[a][((long long)kb * GS + g) * n16 + rt * GQ_ROWS + l16];
                }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
                const long long t = t0 + 16 * j + l16;
                const long long col = (long long)kb * GQ_COLS + 8 * c;
                if (t < A.T) {
                    if ((long long)(kb + 1) * GQ_COLS <= A.m) {                   // a whole block: nothing to look at lane by lane
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[u][k][j].load_whole(A.x, t * A.ldx + col + 32 * k);
                    } else {
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[u][k][j].template load<VEC>(A.x, t * A.ldx, col + 32 * k, A.m);
                    }
                }
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (first + u * nw >= kbs) continue;
#pragma unroll
            for (int g = 0; g < GS; ++g) {
                gq_float4 d[MATS] = {};
                uint32_t power[MATS];                         // exponent field, in place
                if constexpr (LATE) {
#pragma unroll
                    for (int a = 0; a < MATS; ++a) power[a] = min(s[u][a][0][g] & 0x7F80u, (uint32_t)(FEW_POWER + 127) << 7);
                }
#pragma unroll
                for (int k = g * (4 / GS); k < (g + 1) * (4 / GS); ++k) {
                    gq_bf16x8 b[NT];
#pragma unroll
                    for (int j = 0; j < NT; ++j) b[j] = x[u][k][j].operand();
#pragma unroll
                    for (int a = 0; a < MATS; ++a) {
                        if constexpr (LATE) {
                            d[a] = mfma(b[0], code_operand(w[u][a][0][k], gq_scale(power[a] + (9u << 7))), d[a]);
                        } else {
#pragma unroll
                            for (int r = 0; r < RT; ++r) {
                                const gq_bf16x8 q = __builtin_bit_cast(gq_bf16x8, weight_operand(w[u][a][r][k], gq_scale(s[u][a][r][g])));
#pragma unroll
                                for (int j = 0; j < NT; ++j) acc[a][r][j] = mfma(q, b[j], acc[a][r][j]);
                            }
                        }
                    }
                }
                if constexpr (LATE) {
#pragma unroll
                    for (int a = 0; a < MATS; ++a) {
                        const float f = gq_scale(s[u][a][0][g]) * gq_scale((254u << 7) - power[a]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[a][0][0][i] = fmaf(f, d[a][i], acc[a][0][0][i]);
                    }
                }
            }
        }
    }
    constexpr int E = RT * NT * 64;      // fours of a wavefront's sums, for one matrix: of 4 rows of a token each
    constexpr int ROOM = LATE ? 16 * FEW_TOKEN / 4 : E;
    gq_float4 *red = (gq_float4 *)few_lds;
    if constexpr (LATE) {                // (a lane has 4 tokens of its row)
#pragma unroll
        for (int a = 0; a < MATS; ++a)
#pragma unroll
            for (int i = 0; i < 4; ++i) ((float *)(red + (wave * MATS + a) * ROOM))[(4 * c + i) * FEW_TOKEN + l16] = acc[a][0][0][i];
    } else {
#pragma unroll
        for (int a = 0; a < MATS; ++a)
#pragma unroll
            for (int r = 0; r < RT; ++r)
#pragma unroll
                for (int j = 0; j < NT; ++j) red[(wave * MATS + a) * ROOM + (r * NT + j) * 64 + lane] = acc[a][r][j];
    }
    __syncthreads();
    for (int e = tid; e < E; e += blockDim.x) {
        gq_float4 v[MATS] = {};
        const int el = e & 63, at = LATE ? (el & 15) * (FEW_TOKEN / 4) + (el >> 4) : e;
#pragma unroll
        for (int a = 0; a < MATS; ++a)
            for (int w = 0; w < nw; ++w) v[a] += red[(w * MATS + a) * ROOM + at];
        const long long t = t0 + 16 * ((e >> 6) % NT) + (el & 15), rt = rt0 + (e >> 6) / NT;
        if (t < A.T)
            finish4<MODE>(A, t, rt * GQ_ROWS + 4 * (el >> 4), A.n, v[0], v[MATS - 1], XT == SKIM_E4M3 ? A.x_scales[t] : 1.f);
    }
}

// ---- many tokens -----------------------------------------------------------------------------------------------------------

// y = x W^T, the gated block and its backward pass, and dx = dy W (+ dy2 W2), on tiles of the matrix cores.  Four wavefronts side by side make
// 256 rows of W (128 of gate and the same of up; for dx 256 columns) for 128 tokens, each 64 of them: 2 x 4 accumulator
// tiles of 32 x 32.
// The tokens' operand: 128 columns of x (for dx as many values of dy) go straight to LDS a block ahead.  The weights' operand never is in
// memory: codes come into registers a block ahead, one 16-byte load for 32 of them, and are taken apart there, times their scale, into
// operands, those of the next 16 columns between the matrix instructions of these (19 operations for 8 weights).  For dx, where a lane
// needs 8 rows of one column, they pass through LDS of the wavefront's own and come back by the transposing read.
// LDS rows of a token are 256 bytes; its 16-byte unit u is at place u ^ (token % 16), so that 16 tokens' units of one column octet lie in different banks.
// 32 x 32 instructions: half as many as of 16 x 16 for the same product.  No wait stands between a load and the end of its block: a value that is
// shifted or combined as it arrives is waited for at once, which cost 20 % when it happened to the scales.
// Bound by the matrix cores and the power they draw: 2048 tokens on 8192 x 11008 run at 1.15-1.24 PFLOP/s (matrix products of bfloat16 matrices at
// 1.45-1.5), on x of zeros at 1.46, without the taking apart at 1.33; two wavefronts a SIMD, 256 registers each, leave no room for tiles that would share it more.
constexpr int WIDE_R = 4, WIDE_THREADS = 64 * WIDE_R;
constexpr int wide_x_bytes(int tt) { return 32 * tt * GQ_COLS * 2; }     // of one block: 32 KB for 128 tokens
constexpr int WIDE_A_ROW = 144, WIDE_A_BYTES = 16 * WIDE_A_ROW;      // dx: a wavefront's 16 rows x 64 columns; rows 16 bytes further apart than they are long, for the banks

// The other lane's of a pair.
__device__ __forceinline__ float neighbour(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xF, 0xF, true)); }

// Four sums of either row tile of wavefront `w` (counted through all tiles) for token t, those `in` rows down the tile.
template <bool DX, int MODE>
__device__ __forceinline__ void wide_finish(const MmArgs &A, long long w, long long t, int in, gq_float4 v0, gq_float4 v1) {
    if (DX && A.paired) {                            // a token's two rows are two lanes'
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v0[i] += neighbour(v0[i]);
            v1[i] += neighbour(v1[i]);
        }
        if (t >= A.T || (t & 1)) return;
        t >>= 1;
    } else if (t >= A.T) {
        return;
    }
    const float by = A.x_scales ? A.x_scales[t] : 1.f;
    if constexpr (MODE == MM_PLAIN) {
        finish4<MODE>(A, t, w * 64 + in, DX ? A.m : A.n, v0, gq_float4{}, by);
        finish4<MODE>(A, t, w * 64 + 32 + in, DX ? A.m : A.n, v1, gq_float4{}, by);
    } else {
        finish4<MODE>(A, t, w * 32 + in, A.n, v0, v1, by);
    }
}

// Four wavefronts side by side; with KS = 2 four more sum the other half of the columns, and the halves meet in LDS at the end.  `parts`
// workgroups share a tile's columns further: their sums go to `partial`, and group_join_kernel adds them up.
template <bool DX, int MODE, int KS, int TT>
__global__ void __launch_bounds__(WIDE_THREADS *KS) __attribute__((amdgpu_waves_per_eu(2, 2)))
group_wide_kernel(MmArgs A, int group, int mats, int ttiles, int tile0, int whole, int rest, int rest_parts, gq_float4 *partial) {
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int TOKENS = 32 * TT, X_BYTES = wide_x_bytes(TT);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane >> 4, l16 = lane & 15;
    const int kg = wave / WIDE_R, rg = wave % WIDE_R;
    // the first `whole` workgroups take a tile each, the others a part of one of the `rest`
    const bool shared = (int)blockIdx.x >= whole;
    const int work = shared ? xcd_order(blockIdx.x - whole, gridDim.x - whole) : xcd_order(blockIdx.x, whole);
    const int parts = shared ? rest_parts : 1, part = shared ? work / rest : 0, nth = work - part * rest, tile = tile0 + (shared ? whole + nth : work);
    const long long ob = tile / ttiles, t0 = (long long)(tile % ttiles) * TOKENS;
    const long long kbs = gq_col_blocks(A.m), rbs = gq_row_blocks(A.n), n16 = rbs * GQ_ROWS;
    const long long depth = DX ? A.n : A.m;                          // summed over
    const int blocks = (int)((depth + 127) / 128), total = DX ? blocks * mats : blocks;
    const int per = GQ_COLS / group;
    const int share = part * KS + kg, shares = parts * KS;
    const int kb0 = (int)((long long)total * share / shares), kb1 = (int)((long long)total * (share + 1) / shares);
    const int rounds = (total + shares - 1) / shares;                // (of the longest share: all wavefronts meet at every barrier)

    // ---- the tokens' operand: 2 TT copies of 1 KB a wavefront and block, 4 tokens of 16 units each
    unsigned char *const xbuf = smem + kg * 2 * X_BYTES;
    const uint32_t lds_x = (uint32_t)(uintptr_t)(lds_byte *)xbuf + (uint32_t)(rg * 2 * TT * 1024);
    const uint32_t ldb = (uint32_t)(A.ldx * 2), voff0 = (uint32_t)(rg * 8 * TT + c) * ldb;       // of the token of copy 0
    const int unit0 = l16 ^ c;                                                               // its unit
    auto stage = [&](int kb, int place) {
        const int a = DX && kb >= blocks ? 1 : 0;
        const long long col = (long long)(kb - a * blocks) * GQ_COLS;
        const int left = (int)min(depth - col, (long long)GQ_COLS);
        // (rows come in whole octets; tokens past the last lie past the end of x, where zeros arrive from)
        const LdsSource src{(uint64_t)(uintptr_t)((const uint16_t *)(a ? A.x2 : A.x) + t0 * A.ldx + col), ((A.T - 1 - t0) * A.ldx + (depth + 7) / 8 * 8 - col) * 2};
        const int4v rs = src.rsrc();
#pragma unroll
        for (int i = 0; i < 2 * TT; ++i) {
            const int u = unit0 ^ 4 * (i & 3);
            copy_to_lds(lds_x + place * X_BYTES + i * 1024, u * 8 < left ? voff0 + (uint32_t)(4 * i) * ldb + (uint32_t)(u * 16) : 0x80000000u, rs);
        }
    };

    // ---- the weights' operand.  Half step s of a block: 16 columns (rows for dx) of all 64 rows (columns).
    const int hi = lane >> 5;
    constexpr int PAIR = MODE == MM_PLAIN ? 4 : 2;                   // row blocks of a wavefront, of one matrix
    const long long rb0 = (ob * WIDE_R + rg) * PAIR;
    const long long cb = min((ob * WIDE_R + rg) >> 1, kbs - 1);           // dx: column block, and which half of it
    const int half = rg & 1;
    gq_word4 next[4], cur[4];        // forward: [2 row tile + p], p: columns 16 p + 8 hi of every 32; dx: two row blocks of two words each
    // The block's scales.  Forward: [2 row tile + w]: those of words 2 w and 2 w + 1.  dx: [row / 64]: those of the two words.  They come two rows a
    // register, [4 row tile + group] or [2 (row / 64) + group], and stay so until take_codes: anything done to them earlier would wait for them.
    uint32_t nscale[8], cscale[4];
    // (addresses: a wavefront's own, and 32-bit places of the lanes)
    uint32_t wplace[2], splace[2];
    long long rbu[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        rbu[i] = min(rb0 + (MODE == MM_PLAIN ? 2 * i : 0), rbs - 1);
        const int second = rbu[i] + 1 < rbs ? c & 1 : 0;
        wplace[i] = DX ? (uint32_t)(lane * 16 + 8 * half) : (uint32_t)(second * kbs) * 1024u + (uint32_t)(16 * hi + l16) * 16u;
        splace[i] = DX ? (uint32_t)(lane & ~1) : (uint32_t)(second * 16 + (l16 & ~1)) * 2u;
    }
    auto load_codes = [&](int kb) {
        if constexpr (DX) {
            const int a = kb >= blocks ? 1 : 0;
            const long long rb = (long long)(kb - a * blocks) * 8;
            const char *w = (const char *)A.codes[a] + (rb * kbs + cb) * 1024;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                gq_word2 v = {};
                if (rb + j < rbs) v = *(const gq_word2 *)(w + j * kbs * 1024 + wplace[0]);
                next[j >> 1][2 * (j & 1)] = v[0];
                next[j >> 1][2 * (j & 1) + 1] = v[1];
            }
            const char *s = (const char *)(A.scales[a] + (cb * per + 64 * half / group) * n16 + rb * GQ_ROWS);
            const uint32_t last = (uint32_t)min(n16 - rb * GQ_ROWS, 128ll) - 2;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t row = min(splace[0] + 64u * q, last);
                nscale[2 * q] = *(const uint32_t *)(s + row * 2);
                if (group == 32) nscale[2 * q + 1] = *(const uint32_t *)(s + n16 * 2 + row * 2);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int m = MODE == MM_PLAIN ? 0 : i;
                const char *w = (const char *)A.codes[m] + (rbu[i] * kbs + kb) * 1024;
                next[2 * i] = *(const gq_word4 *)(w + wplace[i]);
                next[2 * i + 1] = *(const gq_word4 *)(w + wplace[i] + 512);
                const char *s = (const char *)(A.scales[m] + (long long)kb * per * n16 + rbu[i] * GQ_ROWS);
                nscale[4 * i] = *(const uint32_t *)(s + splace[i]);
                if (group <= 64) nscale[4 * i + 1] = *(const uint32_t *)(s + n16 * 2 + splace[i]);
                if (group == 32) {
                    nscale[4 * i + 2] = *(const uint32_t *)(s + n16 * 4 + splace[i]);
                    nscale[4 * i + 3] = *(const uint32_t *)(s + n16 * 6 + splace[i]);
                }
            }
        }
    };
    unsigned char *mine = smem + 2 * KS * X_BYTES + wave * WIDE_A_BYTES;
    auto operands = [&](int s, gq_bf16x8 (&a)[2]) {
        if constexpr (DX) {
            const uint32_t f = (uint32_t)__shfl((int)cscale[s >> 2], 16 * (s & 3) + l16, 64);
            // (one place for all half steps: a wavefront's accesses to LDS stay in their order)
#pragma unroll
            for (int q = 0; q < 2; ++q)
                *(gq_word4 *)(mine + l16 * WIDE_A_ROW + c * 16 + q * 64) =
                    weight_operand(cur[s >> 1][2 * (s & 1) + q], q ? __uint_as_float(f & 0xFFFF0000u) : __uint_as_float(f << 16));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                // 16 lanes read 4 rows of 16 columns and get 4 rows of one column each; a lane's operand: column lane % 32, rows 8 hi .. 8 hi + 7
                const unsigned char *from = mine + (8 * hi + (l16 >> 2)) * WIDE_A_ROW + (c & 1) * 32 + (l16 & 3) * 8 + i * 64;
                const gq_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)from);
                const gq_short4 up = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(from + 4 * WIDE_A_ROW));
                a[i] = __builtin_bit_cast(gq_bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        } else {
            const int k = s >> 1;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t f = cscale[2 * i + (k >> 1)];
                a[i] = __builtin_bit_cast(gq_bf16x8, weight_operand(cur[2 * i + (s & 1)][k], k & 1 ? __uint_as_float(f & 0xFFFF0000u) : __uint_as_float(f << 16)));
            }
        }
    };
    // the next block's codes have come (and all copies with them)
    auto take_codes = [&]() {
        asm volatile("s_waitcnt vmcnt(0)"
                     : "+v"(next[0]), "+v"(next[1]), "+v"(next[2]), "+v"(next[3]), "+v"(nscale[0]), "+v"(nscale[1]), "+v"(nscale[2]), "+v"(nscale[3])
                     :
                     : "memory");
        if constexpr (!DX) asm volatile("" : "+v"(nscale[4]), "+v"(nscale[5]), "+v"(nscale[6]), "+v"(nscale[7]));
#pragma unroll
        for (int i = 0; i < 4; ++i) cur[i] = next[i];
        const uint32_t pick = lane & 1 ? 0x03020302u : 0x01000100u, both = lane & 1 ? 0x07060302u : 0x05040100u;       // the lane's row; of two registers
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            if constexpr (DX) {
                cscale[i] = group == 32 ? __builtin_amdgcn_perm(nscale[2 * i + 1], nscale[2 * i], both) : __builtin_amdgcn_perm(0u, nscale[2 * i], pick);
            } else if (group == 128) {
                cscale[2 * i] = cscale[2 * i + 1] = __builtin_amdgcn_perm(0u, nscale[4 * i], pick);
            } else if (group == 64) {
                cscale[2 * i] = __builtin_amdgcn_perm(0u, nscale[4 * i], pick);
                cscale[2 * i + 1] = __builtin_amdgcn_perm(0u, nscale[4 * i + 1], pick);
            } else {
                cscale[2 * i] = __builtin_amdgcn_perm(nscale[4 * i + 1], nscale[4 * i], both);
                cscale[2 * i + 1] = __builtin_amdgcn_perm(nscale[4 * i + 3], nscale[4 * i + 2], both);
            }
        }
    };

    floatx16 acc[2][TT] = {};
    gq_bf16x8 a[2][2], b[2][TT];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        next[i] = gq_word4{};
        nscale[i] = nscale[4 + i] = 0;
    }
    if (kb0 < kb1) {
        stage(kb0, 0);
        load_codes(kb0);
    }
    take_codes();
    operands(0, a[0]);
    for (int r = 0; r < rounds; ++r) {
        const int kb = kb0 + r, now = r & 1;                         // block, and which of the two places in LDS it is in
        // this block's copies have landed, and everybody is done with the block before, whose place the next one takes
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (kb >= kb1) continue;                                     // (a share that is one block shorter)
        if (kb + 1 < kb1) {
            stage(kb + 1, now ^ 1);
            load_codes(kb + 1);
        }
        const unsigned char *xb = xbuf + now * X_BYTES + (lane & 31) * (GQ_COLS * 2);
        auto read_x = [&](int s, gq_bf16x8 (&v)[TT]) {
            const int place = (2 * s + hi) ^ l16;
#pragma unroll
            for (int j = 0; j < TT; ++j) v[j] = *(const gq_bf16x8 *)(xb + j * 32 * GQ_COLS * 2 + place * 16);
        };
        read_x(0, b[0]);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            if (s < 7) {
                read_x(s + 1, b[(s + 1) & 1]);
                operands(s + 1, a[(s + 1) & 1]);
            } else {
                take_codes();
                operands(0, a[0]);
            }
#pragma unroll
            for (int j = 0; j < TT; ++j)
#pragma unroll
                for (int i = 0; i < 2; ++i) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[s & 1][i], b[s & 1][j], acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            // (a wavefront ahead of the other on its SIMD for every second half step: they take turns at the matrix cores and at taking codes apart; 315 ->
            // 298 us where two workgroups share a compute unit)
            if (s & 1) __builtin_amdgcn_s_setprio(0);
            else __builtin_amdgcn_s_setprio(1);
        }
    }
    int j0 = 0, j1 = TT;
    if constexpr (KS == 2) {                                         // each four give half of their sums and finish the others
        constexpr int H = TT / 2;
        floatx16 *give = (floatx16 *)smem + (size_t)wave * (2 * H * 64) + lane;
        const floatx16 *take = (const floatx16 *)smem + (size_t)(wave ^ WIDE_R) * (2 * H * 64) + lane;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) give[(i * H + j) * 64] = kg == 0 ? acc[i][j + H] : acc[i][j];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < H; ++j) {
                const floatx16 o = take[(i * H + j) * 64];
                if (kg == 0) acc[i][j] += o;
                else acc[i][j + H] += o;
            }
        j0 = H * kg;
        j1 = j0 + H;
    }
#pragma unroll
    for (int j = 0; j < TT; ++j) {
        if (j < j0 || j >= j1 || t0 + 32 * j >= A.T) continue;
        auto four = [&](int i, int q) { return gq_float4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}; };
        if (parts > 1) {
            gq_float4 *p = partial + ((((size_t)part * rest + nth) * WIDE_R + rg) * TT + j) * 512 + lane;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int i = 0; i < 2; ++i) p[(2 * q + i) * 64] = four(i, q);
        } else {
#pragma unroll
            for (int q = 0; q < 4; ++q) wide_finish<DX, MODE>(A, ob * WIDE_R + rg, t0 + 32 * j + (lane & 31), 8 * q + 4 * hi, four(0, q), four(1, q));
        }
    }
}

// The parts of a tile added up in their order, and finished: one wavefront for 32 tokens and 16 of a wavefront's rows.
template <bool DX, int MODE, int TT>
__global__ void __launch_bounds__(256) group_join_kernel(MmArgs A, int ttiles, int first, int rest, int parts, const gq_float4 *__restrict__ partial) {
    const int lane = threadIdx.x & 63, q = threadIdx.x >> 6;
    const int nth = blockIdx.x / (TT * WIDE_R), tile = first + nth, rg = blockIdx.x / TT % WIDE_R, j = blockIdx.x % TT;
    const long long ob = tile / ttiles, t0 = (long long)(tile % ttiles) * (32 * TT);
    if (t0 + 32 * j >= A.T) return;
    const gq_float4 *p = partial + (((size_t)nth * WIDE_R + rg) * TT + j) * 512 + 2 * q * 64 + lane;
    const size_t step = (size_t)rest * WIDE_R * TT * 512;
    gq_float4 v0 = p[0], v1 = p[64];
    for (int i = 1; i < parts; ++i) {
        v0 += p[i * step];
        v1 += p[i * step + 64];
    }
    wide_finish<DX, MODE>(A, ob * WIDE_R + rg, t0 + 32 * j + (lane & 31), 8 * q + 4 * (lane >> 5), v0, v1);
}

// x as the tiles take it: bfloat16, rows of `columns` values on 16-byte borders.  (In the tiles themselves the conversion of e4m3 through registers
// cost 40 % of their time, for want of registers; this pass, bound by the 3 bytes a value, costs 3 to 5 % of it on 512 tokens of 4096 values.)
template <int XT>
__global__ void __launch_bounds__(256) group_widen_kernel(const void *x, long long ldx, long long T, int m, int columns, uint16_t *out) {
    const long long octets = columns / 8, at = (long long)blockIdx.x * 256 + threadIdx.x;
    if (at >= T * octets) return;
    const long long t = at / octets, col = (at - t * octets) * 8;
    XOctet<XT> v;
    v.template load<false>(x, t * ldx, col, m);
    *(gq_bf16x8 *)(out + t * columns + col) = v.operand();
}

// ---- host ------------------------------------------------------------------------------------------------------------------

// Forward, tiles from so many tokens on.  The few-token kernel reads all codes once for every 32 tokens, the tiles once for 128, with a launch or two more and scratch.
// us, few / tiles: 4096 x 4096 17 tokens 9.8 / 19.2, 64 11.6 / 21.1; 4096 x 11008 17 17 / 25, 64 25.2 / 27.5; gated 11008 x 4096 17 19.6 / 38, 64 33 / 39.5, from e4m3
// 34 / 42.  Beyond 64: 4096 x 11008 65 46 / 28; gated 11008 x 4096 65 40 / 41, 96 51 / 42; on small matrices the tiles are behind for longer (1021 x 2999 65 12 / 20, 128
// 12 / 21; 4096 x 4096 65 19.5 / 23.5), where a border that goes by their size would gain.
constexpr int64_t WIDE_FROM = 65;

bool all_on(int64_t border, std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if ((uintptr_t)p % border) return false;
    return true;
}

// How the tiles of a product are shared out.  `pairs` tiles by four wavefronts a workgroup, two workgroups a compute unit.  Then `whole` tiles and `parts`
// of each of the `rest` by eight wavefronts a workgroup, one workgroup a compute unit.
// us with all tiles of the first kind / with the second: 64 tiles (512 tokens on 4096 x 4096) 70 / 39, 256 (2048 on 4096 x 11008) 178 / 164, 344 (512 on
// gated 11008 x 4096) 105 / 103, 512 (2048 on 8192 x 11008) 299 / 330; with the second for what full rounds of the first leave: 4 of 516 (1500 on 11008 x
// 4096) 175 / 136, 176 of 688 (1024 on gated 11008 x 4096) 180 / 184.  So the first by full rounds, and the second for the rest where it is at most half a
// tile, or one and a half, for every compute unit; alone also up to one.  Its tiles beyond a whole number for every unit are cut along the sum into as
// many parts as there are units left for each, of at least 4 blocks of 128.
// Tiles of 64 tokens (gradients; forward there are always more) where there are no more: 64 on 4096 x 11008 25 us, 29 with half-empty ones.
struct WidePlan {
    int64_t ttiles, pairs, whole, rest;
    int parts, tt;
    size_t scratch() const { return parts > 1 ? (size_t)rest * parts * WIDE_R * tt * 512 * sizeof(gq_float4) : 0; }
    void join_none() { whole += rest, rest = 0, parts = 1; }
};
WidePlan wide_plan(const skim_ctx *ctx, int64_t out, int64_t per, int64_t blocks, int64_t T) {
    WidePlan p;
    static_assert(WIDE_FROM > 64, "forward tiles are of 128 tokens only, and so are the partial sums they write");
    p.tt = T <= 64 ? 2 : 4;
    p.ttiles = (T + 32 * p.tt - 1) / (32 * p.tt);
    const int64_t cu = ctx->num_cu, tiles = (out + per - 1) / per * p.ttiles, left = tiles % (2 * cu);
    const bool second = blocks >= 4 && (tiles <= cu || (2 * left <= 3 * cu && 2 * (left % cu) <= cu));
    p.pairs = second ? tiles - left : tiles;
    p.whole = tiles - p.pairs;
    p.rest = 0;
    p.parts = 1;
    const int64_t rest = p.whole % cu, parts = rest ? std::min<int64_t>(cu / rest, blocks / 4) : 1;
    if (parts > 1) p.whole -= rest, p.rest = rest, p.parts = (int)parts;
    return p;
}

// Whether the tiles can copy rows of x as they are.  (A tile's 128 rows lie within the 2^31 bytes that a copy's offset reaches, which also limits the
// matrices: their widened rows are as long.)
static_assert(127ll * SKIM_GROUP_MAX * 2 + 2 * GQ_COLS < (1ll << 31));
bool wide_takes(const void *x, int x_type, int64_t ldx, int64_t depth) {
    return x_type == SKIM_BF16 && depth % 8 == 0 && ldx % 8 == 0 && ldx <= SKIM_GROUP_MAX && all_on(16, {x});
}
int64_t wide_columns(int64_t depth) { return (depth + 7) / 8 * 8; }
size_t widened_bytes(int64_t depth, int64_t T) { return ((size_t)wide_columns(depth) * T * 2 + 255) / 256 * 256; }

// Of dgate and dup in two pieces: dx in float32, and any dx of up to PIECES_TO tokens, is made of 16 bits of them, as pairs of rows of the tiles.  So few
// tokens leave half a tile empty anyway (gated 11008 x 4096: 1 token 45.6 us, 32 59, 64 82, as stored 44.2, 55 and 69), and their errors do not average: dx of rounded
// gradients is 1.2 to 1.8 times as far off as its own rounding makes it.  For more tokens that is 1.4 times throughout, and the pieces are twice the
// products (65 tokens 80 us as stored, 100 in pieces; 1024 378 and 614): who wants them asks for float32.
constexpr int64_t PIECES_TO = 64;
bool takes_pieces(int64_t T, int dx_type) { return T <= PIECES_TO || dx_type == SKIM_F32; }
size_t piece_bytes(int64_t n, int64_t T) { return ((size_t)gq_row_blocks(n) * GQ_ROWS * 2 * 2 * T * 2 + 255) / 256 * 256; }

skim_status widen_x(skim_ctx *ctx, const void *x, int x_type, int64_t ldx, int64_t T, int64_t depth, void *out) {
    const int64_t columns = wide_columns(depth), groups = (T * (columns / 8) + 255) / 256;
    if (groups > 0xffffff) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%lld tokens of %lld values are too many for one call", (long long)T, (long long)depth);
    if (x_type == SKIM_BF16)
        hipLaunchKernelGGL(group_widen_kernel<SKIM_BF16>, dim3((unsigned)groups), dim3(256), 0, ctx->stream, x, (long long)ldx, (long long)T, (int)depth, (int)columns,
                           (uint16_t *)out);
    else
        hipLaunchKernelGGL(group_widen_kernel<SKIM_E4M3>, dim3((unsigned)groups), dim3(256), 0, ctx->stream, x, (long long)ldx, (long long)T, (int)depth, (int)columns,
                           (uint16_t *)out);
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
}

template <bool DX, int MODE>
skim_status launch_wide(skim_ctx *ctx, MmArgs A, int group, int x_type, int mats, void *scratch, size_t scratch_bytes) {
    const int64_t depth = DX ? A.n : A.m;
    char *room = (char *)scratch;
    if (A.paired) {                                                  // (rows of ours, zeros past the matrix)
    } else if (!wide_takes(A.x, x_type, A.ldx, depth) || (mats == 2 && !wide_takes(A.x2, x_type, A.ldx, depth))) {
        const size_t each = widened_bytes(depth, A.T), need = each * mats;
        if (need > scratch_bytes)
            SKIM_FAIL(ctx, SKIM_ERR_WORKSPACE, "%lld tokens of this type, stride or alignment need %zu bytes of scratch, %zu given", A.T, need, scratch_bytes);
        skim_status st;
        if ((st = widen_x(ctx, A.x, x_type, A.ldx, A.T, depth, room)) != SKIM_OK) return st;
        if (mats == 2 && (st = widen_x(ctx, A.x2, x_type, A.ldx, A.T, depth, room + each)) != SKIM_OK) return st;
        A.x = room;
        A.x2 = room + each;
        A.ldx = wide_columns(depth);
        room += need;
        scratch_bytes -= need;
    }
    // (a launch has fewer than 2^32 threads)
    WidePlan p = wide_plan(ctx, DX ? A.m : A.n, MODE == MM_PLAIN ? 256 : 128, (depth + 127) / 128 * mats, A.T);
    if (p.scratch() > scratch_bytes) p.join_none();
    if (p.pairs > 0xffffff) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%lld tokens are too many for one call", A.T);
    auto go = [&](auto split, auto tokens) -> hipError_t {
        constexpr int KS = decltype(split)::value, TT = decltype(tokens)::value;
        const size_t lds = KS * (2 * wide_x_bytes(TT) + (DX ? 4 * WIDE_A_BYTES : 0));
        auto *k = &group_wide_kernel<DX, MODE, KS, TT>;
        hipError_t e = hipSuccess;
        const unsigned bit = 1u << (DX ? 2 * (KS - 1) + (TT == 4) : 4 + MODE);       // (forward four wavefronts need no more than 64 KB)
        if (lds > 64 * 1024 && !(ctx->wide_lds_enabled & bit)) {
            e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
            if (e == hipSuccess) ctx->wide_lds_enabled |= bit;
        }
        if (e != hipSuccess) return e;
        if (KS == 1)
            hipLaunchKernelGGL(k, dim3((unsigned)p.pairs), dim3(WIDE_THREADS), lds, ctx->stream, A, group, mats, (int)p.ttiles, 0, (int)p.pairs, 0, 1,
                               (gq_float4 *)nullptr);
        else
            hipLaunchKernelGGL(k, dim3((unsigned)(p.whole + p.rest * p.parts)), dim3(2 * WIDE_THREADS), lds, ctx->stream, A, group, mats, (int)p.ttiles, (int)p.pairs,
                               (int)p.whole, (int)p.rest, p.parts, (gq_float4 *)room);
        if (KS == 2 && p.parts > 1)
            hipLaunchKernelGGL((group_join_kernel<DX, MODE, TT>), dim3((unsigned)(p.rest * WIDE_R * TT)), dim3(256), 0, ctx->stream, A, (int)p.ttiles,
                               (int)(p.pairs + p.whole), (int)p.rest, p.parts, (const gq_float4 *)room);
        return hipGetLastError();
    };
    auto by_tokens = [&](auto split) {
        if constexpr (DX)
            if (p.tt == 2) return go(split, std::integral_constant<int, 2>{});
        return go(split, std::integral_constant<int, 4>{});
    };
    if (p.pairs) SKIM_HIP(ctx, by_tokens(std::integral_constant<int, 1>{}));
    if (p.whole + p.rest) SKIM_HIP(ctx, by_tokens(std::integral_constant<int, 2>{}));
    return SKIM_OK;
}

template <int MODE>
skim_status launch_forward(skim_ctx *ctx, MmArgs A, int group, int x_type, void *scratch, size_t scratch_bytes) {
    A.quads = A.n % 4 == 0 && all_on(16, {A.y, A.dgate, A.dup}) && (!A.da || (A.ldda % 4 == 0 && all_on(8, {A.da})));
    constexpr int MATS = MODE == MM_PLAIN ? 1 : 2;
    if (A.T >= WIDE_FROM) return launch_wide<false, MODE>(ctx, A, group, x_type, 1, scratch, scratch_bytes);
    // 16 rows a workgroup, 32 where every row block reads more than 16 tokens; enough wavefronts for 16 a compute unit, no more than there are blocks
    const int nt = A.T <= 16 ? 1 : 2, rt = nt;
    const int64_t chunks = (A.T + 16 * nt - 1) / (16 * nt), groups = (gq_row_blocks(A.n) + rt - 1) / rt * chunks;
    if (groups > 0x7fffffff) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%lld tokens on %lld rows are too many for one call", A.T, A.n);
    int nw = 4;
    while (nw < (nt == 1 ? 16 : 8) && groups * nw < 16ll * ctx->num_cu && nw < gq_col_blocks(A.m)) nw *= 2;
    const size_t lds = (size_t)nw * MATS * (nt == 1 ? 16 * FEW_TOKEN * 4 : rt * nt * 1024);
    const int64_t octet = x_type == SKIM_BF16 ? 16 : 8, es = x_type == SKIM_BF16 ? 2 : 1;
    const bool vec = A.m % 8 == 0 && (A.ldx * es) % octet == 0 && (uintptr_t)A.x % octet == 0;
    with_group(group, [&](auto g) {
        auto go = [&](auto xt, auto ntc, auto v) {
            constexpr int NT = decltype(ntc)::value;
            hipLaunchKernelGGL((group_few_kernel<decltype(xt)::value, NT, decltype(g)::value, MODE, decltype(v)::value>), dim3((unsigned)groups),
                               dim3(64 * nw), lds, ctx->stream, A, (int)chunks);
        };
        auto by_nt = [&](auto xt, auto v) {
            if (nt == 1) go(xt, std::integral_constant<int, 1>{}, v);
            else go(xt, std::integral_constant<int, 2>{}, v);
        };
        auto by_vec = [&](auto xt) {
            if (vec) by_nt(xt, std::true_type{});
            else by_nt(xt, std::false_type{});
        };
        if (x_type == SKIM_BF16) by_vec(std::integral_constant<int, SKIM_BF16>{});
        else by_vec(std::integral_constant<int, SKIM_E4M3>{});
    });
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
}

skim_status launch_dx(skim_ctx *ctx, MmArgs A, int group, int mats, void *scratch, size_t scratch_bytes) {
    A.quads = A.m % 4 == 0 && all_on(16, {A.y});
    return launch_wide<true, MM_PLAIN>(ctx, A, group, SKIM_BF16, mats, scratch, scratch_bytes);
}

skim_status check_x(skim_ctx *ctx, const void *x, int x_type, int64_t ldx, const float *x_scales, int64_t T, int64_t m, const char *who) {
    if (x_type != SKIM_BF16 && x_type != SKIM_E4M3) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: x_type %d is neither SKIM_BF16 nor SKIM_E4M3", who, x_type);
    if (T < 0 || T > 0x7fffffff || ldx < m) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%s: bad shape T=%lld m=%lld ldx=%lld", who, (long long)T, (long long)m, (long long)ldx);
    if (T > 0 && (!x || (x_type == SKIM_E4M3) != (x_scales != nullptr)))
        SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: x must not be NULL, and x_scales is given with e4m3 and only then", who);
    return SKIM_OK;
}

skim_status check_scratch(skim_ctx *ctx, const void *scratch, size_t bytes, const char *who) {
    if ((bytes && !scratch) || ((uintptr_t)scratch & 15)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: scratch must be 16-byte aligned, and not NULL where it has a size", who);
    return SKIM_OK;
}

skim_status check_out(skim_ctx *ctx, const void *y, int y_type, int64_t T, const char *who) {
    if (y_type != SKIM_BF16 && y_type != SKIM_F32) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: the result's type %d is neither SKIM_BF16 nor SKIM_F32", who, y_type);
    if (T > 0 && !y) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: the result must not be NULL", who);
    return SKIM_OK;
}

MmArgs matrix_args(const uint32_t *codes, const uint16_t *scales, const uint32_t *codes2, const uint16_t *scales2, int64_t n, int64_t m) {
    MmArgs A = {};
    A.codes[0] = (const gq_word4 *)codes;
    A.codes[1] = (const gq_word4 *)codes2;
    A.scales[0] = scales;
    A.scales[1] = scales2;
    A.n = n;
    A.m = m;
    return A;
}

}  // namespace

namespace {

bool sizes_taken(const skim_ctx *ctx, int64_t n, int64_t m, int64_t T, int gradients) {
    return ctx && n >= 1 && n <= SKIM_GROUP_MAX && m >= 1 && m <= SKIM_GROUP_MAX && T >= 1 && T <= 0x7fffffff && gradients >= 0 && gradients <= 2;
}
// `convert`: x (to the input: its gradient) goes to the tiles through a copy of its own.
size_t scratch_bytes_of(const skim_ctx *ctx, int64_t n, int64_t m, int64_t T, int gradients, bool convert, int dx_type) {
    const int64_t over_m = (m + 127) / 128, over_n = (n + 127) / 128;
    // forward: that copy, and the partial sums
    const size_t forward = T < WIDE_FROM ? 0
                                         : (convert ? widened_bytes(m, T) : 0) +
                                               std::max(wide_plan(ctx, n, 256, over_m, T).scratch(), wide_plan(ctx, n, 128, over_m, T).scratch());
    if (gradients == 0) return forward;
    // to the input: the same for one gradient, or for two whose rows may not be multiples of 8
    if (gradients == 1) return (convert ? widened_bytes(n, T) : 0) + wide_plan(ctx, m, 256, over_n, T).scratch();
    if (takes_pieces(T, dx_type)) return piece_bytes(n, T) + std::max(forward, wide_plan(ctx, m, 256, 2 * over_n, 2 * T).scratch());
    return std::max(forward, (n % 8 ? 2 * widened_bytes(n, T) : 0) + wide_plan(ctx, m, 256, 2 * over_n, T).scratch());
}

}  // namespace

extern "C" size_t skim_group_scratch_bytes(const skim_ctx *ctx, int64_t n, int64_t m, int64_t T, int gradients) {
    return sizes_taken(ctx, n, m, T, gradients) ? scratch_bytes_of(ctx, n, m, T, gradients, true, SKIM_BF16) : 0;
}

extern "C" size_t skim_group_scratch_bytes_for(const skim_ctx *ctx, int64_t n, int64_t m, int64_t T, int gradients, const void *x, int x_type, int64_t ldx,
                                               int dx_type) {
    const int64_t columns = gradients == 1 ? n : m;
    if (!sizes_taken(ctx, n, m, T, gradients) || (x_type != SKIM_BF16 && (x_type != SKIM_E4M3 || gradients == 1)) || ldx < columns) return 0;
    if (gradients && dx_type != SKIM_BF16 && dx_type != SKIM_F32) return 0;
    return scratch_bytes_of(ctx, n, m, T, gradients, !wide_takes(x, x_type, ldx, columns), dx_type);
}

extern "C" skim_status skim_group_matmul(skim_ctx *ctx, const uint32_t *codes, const uint16_t *scales_bf16, int64_t n, int64_t m, int group,
                                         const void *x, int x_type, int64_t ldx, const float *x_scales, int64_t T, void *y, int y_type,
                                         void *scratch, size_t scratch_bytes) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_matmul";
    if ((st = skim_group_check(ctx, codes, scales_bf16, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, x, x_type, ldx, x_scales, T, m, who)) != SKIM_OK) return st;
    if ((st = check_out(ctx, y, y_type, T, who)) != SKIM_OK) return st;
    if ((st = check_scratch(ctx, scratch, scratch_bytes, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    MmArgs A = matrix_args(codes, scales_bf16, nullptr, nullptr, n, m);
    A.x = x, A.ldx = ldx, A.x_scales = x_scales, A.T = T, A.y = y, A.y_f32 = y_type == SKIM_F32;
    return launch_forward<MM_PLAIN>(ctx, A, group, x_type, scratch, scratch_bytes);
}

extern "C" skim_status skim_group_matmul_dx(skim_ctx *ctx, const uint32_t *codes, const uint16_t *scales_bf16, int64_t n, int64_t m, int group,
                                            const uint16_t *dy_bf16, int64_t lddy, int64_t T, void *dx, int dx_type, void *scratch, size_t scratch_bytes) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_matmul_dx";
    if ((st = skim_group_check(ctx, codes, scales_bf16, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, dy_bf16, SKIM_BF16, lddy, nullptr, T, n, who)) != SKIM_OK) return st;
    if ((st = check_out(ctx, dx, dx_type, T, who)) != SKIM_OK) return st;
    if ((st = check_scratch(ctx, scratch, scratch_bytes, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    MmArgs A = matrix_args(codes, scales_bf16, nullptr, nullptr, n, m);
    A.x = dy_bf16, A.ldx = lddy, A.T = T, A.y = dx, A.y_f32 = dx_type == SKIM_F32;
    return launch_dx(ctx, A, group, 1, scratch, scratch_bytes);
}

extern "C" skim_status skim_group_glu(skim_ctx *ctx, const uint32_t *gate_codes, const uint16_t *gate_scales, const uint32_t *up_codes,
                                      const uint16_t *up_scales, int64_t n, int64_t m, int group, const void *x, int x_type, int64_t ldx,
                                      const float *x_scales, int64_t T, void *a, int a_type, void *scratch, size_t scratch_bytes) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_glu";
    if ((st = skim_group_check(ctx, gate_codes, gate_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = skim_group_check(ctx, up_codes, up_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, x, x_type, ldx, x_scales, T, m, who)) != SKIM_OK) return st;
    if ((st = check_out(ctx, a, a_type, T, who)) != SKIM_OK) return st;
    if ((st = check_scratch(ctx, scratch, scratch_bytes, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    MmArgs A = matrix_args(gate_codes, gate_scales, up_codes, up_scales, n, m);
    A.x = x, A.ldx = ldx, A.x_scales = x_scales, A.T = T, A.y = a, A.y_f32 = a_type == SKIM_F32;
    return launch_forward<MM_GLU>(ctx, A, group, x_type, scratch, scratch_bytes);
}

extern "C" skim_status skim_group_glu_backward(skim_ctx *ctx, const uint32_t *gate_codes, const uint16_t *gate_scales, const uint32_t *up_codes,
                                               const uint16_t *up_scales, int64_t n, int64_t m, int group, const void *x, int x_type,
                                               int64_t ldx, const float *x_scales, int64_t T, const uint16_t *da_bf16, int64_t ldda,
                                               uint16_t *dgate_bf16, uint16_t *dup_bf16, void *dx, int dx_type, void *scratch, size_t scratch_bytes) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_glu_backward";
    if ((st = skim_group_check(ctx, gate_codes, gate_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = skim_group_check(ctx, up_codes, up_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, x, x_type, ldx, x_scales, T, m, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, da_bf16, SKIM_BF16, ldda, nullptr, T, n, who)) != SKIM_OK) return st;
    if (dx_type != SKIM_BF16 && dx_type != SKIM_F32) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: the result's type %d is neither SKIM_BF16 nor SKIM_F32", who, dx_type);
    if ((st = check_scratch(ctx, scratch, scratch_bytes, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    if (!dgate_bf16 || !dup_bf16 || !all_on(16, {dgate_bf16, dup_bf16}))
        SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: dgate and dup must not be NULL, and 16-byte aligned", who);
    MmArgs A = matrix_args(gate_codes, gate_scales, up_codes, up_scales, n, m);
    A.x = x, A.ldx = ldx, A.x_scales = x_scales, A.T = T, A.da = da_bf16, A.ldda = ldda, A.dgate = dgate_bf16, A.dup = dup_bf16;
    // (the pieces where there is room for them next to the copy of x that the projections cannot do without)
    const size_t pieces = dx && takes_pieces(T, dx_type) ? piece_bytes(n, T) : 0;
    if (pieces && pieces + (T < WIDE_FROM || wide_takes(x, x_type, ldx, m) ? 0 : widened_bytes(m, T)) <= scratch_bytes) {
        A.pieces = (uint16_t *)scratch, A.ldp = gq_row_blocks(n) * GQ_ROWS;
        scratch = (char *)scratch + pieces;
        scratch_bytes -= pieces;
    }
    // (refused before anything is written: rows of dgate and dup that the tiles cannot copy need one of their own)
    if (dx && !A.pieces && n % 8 && 2 * widened_bytes(n, T) > scratch_bytes)
        SKIM_FAIL(ctx, SKIM_ERR_WORKSPACE, "%s: dx of %lld tokens on %lld rows needs %zu bytes of scratch, %zu given", who, (long long)T, (long long)n, 2 * widened_bytes(n, T),
                  scratch_bytes);
    if ((st = launch_forward<MM_GLU_BACK>(ctx, A, group, x_type, scratch, scratch_bytes)) != SKIM_OK || !dx) return st;
    A.x = dgate_bf16, A.x2 = dup_bf16, A.ldx = n, A.x_scales = nullptr, A.y = dx, A.y_f32 = dx_type == SKIM_F32;
    if (A.pieces) A.x = A.pieces, A.x2 = A.pieces + 2 * T * A.ldp, A.ldx = A.ldp, A.T = 2 * T, A.paired = true;
    return launch_dx(ctx, A, group, 2, scratch, scratch_bytes);
}
