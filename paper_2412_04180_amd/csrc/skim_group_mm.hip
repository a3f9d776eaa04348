// Products with 4-bit weights and group scales (layout: skim_group.h), for one token to many:
//   y = x W^T,   a = silu(x Wg^T) * (x Wu^T),   dx = dy W,   and the backward pass of a.
// All of them run on the matrix cores with exact operands: a code is a whole number, a code times its scale a bfloat16, and x comes in
// bfloat16 or e4m3.  Sums are float32; the one rounding is that of a result to its type.
#include "skim_group.h"
#include "skim_tiles.h"

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
    bool quads;                  // results (and da) can be taken in fours
};

enum { MM_PLAIN, MM_GLU, MM_GLU_BACK };

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float from_bf16(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + expf(-g)); }

// Four neighbouring results of a token, of rows `row` .. row + 3 of `rows`; the token is inside.  Sums come times `by`.
template <int MODE>
__device__ __forceinline__ void finish4(const MmArgs &A, long long t, long long row, long long rows, gq_float4 g, gq_float4 u, float by) {
    if (row >= rows) return;
    const long long at = t * rows + row;
    const bool quad = A.quads;                    // rows come in fours, everything on borders of fours
    if constexpr (MODE == MM_GLU_BACK) {
        gq_short4 d = {}, dg, du;
        const uint16_t *p = A.da + t * A.ldda + row;
        if (quad) d = *(const gq_short4 *)p;
        else
            for (int i = 0; i < 4; ++i)
                if (row + i < rows) d[i] = (short)p[i];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float gi = g[i] * by, ui = u[i] * by, di = from_bf16((uint16_t)d[i]), s = sigmoid(gi);
            dg[i] = (short)to_bf16(di * ui * s * fmaf(gi, 1.f - s, 1.f));
            du[i] = (short)to_bf16(di * gi * s);
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

// The codes of a word, whole numbers in bfloat16.
__device__ __forceinline__ gq_bf16x8 code_operand(uint32_t w) {
    const uint32_t lo = gq_low(w), hi = gq_high(w);
    const gq_word4 u{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false)),
                     __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true))};
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

// 8 values of a row of x from column col on as a matrix operand, zeros past column m.  VEC: rows start on borders of the octet's size and m is a
// multiple of 8.
template <int XT, bool VEC>
__device__ __forceinline__ gq_bf16x8 load_x(const void *x, long long row0, long long col, long long m) {
    typedef std::conditional_t<XT == SKIM_BF16, uint16_t, uint8_t> E;
    typedef std::conditional_t<XT == SKIM_BF16, gq_word4, gq_word2> V;
    const E *p = (const E *)x + row0 + col;
    V v = {};
    if constexpr (VEC) {
        if (col < m) v = *(const V *)p;
    } else {
        if (col + 8 <= m) {
            __builtin_memcpy(&v, p, sizeof(v));              // (one load, of any alignment)
        } else {
            E e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = col + i < m ? p[i] : (E)0;
            __builtin_memcpy(&v, e, sizeof(v));
        }
    }
    if constexpr (XT == SKIM_BF16) return __builtin_bit_cast(gq_bf16x8, v);
    else return widen(v);
}

// ---- few tokens ----------------------------------------------------------------------------------------------------------

// A workgroup makes 16 rows of the result for 16 NT tokens; its wavefronts share the columns block by block, and their sums are added
// up in LDS in the order of the wavefronts.
template <int XT, int NT, int G, int MODE, bool VEC>
__global__ void __launch_bounds__(1024) group_few_kernel(MmArgs A, int chunks) {
    constexpr int MATS = MODE == MM_PLAIN ? 1 : 2;
    extern __shared__ __align__(16) unsigned char few_lds[];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, nw = blockDim.x >> 6;
    const int c = lane >> 4, l16 = lane & 15;
    const long long rt = blockIdx.x / chunks, t0 = (long long)(blockIdx.x % chunks) * (16 * NT);
    const long long kbs = gq_col_blocks(A.m), n16 = gq_row_blocks(A.n) * GQ_ROWS;
    long long xrow[NT];
#pragma unroll
    for (int j = 0; j < NT; ++j) xrow[j] = min(t0 + 16 * j + l16, A.T - 1) * A.ldx;
    gq_float4 acc[MATS][NT] = {};
    for (long long kb = wave; kb < kbs; kb += nw) {
        gq_word4 w[MATS];
#pragma unroll
        for (int a = 0; a < MATS; ++a) w[a] = A.codes[a][(rt * kbs + kb) * 64 + lane];
#pragma unroll
        for (int g = 0; g < GQ_COLS / G; ++g) {
            gq_float4 d[MATS][NT] = {};
#pragma unroll
            for (int k = g * (G / 32); k < (g + 1) * (G / 32); ++k) {
                gq_bf16x8 b[NT];
#pragma unroll
                for (int j = 0; j < NT; ++j) b[j] = load_x<XT, VEC>(A.x, xrow[j], kb * GQ_COLS + 32 * k + 8 * c, A.m);
#pragma unroll
                for (int a = 0; a < MATS; ++a) {
                    const gq_bf16x8 q = code_operand(w[a][k]);
#pragma unroll
                    for (int j = 0; j < NT; ++j) d[a][j] = mfma(q, b[j], d[a][j]);
                }
            }
#pragma unroll
            for (int a = 0; a < MATS; ++a) {
                const gq_word2 s = *(const gq_word2 *)(A.scales[a] + (kb * (GQ_COLS / G) + g) * n16 + rt * GQ_ROWS + 4 * c);
                const gq_float4 f{gq_scale(s[0] & 0xFFFF), __uint_as_float(s[0] & 0xFFFF0000u), gq_scale(s[1] & 0xFFFF), __uint_as_float(s[1] & 0xFFFF0000u)};
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[a][j][i] = fmaf(f[i], d[a][j][i], acc[a][j][i]);
            }
        }
    }
    constexpr int E = NT * 64;           // fours of a wavefront's sums, for one matrix
    gq_float4 *red = (gq_float4 *)few_lds;
#pragma unroll
    for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int j = 0; j < NT; ++j) red[((wave * MATS + a) * NT + j) * 64 + lane] = acc[a][j];
    __syncthreads();
    for (int e = tid; e < E; e += blockDim.x) {
        gq_float4 v[MATS] = {};
#pragma unroll
        for (int a = 0; a < MATS; ++a)
            for (int w = 0; w < nw; ++w) v[a] += red[(w * MATS + a) * E + e];
        const int el = e & 63;
        const long long t = t0 + 16 * (e >> 6) + (el & 15);
        if (t < A.T) finish4<MODE>(A, t, rt * GQ_ROWS + 4 * (el >> 4), A.n, v[0], v[MATS - 1], XT == SKIM_E4M3 ? A.x_scales[t] : 1.f);
    }
}

// ---- many tokens -----------------------------------------------------------------------------------------------------------

// y = x W^T, the gated block and its backward pass, and dx = dy W (+ dy2 W2), on tiles of the matrix cores.  A workgroup of four wavefronts makes
// 256 rows of W (128 of gate and the same of up; for dx 256 columns) for 128 tokens, a wavefront 64 of them: 4 x 8 accumulator
// tiles of 16 x 16.
// The tokens' operand: 128 columns of x (rows of dy's matrix for dx) go to LDS a block ahead, in bfloat16.  The weights' operand never is in
// memory: codes come into registers a block ahead, one 16-byte load for 32 of them, and are taken apart there, times their scale, into
// operands.  For dx, where a lane needs 8 rows of one column, they pass through 4 KB of LDS of the wavefront's own and come back by the transposing read.
// LDS rows of a token are 256 bytes; its 16-byte unit u is at place u ^ (token % 16), so that 16 tokens' units of one column octet lie in different banks.
constexpr int WIDE_TOKENS = 128, WIDE_THREADS = 256, WIDE_TT = WIDE_TOKENS / 16, WIDE_RT = 4;
constexpr int WIDE_X_BYTES = WIDE_TOKENS * GQ_COLS * 2;              // of one block: 32 KB
constexpr int WIDE_A_BYTES = 32 * 64 * 2;                            // dx: a wavefront's 32 rows x 64 columns
constexpr int WIDE_UNITS = WIDE_X_BYTES / 16 / WIDE_THREADS;         // 16-byte units of a thread: 8

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

enum { STAGE_COPY, STAGE_BF16, STAGE_E4M3 };       // straight into LDS; through registers: bfloat16 of any alignment, e4m3

template <bool DX, int MODE, int STAGE>
__global__ void __launch_bounds__(WIDE_THREADS) __attribute__((amdgpu_waves_per_eu(2, 2))) group_wide_kernel(MmArgs A, int group, int mats, int ttiles) {
    extern __shared__ __align__(16) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane >> 4, l16 = lane & 15;
    const int tile = xcd_order(blockIdx.x, gridDim.x);
    const long long ob = tile / ttiles, t0 = (long long)(tile % ttiles) * WIDE_TOKENS;
    const long long kbs = gq_col_blocks(A.m), rbs = gq_row_blocks(A.n), n16 = rbs * GQ_ROWS;
    const long long depth = DX ? A.n : A.m;                          // summed over
    const int blocks = (int)((depth + 127) / 128), total = DX ? blocks * mats : blocks;
    const int per = GQ_COLS / group;

    // ---- the tokens' operand
    const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_byte *)smem;
    const int es = STAGE == STAGE_E4M3 ? 1 : 2;
    uint32_t voff[WIDE_UNITS];
    gq_word2 held[WIDE_UNITS];                                       // e4m3: the next block's units on their way
#pragma unroll
    for (int i = 0; i < WIDE_UNITS; ++i) {
        const int t = (wave * WIDE_UNITS + i) * 4 + c;               // (copies: 4 tokens of 16 units each)
        voff[i] = (uint32_t)(min((long long)t, A.T - 1 - t0) * A.ldx * es) + (uint32_t)((l16 ^ (t & 15)) * 8 * es);
    }
    auto xbase = [&](int kb) -> const unsigned char * {
        const int a = DX ? kb / blocks : 0;
        return (const unsigned char *)(a ? A.x2 : A.x) + (t0 * A.ldx + (long long)(kb - a * blocks) * GQ_COLS) * es;
    };
    auto columns_left = [&](int kb) -> int { return (int)min(depth - (long long)(kb % blocks) * GQ_COLS, 128ll); };
    auto unit_column = [&](int i) -> int { return (l16 ^ ((i * 4 + c) & 15)) * 8; };
    auto stage = [&](int kb) {
        const int left = columns_left(kb);
        const uint32_t dst = lds0 + (uint32_t)(kb & 1) * WIDE_X_BYTES + (uint32_t)wave * (WIDE_X_BYTES / 4);
        if constexpr (STAGE == STAGE_COPY) {
            const LdsSource src{(uint64_t)(uintptr_t)xbase(kb), 0x7FFFFFFF};
            const int4v rs = src.rsrc();
#pragma unroll
            for (int i = 0; i < WIDE_UNITS; ++i) copy_to_lds(dst + i * 1024, unit_column(i) < left ? voff[i] : 0x80000000u, rs);
        } else if constexpr (STAGE == STAGE_E4M3) {
            const unsigned char *x = xbase(kb);
#pragma unroll
            for (int i = 0; i < WIDE_UNITS; ++i) {
                held[i] = gq_word2{};
                const int over = unit_column(i) - left;
                if (over <= -8) __builtin_memcpy(&held[i], x + voff[i], 8);
                else if (over < 0) {
                    uint8_t e[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) e[q] = over + q < 0 ? x[voff[i] + q] : (uint8_t)0;
                    __builtin_memcpy(&held[i], e, 8);
                }
            }
        } else {
            const unsigned char *x = xbase(kb);
#pragma unroll
            for (int i = 0; i < WIDE_UNITS; ++i) {
                gq_word4 v = {};
                const int over = unit_column(i) - left;
                if (over <= -8) __builtin_memcpy(&v, x + voff[i], 16);
                else if (over < 0) {
                    uint16_t e[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) e[q] = over + q < 0 ? ((const uint16_t *)(x + voff[i]))[q] : (uint16_t)0;
                    __builtin_memcpy(&v, e, 16);
                }
                *(gq_word4 *)(smem + (dst - lds0) + i * 1024 + lane * 16) = v;
            }
        }
    };
    auto store_held = [&](int kb) {
        unsigned char *dst = smem + (kb & 1) * WIDE_X_BYTES + wave * (WIDE_X_BYTES / 4);
#pragma unroll
        for (int i = 0; i < WIDE_UNITS; ++i) *(gq_bf16x8 *)(dst + i * 1024 + lane * 16) = widen(held[i]);
    };

    // ---- the weights' operand
    constexpr int PAIR = MODE == MM_PLAIN ? 4 : 2;                   // row blocks of a wavefront, of one matrix
    const long long rb0 = (ob * 4 + wave) * PAIR;
    const long long cb = min(ob * 2 + (wave >> 1), kbs - 1);         // dx: column block, and which half of it
    const int half = wave & 1;
    gq_word4 next[4];
    uint32_t nscale[4];
    auto load_codes = [&](int kb) {
        if constexpr (DX) {
            const int a = kb / blocks;
            const long long rb = (long long)(kb - a * blocks) * 8;
            const uint32_t *w = (const uint32_t *)A.codes[a] + (cb * 64 + lane) * 4 + 2 * half;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                gq_word2 v = {};
                if (rb + j < rbs) v = *(const gq_word2 *)(w + (rb + j) * kbs * 256);
                next[j >> 1][2 * (j & 1)] = v[0];
                next[j >> 1][2 * (j & 1) + 1] = v[1];
            }
#pragma unroll
            for (int q = 0; q < 4; ++q)                              // word q / 2 of the half, rows q % 2 * 64 + lane
                nscale[q] = A.scales[a][(cb * per + (64 * half + 32 * (q >> 1)) / group) * n16 + min(rb * GQ_ROWS + 64 * (q & 1) + lane, n16 - 1)];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) next[i] = A.codes[i / PAIR][(min(rb0 + i % PAIR, rbs - 1) * kbs + kb) * 64 + lane];
            const uint16_t *s = A.scales[c / PAIR] + min(rb0 + c % PAIR, rbs - 1) * GQ_ROWS + l16;
#pragma unroll
            for (int q = 0; q < 4; ++q) nscale[q] = s[((long long)kb * per + 32 * q / group) * n16];
        }
    };
    gq_word4 cur[4];
    uint32_t cscale[4];
    unsigned char *mine = smem + 2 * WIDE_X_BYTES + wave * WIDE_A_BYTES;
    auto flip = [](int row) { return (2 * (row & 3)) ^ ((row >> 2) & 1); };    // dx: unit u of a row is at u ^ flip(row)
    auto operands = [&](int k, gq_bf16x8 (&a)[4]) {
        if constexpr (DX) {
#pragma unroll
            for (int p = 0; p < 4; ++p) {                            // row block p / 2 of the step, word p % 2
                const int j = 2 * k + (p >> 1), q = p & 1;
                const float s = gq_scale((uint32_t)__shfl((int)cscale[2 * q + (j >> 2)], 16 * (j & 3) + l16, 64));
                const int row = 16 * (p >> 1) + l16;
                *(gq_word4 *)(mine + row * 128 + ((4 * q + c) ^ flip(row)) * 16) = weight_operand(cur[j >> 1][2 * (j & 1) + q], s);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = 8 * c + (l16 >> 2), u = 2 * i + ((l16 & 3) >> 1);
                const gq_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(mine + row * 128 + (u ^ flip(row)) * 16 + (l16 & 1) * 8));
                const gq_short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)(mine + (row + 4) * 128 + (u ^ flip(row + 4)) * 16 + (l16 & 1) * 8));
                a[i] = __builtin_bit_cast(gq_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float s = gq_scale((uint32_t)__shfl((int)cscale[k], 16 * i + l16, 64));
                a[i] = __builtin_bit_cast(gq_bf16x8, weight_operand(cur[i][k], s));
            }
        }
    };

    gq_float4 acc[WIDE_RT][WIDE_TT] = {};
    stage(0);
    load_codes(0);
    if constexpr (STAGE == STAGE_E4M3) store_held(0);
    for (int kb = 0; kb < total; ++kb) {
        // this block's copies have landed, its codes too, and everybody is done with the block before, whose place the next one takes
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cur[i] = next[i];
            cscale[i] = nscale[i];
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier"
                     : "+v"(cur[0]), "+v"(cur[1]), "+v"(cur[2]), "+v"(cur[3]), "+v"(cscale[0]), "+v"(cscale[1]), "+v"(cscale[2]), "+v"(cscale[3])
                     :
                     : "memory");
        if (kb + 1 < total) {
            stage(kb + 1);
            load_codes(kb + 1);
        }
        const unsigned char *xb = smem + (kb & 1) * WIDE_X_BYTES + l16 * 256;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            gq_bf16x8 a[4];
            operands(k, a);
#pragma unroll
            for (int j = 0; j < WIDE_TT; ++j) {
                const gq_bf16x8 b = *(const gq_bf16x8 *)(xb + j * 4096 + (((4 * k + c) ^ l16) << 4));
#pragma unroll
                for (int i = 0; i < WIDE_RT; ++i) acc[i][j] = mfma(a[i], b, acc[i][j]);
            }
        }
        if constexpr (STAGE == STAGE_E4M3) {
            if (kb + 1 < total) store_held(kb + 1);
        }
    }
#pragma unroll
    for (int j = 0; j < WIDE_TT; ++j) {
        const long long t = t0 + 16 * j + l16;
        if (t >= A.T) continue;
        const float by = STAGE == STAGE_E4M3 ? A.x_scales[t] : 1.f;
        if constexpr (DX) {
#pragma unroll
            for (int i = 0; i < 4; ++i) finish4<MM_PLAIN>(A, t, (ob * 4 + wave) * 64 + 16 * i + 4 * c, A.m, acc[i][j], acc[i][j], 1.f);
        } else {
#pragma unroll
            for (int i = 0; i < PAIR; ++i) finish4<MODE>(A, t, (rb0 + i) * GQ_ROWS + 4 * c, A.n, acc[i][j], acc[MODE == MM_PLAIN ? i : i + PAIR][j], by);
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

template <typename F>
void with_group(int group, F &&f) {
    if (group == 32) f(std::integral_constant<int, 32>{});
    else if (group == 64) f(std::integral_constant<int, 64>{});
    else f(std::integral_constant<int, 128>{});
}

// From so many tokens on the tiles of 128 pay.
constexpr int64_t WIDE_FROM = 65;

bool all_on(int64_t border, std::initializer_list<const void *> ps) {
    for (const void *p : ps)
        if ((uintptr_t)p % border) return false;
    return true;
}

template <bool DX, int MODE>
skim_status launch_wide(skim_ctx *ctx, const MmArgs &A, int group, int x_type, int mats) {
    const int64_t out = DX ? A.m : A.n, per = MODE == MM_PLAIN ? 256 : 128;
    const int64_t ttiles = (A.T + WIDE_TOKENS - 1) / WIDE_TOKENS, tiles = (out + per - 1) / per * ttiles, depth = DX ? A.n : A.m;
    if (tiles > 0x7fffffff || A.ldx >= (1 << 23) || depth > (1 << 24))
        SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%lld tokens of row stride %lld are too many for one call", A.T, A.ldx);
    const size_t lds = 2 * WIDE_X_BYTES + (DX ? 4 * WIDE_A_BYTES : 0);
    const bool copy = x_type == SKIM_BF16 && depth % 8 == 0 && A.ldx % 8 == 0 && all_on(16, {A.x, A.x2});
    auto go = [&](auto stage) -> hipError_t {
        auto *k = &group_wide_kernel<DX, MODE, decltype(stage)::value>;
        hipError_t e = hipSuccess;
        if (lds > 64 * 1024) e = hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (e == hipSuccess) hipLaunchKernelGGL(k, dim3((unsigned)tiles), dim3(WIDE_THREADS), lds, ctx->stream, A, group, mats, (int)ttiles);
        return e;
    };
    hipError_t e;
    if (copy) e = go(std::integral_constant<int, STAGE_COPY>{});
    else if (x_type == SKIM_BF16) e = go(std::integral_constant<int, STAGE_BF16>{});
    else if constexpr (!DX) e = go(std::integral_constant<int, STAGE_E4M3>{});
    else SKIM_FAIL(ctx, SKIM_ERR_ARG, "gradients are bfloat16");
    SKIM_HIP(ctx, e);
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
}

template <int MODE>
skim_status launch_forward(skim_ctx *ctx, MmArgs A, int group, int x_type) {
    A.quads = A.n % 4 == 0 && all_on(16, {A.y, A.dgate, A.dup}) && (!A.da || (A.ldda % 4 == 0 && all_on(8, {A.da})));
    constexpr int MATS = MODE == MM_PLAIN ? 1 : 2;
    if (A.T >= WIDE_FROM) return launch_wide<false, MODE>(ctx, A, group, x_type, 1);
    const int nt = A.T <= 16 ? 1 : A.T <= 32 ? 2 : 4;
    const int64_t chunks = (A.T + 16 * nt - 1) / (16 * nt), groups = gq_row_blocks(A.n) * chunks;
    if (groups > 0x7fffffff) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%lld tokens on %lld rows are too many for one call", A.T, A.n);
    int nw = 4;
    while (nw < 16 && groups * nw < 8ll * ctx->num_cu && nw < gq_col_blocks(A.m) && nw * MATS * nt * 2048 <= 65536) nw *= 2;
    const size_t lds = (size_t)nw * MATS * nt * 1024;
    const int64_t octet = x_type == SKIM_BF16 ? 16 : 8, es = x_type == SKIM_BF16 ? 2 : 1;
    const bool vec = A.m % 8 == 0 && (A.ldx * es) % octet == 0 && (uintptr_t)A.x % octet == 0;
    with_group(group, [&](auto g) {
        auto go = [&](auto xt, auto ntc, auto v) {
            hipLaunchKernelGGL((group_few_kernel<decltype(xt)::value, decltype(ntc)::value, decltype(g)::value, MODE, decltype(v)::value>), dim3((unsigned)groups),
                               dim3(64 * nw), lds, ctx->stream, A, (int)chunks);
        };
        auto by_nt = [&](auto xt, auto v) {
            if (nt == 1) go(xt, std::integral_constant<int, 1>{}, v);
            else if (nt == 2) go(xt, std::integral_constant<int, 2>{}, v);
            else go(xt, std::integral_constant<int, 4>{}, v);
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

skim_status launch_dx(skim_ctx *ctx, MmArgs A, int group, int mats) {
    A.quads = A.m % 4 == 0 && all_on(16, {A.y});
    return launch_wide<true, MM_PLAIN>(ctx, A, group, SKIM_BF16, mats);
}

skim_status check_x(skim_ctx *ctx, const void *x, int x_type, int64_t ldx, const float *x_scales, int64_t T, int64_t m, const char *who) {
    if (x_type != SKIM_BF16 && x_type != SKIM_E4M3) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: x_type %d is neither SKIM_BF16 nor SKIM_E4M3", who, x_type);
    if (T < 0 || T > 0x7fffffff || ldx < m) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%s: bad shape T=%lld m=%lld ldx=%lld", who, (long long)T, (long long)m, (long long)ldx);
    if (T > 0 && (!x || (x_type == SKIM_E4M3) != (x_scales != nullptr)))
        SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: x must not be NULL, and x_scales is given with e4m3 and only then", who);
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

extern "C" skim_status skim_group_matmul(skim_ctx *ctx, const uint32_t *codes, const uint16_t *scales_bf16, int64_t n, int64_t m, int group,
                                         const void *x, int x_type, int64_t ldx, const float *x_scales, int64_t T, void *y, int y_type) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_matmul";
    if ((st = skim_group_check(ctx, codes, scales_bf16, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, x, x_type, ldx, x_scales, T, m, who)) != SKIM_OK) return st;
    if ((st = check_out(ctx, y, y_type, T, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    MmArgs A = matrix_args(codes, scales_bf16, nullptr, nullptr, n, m);
    A.x = x, A.ldx = ldx, A.x_scales = x_scales, A.T = T, A.y = y, A.y_f32 = y_type == SKIM_F32;
    return launch_forward<MM_PLAIN>(ctx, A, group, x_type);
}

extern "C" skim_status skim_group_matmul_dx(skim_ctx *ctx, const uint32_t *codes, const uint16_t *scales_bf16, int64_t n, int64_t m, int group,
                                            const uint16_t *dy_bf16, int64_t lddy, int64_t T, void *dx, int dx_type) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_matmul_dx";
    if ((st = skim_group_check(ctx, codes, scales_bf16, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, dy_bf16, SKIM_BF16, lddy, nullptr, T, n, who)) != SKIM_OK) return st;
    if ((st = check_out(ctx, dx, dx_type, T, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    MmArgs A = matrix_args(codes, scales_bf16, nullptr, nullptr, n, m);
    A.x = dy_bf16, A.ldx = lddy, A.T = T, A.y = dx, A.y_f32 = dx_type == SKIM_F32;
    return launch_dx(ctx, A, group, 1);
}

extern "C" skim_status skim_group_glu(skim_ctx *ctx, const uint32_t *gate_codes, const uint16_t *gate_scales, const uint32_t *up_codes,
                                      const uint16_t *up_scales, int64_t n, int64_t m, int group, const void *x, int x_type, int64_t ldx,
                                      const float *x_scales, int64_t T, void *a, int a_type) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_glu";
    if ((st = skim_group_check(ctx, gate_codes, gate_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = skim_group_check(ctx, up_codes, up_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, x, x_type, ldx, x_scales, T, m, who)) != SKIM_OK) return st;
    if ((st = check_out(ctx, a, a_type, T, who)) != SKIM_OK) return st;
    if (T == 0) return SKIM_OK;
    MmArgs A = matrix_args(gate_codes, gate_scales, up_codes, up_scales, n, m);
    A.x = x, A.ldx = ldx, A.x_scales = x_scales, A.T = T, A.y = a, A.y_f32 = a_type == SKIM_F32;
    return launch_forward<MM_GLU>(ctx, A, group, x_type);
}

extern "C" skim_status skim_group_glu_backward(skim_ctx *ctx, const uint32_t *gate_codes, const uint16_t *gate_scales, const uint32_t *up_codes,
                                               const uint16_t *up_scales, int64_t n, int64_t m, int group, const void *x, int x_type,
                                               int64_t ldx, const float *x_scales, int64_t T, const uint16_t *da_bf16, int64_t ldda,
                                               uint16_t *dgate_bf16, uint16_t *dup_bf16, void *dx, int dx_type) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    const char *who = "skim_group_glu_backward";
    if ((st = skim_group_check(ctx, gate_codes, gate_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = skim_group_check(ctx, up_codes, up_scales, n, m, group, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, x, x_type, ldx, x_scales, T, m, who)) != SKIM_OK) return st;
    if ((st = check_x(ctx, da_bf16, SKIM_BF16, ldda, nullptr, T, n, who)) != SKIM_OK) return st;
    if (dx_type != SKIM_BF16 && dx_type != SKIM_F32) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: the result's type %d is neither SKIM_BF16 nor SKIM_F32", who, dx_type);
    if (T == 0) return SKIM_OK;
    if (!dgate_bf16 || !dup_bf16) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: dgate and dup must not be NULL", who);
    MmArgs A = matrix_args(gate_codes, gate_scales, up_codes, up_scales, n, m);
    A.x = x, A.ldx = ldx, A.x_scales = x_scales, A.T = T, A.da = da_bf16, A.ldda = ldda, A.dgate = dgate_bf16, A.dup = dup_bf16;
    if ((st = launch_forward<MM_GLU_BACK>(ctx, A, group, x_type)) != SKIM_OK || !dx) return st;
    A.x = dgate_bf16, A.x2 = dup_bf16, A.ldx = n, A.y = dx, A.y_f32 = dx_type == SKIM_F32;
    return launch_dx(ctx, A, group, 2);
}
