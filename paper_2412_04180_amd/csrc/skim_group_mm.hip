// Products with 4-bit weights and group scales (layout: skim_group.h), for one token to many:
//   y = x W^T,   a = silu(x Wg^T) * (x Wu^T),   dx = dy W,   and the backward pass of a.
// All of them run on the matrix cores with exact operands: a code is a whole number, a code times its scale a bfloat16, and x comes in
// bfloat16 or e4m3.  Sums are float32; the one rounding is that of a result to its type.
#include "skim_group.h"

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
};

enum { MM_PLAIN, MM_GLU, MM_GLU_BACK };

__device__ __forceinline__ uint16_t to_bf16(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float from_bf16(uint16_t b) { return __uint_as_float((uint32_t)b << 16); }
__device__ __forceinline__ float sigmoid(float g) { return 1.f / (1.f + expf(-g)); }

// One result: row and token are inside.
template <int MODE>
__device__ __forceinline__ void finish(const MmArgs &A, long long t, long long row, float g, float u) {
    if (MODE == MM_GLU_BACK) {
        const float d = from_bf16(A.da[t * A.ldda + row]), s = sigmoid(g);
        A.dgate[t * A.n + row] = to_bf16(d * u * s * fmaf(g, 1.f - s, 1.f));
        A.dup[t * A.n + row] = to_bf16(d * g * s);
        return;
    }
    const float v = MODE == MM_GLU ? g * sigmoid(g) * u : g;
    if (A.y_f32) ((float *)A.y)[t * A.n + row] = v;
    else ((uint16_t *)A.y)[t * A.n + row] = to_bf16(v);
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
        E e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = col + i < m ? p[i] : (E)0;
        __builtin_memcpy(&v, e, sizeof(v));
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
    extern __shared__ float red[];
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
    constexpr int E = NT * 4 * 64;       // sums of a wavefront, for one matrix
#pragma unroll
    for (int a = 0; a < MATS; ++a)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) red[((wave * MATS + a) * NT + j) * 256 + i * 64 + lane] = acc[a][j][i];
    __syncthreads();
    for (int e = tid; e < E; e += blockDim.x) {
        float v[MATS];
#pragma unroll
        for (int a = 0; a < MATS; ++a) {
            v[a] = 0.f;
            for (int w = 0; w < nw; ++w) v[a] += red[(w * MATS + a) * E + e];
        }
        const int el = e & 63;
        const long long t = t0 + 16 * (e >> 8) + (el & 15), row = rt * GQ_ROWS + 4 * (el >> 4) + ((e >> 6) & 3);
        if (t < A.T && row < A.n) {
            const float by = XT == SKIM_E4M3 ? A.x_scales[t] : 1.f;
            finish<MODE>(A, t, row, v[0] * by, MATS == 2 ? v[MATS - 1] * by : 0.f);
        }
    }
}

// ---- gradient to the input -------------------------------------------------------------------------------------------------

// dx = dy W (+ dy2 W2): a workgroup makes 128 columns for 64 tokens, a wavefront 32 of them.  32 rows a step: the codes of two row blocks
// become scaled bfloat16 values in LDS, and the transposing reads give each lane 8 rows of its column.
template <int G, bool VEC>
__global__ void __launch_bounds__(256) group_dx_kernel(MmArgs A, int mats, int chunks) {
    __shared__ __align__(16) uint16_t tile[4][32][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane >> 4, l16 = lane & 15;
    const long long kb = blockIdx.x / chunks, t0 = (long long)(blockIdx.x % chunks) * 64;
    const long long kbs = gq_col_blocks(A.m), rbs = gq_row_blocks(A.n), n16 = rbs * GQ_ROWS;
    long long xrow[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) xrow[j] = min(t0 + 16 * j + l16, A.T - 1) * A.ldx;
    gq_float4 acc[2][4] = {};
    for (int a = 0; a < mats; ++a) {
        for (long long rb = 0; rb < rbs; rb += 2) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                gq_word4 v = {};
                if (rb + h < rbs) {
                    const uint32_t w = A.codes[a][((rb + h) * kbs + kb) * 64 + lane][wave];
                    const float s = gq_scale(A.scales[a][(kb * (GQ_COLS / G) + 32 * wave / G) * n16 + (rb + h) * GQ_ROWS + l16]);
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const uint32_t bytes = p < 2 ? gq_low(w) : gq_high(w);
                        const gq_float2 f = p & 1 ? __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bytes, 512.f, true)
                                                  : __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bytes, 512.f, false);
                        v[p] = __builtin_amdgcn_perm(__float_as_uint(s * f.y), __float_as_uint(s * f.x), 0x07060302u);
                    }
                }
                *(gq_word4 *)&tile[wave][16 * h + l16][8 * c] = v;
            }
            __syncthreads();
            gq_bf16x8 b[4];
            const void *x = a ? A.x2 : A.x;
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = load_x<SKIM_BF16, VEC>(x, xrow[j], rb * GQ_ROWS + 8 * c, A.n);
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const gq_short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)&tile[wave][8 * c + (l16 >> 2)][16 * p + 4 * (l16 & 3)]);
                const gq_short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4 *)&tile[wave][8 * c + 4 + (l16 >> 2)][16 * p + 4 * (l16 & 3)]);
                const gq_bf16x8 q = __builtin_bit_cast(gq_bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[p][j] = mfma(q, b[j], acc[p][j]);
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const long long t = t0 + 16 * j + l16, col = kb * GQ_COLS + 32 * wave + 16 * p + 4 * c + i;
                if (t < A.T && col < A.m) {
                    if (A.y_f32) ((float *)A.y)[t * A.m + col] = acc[p][j][i];
                    else ((uint16_t *)A.y)[t * A.m + col] = to_bf16(acc[p][j][i]);
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

template <int MODE>
skim_status launch_forward(skim_ctx *ctx, const MmArgs &A, int group, int x_type) {
    constexpr int MATS = MODE == MM_PLAIN ? 1 : 2;
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

skim_status launch_dx(skim_ctx *ctx, const MmArgs &A, int group, int mats) {
    const int64_t chunks = (A.T + 63) / 64, groups = gq_col_blocks(A.m) * chunks;
    if (groups > 0x7fffffff) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%lld tokens on %lld columns are too many for one call", A.T, A.m);
    const bool vec = A.n % 8 == 0 && A.ldx % 8 == 0 && (((uintptr_t)A.x | (uintptr_t)A.x2) & 15) == 0;
    with_group(group, [&](auto g) {
        auto go = [&](auto v) {
            hipLaunchKernelGGL((group_dx_kernel<decltype(g)::value, decltype(v)::value>), dim3((unsigned)groups), dim3(256), 0, ctx->stream, A, mats, (int)chunks);
        };
        if (vec) go(std::true_type{});
        else go(std::false_type{});
    });
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
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
