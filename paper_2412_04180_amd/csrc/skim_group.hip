// Weights in 4 bits with one scale a group of columns: written from a dense matrix, and read back.  The products with them
// are in skim_group_mm.hip.
#include "skim_group.h"

#include <algorithm>

namespace {

constexpr int GQ_WAVES = 4;

// One wavefront a block of 16 rows x 128 columns; lane (c, r) takes the columns of its place.
// s = the least number of 5 significant bits >= max |w| / 7 (at least the least normal number, 0 for a group of zeros): found
// in float64, where the quotient of a float32 and 7 can be told from the numbers of 5 bits next to it, by adding all ones
// below the 4 bits that stay and cutting them off.  q = w / s rounded to a whole number, ties to even; |w| / s <= 7, so no
// code needs clamping and |w - s q| <= s / 2.
// Bound by memory: 4 bytes of a weight in, 1/2 out; 11008 x 4096 in 43 us, 4.7 TB/s.
template <int G, bool VEC>
__global__ void __launch_bounds__(64 * GQ_WAVES) group_quantize_kernel(const float *__restrict__ W, long long n, long long m, long long ld, long long nblocks,
                                                                       uint32_t *__restrict__ codes, uint16_t *__restrict__ scales) {
    const long long block = (long long)blockIdx.x * GQ_WAVES + (threadIdx.x >> 6);
    if (block >= nblocks) return;
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const long long kbs = gq_col_blocks(m), rt = block / kbs, kb = block - rt * kbs;
    const long long row = rt * GQ_ROWS + r, n16 = gq_row_blocks(n) * GQ_ROWS;
    float w[4][8];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const long long col = kb * GQ_COLS + 32 * k + 8 * c;
        const float *p = W + row * ld + col;
#pragma unroll
        for (int i = 0; i < 8; ++i) w[k][i] = 0.f;
        if constexpr (VEC) {
            if (row < n && col < m) {
                const float4 a = *(const float4 *)p, b = *(const float4 *)(p + 4);
                w[k][0] = a.x, w[k][1] = a.y, w[k][2] = a.z, w[k][3] = a.w;
                w[k][4] = b.x, w[k][5] = b.y, w[k][6] = b.z, w[k][7] = b.w;
            }
        } else {
            if (row < n) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (col + i < m) w[k][i] = p[i];
            }
        }
    }
    gq_word4 out;
    constexpr int KG = G / 32;                    // words of a group
#pragma unroll
    for (int g = 0; g < 4 / KG; ++g) {
        float top = 0.f;
#pragma unroll
        for (int k = g * KG; k < (g + 1) * KG; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(w[k][i]));
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const long long up = (__double_as_longlong((double)top / 7.0) + ((1ll << 48) - 1)) & ~((1ll << 48) - 1);
        const double s = top > 0.f ? fmax(__longlong_as_double(up), 0x1p-126) : 0.0;
        const double by = top > 0.f ? s : 1.0;
        if (c == 0) scales[(kb * (GQ_COLS / G) + g) * n16 + row] = (uint16_t)(__float_as_uint((float)s) >> 16);
#pragma unroll
        for (int k = g * KG; k < (g + 1) * KG; ++k) {
            uint32_t word = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int q = (int)rint((double)w[k][i] / by), b = i & 3;
                const uint32_t size = (uint32_t)abs(q) & 7u, sign = q < 0 ? 1u : 0u;
                word |= i < 4 ? size << (8 * b) | sign << (8 * b + 7) : size << (8 * b + 4) | sign << (8 * ((b + 1) & 3) + 3);
            }
            out[k] = word;
        }
    }
    ((gq_word4 *)codes)[block * 64 + lane] = out;
}

// The dense matrix, bound by the 4 bytes written per weight: 11008 x 4096 in 35-40 us, 5.1-5.8 TB/s.
template <int G, bool VEC>
__global__ void __launch_bounds__(64 * GQ_WAVES) group_unpack_kernel(const uint32_t *__restrict__ codes, const uint16_t *__restrict__ scales, long long n,
                                                                     long long m, long long nblocks, float *__restrict__ Wq) {
    const long long block = (long long)blockIdx.x * GQ_WAVES + (threadIdx.x >> 6);
    if (block >= nblocks) return;
    const int lane = threadIdx.x & 63, r = lane & 15, c = lane >> 4;
    const long long kbs = gq_col_blocks(m), rt = block / kbs, kb = block - rt * kbs;
    const long long row = rt * GQ_ROWS + r, n16 = gq_row_blocks(n) * GQ_ROWS;
    const gq_word4 in = ((const gq_word4 *)codes)[block * 64 + lane];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float s = gq_scale(scales[(kb * (GQ_COLS / G) + 32 * k / G) * n16 + row]);
        const long long col = kb * GQ_COLS + 32 * k + 8 * c;
        float v[8];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t bytes = h ? gq_high(in[k]) : gq_low(in[k]);
            const gq_float2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bytes, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(bytes, 512.f, true);
            v[4 * h] = s * a.x, v[4 * h + 1] = s * a.y, v[4 * h + 2] = s * b.x, v[4 * h + 3] = s * b.y;
        }
        if (row >= n) continue;
        float *p = Wq + row * m + col;
        if constexpr (VEC) {
            if (col < m) {
                *(float4 *)p = make_float4(v[0], v[1], v[2], v[3]);
                *(float4 *)(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < m) p[i] = v[i];
        }
    }
}

// Input validation (off unless the caller asks for it): 1 for a weight that is not finite, or of 2^127 and more.
__global__ void group_validate_clear_kernel(int *flag) { *flag = 0; }
__global__ void __launch_bounds__(256) group_validate_kernel(const float *__restrict__ W, long long n, long long m, long long ld, int *flag) {
    int bad = 0;
    for (long long row = blockIdx.x; row < n; row += gridDim.x)
        for (long long j = threadIdx.x; j < m; j += 256)
            if (!(fabsf(W[row * ld + j]) < 0x1p127f)) bad = 1;
    if (bad) atomicOr(flag, 1);
}
skim_status validate_weights(skim_ctx *ctx, const float *W, int64_t n, int64_t m, int64_t ld) {
    if (!ctx->validate) return SKIM_OK;
    int *const on_device = ctx->sort_counters + SKIM_GROUP_FLAG;
    hipLaunchKernelGGL(group_validate_clear_kernel, dim3(1), dim3(1), 0, ctx->stream, on_device);
    hipLaunchKernelGGL(group_validate_kernel, dim3((unsigned)std::min<int64_t>(n, 8ll * ctx->num_cu)), dim3(256), 0, ctx->stream, W, (long long)n, (long long)m, (long long)ld,
                       on_device);
    SKIM_HIP(ctx, hipGetLastError());
    int flag = 0;
    SKIM_HIP(ctx, hipMemcpyAsync(&flag, on_device, sizeof(int), hipMemcpyDeviceToHost, ctx->stream));
    SKIM_HIP(ctx, hipStreamSynchronize(ctx->stream));
    if (flag) SKIM_FAIL(ctx, SKIM_ERR_NONFINITE, "skim_group_quantize: W holds a value that is not finite, or of 2^127 or more");
    return SKIM_OK;
}

}  // namespace

skim_status skim_group_check(skim_ctx *ctx, const void *codes, const void *scales, int64_t n, int64_t m, int group, const char *who) {
    if (!codes || !scales) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: NULL argument", who);
    if (((uintptr_t)codes & 15) || ((uintptr_t)scales & 15)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: codes and scales must be 16-byte aligned", who);
    if (group != 32 && group != 64 && group != 128) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: group %d is none of 32, 64, 128", who, group);
    if (n < 1 || n > SKIM_GROUP_MAX || m < 1 || m > SKIM_GROUP_MAX)
        SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%s: bad shape n=%lld m=%lld", who, (long long)n, (long long)m);
    if (gq_row_blocks(n) * gq_col_blocks(m) > 0x7fffffffll)
        SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%s: n=%lld m=%lld is over 2^31 blocks", who, (long long)n, (long long)m);
    return SKIM_OK;
}

extern "C" int64_t skim_group_code_words(int64_t n, int64_t m) {
    if (n < 1 || n > SKIM_GROUP_MAX || m < 1 || m > SKIM_GROUP_MAX) return -1;
    return gq_row_blocks(n) * gq_col_blocks(m) * 256;
}

extern "C" int64_t skim_group_scale_entries(int64_t n, int64_t m, int group) {
    if (n < 1 || n > SKIM_GROUP_MAX || m < 1 || m > SKIM_GROUP_MAX || (group != 32 && group != 64 && group != 128)) return -1;
    return gq_row_blocks(n) * GQ_ROWS * gq_col_blocks(m) * (GQ_COLS / group);
}

extern "C" skim_status skim_group_quantize(skim_ctx *ctx, const float *W, int64_t n, int64_t m, int64_t ld, int group, uint32_t *codes,
                                           uint16_t *scales_bf16) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    if ((st = skim_group_check(ctx, codes, scales_bf16, n, m, group, "skim_group_quantize")) != SKIM_OK) return st;
    if (!W) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_group_quantize: W must not be NULL");
    if (ld < m) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "skim_group_quantize: ld=%lld is less than m=%lld", (long long)ld, (long long)m);
    if ((st = validate_weights(ctx, W, n, m, ld)) != SKIM_OK) return st;
    const long long nblocks = gq_row_blocks(n) * gq_col_blocks(m);
    const bool vec = m % 8 == 0 && ld % 4 == 0 && ((uintptr_t)W & 15) == 0;
    with_group(group, [&](auto g) {
        constexpr int G = decltype(g)::value;
        auto launch = [&](auto v) {
            hipLaunchKernelGGL((group_quantize_kernel<G, decltype(v)::value>), dim3((unsigned)((nblocks + GQ_WAVES - 1) / GQ_WAVES)), dim3(64 * GQ_WAVES), 0,
                               ctx->stream, W, (long long)n, (long long)m, (long long)ld, nblocks, codes, scales_bf16);
        };
        if (vec) launch(std::true_type{});
        else launch(std::false_type{});
    });
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
}

extern "C" skim_status skim_group_unpack(skim_ctx *ctx, const uint32_t *codes, const uint16_t *scales_bf16, int64_t n, int64_t m, int group, float *Wq) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    if ((st = skim_group_check(ctx, codes, scales_bf16, n, m, group, "skim_group_unpack")) != SKIM_OK) return st;
    if (!Wq) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_group_unpack: Wq must not be NULL");
    const long long nblocks = gq_row_blocks(n) * gq_col_blocks(m);
    const bool vec = m % 8 == 0 && ((uintptr_t)Wq & 15) == 0;
    with_group(group, [&](auto g) {
        constexpr int G = decltype(g)::value;
        auto launch = [&](auto v) {
            hipLaunchKernelGGL((group_unpack_kernel<G, decltype(v)::value>), dim3((unsigned)((nblocks + GQ_WAVES - 1) / GQ_WAVES)), dim3(64 * GQ_WAVES), 0,
                               ctx->stream, codes, scales_bf16, (long long)n, (long long)m, nblocks, Wq);
        };
        if (vec) launch(std::true_type{});
        else launch(std::false_type{});
    });
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
}
