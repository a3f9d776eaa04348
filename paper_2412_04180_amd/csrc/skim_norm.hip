// Root-mean-square norm of a decoder block with the residual's addition and an 8-bit output, and its backward pass.
#include "skim_common.h"

#include <type_traits>

namespace {

constexpr int NORM_OCTET = 8;          // neighbouring columns of a thread: 16 bytes of bfloat16
constexpr int NORM_MAX_THREADS = 1024;
constexpr double E4M3_MAX = 448.0;

typedef float float8v __attribute__((ext_vector_type(8)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t f32_to_bf16(float v) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v); }

// Eight values of a row from column c on (zeros past column m).  VEC: the row starts on a 16-byte border and m is a
// multiple of 8, so that an octet is whole or not there.
template <typename T, bool VEC>
__device__ __forceinline__ float8v load8(const T *row, int c, int m) {
    float8v v = {};
    if constexpr (VEC) {
        if (c < m) {
            if constexpr (sizeof(T) == 2) {
                const uint4v u = *(const uint4v *)(row + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[2 * i] = __uint_as_float(u[i] << 16);
                    v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
                }
            } else {
                const float4 a = *(const float4 *)(row + c), b = *(const float4 *)(row + c + 4);
                v = float8v{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < m) {
                if constexpr (sizeof(T) == 2) v[i] = bf16_to_f32(row[c + i]);
                else v[i] = row[c + i];
            }
    }
    return v;
}

template <typename T, bool VEC>
__device__ __forceinline__ void store8(T *row, int c, int m, const float8v &v) {
    if constexpr (sizeof(T) == 2) {
        if constexpr (VEC) {
            if (c < m) {
                uint4v u;
#pragma unroll
                for (int i = 0; i < 4; ++i) u[i] = f32_to_bf16(v[2 * i]) | f32_to_bf16(v[2 * i + 1]) << 16;
                *(uint4v *)(row + c) = u;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < m) row[c + i] = (uint16_t)f32_to_bf16(v[i]);
        }
    } else {
        if constexpr (VEC) {
            if (c < m) {
                *(float4 *)(row + c) = make_float4(v[0], v[1], v[2], v[3]);
                *(float4 *)(row + c + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < m) row[c + i] = v[i];
        }
    }
}

// The value that T holds of v.
template <typename T>
__device__ __forceinline__ float as_stored(float v) {
    if constexpr (sizeof(T) == 2) return bf16_to_f32(f32_to_bf16(v));
    return v;
}

// v (at most 448 in size) in float32 rounded to odd: what is rounded once more, to e4m3, then comes out as if it had been
// rounded once.
__device__ __forceinline__ float to_odd(double v) {
    const float f = (float)v;
    const double d = (double)f;
    uint32_t u = __float_as_uint(f);
    u -= fabs(d) > fabs(v) ? 1u : 0u;
    u |= d != v ? 1u : 0u;
    return __uint_as_float(u);
}

// h = x + residual (stored as x is), rstd = 1 / sqrt(mean h^2 + eps), y = h rstd weight, and y in e4m3 with one scale a row,
// max |y| / 448.
// Bound by memory: bfloat16 x, residual in, h and the 8-bit output out are 7 bytes a value.  One workgroup a row, the row in registers
// (R octets a thread), both statistics in one reduction: max |h weight| does not need rstd.  They and the quotient that is rounded
// to 8 bits are float64: a code is then the one that the definition gives, also next to a border, and nobody can see in which
// order the row was summed.  The float64 units do as many operations a clock as the float32 ones here, and about 20 a value are
// half of what the memory takes.
template <typename T, int R, bool VEC>
__global__ void __launch_bounds__(NORM_MAX_THREADS)
rms_norm_kernel(const T *x, long long ldx, const T *residual, long long ldr, const float *__restrict__ weight, float eps,
                int m, T *h, T *y, uint8_t *q, float *scales, float *rstd_out) {
    __shared__ double red[2][NORM_MAX_THREADS / 64];
    const long long t = blockIdx.x;
    const int tid = threadIdx.x, nth = blockDim.x;
    float8v v[R], w[R];
    double sum = 0.0, top = 0.0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * nth + tid) * NORM_OCTET;
        v[r] = load8<T, VEC>(x + t * ldx, c, m);
        if (weight) w[r] = load8<float, VEC>(weight, c, m);
        else w[r] = float8v{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
        if (residual) {
            const float8v e = load8<T, VEC>(residual + t * ldr, c, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[r][i] = as_stored<T>(v[r][i] + e[i]);
            store8<T, VEC>(h + t * m, c, m, v[r]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double d = (double)v[r][i];
            sum = fma(d, d, sum);
            top = fmax(top, fabs(d * (double)w[r][i]));
        }
    }
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        sum += __shfl_xor(sum, d, 64);
        top = fmax(top, __shfl_xor(top, d, 64));
    }
    if ((tid & 63) == 0) {
        red[0][tid >> 6] = sum;
        red[1][tid >> 6] = top;
    }
    __syncthreads();
    sum = top = 0.0;
    for (int i = 0; i < nth / 64; ++i) {
        sum += red[0][i];
        top = fmax(top, red[1][i]);
    }
    const double rstd = 1.0 / sqrt(sum / (double)m + (double)eps);
    // (a scale below the least normal number would have digits missing; one row of zeros has none: 1)
    const float scale = top > 0.0 ? fmaxf((float)(top * rstd / E4M3_MAX), 1.17549435e-38f) : 1.f;
    if (tid == 0) {
        if (rstd_out) rstd_out[t] = (float)rstd;
        if (q) scales[t] = scale;
    }
    const double k = rstd / (double)scale;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int c = (r * nth + tid) * NORM_OCTET;
        if (c >= m) continue;
        if (y) {
            float8v o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = (float)((double)v[r][i] * (double)w[r][i] * rstd);
            store8<T, VEC>(y + t * m, c, m, o);
        }
        if (q) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double e = (double)v[r][i] * (double)w[r][i] * k;
                o[i] = to_odd(fmin(fmax(e, -E4M3_MAX), E4M3_MAX));
            }
            int lo = __builtin_amdgcn_cvt_pk_fp8_f32(o[0], o[1], 0, false);
            lo = __builtin_amdgcn_cvt_pk_fp8_f32(o[2], o[3], lo, true);
            int hi = __builtin_amdgcn_cvt_pk_fp8_f32(o[4], o[5], 0, false);
            hi = __builtin_amdgcn_cvt_pk_fp8_f32(o[6], o[7], hi, true);
            uint8_t *p = q + t * m + c;
            if constexpr (VEC) {
                *(uint2v *)p = uint2v{(uint32_t)lo, (uint32_t)hi};
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c + i < m) p[i] = (uint8_t)((uint32_t)(i < 4 ? lo : hi) >> (8 * (i & 3)));
            }
        }
    }
}

// With g = dy weight and n = h rstd:  dx = rstd (g - n mean(g n)) + dh,  dweight = sum over the rows of dy n.
// Bound by memory: dy, h, dh in and dx out, 8 bytes a value in bfloat16.  A workgroup takes a run of rows and keeps the columns'
// shares of dweight in registers: one partial row a workgroup goes to memory, and norm_columns_kernel adds them up in a fixed order.
template <typename T, int R, bool VEC>
__global__ void __launch_bounds__(NORM_MAX_THREADS)
rms_norm_back_kernel(const T *__restrict__ dy, long long lddy, const T *__restrict__ h, long long ldh, const T *__restrict__ dh, long long lddh,
                     const float *__restrict__ rstd, const float *__restrict__ weight, long long rows, int m, T *dx, float *partial) {
    __shared__ float red[2][NORM_MAX_THREADS / 64];
    const int tid = threadIdx.x, nth = blockDim.x;
    const long long t0 = rows * blockIdx.x / gridDim.x, t1 = rows * (blockIdx.x + 1) / gridDim.x;
    float8v w[R], dw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        dw[r] = float8v{};
        if (weight) w[r] = load8<float, VEC>(weight, (r * nth + tid) * NORM_OCTET, m);
        else w[r] = float8v{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    }
    for (long long t = t0; t < t1; ++t) {
        const float rs = rstd[t];
        float8v g[R], n[R];
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * nth + tid) * NORM_OCTET;
            g[r] = load8<T, VEC>(dy + t * lddy, c, m);
            n[r] = load8<T, VEC>(h + t * ldh, c, m) * rs;
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[r][i] = fmaf(g[r][i], n[r][i], dw[r][i]);
                g[r][i] *= w[r][i];
                part = fmaf(g[r][i], n[r][i], part);
            }
            sum += part;
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
        const int turn = (int)(t & 1);                   // (two sets: a row's sums are read while the next row's are written)
        if ((tid & 63) == 0) red[turn][tid >> 6] = sum;
        __syncthreads();
        sum = 0.f;
        for (int i = 0; i < nth / 64; ++i) sum += red[turn][i];
        const float mean = sum / (float)m;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * nth + tid) * NORM_OCTET;
            float8v o;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] = rs * fmaf(-n[r][i], mean, g[r][i]);
            if (dh) o += load8<T, VEC>(dh + t * lddh, c, m);
            store8<T, VEC>(dx + t * m, c, m, o);
        }
    }
    if (partial) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * nth + tid) * NORM_OCTET;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < m) partial[(long long)blockIdx.x * m + c + i] = dw[r][i];
        }
    }
}

// dweight: the partial rows added up, 64 columns a workgroup, its wavefronts taking every 16th row.
constexpr int NORM_COL_WAVES = 16;
__global__ void __launch_bounds__(64 * NORM_COL_WAVES) norm_columns_kernel(const float *__restrict__ partial, int parts, int m, float *dweight) {
    __shared__ float red[NORM_COL_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = blockIdx.x * 64 + lane;
    float sum = 0.f;
    if (c < m)
        for (int p = wave; p < parts; p += NORM_COL_WAVES) sum += partial[(long long)p * m + c];
    red[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && c < m) {
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < NORM_COL_WAVES; ++i) sum += red[i][lane];
        dweight[c] = sum;
    }
}

// Octets a thread keeps of a row and threads a workgroup: one octet up to 8192 columns, then up to four.
int norm_octets(int64_t m) { return m <= 8192 ? 1 : m <= 16384 ? 2 : 4; }
int norm_threads(int64_t m, int r) {
    const int64_t per = 64ll * NORM_OCTET * r;
    return (int)((m + per - 1) / per * 64);
}

// Workgroups of the backward pass: two of 512 threads a compute unit, more of smaller ones, and no more than there are rows.
int64_t norm_back_groups(const skim_ctx *ctx, int64_t rows, int64_t m) {
    const int nth = norm_threads(m, norm_octets(m));
    const int64_t most = (int64_t)ctx->num_cu * (nth >= 1024 ? 1 : nth >= 512 ? 2 : 4);
    return rows < most ? rows : most;
}

template <typename F>
void with_shape(int64_t m, bool vec, F &&f) {
    auto pick = [&](auto v) {
        switch (norm_octets(m)) {
            case 1: f(std::integral_constant<int, 1>{}, v); break;
            case 2: f(std::integral_constant<int, 2>{}, v); break;
            default: f(std::integral_constant<int, 4>{}, v); break;
        }
    };
    if (vec) pick(std::true_type{});
    else pick(std::false_type{});
}

bool on16(const void *p) { return ((uintptr_t)p & 15) == 0; }

skim_status check_norm(skim_ctx *ctx, int type, int64_t rows, int64_t m, const char *who) {
    if (type != SKIM_BF16 && type != SKIM_F32) SKIM_FAIL(ctx, SKIM_ERR_ARG, "%s: type %d is neither SKIM_BF16 nor SKIM_F32", who, type);
    if (rows < 0 || rows > 0x7fffffff || m < 1 || m > SKIM_MAX_M)
        SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "%s: bad shape rows=%lld m=%lld", who, (long long)rows, (long long)m);
    return SKIM_OK;
}

}  // namespace

extern "C" skim_status skim_rms_norm(skim_ctx *ctx, const void *x, int64_t ldx, const void *residual, int64_t ldr, int type,
                                     const float *weight, float eps, int64_t rows, int64_t m, void *h, void *y, uint8_t *q_e4m3,
                                     float *scales, float *rstd) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    if ((st = check_norm(ctx, type, rows, m, "skim_rms_norm")) != SKIM_OK) return st;
    if (ldx < m || (residual && ldr < m)) SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "skim_rms_norm: row strides must be at least m=%lld", (long long)m);
    if (!(eps > 0.f && eps <= __FLT_MAX__)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_rms_norm: eps must be positive and finite");
    if (rows == 0) return SKIM_OK;
    if (!x || (!y && !q_e4m3 && !rstd)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_rms_norm: x and one of the outputs must not be NULL");
    if ((residual != nullptr) != (h != nullptr)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_rms_norm: residual and h are given together");
    if ((q_e4m3 != nullptr) != (scales != nullptr)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_rms_norm: q and scales are given together");
    const int64_t es = type == SKIM_BF16 ? 2 : 4;
    const bool vec = m % 8 == 0 && (ldx * es) % 16 == 0 && (ldr * es) % 16 == 0 && on16(x) && on16(residual) && on16(weight) && on16(h) && on16(y) &&
                     ((uintptr_t)q_e4m3 & 7) == 0;
    auto launch = [&](auto zero) {
        using T = decltype(zero);
        with_shape(m, vec, [&](auto r, auto v) {
            constexpr int R = decltype(r)::value;
            hipLaunchKernelGGL((rms_norm_kernel<T, R, decltype(v)::value>), dim3((unsigned)rows), dim3(norm_threads(m, R)), 0, ctx->stream, (const T *)x,
                               (long long)ldx, (const T *)residual, (long long)ldr, weight, eps, (int)m, (T *)h, (T *)y, q_e4m3, scales, rstd);
        });
    };
    if (type == SKIM_BF16) launch((uint16_t)0);
    else launch(0.f);
    SKIM_HIP(ctx, hipGetLastError());
    return SKIM_OK;
}

extern "C" size_t skim_rms_norm_scratch_bytes(const skim_ctx *ctx, int64_t rows, int64_t m) {
    if (!ctx || rows < 1 || m < 1 || m > SKIM_MAX_M) return 0;
    return (size_t)norm_back_groups(ctx, rows, m) * (size_t)m * sizeof(float);
}

extern "C" skim_status skim_rms_norm_backward(skim_ctx *ctx, const void *dy, int64_t lddy, const void *h, int64_t ldh, const void *dh, int64_t lddh,
                                              int type, const float *rstd, const float *weight, int64_t rows, int64_t m, void *dx,
                                              float *dweight, void *scratch, size_t scratch_bytes) {
    skim_status st = skim_enter(ctx);
    if (st != SKIM_OK) return st;
    if ((st = check_norm(ctx, type, rows, m, "skim_rms_norm_backward")) != SKIM_OK) return st;
    if (lddy < m || ldh < m || (dh && lddh < m))
        SKIM_FAIL(ctx, SKIM_ERR_SHAPE, "skim_rms_norm_backward: row strides must be at least m=%lld", (long long)m);
    if (rows > 0 && (!dy || !h || !rstd || !dx)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_rms_norm_backward: dy, h, rstd and dx must not be NULL");
    const int64_t groups = norm_back_groups(ctx, rows, m);
    if (dweight && rows > 0 && (!scratch || scratch_bytes < skim_rms_norm_scratch_bytes(ctx, rows, m)))
        SKIM_FAIL(ctx, SKIM_ERR_WORKSPACE, "skim_rms_norm_backward: dweight needs %zu bytes of scratch, %zu given",
                  skim_rms_norm_scratch_bytes(ctx, rows, m), scratch ? scratch_bytes : (size_t)0);
    if (dweight && ((uintptr_t)scratch & 3)) SKIM_FAIL(ctx, SKIM_ERR_ARG, "skim_rms_norm_backward: scratch must be 4-byte aligned");
    const int64_t es = type == SKIM_BF16 ? 2 : 4;
    const bool vec = m % 8 == 0 && (lddy * es) % 16 == 0 && (ldh * es) % 16 == 0 && (lddh * es) % 16 == 0 && on16(dy) && on16(h) && on16(dh) &&
                     on16(weight) && on16(dx);
    float *partial = dweight ? (float *)scratch : nullptr;
    auto launch = [&](auto zero) {
        using T = decltype(zero);
        with_shape(m, vec, [&](auto r, auto v) {
            constexpr int R = decltype(r)::value;
            hipLaunchKernelGGL((rms_norm_back_kernel<T, R, decltype(v)::value>), dim3((unsigned)groups), dim3(norm_threads(m, R)), 0, ctx->stream,
                               (const T *)dy, (long long)lddy, (const T *)h, (long long)ldh, (const T *)dh, (long long)lddh, rstd, weight, (long long)rows,
                               (int)m, (T *)dx, partial);
        });
    };
    if (rows > 0) {
        if (type == SKIM_BF16) launch((uint16_t)0);
        else launch(0.f);
        SKIM_HIP(ctx, hipGetLastError());
    }
    if (dweight) {                                       // (no rows: zeros)
        hipLaunchKernelGGL(norm_columns_kernel, dim3((unsigned)((m + 63) / 64)), dim3(64 * NORM_COL_WAVES), 0, ctx->stream, partial, (int)groups, (int)m,
                           dweight);
        SKIM_HIP(ctx, hipGetLastError());
    }
    return SKIM_OK;
}
