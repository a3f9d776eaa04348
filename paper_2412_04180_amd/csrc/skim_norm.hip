// Root-mean-square norm of a decoder block with the residual's addition and an 8-bit output, and its backward pass.
#include "skim_common.h"

#include <algorithm>
#include <type_traits>

namespace {

constexpr int NORM_OCTET = 8;          // neighbouring columns of a thread: 16 bytes of bfloat16
constexpr int NORM_MAX_THREADS = 1024;
constexpr int NORM_RESIDENT = 2048;   // threads of a compute unit
constexpr double E4M3_MAX = 448.0;

typedef float float8v __attribute__((ext_vector_type(8)));
typedef float8v float8u __attribute__((aligned(16)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float bf16_to_f32(uint32_t bits) { return __uint_as_float(bits << 16); }
__device__ __forceinline__ uint32_t f32_to_bf16(float v) { return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)v); }

// Eight values of a row from column c on (zeros past column m).  VEC: the row starts on a 16-byte border and m is a
// multiple of 8, so that an octet is whole or not there.  They stay as they came until they are asked for: what is done to a value waits for it.
template <typename T, bool VEC>
struct Octet {
    std::conditional_t<VEC && sizeof(T) == 2, uint4v, float8v> v;
    __device__ __forceinline__ void load(const T *row, int c, int m) {
        v = decltype(v){};
        if constexpr (VEC) {
            if (c < m) {
                if constexpr (sizeof(T) == 2) v = *(const uint4v *)(row + c);
                else v = *(const float8u *)(row + c);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < m) {
                    if constexpr (sizeof(T) == 2) v[i] = bf16_to_f32(row[c + i]);
                    else v[i] = row[c + i];
                }
        }
    }
    __device__ __forceinline__ float8v get() const {
        if constexpr (VEC && sizeof(T) == 2) {
            float8v o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                o[2 * i] = __uint_as_float(v[i] << 16);
                o[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
            }
            return o;
        } else {
            return v;
        }
    }
};
template <typename T, bool VEC>
__device__ __forceinline__ float8v load8(const T *row, int c, int m) {
    Octet<T, VEC> o;
    o.load(row, c, m);
    return o.get();
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

// Eight values below 464 in size, ahead of their rounding to e4m3: in float32, on the same side of every number halfway between two of e4m3 as
// the float64 value, and on none unless that is.  Those numbers have at most 5 significant bits; where the nearest float32 has no more and is not
// the value, the one next to it towards the value is as good.  (One octet in 16000 of other values comes to that.)
__device__ __forceinline__ void off_ties(const double (&v)[8], float (&o)[8]) {
    bool few = false;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        o[i] = (float)v[i];
        few |= (__float_as_uint(o[i]) & 0x7FFFF) == 0;
    }
    if (few) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t u = __float_as_uint(o[i]);
            // (0: v is 0, or below the least float32 and rounds to 0)
            if ((u & 0x7FFFF) == 0 && o[i] != 0.f && (double)o[i] != v[i]) o[i] = __uint_as_float(u + (fabs((double)o[i]) > fabs(v[i]) ? 0xFFFFFFFFu : 1u));
        }
    }
}

// h = x + residual (stored as x is), rstd = 1 / sqrt(mean h^2 + eps), y = h rstd weight, and y in e4m3 with one scale a row,
// max |y| / 448.
// Bound by memory: bfloat16 x, residual in, h and the 8-bit output out are 7 bytes a value (8192 x 4096 in 44 us, 5.3 TB/s).  A workgroup takes every so many rows, a row at a
// time in registers (R octets a thread) with the weights beside it, and the next row on its way; both statistics in one reduction: max |h weight|
// does not need rstd.  They and the quotient that is rounded
// to 8 bits are float64: a code is then the one that the definition gives, also next to a border, and nobody can see in which
// order the row was summed.
template <typename T, int R, bool VEC>
__global__ void __launch_bounds__(NORM_MAX_THREADS)
rms_norm_kernel(const T *x, long long ldx, const T *residual, long long ldr, const float *__restrict__ weight, float eps, long long rows,
                int m, T *h, T *y, uint8_t *q, float *scales, float *rstd_out) {
    __shared__ double red[2][2][NORM_MAX_THREADS / 64];
    const int tid = threadIdx.x, nth = blockDim.x;
    constexpr bool KEEP = R <= 2, KEEP_P = R == 1, AHEAD = R <= 2;   // weights, products and the next row in registers, where there is room
    const float8v ones{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    auto load_weight = [&](int r) { return weight ? load8<float, VEC>(weight, (r * nth + tid) * NORM_OCTET, m) : ones; };
    float8v v[R], w[R];
    double p[KEEP_P ? R : 1][8];
    if (KEEP) {
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = load_weight(r);
    }
    Octet<T, VEC> xr[R], er[R];
    auto load_row = [&](long long t) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * nth + tid) * NORM_OCTET;
            xr[r].load(x + t * ldx, c, m);
            if (residual) er[r].load(residual + t * ldr, c, m);
        }
    };
    if (AHEAD) load_row(blockIdx.x);
    int turn = 0;
    for (long long t = blockIdx.x; t < rows; t += gridDim.x, turn ^= 1) {
        double sum = 0.0, top = 0.0;
        bool none = false;                               // a product that is no number (also of finite x: with a weight that is not; or 0 times an infinity)
        if (!AHEAD) load_row(t);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * nth + tid) * NORM_OCTET;
            v[r] = xr[r].get();
            if (!KEEP) w[r] = load_weight(r);
            // (kept as float32: the compiler would convert kept weights once for all rows, which with two octets a thread spills 12 to 96 bytes a lane; with the
            // conversion in the loop 8192 x 4096 bfloat16 52.6 -> 50.5 us, 1024 x 11008 float32 53 -> 38)
            if (!KEEP_P) asm("" : "+v"(w[r]));
            if (residual) {
                const float8v e = er[r].get();
#pragma unroll
                for (int i = 0; i < 8; ++i) v[r][i] = as_stored<T>(v[r][i] + e[i]);
                store8<T, VEC>(h + t * m, c, m, v[r]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double d = (double)v[r][i], e = d * (double)w[r][i];
                sum = fma(d, d, sum);
                top = fmax(top, fabs(e));                // (passes NaNs over)
                none |= e != e;
                if (KEEP_P) p[r][i] = e;
            }
        }
        if (AHEAD && t + gridDim.x < rows) load_row(t + gridDim.x);
        auto product = [&](int r, int i) { return KEEP_P ? p[r][i] : (double)v[r][i] * (double)w[r][i]; };
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            sum += __shfl_xor(sum, d, 64);
            top = fmax(top, __shfl_xor(top, d, 64));
        }
        const bool some = __any(none);
        if ((tid & 63) == 0) {                           // (two sets: a row's are read while the next row's are written)
            red[turn][0][tid >> 6] = sum;
            red[turn][1][tid >> 6] = some ? __builtin_nan("") : top;
        }
        __syncthreads();
        sum = top = 0.0;
        none = false;
        for (int i = 0; i < nth / 64; ++i) {
            const double o = red[turn][1][i];
            sum += red[turn][0][i];
            top = fmax(top, o);
            none |= o != o;
        }
        const double rstd = 1.0 / sqrt(sum / (double)m + (double)eps);
        // (a scale below the least normal number would have digits missing; a row of zeros has none: 1; that of a row with a NaN or an infinity is NaN, and
        // so is one with a product that is none)
        const double unit = none ? __builtin_nan("") : top * rstd / E4M3_MAX;
        const float scale = top == 0.0 && unit == 0.0 ? 1.f : unit < 0x1p-126 ? 0x1p-126f : (float)unit;
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
                for (int i = 0; i < 8; ++i) o[i] = (float)(product(r, i) * rstd);
                store8<T, VEC>(y + t * m, c, m, o);
            }
            if (q) {
                double e[8];
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = product(r, i) * k;               // (at most 448 (1 + 2^-23))
                off_ties(e, o);
                int lo = __builtin_amdgcn_cvt_pk_fp8_f32(o[0], o[1], 0, false);
                lo = __builtin_amdgcn_cvt_pk_fp8_f32(o[2], o[3], lo, true);
                int hi = __builtin_amdgcn_cvt_pk_fp8_f32(o[4], o[5], 0, false);
                hi = __builtin_amdgcn_cvt_pk_fp8_f32(o[6], o[7], hi, true);
                uint8_t *to = q + t * m + c;
                if constexpr (VEC) {
                    *(uint2v *)to = uint2v{(uint32_t)lo, (uint32_t)hi};
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (c + i < m) to[i] = (uint8_t)((uint32_t)(i < 4 ? lo : hi) >> (8 * (i & 3)));
                }
            }
        }
    }
}

// With g = dy weight and n = h rstd:  dx = rstd (g - n mean(g n)) + dh,  dweight = sum over the rows of dy n.
// Bound by memory: dy, h, dh in and dx out, 8 bytes a value in bfloat16 (4096 x 4096 in 30 us, 4.5 TB/s, and 4 for norm_columns_kernel).  A workgroup takes a run of rows and keeps the columns'
// shares of dweight in registers: one partial row a workgroup goes to memory, and norm_columns_kernel adds them up in a fixed order.
template <typename T, int R, bool VEC>
__global__ void __launch_bounds__(NORM_MAX_THREADS)
rms_norm_back_kernel(const T *__restrict__ dy, long long lddy, const T *__restrict__ h, long long ldh, const T *__restrict__ dh, long long lddh,
                     const float *__restrict__ rstd, const float *__restrict__ weight, long long rows, int m, T *dx, float *partial) {
    __shared__ float red[2][NORM_MAX_THREADS / 64];
    const int tid = threadIdx.x, nth = blockDim.x;
    const long long t0 = rows * blockIdx.x / gridDim.x, t1 = rows * (blockIdx.x + 1) / gridDim.x;
    constexpr bool KEEP = R <= 2;                        // the weights in registers, where there is room; and with one octet a thread the next row
    const float8v ones{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    auto load_weight = [&](int r) { return weight ? load8<float, VEC>(weight, (r * nth + tid) * NORM_OCTET, m) : ones; };
    float8v w[KEEP ? R : 1], dw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        dw[r] = float8v{};
        if (KEEP) w[r] = load_weight(r);
    }
    Octet<T, VEC> gr[R], nr[R], er[1];
    float rs1 = 0.f;
    auto load_row = [&](long long t) {
        rs1 = rstd[t];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (r * nth + tid) * NORM_OCTET;
            gr[r].load(dy + t * lddy, c, m);
            nr[r].load(h + t * ldh, c, m);
            if (R == 1 && dh) er[0].load(dh + t * lddh, c, m);
        }
    };
    if (R == 1 && t0 < t1) load_row(t0);
    for (long long t = t0; t < t1; ++t) {
        if (R > 1) load_row(t);
        float8v g[R], n[R], e = {};
        const float rs = rs1;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            g[r] = gr[r].get();
            n[r] = nr[r].get() * rs;
            const float8v wr = KEEP ? w[KEEP ? r : 0] : load_weight(r);
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                dw[r][i] = fmaf(g[r][i], n[r][i], dw[r][i]);
                g[r][i] *= wr[i];
                part = fmaf(g[r][i], n[r][i], part);
            }
            sum += part;
        }
        if (R == 1) {
            if (dh) e = er[0].get();
            if (t + 1 < t1) load_row(t + 1);
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
            if (dh) o += R == 1 ? e : load8<T, VEC>(dh + t * lddh, c, m);
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

// dweight: the partial rows added up, 16 columns a workgroup, its 64 groups of lanes taking every 64th row.
constexpr int NORM_COL_GROUPS = 64;
__global__ void __launch_bounds__(16 * NORM_COL_GROUPS) norm_columns_kernel(const float *__restrict__ partial, int parts, int m, float *dweight) {
    __shared__ float red[NORM_COL_GROUPS][17];
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4, c = blockIdx.x * 16 + lane;
    float sum = 0.f;
    if (c < m)
        for (int p = group; p < parts; p += NORM_COL_GROUPS) sum += partial[(long long)p * m + c];
    red[group][lane] = sum;
    __syncthreads();
    if (group < 16) {                                    // column `group`: 16 lanes add 4 each, then each other's
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < NORM_COL_GROUPS / 16; ++i) sum += red[lane + 16 * i][group];
#pragma unroll
        for (int d = 8; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 16);
        if (lane == 0 && blockIdx.x * 16 + group < m) dweight[blockIdx.x * 16 + group] = sum;
    }
}

// Octets a thread keeps of a row: one up to 8192 columns, then up to four.  Forward, where there are rows for every compute unit, two from 512
// columns on: the reductions, the root and the divisions cost a wavefront as much as an octet.  (float32 rows are bound by memory as they are.)
int norm_octets(int64_t m) { return m <= 8192 ? 1 : m <= 16384 ? 2 : 4; }
int norm_forward_octets(const skim_ctx *ctx, int type, int64_t rows, int64_t m) {
    return type == SKIM_BF16 && m > 512 && m <= 8192 && rows >= 2 * ctx->num_cu ? 2 : norm_octets(m);
}
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
void with_shape(int octets, bool vec, F &&f) {
    auto pick = [&](auto v) {
        switch (octets) {
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
        with_shape(norm_forward_octets(ctx, type, rows, m), vec, [&](auto r, auto v) {
            constexpr int R = decltype(r)::value;
            const int nth = norm_threads(m, R);
            const int64_t groups = std::min<int64_t>(rows, (int64_t)ctx->num_cu * NORM_RESIDENT / nth);
            hipLaunchKernelGGL((rms_norm_kernel<T, R, decltype(v)::value>), dim3((unsigned)groups), dim3(nth), 0, ctx->stream, (const T *)x, (long long)ldx,
                               (const T *)residual, (long long)ldr, weight, eps, (long long)rows, (int)m, (T *)h, (T *)y, q_e4m3, scales, rstd);
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
        with_shape(norm_octets(m), vec, [&](auto r, auto v) {
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
        hipLaunchKernelGGL(norm_columns_kernel, dim3((unsigned)((m + 15) / 16)), dim3(16 * NORM_COL_GROUPS), 0, ctx->stream, partial, (int)groups, (int)m,
                           dweight);
        SKIM_HIP(ctx, hipGetLastError());
    }
    return SKIM_OK;
}
