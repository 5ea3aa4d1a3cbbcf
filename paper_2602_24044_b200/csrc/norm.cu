// Residual addition and root-mean-square norm of rows, to bf16 rows and to e4m3 codes with scales.
//
// s = x + r ; y_i = s_i * (1 / sqrt(mean(s^2) + eps)) * w_i.  A stream: every input is read once and every
// output written once; a row stays in registers between its sum and its outputs, 8 values (16 bytes) a
// thread and vector, consecutive lanes on consecutive vectors.
//
// The sum of squares: eight neighbours in fp32, every operation rounded by itself, as a tree; the sums of
// eight then in fp64.  So any split of a row over threads gives the same sum but for the last bits of the
// fp64 one, and the codes, which a difference in the last bit of fp32 could turn, do not depend on the
// launch (rounding the fp64 sum to fp32 hides them but once in 10^8 rows).  All of it in fp64 would cost a
// conversion a value, 16 a cycle and SM: more than the rest of the row.
//
// 12937 rows of 4096 with a residual: 67.4 us (6.29 TB/s, 0.98 of a copy's rate), with e4m3 codes and a scale for
// each 128 values 77.9 us (6.14 TB/s).  16 rows: 8 us, which is the call.
#include <cuda_fp8.h>

#include <cmath>

#include "kv_common.cuh"

namespace lora {

enum { NORM_PLAIN = 0, NORM_ROW = 1, NORM_128 = 2, NORM_32 = 3 };     // how codes are scaled
constexpr int NORM_MAX_THREADS = 512, NORM_MAX_WIDTH = 8 * 8 * NORM_MAX_THREADS;

struct NormParams {
    const __nv_bfloat16 *x, *w, *r;
    __nv_bfloat16 *r_out, *out;
    unsigned char *codes;
    void *scales;
    int64_t ldx, ldr, ldro, ldo, ldc, lds;
    int32_t T, vecs;       // rows; 16-byte vectors of a row
    float eps, inv_n;
};

__device__ __forceinline__ void unpack_row8(const uint4 &u, float (&f)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack_row8(const float (&f)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float larger(float a, float b) {      // NaN where either is
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
// What codes are multiplied by, and the scale as it is stored, from a group's largest |y|.
__device__ __forceinline__ float code_scale(float top, float &scale) {
    if (!(top < INFINITY)) { scale = __uint_as_float(0x7fc00000u); return 0.0f; }
    scale = __fmul_rn(top, 1.0f / 448.0f);
    if (scale < 1.17549435e-38f) scale = 0.0f;
    return scale == 0.0f ? 0.0f : __frcp_rn(scale);
}
// The smallest power of two 2^e with top <= 448 * 2^e (448 = 1.75 * 2^8), as the byte e + 127.
__device__ __forceinline__ float code_power(float top, uint32_t &byte) {
    if (!(top < INFINITY)) { byte = 255u; return 0.0f; }
    if (top == 0.0f) { byte = 0u; return 1.0f; }
    // below the normal numbers the bits count too low an exponent: 127 - 2^-126 / 448 is clamped all the same
    const uint32_t bits = __float_as_uint(top);
    const int e = min(max((int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u), -127), 127);
    byte = (uint32_t)(e + 127);
    return e == 127 ? __uint_as_float(0x00400000u) : __uint_as_float((uint32_t)(127 - e) << 23);   // 2^-e
}
__device__ __forceinline__ uint2 codes8(const float (&y)[8], float inv, bool bad) {
    uint32_t h[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        h[i] = __nv_cvt_float2_to_fp8x2(make_float2(__fmul_rn(y[2 * i], inv), __fmul_rn(y[2 * i + 1], inv)),
                                        __NV_SATFINITE, __NV_E4M3);
    return bad ? make_uint2(0u, 0u) : make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}

// NV vectors a thread.  WARP: a row is a warp's, eight rows a block; else a row is a block's.
template <int NV, bool WARP, int Q>
__global__ void __launch_bounds__(WARP ? 256 : NORM_MAX_THREADS) norm_kernel(const NormParams P) {
    __shared__ double part[NORM_MAX_THREADS / 32];
    __shared__ float part_top[NORM_MAX_THREADS / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int me = WARP ? lane : threadIdx.x, step = WARP ? 32 : blockDim.x;
    const int64_t t = WARP ? (int64_t)blockIdx.x * 8 + warp : blockIdx.x;
    if (WARP && t >= P.T) return;
    const uint4 *x = reinterpret_cast<const uint4 *>(P.x + t * P.ldx);
    const uint4 *r = reinterpret_cast<const uint4 *>(P.r + t * P.ldr);
    uint4 raw[NV], res[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = me + i * step;
        raw[i] = res[i] = make_uint4(0u, 0u, 0u, 0u);
        if (v < P.vecs) {
            raw[i] = x[v];
            if (P.r) res[i] = r[v];
        }
    }
    float s[NV][8];
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = me + i * step;
        unpack_row8(raw[i], s[i]);
        if (P.r) {
            float f[8];
            unpack_row8(res[i], f);
#pragma unroll
            for (int k = 0; k < 8; ++k) s[i][k] = __fadd_rn(s[i][k], f[k]);
            if (P.r_out && v < P.vecs) reinterpret_cast<uint4 *>(P.r_out + t * P.ldro)[v] = pack_row8(s[i]);
        }
        float q[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) q[k] = __fmul_rn(s[i][k], s[i][k]);
        sum += (double)__fadd_rn(__fadd_rn(__fadd_rn(q[0], q[1]), __fadd_rn(q[2], q[3])),
                                 __fadd_rn(__fadd_rn(q[4], q[5]), __fadd_rn(q[6], q[7])));
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (!WARP) {
        if (lane == 0) part[warp] = sum;
        __syncthreads();
        sum = 0.0;
        for (int i = 0; i < (int)blockDim.x / 32; ++i) sum += part[i];
    }
    const float n = __frcp_rn(__fsqrt_rn(__fadd_rn(__fmul_rn(__double2float_rn(sum), P.inv_n), P.eps)));
    float row_top = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int v = me + i * step;
        const bool in = v < P.vecs;
        if (P.w) {
            float w[8];
            unpack_row8(in ? __ldg(reinterpret_cast<const uint4 *>(P.w) + v) : make_uint4(0u, 0u, 0u, 0u), w);
#pragma unroll
            for (int k = 0; k < 8; ++k) s[i][k] = __fmul_rn(__fmul_rn(s[i][k], n), w[k]);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) s[i][k] = __fmul_rn(s[i][k], n);
        }
        if (P.out && in) reinterpret_cast<uint4 *>(P.out + t * P.ldo)[v] = pack_row8(s[i]);
        if (Q != NORM_PLAIN) {
            float top = 0.0f;
            if (in) {
#pragma unroll
                for (int k = 0; k < 8; ++k) top = larger(top, fabsf(s[i][k]));
            }
            if (Q == NORM_ROW) row_top = larger(row_top, top);
            if (Q == NORM_128 || Q == NORM_32) {
                // a group is 16 or 4 lanes, all of them inside the row or none
#pragma unroll
                for (int d = 1; d < (Q == NORM_128 ? 16 : 4); d <<= 1) top = larger(top, __shfl_xor_sync(0xffffffffu, top, d));
                float scale = 0.0f, inv;
                uint32_t byte = 0;
                if (Q == NORM_128) inv = code_scale(top, scale); else inv = code_power(top, byte);
                if (in) {
                    *reinterpret_cast<uint2 *>(P.codes + t * P.ldc + (int64_t)v * 8) = codes8(s[i], inv, !(top < INFINITY));
                    if (Q == NORM_128 && v % 16 == 0) reinterpret_cast<float *>(P.scales)[t * P.lds + v / 16] = scale;
                    if (Q == NORM_32 && v % 4 == 0) reinterpret_cast<unsigned char *>(P.scales)[t * P.lds + v / 4] = (unsigned char)byte;
                }
            }
        }
    }
    if (Q == NORM_ROW) {
#pragma unroll
        for (int d = 16; d; d >>= 1) row_top = larger(row_top, __shfl_xor_sync(0xffffffffu, row_top, d));
        if (!WARP) {
            if (lane == 0) part_top[warp] = row_top;
            __syncthreads();
            row_top = 0.0f;
            for (int i = 0; i < (int)blockDim.x / 32; ++i) row_top = larger(row_top, part_top[i]);
        }
        float scale;
        const float inv = code_scale(row_top, scale);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int v = me + i * step;
            if (v < P.vecs)
                *reinterpret_cast<uint2 *>(P.codes + t * P.ldc + (int64_t)v * 8) = codes8(s[i], inv, !(row_top < INFINITY));
        }
        if (me == 0) reinterpret_cast<float *>(P.scales)[t * P.lds] = scale;
    }
}

// ---------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------
struct NormRows { const void *p; int64_t row, ld; };       // bytes

static lora_status_t check_norm_rows(const void *p, int64_t ld, int64_t width, int align) {
    if ((uintptr_t)p & (align - 1)) return LORA_ERR_INVALID_ARG;
    if (ld < width || ld % 8) return LORA_ERR_SHAPE;
    return LORA_OK;
}

static lora_status_t fill_norm(const lora_norm_args_t *a, int32_t T, NormParams *P, int *q) {
    if (!a) return LORA_ERR_INVALID_ARG;
    const int64_t n = a->width;
    if (T < 0 || n < 8 || n % 8 || n > NORM_MAX_WIDTH) return LORA_ERR_SHAPE;
    if (!(a->eps >= 0.0f) || !std::isfinite(a->eps)) return LORA_ERR_INVALID_ARG;
    *q = a->group == 0 ? NORM_PLAIN : a->group == 32 ? NORM_32 : a->group == 128 ? NORM_128 : NORM_ROW;
    if (*q == NORM_ROW && a->group != n) return LORA_ERR_SHAPE;
    if (*q != NORM_PLAIN && n % a->group) return LORA_ERR_SHAPE;
    if (T == 0) return LORA_OK;
    if (!a->x || (a->residual_out && !a->residual)) return LORA_ERR_INVALID_ARG;
    if ((*q != NORM_PLAIN) != (a->codes != nullptr) || (a->codes != nullptr) != (a->scales != nullptr)) return LORA_ERR_INVALID_ARG;
    if (!a->out && !a->codes && !a->residual_out) return LORA_ERR_INVALID_ARG;
    if ((uintptr_t)a->weight & 15) return LORA_ERR_INVALID_ARG;
    lora_status_t s;
    if ((s = check_norm_rows(a->x, a->ldx, n, 16)) != LORA_OK) return s;
    if (a->residual && (s = check_norm_rows(a->residual, a->ldr, n, 16)) != LORA_OK) return s;
    if (a->residual_out && (s = check_norm_rows(a->residual_out, a->ldro, n, 16)) != LORA_OK) return s;
    if (a->out && (s = check_norm_rows(a->out, a->ldo, n, 16)) != LORA_OK) return s;
    if (a->codes && (s = check_norm_rows(a->codes, a->ldc, n, 8)) != LORA_OK) return s;
    const int64_t unit = *q == NORM_32 ? 1 : 4, groups = *q == NORM_PLAIN ? 0 : n / a->group;
    if (a->scales && ((uintptr_t)a->scales & (unit - 1))) return LORA_ERR_INVALID_ARG;
    if (a->scales && a->lds < groups) return LORA_ERR_SHAPE;
    // an output may be an input in place (each value is read by the thread that writes it); else no two touch
    const NormRows in[3] = {{a->x, 2 * n, 2 * a->ldx}, {a->residual, 2 * n, 2 * a->ldr}, {a->weight, 2 * n, 2 * n}};
    const NormRows out[4] = {{a->residual_out, 2 * n, 2 * a->ldro}, {a->out, 2 * n, 2 * a->ldo},
                             {a->codes, n, a->ldc}, {a->scales, groups * unit, a->lds * unit}};
    for (int o = 0; o < 4; ++o) {
        if (!out[o].p) continue;
        for (int i = 0; i < 3; ++i) {
            if (!in[i].p || (o < 2 && i < 2 && out[o].p == in[i].p && out[o].ld == in[i].ld)) continue;
            const NormRows w = {in[i].p, in[i].row, in[i].ld};
            if (i == 2 ? rows_overlap(out[o].p, out[o].row + (T - 1) * out[o].ld, out[o].row + (T - 1) * out[o].ld, w.p, w.row, w.ld, 1)
                       : rows_overlap(out[o].p, out[o].row, out[o].ld, w.p, w.row, w.ld, T))
                return LORA_ERR_INVALID_ARG;
        }
        for (int i = 0; i < o; ++i)
            if (out[i].p && rows_overlap(out[o].p, out[o].row, out[o].ld, out[i].p, out[i].row, out[i].ld, T))
                return LORA_ERR_INVALID_ARG;
    }
    P->x = (const __nv_bfloat16 *)a->x;
    P->w = (const __nv_bfloat16 *)a->weight;
    P->r = (const __nv_bfloat16 *)a->residual;
    P->r_out = (__nv_bfloat16 *)a->residual_out;
    P->out = (__nv_bfloat16 *)a->out;
    P->codes = (unsigned char *)a->codes;
    P->scales = a->scales;
    P->ldx = a->ldx; P->ldr = a->ldr; P->ldro = a->ldro; P->ldo = a->ldo; P->ldc = a->ldc; P->lds = a->lds;
    P->T = T;
    P->vecs = (int32_t)(n / 8);
    P->eps = a->eps;
    P->inv_n = (float)(1.0 / (double)n);
    return LORA_OK;
}

template <int NV, bool WARP>
static void launch_norm(const NormParams &P, int q, cudaStream_t s) {
    const unsigned grid = WARP ? (unsigned)(((int64_t)P.T + 7) / 8) : (unsigned)P.T;
    const int threads = WARP ? 256 : ((P.vecs + NV - 1) / NV + 31) / 32 * 32;
    if (q == NORM_PLAIN) norm_kernel<NV, WARP, NORM_PLAIN><<<grid, threads, 0, s>>>(P);
    else if (q == NORM_ROW) norm_kernel<NV, WARP, NORM_ROW><<<grid, threads, 0, s>>>(P);
    else if (q == NORM_128) norm_kernel<NV, WARP, NORM_128><<<grid, threads, 0, s>>>(P);
    else norm_kernel<NV, WARP, NORM_32><<<grid, threads, 0, s>>>(P);
}

}  // namespace lora

using namespace lora;

extern "C" lora_status_t lora_add_norm(const lora_norm_args_t *args, int32_t T, void *stream) {
    NormParams P;
    int q = NORM_PLAIN;
    lora_status_t s = fill_norm(args, T, &P, &q);
    if (s != LORA_OK || T == 0) return s;
    DeviceGuard g(args->device);
    if (!g.ok) return cuda_fail(cudaErrorInvalidDevice);
    cudaStream_t st = (cudaStream_t)stream;
    // As many threads a row as it has vectors while rows are few: the time is one row's.  With many rows a
    // thread takes several vectors, whose loads are in flight together.
    const bool many = (int64_t)P.T * P.vecs >= 148 * 2048;
    if (P.vecs <= 32) launch_norm<1, true>(P, q, st);
    else if (many && P.vecs <= 128) launch_norm<4, true>(P, q, st);
    else if (P.vecs > 4 * NORM_MAX_THREADS) launch_norm<8, false>(P, q, st);
    else if (many || P.vecs > 2 * NORM_MAX_THREADS) launch_norm<4, false>(P, q, st);
    else if (P.vecs > NORM_MAX_THREADS) launch_norm<2, false>(P, q, st);
    else launch_norm<1, false>(P, q, st);
    return count_launch();
}
