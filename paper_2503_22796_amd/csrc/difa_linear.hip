// out = residual + gate * act(x W^T + bias): the matrix product around the attention of a layer.
#include <math.h>

#include "difa_layer.h"

namespace difa {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- epilogue.  Every kernel computes the product transposed, W X^T, so that a lane of a 16x16 accumulator holds four
// consecutive output features of one row of x: bias, gate and residual are read, and the result is written, four at a time.
__device__ __forceinline__ float activated(float y, int act) {
    if (act == DIFA_ACT_GELU_TANH) {
        // 0.5 y (1 + tanh u) = y / (1 + exp(-2 u)), u = sqrt(2 / pi) (y + 0.044715 y^3)
        const float u = y * fmaf(0.044715f * y, y, 1.f);
        return y / (1.f + exp2f(-2.30220819813f * u));            // 2 sqrt(2 / pi) log2(e)
    }
    if (act == DIFA_ACT_GELU_ERF) return 0.5f * y * (1.f + erff(y * 0.70710678118f));
    if (act == DIFA_ACT_SILU) return y / (1.f + exp2f(-1.44269504089f * y));
    return y;
}

template <typename T> struct Four;      // four consecutive values
template <> struct Four<__bf16> {
    static __device__ __forceinline__ f32x4 load(const __bf16* p) {
        const u32x2 r = *(const u32x2*)p;
        const unsigned a = r[0], b = r[1];
        return f32x4{__builtin_bit_cast(float, a << 16), __builtin_bit_cast(float, a & 0xffff0000u),
                     __builtin_bit_cast(float, b << 16), __builtin_bit_cast(float, b & 0xffff0000u)};
    }
    static __device__ __forceinline__ void store(__bf16* p, f32x4 v) {
        const bf16x2 a = {(__bf16)v[0], (__bf16)v[1]}, b = {(__bf16)v[2], (__bf16)v[3]};
        *(u32x2*)p = u32x2{__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b)};
    }
};
template <> struct Four<float> {
    static __device__ __forceinline__ f32x4 load(const float* p) { return *(const f32x4*)p; }
    static __device__ __forceinline__ void store(float* p, f32x4 v) { *(f32x4*)p = v; }
};

// Rows m and features n .. n + 3 of the result from the product's sums.  `vec`: all the epilogue's rows start at multiples of
// four elements and n is a multiple of four, so that four at a time are aligned and inside.
template <typename T>
__device__ __forceinline__ void finish(const LinearArgs& a, bool vec, int m, int n, f32x4 y) {
    if (m >= a.m || n >= a.n) return;
    const int b = m / a.rows, t = m - b * a.rows;
    const T* bias = (const T*)a.bias;
    const T* gate = a.gate ? (const T*)a.gate + b * a.gate_stride_b : nullptr;
    const T* res = a.residual ? (const T*)a.residual + b * a.res_stride_b + t * a.res_stride_n : nullptr;
    T* out = (T*)a.out + b * a.out_stride_b + t * a.out_stride_n;
    if (vec) {
        if (bias) y += Four<T>::load(bias + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = activated(y[i], a.activation);
        if (gate) y *= Four<T>::load(gate + n);
        if (res) y += Four<T>::load(res + n);
        Four<T>::store(out + n, y);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (n + i >= a.n) return;
        float v = y[i];
        if (bias) v += (float)bias[n + i];
        v = activated(v, a.activation);
        if (gate) v *= (float)gate[n + i];
        if (res) v += (float)res[n + i];
        out[n + i] = (T)v;
    }
}

// ---- any sizes, strides and alignments: 64 x 64 tiles, 32 features of k at a time through LDS, four wavefronts of 32 x 32.
template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    static constexpr int PER = 8;        // values of k a lane holds of a 32-deep step
    static __device__ __forceinline__ void mul(f32x4& d, const __bf16* w, const __bf16* x) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)w, *(const bf16x8*)x, d, 0, 0, 0);
    }
};
template <> struct Mfma<float> {
    static constexpr int PER = 8;
    static __device__ __forceinline__ void mul(f32x4& d, const float* w, const float* x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[i], d, 0, 0, 0);
    }
};

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void linear_any_kernel(LinearArgs a, bool vec_out, int n_tiles) {
    constexpr int BT = 64, BK = 32, PAD = 16 / (int)sizeof(T), LD = BK + PAD;
    __shared__ __attribute__((aligned(16))) T ws[BT * LD], xs[BT * LD];
    const int tile_n = blockIdx.x % n_tiles, tile_m = blockIdx.x / n_tiles;
    const int m0 = tile_m * BT, n0 = tile_n * BT;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    // staging: four threads a row, eight values each
    const int sr = tid >> 2, sc = (tid & 3) * 8;
    const T* wrow = nullptr;
    const T* xrow = nullptr;
    if (n0 + sr < a.n) wrow = (const T*)a.w + (int64_t)(n0 + sr) * a.w_stride;
    if (m0 + sr < a.m) {
        const int b = (m0 + sr) / a.rows, t = m0 + sr - b * a.rows;
        xrow = (const T*)a.x + b * a.x_stride_b + t * a.x_stride_n;
    }
    auto fetch = [&](const T* row, int k, T (&v)[8]) {
        if (VEC && row && k + 8 <= a.k) {
            constexpr int NV = (int)sizeof(T) / 2;
#pragma unroll
            for (int i = 0; i < NV; ++i) *(u32x4*)&v[i * 8 / NV] = *(const u32x4*)(row + k + i * 8 / NV);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = row && k + i < a.k ? row[k + i] : (T)0.f;
        }
    };
    auto put = [&](T* to, const T (&v)[8]) {
        constexpr int NV = (int)sizeof(T) / 2;
#pragma unroll
        for (int i = 0; i < NV; ++i) *(u32x4*)(to + i * 8 / NV) = *(const u32x4*)&v[i * 8 / NV];
    };
    const int wn = (wave & 1) * 32, wm = (wave >> 1) * 32;      // the wavefront's corner of the tile
    const int fr = lane & 15, fk = (lane >> 4) * 8;
    f32x4 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    __attribute__((aligned(16))) T wv[8];
    __attribute__((aligned(16))) T xv[8];
    fetch(wrow, sc, wv);
    fetch(xrow, sc, xv);
    for (int k0 = 0; k0 < a.k; k0 += BK) {
        __syncthreads();
        put(ws + sr * LD + sc, wv);
        put(xs + sr * LD + sc, xv);
        __syncthreads();
        if (k0 + BK < a.k) {
            fetch(wrow, k0 + BK + sc, wv);
            fetch(xrow, k0 + BK + sc, xv);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                Mfma<T>::mul(acc[i][j], ws + (wn + 16 * i + fr) * LD + fk, xs + (wm + 16 * j + fr) * LD + fk);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            finish<T>(a, vec_out, m0 + wm + 16 * j + fr, n0 + wn + 16 * i + (lane >> 4) * 4, acc[i][j]);
}

}  // namespace

int64_t linear_workspace_bytes(int dtype, int64_t m, int64_t n, int64_t k) {
    (void)dtype; (void)m; (void)n; (void)k;
    return 0;
}

hipError_t launch_linear(const LinearArgs& a, int dtype, hipStream_t stream) {
    const int64_t es = dtype == DIFA_DTYPE_BF16 ? 2 : 4;
    auto aligned = [&](const void* p, int64_t s0, int64_t s1, int64_t to) {
        return ((uintptr_t)p % to) == 0 && s0 * es % to == 0 && s1 * es % to == 0;
    };
    const bool vec_in = aligned(a.x, a.x_stride_b, a.x_stride_n, 16) && aligned(a.w, a.w_stride, 0, 16);
    const int64_t four = 4 * es;
    const bool vec_out = a.n % 4 == 0 && aligned(a.out, a.out_stride_b, a.out_stride_n, four) && aligned(a.bias, 0, 0, four) &&
                         aligned(a.gate, a.gate_stride_b, 0, four) && aligned(a.residual, a.res_stride_b, a.res_stride_n, four);
    const int64_t n_tiles = ((int64_t)a.n + 63) / 64, tiles = n_tiles * (((int64_t)a.m + 63) / 64);
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)tiles), threads(256);
    if (dtype == DIFA_DTYPE_BF16) {
        if (vec_in) linear_any_kernel<__bf16, true><<<grid, threads, 0, stream>>>(a, vec_out, (int)n_tiles);
        else linear_any_kernel<__bf16, false><<<grid, threads, 0, stream>>>(a, vec_out, (int)n_tiles);
    } else {
        if (vec_in) linear_any_kernel<float, true><<<grid, threads, 0, stream>>>(a, vec_out, (int)n_tiles);
        else linear_any_kernel<float, false><<<grid, threads, 0, stream>>>(a, vec_out, (int)n_tiles);
    }
    return hipGetLastError();
}

}  // namespace difa
