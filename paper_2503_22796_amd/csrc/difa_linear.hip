// out = residual + gate * act(x W^T + bias): the matrix product around the attention of a layer.
//   linear_tile_kernel   tiles of 256 x 256, 128 x 128 or (fp32) 64 x 128 and 64 x 64 sums; x and w by loads that write LDS
//   linear_rows_kernel   up to 32 rows of x: w straight into operands
//   linear_any_kernel    any alignment, any stride; linear_pad_kernel copies bf16 rows that do not start at multiples of 16
//                        bytes for the other two where a workspace has room
// Sums are held in fp32 and rounded once, behind the epilogue.  What bounds them, and what was tried, stands at each.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "difa_layer.h"

namespace difa {

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// ---- epilogue
// The activation of eight sums.  bf16's erf: Abramowitz and Stegun 7.1.26, within 1.5e-7, so that the activation is within 2^-23 of
// its argument; fp32 takes the complement, which is as exact on the negative side, where little is left.  So are fp32's SiLU and
// GELU tanh, v / (1 + exp(-z)), within 7 half steps of the result, where an exponent rounded to 32 bits costs |z| of them
// (4096 x 1536 -> 6144 548 and 551 us so, 557 and 562 as here; 4096 x 64 -> 4096 36 and 40, 41).
// |z| log2(e) = hi + lo; below: z < 0, the result is v exp(-|z|) / (1 + exp(-|z|)).
__device__ __forceinline__ float times_logistic(float v, bool below, float hi, float lo) {
    // The instruction knows no numbers below 2^-126: far out it gives 2^24 times as much (exactly: hi's steps are coarser than
    // the difference's).
    const bool tiny = hi > 100.f;
    float e = __builtin_amdgcn_exp2f((tiny ? 24.f : 0.f) - hi);
    e = fmaf(e, -0.69314718056f * lo, e);
    const float n = below ? e : 1.f, d = 1.f + e, r = __builtin_amdgcn_rcpf(d), q = n * r;
    const float y = v * fmaf(fmaf(-q, d, n), r, q);
    return tiny && below ? y * 0x1p-24f : y;
}
template <typename T> __device__ __forceinline__ void activate(int act, float (&v)[8]) {
    if (act == DIFA_ACT_GELU_TANH && sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // z log2(e), z = 2 sqrt(2 / pi) (y + 0.044715 y^3), in 64 bits, up to where exp(-z) is 0
            const double y = v[i], z = fmin(fabs(y * fma(y * y, 0.10294323958002349, 2.3022081981443248)), 200.0);
            const float hi = (float)z;
            v[i] = times_logistic(v[i], v[i] < 0.f, hi, (float)(z - (double)hi));
        }
    } else if (act == DIFA_ACT_SILU && sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // log2(e) in two parts; hi is rounded, whatever it is added to
#pragma clang fp contract(off)
            const float z = fminf(fabsf(v[i]), 140.f), hi = z * 1.44269502f;
            v[i] = times_logistic(v[i], v[i] < 0.f, hi, fmaf(z, 1.92596299e-08f, fmaf(z, 1.44269502f, -hi)));
        }
    } else if (act == DIFA_ACT_GELU_TANH) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // 0.5 y (1 + tanh u) = y / (1 + exp(-2 u)), u = sqrt(2 / pi) (y + 0.044715 y^3), in powers of two:
            // 2 sqrt(2 / pi) log2(e) = 2.3022082, times 0.044715 = 0.10294324
            const float z = v[i] * fmaf(v[i] * v[i], -0.10294324f, -2.3022082f);
            v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z));
        }
    } else if (act == DIFA_ACT_GELU_ERF && sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= 0.5f * erfcf(-0.70710678118f * v[i]);
    } else if (act == DIFA_ACT_GELU_ERF) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float z = fabsf(v[i]) * 0.70710678118f, t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, z, 1.f));
            float p = fmaf(1.061405429f, t, -1.453152027f);
            p = fmaf(p, t, 1.421413741f);
            p = fmaf(p, t, -0.284496736f);
            p = fmaf(p, t, 0.254829592f);
            const float tail = 0.5f * p * t * __builtin_amdgcn_exp2f(-1.44269504089f * z * z);       // erfc(z) / 2
            v[i] *= v[i] < 0.f ? tail : 1.f - tail;
        }
    } else if (act == DIFA_ACT_SILU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504089f * v[i]));
    }
}

template <typename T> struct Eight;      // eight consecutive values, 16-byte aligned
template <> struct Eight<__bf16> {
    static __device__ __forceinline__ void load(const __bf16* p, float (&v)[8]) {
        const u32x4 r = *(const u32x4*)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned u = r[i];
            v[2 * i] = __builtin_bit_cast(float, u << 16);
            v[2 * i + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
        }
    }
    static __device__ __forceinline__ void store(__bf16* p, const float (&v)[8]) {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 h = {(__bf16)v[2 * i], (__bf16)v[2 * i + 1]};
            r[i] = __builtin_bit_cast(unsigned, h);
        }
        // past the caches, which the loads need: 32768 x 6144 x 1536 534 us -> 494, 8192^3 770 -> 720
        __builtin_nontemporal_store(r, (u32x4*)p);
    }
};
template <> struct Eight<float> {
    static __device__ __forceinline__ void load(const float* p, float (&v)[8]) {
        const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    }
    static __device__ __forceinline__ void store(float* p, const float (&v)[8]) {
        *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
    }
};

// Features n .. n + 7 of row m of the result from the product's sums.  `vec`: all the epilogue's rows start at multiples of 16
// bytes and n is a multiple of eight, so that eight at a time are aligned and inside.
template <typename T>
__device__ __forceinline__ void finish(const LinearArgs& a, bool vec, int m, int n, float (&v)[8]) {
    if (m >= a.m || n >= a.n) return;
    const int b = a.batch == 1 ? 0 : m / a.rows, t = m - b * a.rows;
    const T* bias = (const T*)a.bias;
    const T* gate = a.gate ? (const T*)a.gate + b * a.gate_stride_b : nullptr;
    const T* res = a.residual ? (const T*)a.residual + b * a.res_stride_b + t * a.res_stride_n : nullptr;
    T* out = (T*)a.out + b * a.out_stride_b + t * a.out_stride_n;
    float e[8];
    if (vec) {
        float r[8];
        if (res) Eight<T>::load(res + n, r);
        if (bias) {
            Eight<T>::load(bias + n, e);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += e[i];
        }
        activate<T>(a.activation, v);
        if (gate) {
            Eight<T>::load(gate + n, e);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= e[i];
        }
        if (res) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += r[i];
        }
        Eight<T>::store(out + n, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (bias && n + i < a.n) v[i] += (float)bias[n + i];
    activate<T>(a.activation, v);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (n + i < a.n) {
            if (gate) v[i] *= (float)gate[n + i];
            if (res) v[i] += (float)res[n + i];
            out[n + i] = (T)v[i];
        }
}

// The same for rows of one batch entry that a lane meets one after the other, always at the same eight features: bias and gate
// stay in registers and the row's place moves on by additions.  A tile is finished while its workgroup's matrix cores stand
// still, and the vector units take four clocks an instruction (32768 x 6144 x 1536 540 us with `finish`, 534 so).
template <typename T> struct Columns {
    float bias[8], gate[8];
    const T *res;
    T* out;
    int64_t res_step, out_step;
    // features n .. n + 7 of row t of batch entry b, then every `step`th row
    __device__ __forceinline__ Columns(const LinearArgs& a, int b, int t, int n, int step) {
        if (a.bias) Eight<T>::load((const T*)a.bias + n, bias);
        if (a.gate) Eight<T>::load((const T*)a.gate + b * a.gate_stride_b + n, gate);
        out = (T*)a.out + b * a.out_stride_b + t * a.out_stride_n + n;
        out_step = step * a.out_stride_n;
        res = (const T*)a.residual + b * a.res_stride_b + t * a.res_stride_n + n;
        res_step = step * a.res_stride_n;
    }
    __device__ __forceinline__ void finish(const LinearArgs& a, bool inside, float (&v)[8]) {
        float r[8];
        if (a.residual && inside) Eight<T>::load(res, r);
        if (a.bias) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += bias[i];
        }
        activate<T>(a.activation, v);
        if (a.gate) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= gate[i];
        }
        if (a.residual) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += r[i];
        }
        if (inside) Eight<T>::store(out, v);
        out += out_step;
        res += res_step;
    }
};

// ---- any sizes, strides and alignments: 64 x 64 tiles, 32 features of k at a time through LDS, four wavefronts of 32 x 32.  Bound by
// its loads, one value at a time where rows are not aligned (8000 x 5000 x 3001, bf16: 4651 us, by way of copies 250): it serves
// what is small, or comes without a workspace.  A lane's eight values of k are consecutive for both operands, so it
// does not matter which of them the matrix instruction takes for which.
template <typename T> struct Mfma;
template <> struct Mfma<__bf16> {
    static __device__ __forceinline__ void mul(f32x4& d, const __bf16* w, const __bf16* x) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8*)w, *(const bf16x8*)x, d, 0, 0, 0);
    }
};
template <> struct Mfma<float> {
    static __device__ __forceinline__ void mul(f32x4& d, const float* w, const float* x) {
#pragma unroll
        for (int i = 0; i < 8; ++i) d = __builtin_amdgcn_mfma_f32_16x16x4f32(w[i], x[i], d, 0, 0, 0);
    }
};

template <typename T, bool VEC>                          // VEC: x and w can be read 16 bytes at a time
__global__ __launch_bounds__(256) void linear_any_kernel(LinearArgs a, bool vec_out, unsigned first, int n_tiles) {
    constexpr int BT = 64, BK = 32, PAD = 16 / (int)sizeof(T), LD = BK + PAD;
    __shared__ __attribute__((aligned(16))) char lds[2 * BT * LD * sizeof(T) > BT * (BT + 4) * 4 ? 2 * BT * LD * sizeof(T) : BT * (BT + 4) * 4];
    T *ws = (T*)lds, *xs = ws + BT * LD;
    float* sums = (float*)lds;
    const unsigned place = first + blockIdx.x;
    const int tile_n = place % n_tiles, tile_m = place / n_tiles;
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
    f32x4 total[2][2];                                     // fp32: sums of 512 products at a time, see linear_tile_kernel
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) total[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < a.k; k0 += BK) {
        if (sizeof(T) == 4 && k0 % 512 == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    total[i][j] += acc[i][j];
                    acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
        }
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
    // through LDS, so that a thread finishes eight features of a row
    __syncthreads();
    constexpr int LS = BT + 4;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) *(f32x4*)(sums + (wm + 16 * j + fr) * LS + wn + 16 * i + (lane >> 4) * 4) = acc[i][j] + total[i][j];
    __syncthreads();
#pragma unroll 1
    for (int r = tid >> 3; r < BT; r += 32) {
        float v[8];
        Eight<float>::load(sums + r * LS + (tid & 7) * 8, v);
        finish<T>(a, vec_out, m0 + r, n0 + (tid & 7) * 8, v);
    }
}

// A 16-byte operand: products of 16 features and 16 rows over its chunk of k.  The matrix instruction counts k in another order,
// the same one for both operands.
template <typename T> struct Operand;
template <> struct Operand<__bf16> {
    typedef bf16x8 type;
    static constexpr int PARTS = 1;
    static __device__ __forceinline__ void multiply(f32x4& d, const bf16x8& w, const bf16x8& x, int) {
        d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, d, 0, 0, 0);
    }
};
template <> struct Operand<float> {
    typedef f32x4 type;
    static constexpr int PARTS = 4;
    static __device__ __forceinline__ void multiply(f32x4& d, const f32x4& w, const f32x4& x, int part) {
        d = __builtin_amdgcn_mfma_f32_16x16x4f32(w[part], x[part], d, 0, 0, 0);
    }
};

// ---- few rows: up to 16 * MB.  w is read once, straight into operands, by workgroups of 16 features whose wavefronts share k
// out; their sums meet in LDS.  Bound by w's bytes, so what counts is that every load is on its way early: sixteen 16-byte
// loads of w and of x a lane (eight and sixteen for up to 32 rows) before the first product.  2 rows, 1536 -> 9216: 8.8 us
// a call among others, 7.9 to 9.4 in the kernel, 3.1 TB/s; eight wavefronts a workgroup instead of four 10.8, w read past the caches 9.7.
template <typename T, int MB>
__global__ __launch_bounds__(512) void linear_rows_kernel(LinearArgs a, bool vec_out, unsigned first) {
    typedef typename Operand<T>::type Op;
    constexpr int CHUNK = 16 / sizeof(T), STEP = 4 * CHUNK, DEPTH = MB == 1 ? 16 : 8, LS = 20;    // LS: floats between rows of a block in LDS
    extern __shared__ __attribute__((aligned(16))) float sums[];                    // [wavefront][row][LS]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
    const int n0 = (int)(first + blockIdx.x) * 16, chunk = (lane >> 4) * CHUNK;
    // whole lines of k for every wavefront
    const int lines = (a.k + 2 * STEP - 1) / (2 * STEP);
    const int k0 = (int)((int64_t)lines * wave / n_waves) * 2 * STEP, k1 = (int)((int64_t)lines * (wave + 1) / n_waves) * 2 * STEP;
    const int end = k1 < a.k ? k1 : a.k;
    const int r = n0 + (lane & 15);
    const T* w = (const T*)a.w + (int64_t)(r < a.n ? r : a.n - 1) * a.w_stride + chunk;      // past the end: read, not kept
    const T* x[MB];
#pragma unroll
    for (int j = 0; j < MB; ++j) {
        const int m = j * 16 + (lane & 15) < a.m ? j * 16 + (lane & 15) : a.m - 1, b = m / a.rows, t = m - b * a.rows;
        x[j] = (const T*)a.x + b * a.x_stride_b + t * a.x_stride_n + chunk;
    }
    f32x4 acc[MB], total[MB];                              // fp32: sums of DEPTH * STEP products at a time, see linear_tile_kernel
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[j] = total[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    const Op zero = {};
#pragma unroll 1
    for (int k = k0; k < end; k += DEPTH * STEP) {
        Op wv[DEPTH], xv[DEPTH][MB];
#pragma unroll
        for (int i = 0; i < DEPTH; ++i) {
            const bool in = k + i * STEP + chunk < end;
            wv[i] = in ? *(const Op*)(w + k + i * STEP) : zero;
#pragma unroll
            for (int j = 0; j < MB; ++j) xv[i][j] = in ? *(const Op*)(x[j] + k + i * STEP) : zero;
        }
#pragma unroll
        for (int i = 0; i < DEPTH; ++i)
#pragma unroll
            for (int part = 0; part < Operand<T>::PARTS; ++part)
#pragma unroll
                for (int j = 0; j < MB; ++j) Operand<T>::multiply(acc[j], wv[i], xv[i][j], part);
        if (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < MB; ++j) {
                total[j] += acc[j];
                acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            }
        }
    }
#pragma unroll
    for (int j = 0; j < MB; ++j) *(f32x4*)(sums + ((wave * MB + j) * 16 + (lane & 15)) * LS + (lane >> 4) * 4) = sizeof(T) == 4 ? total[j] : acc[j];
    __syncthreads();
    const int m = threadIdx.x / 2, col = threadIdx.x % 2 * 8;
    if (m >= 16 * MB) return;
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < n_waves; ++i) {
        float s[8];
        Eight<float>::load(sums + (i * MB * 16 + m) * LS + col, s);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += s[e];
    }
    finish<T>(a, vec_out, m, n0 + col, v);
}

template <typename T, int MB> hipError_t launch_rows(const LinearArgs& a, bool vec_out, hipStream_t stream) {
    // wavefronts for every compute unit's four SIMDs twice over, each with a line of k at least
    const int groups = (a.n + 15) / 16, lines = (int)((a.k * (int64_t)sizeof(T) + 127) / 128);
    int waves = 2048 / groups;
    waves = waves < 4 ? 4 : waves > 8 ? 8 : waves;
    waves = waves < lines ? waves : lines;
    return in_slices(groups, [&](unsigned first, unsigned blocks) {
        linear_rows_kernel<T, MB><<<dim3(blocks), dim3(64 * waves), waves * MB * 16 * 20 * 4, stream>>>(a, vec_out, first);
        return hipGetLastError();
    });
}

// ---- rows of x and w that start at multiples of 16 bytes: tiles of TN features x TM rows.  (Numbers of values: bf16; fp32 has
// half as many in the same bytes, and four products of v_mfma_f32_16x16x4_f32 for one of 16x16x32.)
//
// 64 values of k at a time come through two LDS stages, written by the loads themselves (buffer_load_dwordx4 ... lds:
// lane l of a wavefront deposits its 16 bytes at M0 + 16 l, so that one instruction fills eight rows of 128 bytes).
// Whole lines: 32 values of k a stage and four stages asked the L2 for half a line at a time, and the L2 serves
// requests, not bytes (8192^3 with 128 x 128 tiles: 14.5 TB/s, one 64-byte request per channel and clock).
// A stage is multiplied in two steps of 32 values of k.  Each step reads the operands of the next one, so that no matrix instruction
// waits for a read; the step that ends a stage's reads ends in the stage's one barrier, which also publishes
// the next stage, and the step after it requests the stage after that into the freed place: a load has two steps to land.
// A b128 operand read is served 16 lanes at a time, and they are not neighbours: lanes 0-3, 12-15 and 20-27, then 4-11, 16-19 and
// 28-31, and the upper half alike.  Chunk c (16 bytes) of row r is stored at c ^ (r / 2) % 8, which puts the 16 rows and two
// chunks of each set into 64 different banks.  The permutation is applied to what each lane fetches.
// Rows past the end and, in the last stage, chunks past k are requested beyond the buffer and arrive as zeros.
// fp32 rows that do not start at multiples of 16 bytes come the same way a value a lane (PIECE = 4 bytes: an instruction fills
// two rows), four times the instructions: 105 x 7587 x 3881 112 (with copies) -> 87 us; with aligned rows of 3880 68-71.
constexpr int kLine = 128;                  // bytes of a row per stage
constexpr unsigned kOutside = 0x80000000u;  // an offset beyond every buffer

// The grid: `parts` workgroups for every tile, each with its share of k; a launch runs those from number `first` on.
struct TileMap { int n_tiles, m_tiles, parts, per_die, rest; unsigned first; };
struct Tile { int m, n, index, part; };

// Workgroup p runs on die p % 8; each die takes a run of consecutive places (`rest` dies one more than the others): the tiles
// of one part of k, four rows of tiles at a time and feature by feature, so that what runs on a die at one time
// shares x and w in its L2.  8192^3 with 2, 4, 8 and 16 rows: 790, 768, 779 and 795 us.
__device__ __forceinline__ Tile tile_of(const TileMap& map) {
    const unsigned wg = map.first + blockIdx.x;
    const int die = wg % 8, p = die * map.per_die + (die < map.rest ? die : map.rest) + wg / 8;
    const int tiles = map.n_tiles * map.m_tiles, part = p / tiles, t = p - part * tiles;
    constexpr int ROWS = 4;
    const int group = t / (ROWS * map.n_tiles), in = t - group * ROWS * map.n_tiles;
    const int rows = map.m_tiles - group * ROWS < ROWS ? map.m_tiles - group * ROWS : ROWS;
    const int n = in / rows;
    return {group * ROWS + in - n * rows, n, t, part};
}

// Workspace: a ticket per tile, zero between calls, then the parts' sums.
constexpr int kTickets = 4096;
constexpr int kDeviceCoherent = 16;          // cache policy of the buffer builtins: written through, read around a stale L2 line ("sc1")

template <typename T, int WN, int WM, int NB, int MB, int NS, int PIECE>
__global__ __launch_bounds__(WN * WM * 64, 2) void linear_tile_kernel(LinearArgs a, TileMap map, bool vec_out) {
    constexpr int NW = WN * WM, TN = WN * NB * 16, TM = WM * MB * 16;
    constexpr int ES = sizeof(T), kStage = kLine / ES;         // values per stage
    typedef typename Operand<T>::type Op;
    constexpr int RPI = PIECE / 2;                                         // rows per load instruction
    constexpr int LW = TN / RPI / NW, LX = TM / RPI / NW, LOADS = LW + LX; // load instructions per wavefront and stage
    static_assert(PIECE == 16 || (PIECE == 4 && ES == 4), "");
    static_assert(LW * RPI % 16 == 0 && LX * RPI % 16 == 0, "the chunk a lane fetches goes by the instruction's number");
    constexpr int STAGE = (TN + TM) * kLine;                               // bytes
    // The sums leave through LDS, PASSES parts of the tile's rows one after the other.
    constexpr int LS = TN + 4, PASSES = TM * LS * 4 <= NS * STAGE + 8192 ? 1 : 2, JB = MB / PASSES, ROWS = TM / PASSES;
    __shared__ __attribute__((aligned(1024))) char lds[NS * STAGE > ROWS * LS * 4 ? NS * STAGE : ROWS * LS * 4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Tile tile = tile_of(map);
    const int m0 = tile.m * TM, n0 = tile.n * TN;
    const int all = (a.k + kStage - 1) / kStage;                           // stages of k; this workgroup's: [first, stages)
    const int first = (int)((int64_t)all * tile.part / map.parts), stages = (int)((int64_t)all * (tile.part + 1) / map.parts);

    // ---- where this lane's share of the loads comes from: instruction i fills rows RPI * i and on
    const int left = a.k - (all - 1) * kStage;                             // of k in the last stage
    const int row = PIECE == 16 ? lane >> 3 : lane >> 5;
    auto byte_of = [&](int i) __attribute__((always_inline)) {             // in the row's 128
        return PIECE == 16 ? ((lane & 7) ^ (lane >> 4) ^ (i % 2 * 4)) * 16 : (((lane >> 2) & 7) ^ (i % 8)) * 16 + (lane & 3) * 4;
    };
    unsigned past[16 / RPI];
#pragma unroll
    for (int i = 0; i < 16 / RPI; ++i) past[i] = byte_of(i) < left * ES ? 0u : kOutside;
    const int b0 = m0 / a.rows, t0 = m0 - b0 * a.rows;
    const int64_t x0 = b0 * a.x_stride_b + t0 * a.x_stride_n;
    unsigned from[LOADS];
#pragma unroll
    for (int i = 0; i < LW; ++i) {
        const int r = (wave * LW + i) * RPI + row;
        from[i] = n0 + r < a.n ? (unsigned)(r * a.w_stride * ES) + byte_of(i) : kOutside;
    }
#pragma unroll
    for (int i = 0; i < LX; ++i) {
        const int m = m0 + (wave * LX + i) * RPI + row;
        const int b = m / a.rows, t = m - b * a.rows;
        from[LW + i] = m < a.m ? (unsigned)((b * a.x_stride_b + t * a.x_stride_n - x0) * ES) + byte_of(i) : kOutside;
    }
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const char* wbase = (const char*)a.w + (int64_t)n0 * a.w_stride * ES;
    const char* xbase = (const char*)a.x + x0 * ES;
    u32x4 wr, xr;                                          // descriptors of the stage that is being requested
    bool last;
    auto aim = [&](int stage) __attribute__((always_inline)) {
        const unsigned size = stage < stages ? 0x7fffffffu : 0u;       // behind the last one: nothing is read
        last = stage == all - 1;
        const char* wp = wbase + (int64_t)stage * kLine;
        const char* xp = xbase + (int64_t)stage * kLine;
        wr = u32x4{(unsigned)(uintptr_t)wp, (unsigned)((uintptr_t)wp >> 32) & 0xffffu, size, 0x00020000u};
        xr = u32x4{(unsigned)(uintptr_t)xp, (unsigned)((uintptr_t)xp >> 32) & 0xffffu, size, 0x00020000u};
    };
    auto request = [&](int i, int place) __attribute__((always_inline)) {
        const unsigned to = lds0 + place * STAGE + (i < LW ? wave * LW + i : TN / RPI + wave * LX + i - LW) * (RPI * 128);
        const unsigned off = from[i] | (last ? past[i % (16 / RPI)] : 0u);     // (LW is a multiple)
        if constexpr (PIECE == 16)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" :: "s"(to), "v"(off), "s"(i < LW ? wr : xr) : "memory", "m0");
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" :: "s"(to), "v"(off), "s"(i < LW ? wr : xr) : "memory", "m0");
    };

    // ---- operands: this lane's row and chunk, chunks of the second step 64 bytes away
    const int wn = wave % WN, wm = wave / WN;
    const unsigned at = lds0 + (lane & 15) * 128 + (((lane >> 4) ^ (lane >> 1)) & 7) * 16;
    unsigned wl[2] = {at + wn * NB * 2048, 0}, xl[2] = {at + TN * 128 + wm * MB * 2048, 0};
    wl[1] = wl[0] ^ 64;
    xl[1] = xl[0] ^ 64;
    Op w[2][NB], x[2][MB];
    f32x4 acc[NB][MB];
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int j = 0; j < MB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // operand i of step `half` of the stage in `place`: x's MB blocks first, then w's NB
    auto read = [&](int place, int half, int i) __attribute__((always_inline)) {
        const unsigned p = (i < MB ? xl[half] + i * 2048 : wl[half] + (i - MB) * 2048) + place * STAGE;
        const Op v = *(const __attribute__((address_space(3))) Op*)(uintptr_t)p;
        if (i < MB) x[half][i] = v; else w[half][i - MB] = v;
    };
    // A step is laid out by hand, MB matrix instructions at a time with what runs under them.
    auto step = [&](int place, int half) __attribute__((always_inline)) {
        constexpr int READS = (NB + MB + NB - 2) / (NB - 1);           // per group; the last group has none
        constexpr int REQUESTS = (LOADS + NB - 1) / NB;
#pragma unroll
        for (int i = 0; i < NB; ++i) {
#pragma unroll
            for (int part = 0; part < Operand<T>::PARTS; ++part)
#pragma unroll
                for (int j = 0; j < MB; ++j) Operand<T>::multiply(acc[i][j], w[half][i], x[half][j], part);
            __builtin_amdgcn_sched_barrier(0);
            if (half == 1) {
#pragma unroll
                for (int r = i * REQUESTS; r < (i + 1) * REQUESTS && r < LOADS; ++r) request(r, place);
            }
#pragma unroll
            for (int r = i * READS; r < (i + 1) * READS && r < NB + MB; ++r) read(half ? (place + 1) % NS : place, 1 - half, r);
        }
        if (half == 0) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"((NS - 2) * LOADS) : "memory");
        __builtin_amdgcn_sched_barrier(0);
    };

#pragma unroll
    for (int s = 0; s < NS; ++s) {
        aim(first + s);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) request(i, s);
    }
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"((NS - 1) * LOADS) : "memory");
#pragma unroll
    for (int i = 0; i < NB + MB; ++i) read(0, 0, i);
    auto stage = [&](int s, int place) __attribute__((always_inline)) {
        step(place, 0);
        aim(s + NS);
        step(place, 1);
    };
    // fp32: sums of 512 products are set aside and added up among themselves, so that no chain of roundings grows with k
    // (k = 3512: 1.2e-6 of the result without, where the library has 0.6e-6).  bf16's result is rounded to 4e-3.
    constexpr bool ASIDE = sizeof(T) == 4;
    f32x4 total[ASIDE ? NB : 1][ASIDE ? MB : 1];
    if constexpr (ASIDE) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) total[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    auto set_aside = [&]() __attribute__((always_inline)) {
        if constexpr (ASIDE) {
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) {
                    total[i][j] += acc[i][j];
                    acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
                }
        }
    };
    int s = first;
    for (; s + NS <= stages; s += NS) {
#pragma unroll
        for (int place = 0; place < NS; ++place) stage(s + place, place);
        if (ASIDE && (s - first) % 16 == 16 - NS) set_aside();
    }
#pragma unroll
    for (int place = 0; place < NS - 1; ++place)
        if (s + place < stages) stage(s + place, place);
    if constexpr (ASIDE) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < MB; ++j) acc[i][j] += total[i][j];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");       // nothing may land in LDS that is no longer this workgroup's

    if constexpr (NS > 2) {                                // the deep rings are for few tiles
        if (map.parts > 1) {
            // Every part leaves its sums in the workspace, in the order of the registers, and takes a ticket of the tile; the
            // one that draws the last ticket adds the parts in the order of their numbers and finishes the tile.  Stores and
            // loads are device-coherent: another part may run on another die, with an L2 of its own.
            __shared__ int ticket;
            constexpr int SLOT = TN * TM * 4, MINE = NB * MB * 1024, P = 3;    // P: parts in flight, as the reads come from memory
            char* slots = (char*)a.workspace + kTickets * 4 + (int64_t)tile.index * map.parts * SLOT;
            const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(slots, 0, map.parts * SLOT, 0x00020000);
            const unsigned mine = wave * MINE + __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0)) * 16;
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, acc[i][j]), rsrc, mine + (i * MB + j) * 1024, tile.part * SLOT, kDeviceCoherent);
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
            if (threadIdx.x == 0) ticket = atomicAdd((int*)a.workspace + tile.index, 1);
            __syncthreads();
            if (ticket != map.parts - 1) return;
            if (threadIdx.x == 0) atomicExch((int*)a.workspace + tile.index, 0);
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j < MB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
            for (int p0 = 0; p0 < map.parts; p0 += P) {
                u32x4 q[P][NB][MB];
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const unsigned at = p0 + p < map.parts ? mine : kOutside;  // zeros
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int j = 0; j < MB; ++j)
                            q[p][i][j] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, at + (i * MB + j) * 1024, (p0 + p) * SLOT, kDeviceCoherent);
                }
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int i = 0; i < NB; ++i)
#pragma unroll
                        for (int j = 0; j < MB; ++j) acc[i][j] += __builtin_bit_cast(f32x4, q[p][i][j]);
            }
        }
    }

    // ---- the sums, row by row: a lane has eight features of every STRIDE-th row of a pass
    float* sums = (float*)lds;
    constexpr int PER_ROW = TN / 8, STRIDE = NW * 64 / PER_ROW;
    static_assert(PASSES == 1 || JB * 16 % STRIDE == 0, "");
    // the thread's number made anew: nothing of it is held through the loop above
    const int tid = wave * 64 + __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
    const int row0 = tid / PER_ROW, col = tid % PER_ROW * 8, n = n0 + col;
    // a pass holds rows [pass * JB * 16, ...) of every wm's share of MB * 16
    auto row_in_tile = [&](int pass, int r) { return PASSES == 1 ? r : (r / (JB * 16) * MB + pass * JB) * 16 + r % (JB * 16); };
    const int rows_here = a.m - m0 < TM ? a.m - m0 : TM;
    const bool simple = vec_out && t0 + rows_here <= a.rows;
#pragma unroll 1
    for (int pass = 0; pass < PASSES; ++pass) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NB; ++i)
#pragma unroll
            for (int j = 0; j < JB; ++j) {
                f32x4 v = acc[i][j];
                if (PASSES == 2 && pass == 1) v = acc[i][MB - JB + j];
                *(f32x4*)(sums + ((wm * JB + j) * 16 + (tid & 15)) * LS + (wn * NB + i) * 16 + (tid >> 4) % 4 * 4) = v;
            }
        __syncthreads();
        if (simple) {
            if (n >= a.n) continue;
#pragma unroll 1
            for (int w = 0; w < ROWS; w += PASSES == 1 ? ROWS : JB * 16) {      // runs of rows that follow each other
                const int first_row = row_in_tile(pass, w) + row0;
                Columns<T> columns(a, b0, t0 + first_row, n, STRIDE);
#pragma unroll 2
                for (int r = 0; r < (PASSES == 1 ? ROWS : JB * 16); r += STRIDE) {
                    float v[8];
                    Eight<float>::load(sums + (w + row0 + r) * LS + col, v);
                    columns.finish(a, first_row + r < rows_here, v);
                }
            }
        } else {
#pragma unroll 1
            for (int r = row0; r < ROWS; r += STRIDE) {
                float v[8];
                Eight<float>::load(sums + r * LS + col, v);
                finish<T>(a, vec_out, m0 + row_in_tile(pass, r), n, v);
            }
        }
    }
}

template <typename T, int WN, int WM, int NB, int MB, int NS, int PIECE = 16>
hipError_t launch_tiles(const LinearArgs& a, int parts, bool vec_out, hipStream_t stream) {
    constexpr int TN = WN * NB * 16, TM = WM * MB * 16;
    const int64_t n_tiles = ((int64_t)a.n + TN - 1) / TN, m_tiles = ((int64_t)a.m + TM - 1) / TM, places = n_tiles * m_tiles * parts;
    if (places > 0x7fffffff) return hipErrorInvalidValue;
    return in_slices(places, [&](unsigned first, unsigned blocks) {
        const TileMap map = {(int)n_tiles, (int)m_tiles, parts, (int)(places / 8), (int)(places % 8), first};
        linear_tile_kernel<T, WN, WM, NB, MB, NS, PIECE><<<dim3(blocks), dim3(WN * WM * 64), 0, stream>>>(a, map, vec_out);
        return hipGetLastError();
    });
}

// ---- rows that cannot be read 16 bytes at a time, copied to where they can: x's m rows, then w's n, `padded` values each with
// zeros behind the k-th.  A wavefront moves 512 values of a row, 64 neighbours at a time.
template <typename T>
__global__ __launch_bounds__(256) void linear_pad_kernel(LinearArgs a, unsigned first, T* to, int padded, int pieces) {
    const int lane = threadIdx.x & 63;
    const int64_t item = ((int64_t)first + blockIdx.x) * 4 + (threadIdx.x >> 6), r = item / pieces;
    if (r >= (int64_t)a.m + a.n) return;
    const int c = (int)(item - r * pieces) * 512 + lane;
    const T* from;
    if (r < a.m) {
        const int64_t b = r / a.rows, t = r - b * a.rows;
        from = (const T*)a.x + b * a.x_stride_b + t * a.x_stride_n;
    } else {
        from = (const T*)a.w + (r - a.m) * a.w_stride;
    }
    T v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = c + i * 64 < a.k ? from[c + i * 64] : (T)0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (c + i * 64 < padded) to[r * padded + c + i * 64] = v[i];
}

template <typename T> hipError_t launch_any(const LinearArgs& a, bool vec_in, bool vec_out, hipStream_t stream) {
    const int64_t n_tiles = ((int64_t)a.n + 63) / 64, tiles = n_tiles * (((int64_t)a.m + 63) / 64);
    if (tiles > 0x7fffffff) return hipErrorInvalidValue;
    return in_slices(tiles, [&](unsigned first, unsigned blocks) {
        if (vec_in) linear_any_kernel<T, true><<<dim3(blocks), dim3(256), 0, stream>>>(a, vec_out, first, (int)n_tiles);
        else linear_any_kernel<T, false><<<dim3(blocks), dim3(256), 0, stream>>>(a, vec_out, first, (int)n_tiles);
        return hipGetLastError();
    });
}

}  // namespace

namespace {

// What a product runs on: kernels of 256 x 256 (one workgroup on a compute unit) or 128 x 128 sums (two), two stages
// each, or of 128 x 128 with four stages (one), which a product of few tiles needs, its k cut into parts for more of them; fp32
// also 64 x 128 (features x rows), two stages, and 64 x 64 (two) with four stages and in parts;
// and the kernel for few rows.
constexpr int64_t kFewRows = 32;
enum Form { kRows, kWide, kHalf, kQuarter, kDeep, kSmall };
struct Choice { Form form; int parts; };
struct Sums { int n, m; };                                 // of a tile that takes parts
constexpr Sums sums_of(Form f) { return f == kSmall ? Sums{64, 64} : Sums{128, 128}; }

// The form with the earliest end by what one round of workgroups was measured to take, us: a stage of k and the rest.  bf16, us
// (wide / half / deep, one MI355X, 256 compute units; m x n x k):
//   32768 x 6144 x 1536  526 / 620 / 707    8192 x 4608 x 1536  122 / 122 / 136     8192 x 1536 x 1536  39.8 / 46.9 / 47.0
//   32768 x 1536 x 6144  502 / 594 / 642    8192 x 1536 x 6144  150 / 190 / 172     4096 x 1536 x 1536  36.4 / 25.0 / 29.9
//   2048 x 1536 x 1536   36.1 / 22.0 / 16.0  1333 x 2000 x 3000  65.7 / 42.7 / 33.2  666 x 6144 x 1536   35.5 / 22.1 / 28.0
//   666 x 1536 x 6144    112 / 61.6 / 39.3, deep in two parts 28.7, in three 25.9;  333 x 1536 x 1536 35.4 / 19.9 / 14.2, 14.6, 14.5
// fp32 is bound by its matrix instructions, 1.71 us for a stage of 128 x 128 sums on a compute unit: what counts is that the
// tiles come out even, for which products of few tiles take 64 x 64 in parts (0.47 us a stage, 0.57 for one alone on its unit;
// more requests to the L2 than the larger tiles: 8192 x 1536 x 1536 291 instead of 278).  us, half / quarter / small in parts:
//   666 x 1536 x 6144   367 / 204 / 131 (3)     771 x 2472 x 1616  101 / 101 / 56.5 (1)   642 x 1244 x 1816  116 / 64.7 / 37.8 (1)
//   406 x 232 x 4376    257 / 142 / 18.8 (8)    5416 x 376 x 4640  274 / 276 / 148 (1)    6366 x 148 x 5092  305 / 173 / 113 (3)
// values: fp32 rows that come a value a lane, for which there is the small form.
Choice choose(int dtype, int64_t m, int64_t n, int64_t k, bool values) {
    constexpr int64_t kUnits = 256;
    const bool f32 = dtype != DIFA_DTYPE_BF16;
    if (m <= kFewRows && !values) return {kRows, 1};
    const int64_t stages = (k * (f32 ? 4 : 2) + kLine - 1) / kLine;
    auto tiles = [&](int64_t tn, int64_t tm) { return ((m + tm - 1) / tm) * ((n + tn - 1) / tn); };
    const int64_t half = tiles(128, 128), rest = half % (2 * kUnits);
    Choice c = {kHalf, 1};
    double best;
    if (f32) {
        const int64_t quarter = tiles(64, 128);
        best = (double)((half + kUnits - 1) / kUnits) * 1.71 * stages + 5;
        const double quarters = (double)((quarter + kUnits - 1) / kUnits) * 0.88 * stages + 5;
        if (quarters < best) { best = quarters; c = {kQuarter, 1}; }
        if (values) best = HUGE_VAL;
    } else {
        best = (double)(half / (2 * kUnits)) * (0.94 * stages + 5) + (rest > kUnits ? 0.94 * stages + 5 : rest > 0 ? 0.75 * stages + 5 : 0);
        const double wide = (double)((tiles(256, 256) + kUnits - 1) / kUnits) * (1.5 * stages + 6);
        if (wide <= best) { best = wide; c = {kWide, 1}; }
    }
    for (int64_t parts = 1; !f32 && parts <= 8 && parts * 4 <= std::max<int64_t>(stages, 4); ++parts) {
        if (parts > 1 && half * parts > kUnits) break;
        const double stage = half * parts > kUnits * 5 / 8 ? 0.58 : 0.45;
        const double deep = (double)((half * parts + kUnits - 1) / kUnits) * (stage * ((stages + parts - 1) / parts) + 6) + (parts > 1 ? 6 : 0);
        if (deep < best) { best = deep; c = {kDeep, (int)parts}; }
    }
    if (f32) {
        const int64_t count = tiles(64, 64);
        for (int64_t parts = 1; parts <= 16 && parts * 4 <= std::max<int64_t>(stages, 4); ++parts) {
            if (parts > 1 && count * parts > 4 * kUnits) break;
            const int64_t on_unit = (count * parts + kUnits - 1) / kUnits, stages_here = (stages + parts - 1) / parts;
            const double t = (on_unit == 1 ? 0.57 : on_unit * 0.47) * stages_here + 6 + (parts > 1 ? 4 + 0.002 * count * parts : 0);
            if (t < best) { best = t; c = {kSmall, (int)parts}; }
        }
    }
    return c;
}
bool values_apart(int64_t k, int64_t es) { return es == 4 && k * es % 16 != 0; }
int64_t split_bytes(int64_t m, int64_t n, Choice c) {
    const Sums s = sums_of(c.form);
    return c.parts == 1 ? 0 : kTickets * 4 + ((m + s.m - 1) / s.m) * ((n + s.n - 1) / s.n) * c.parts * (int64_t)(s.m * s.n * 4);
}

// (choose gives a type no form that is the other's)
template <typename T> hipError_t launch_aligned(const LinearArgs& a, Choice c, bool values, bool vec_out, hipStream_t stream) {
    if (c.form == kRows) return a.m <= 16 ? launch_rows<T, 1>(a, vec_out, stream) : launch_rows<T, 2>(a, vec_out, stream);
    if (c.form == kHalf) return launch_tiles<T, 2, 2, 4, 4, 2>(a, 1, vec_out, stream);
    if constexpr (sizeof(T) == 2) {
        if (c.form == kWide) return launch_tiles<T, 2, 4, 8, 4, 2>(a, 1, vec_out, stream);
        if (c.form == kDeep) return launch_tiles<T, 2, 4, 4, 2, 4>(a, c.parts, vec_out, stream);
    } else {
        if (c.form == kQuarter) return launch_tiles<T, 2, 2, 2, 4, 2>(a, 1, vec_out, stream);
        if (c.form == kSmall) return values ? launch_tiles<T, 2, 2, 2, 2, 4, 4>(a, c.parts, vec_out, stream)
                                            : launch_tiles<T, 2, 2, 2, 2, 4>(a, c.parts, vec_out, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace

namespace {

constexpr int64_t padded_k(int64_t k, int64_t es) { return (k * es + kLine - 1) / kLine * kLine / es; }

// Whether a bf16 product whose rows do not start at multiples of 16 bytes is worth copying them: the kernel for any rows takes some 1.3 us
// for 32 values of k and a tile of 64 x 64 on every compute unit, the copies 8 us and their bytes at 3 TB/s.  (Rows that do, and come
// here because they are far apart, take it a quarter of that: 2 x 77 rows of 1536, entries 46 M values apart, 1536 features 19.9 us,
// by copies 22.6, side by side 17.3.)
bool worth_copies(int64_t m, int64_t n, int64_t k, int64_t es) {
    if (es == 4 || padded_k(k, es) > (1 << 20)) return false;              // fp32 has no need of them; the fast kernels' longest row
    const double tiles = (double)((m + 63) / 64) * (double)((n + 63) / 64) / 256;
    return 1.3 * (double)((k + 31) / 32) * (tiles > 1 ? tiles : 1) > 8 + 2e-6 / 3 * (double)(m + n) * (double)(k * es);
}
int64_t copy_bytes(int64_t m, int64_t n, int64_t k, int64_t es) { return (m + n) * padded_k(k, es) * es; }

}  // namespace

int64_t linear_workspace_bytes(int dtype, int64_t m, int64_t n, int64_t k) {
    const int64_t es = dtype == DIFA_DTYPE_BF16 ? 2 : 4;
    if (es == 4 || k * es % 16 == 0) return split_bytes(m, n, choose(dtype, m, n, k, values_apart(k, es)));
    if (!worth_copies(m, n, k, es)) return 0;
    const int64_t split = split_bytes(m, n, choose(dtype, m, n, padded_k(k, es), false));
    return (split ? split : kTickets * 4) + copy_bytes(m, n, k, es);
}

hipError_t launch_linear(const LinearArgs& given, int dtype, hipStream_t stream) {
    LinearArgs a = given;
    // strides that nothing is multiplied by: whatever they are, they cost no call the fast kernels
    if (a.batch == 1) a.x_stride_b = a.out_stride_b = a.res_stride_b = a.gate_stride_b = 0;
    if (a.rows == 1) a.x_stride_n = a.out_stride_n = a.res_stride_n = 0;
    const int64_t es = dtype == DIFA_DTYPE_BF16 ? 2 : 4;
    auto aligned = [&](const void* p, int64_t s0, int64_t s1, int64_t to) {
        return ((uintptr_t)p % to) == 0 && s0 * es % to == 0 && s1 * es % to == 0;
    };
    const bool vec_in = aligned(a.x, a.x_stride_b, a.x_stride_n, 16) && aligned(a.w, a.w_stride, 0, 16);
    const bool vec_out = a.n % 8 == 0 && aligned(a.out, a.out_stride_b, a.out_stride_n, 16) && aligned(a.bias, 0, 0, 16) &&
                         aligned(a.gate, a.gate_stride_b, 0, 16) && aligned(a.residual, a.res_stride_b, a.res_stride_n, 16);
    // Rows are fetched 16 bytes at a time, and the loads' 32-bit offsets span a tile's rows: at most 256, with the gaps between batch
    // entries, counted as if there were as many entries as 256 rows can meet.  Entries whose rows do not follow each other (one x for
    // all, or rows of the entries in turn) would want offsets below zero: these and longer gaps go by way of copies or one by one.
    const int64_t gap = a.batch == 1 ? 0 : a.x_stride_b - a.rows * a.x_stride_n;
    const bool near = a.x_stride_n <= (1 << 20) && a.w_stride <= (1 << 20) && gap >= 0 && gap <= (1 << 27) / (256 / a.rows + 1);
    const bool values = es == 4 && !(vec_in && a.k * es % 16 == 0);
    if (values ? near : vec_in && a.k * es % 16 == 0 && (near || a.m <= kFewRows)) {
        Choice c = choose(dtype, a.m, a.n, a.k, values);
        while (c.parts > 1 && split_bytes(a.m, a.n, c) > a.workspace_bytes) --c.parts;
        return dtype == DIFA_DTYPE_BF16 ? launch_aligned<__bf16>(a, c, false, vec_out, stream) : launch_aligned<float>(a, c, values, vec_out, stream);
    }
    // bf16's other rows: by way of copies where the workspace has room for them and they are worth it
    const int64_t kp = padded_k(a.k, es), pieces = (kp + 511) / 512, items = ((int64_t)a.m + a.n) * pieces, blocks = (items + 3) / 4;
    if (worth_copies(a.m, a.n, a.k, es) && blocks <= 0x7fffffff) {
        Choice c = choose(dtype, a.m, a.n, kp, false);
        const int64_t copies = copy_bytes(a.m, a.n, a.k, es);
        int64_t split = split_bytes(a.m, a.n, c);
        if (split + copies > a.workspace_bytes) { split = 0; c.parts = 1; }
        if (split == 0) split = kTickets * 4;              // the tickets are nobody's room
        if (split + copies <= a.workspace_bytes) {
            LinearArgs p = a;
            char* to = (char*)a.workspace + split;
            p.x = to; p.w = to + a.m * kp * es;
            p.x_stride_n = p.w_stride = kp; p.x_stride_b = a.rows * kp; p.k = (int32_t)kp;
            const hipError_t e = in_slices(blocks, [&](unsigned first, unsigned count) {
                linear_pad_kernel<__bf16><<<dim3(count), dim3(256), 0, stream>>>(a, first, (__bf16*)to, (int)kp, (int)pieces);
                return hipGetLastError();
            });
            return e != hipSuccess ? e : launch_aligned<__bf16>(p, c, false, vec_out, stream);
        }
    }
    return dtype == DIFA_DTYPE_BF16 ? launch_any<__bf16>(a, vec_in, vec_out, stream) : launch_any<float>(a, vec_in, vec_out, stream);
}

}  // namespace difa
