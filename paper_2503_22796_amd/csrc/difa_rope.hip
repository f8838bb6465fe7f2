// Rotary positions and head norms of a layer's queries and keys.
//   rope_table_kernel      cosines and sines of every (row, pair)
//   rotate_kernel          queries and keys turned by them
//   norm_rotate_kernel     RMS norm per head, rotation, and the streams' rows gathered into the joint tensors
//   norm_backward_kernel   its gradients; norm_weight_kernel adds up the weight gradients' partial sums
// All but the first stream their tensors once and are bound by HBM.  D / 8 lanes hold one head row, eight features
// each, arranged so that every lane holds four whole pairs: features 8l .. 8l + 7, or (HALVES) 4l .. 4l + 3 and as
// many from the row's middle on; pair i of a lane is pair 4l + i of the row either way.  A group of such lanes keeps one
// token and walks over a few heads, consecutive groups take consecutive tokens of the same heads.
// Measured (one MI355X; a copy of 1 GiB reaches 5.06 TB/s): with all of a token's heads in one group, and then in as many groups as make
// 65536 workgroups (split): norm of a FLUX-like 2K layer 120 and 117 us (5.3 TB/s), SD3-like 1K 31.3 and 29.7, fp32 rotation of
// a video layer 195 and 186.  What the norm and its gradients write is stored past the caches (stream): 126 and 120 us,
// 35.7 and 31.1; the rotation's is not: 20.5 us and 22.6, where a call reads what an earlier one wrote.
#include <math.h>

#include "difa_layer.h"

namespace difa {

namespace {

typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// Eight features of a row as they are stored: two halves of four (HALVES: D / 2 apart, otherwise adjacent).
template <typename T, int D, bool HALVES> struct Vec;

template <int D, bool HALVES> struct Vec<__bf16, D, HALVES> {
    u32x4 r;
    __device__ __forceinline__ void load(const __bf16* row, int l) {
        if constexpr (HALVES) {
            const u32x2 a = *(const u32x2*)(row + 4 * l), b = *(const u32x2*)(row + D / 2 + 4 * l);
            r = u32x4{a[0], a[1], b[0], b[1]};
        } else {
            r = *(const u32x4*)(row + 8 * l);
        }
    }
    __device__ __forceinline__ void store(__bf16* row, int l) const {
        if constexpr (HALVES) {
            *(u32x2*)(row + 4 * l) = u32x2{r[0], r[1]};
            *(u32x2*)(row + D / 2 + 4 * l) = u32x2{r[2], r[3]};
        } else {
            *(u32x4*)(row + 8 * l) = r;
        }
    }
    __device__ __forceinline__ void stream(__bf16* row, int l) const {
        if constexpr (HALVES) {
            __builtin_nontemporal_store(u32x2{r[0], r[1]}, (u32x2*)(row + 4 * l));
            __builtin_nontemporal_store(u32x2{r[2], r[3]}, (u32x2*)(row + D / 2 + 4 * l));
        } else {
            __builtin_nontemporal_store(r, (u32x4*)(row + 8 * l));
        }
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned u = r[i];
            x[2 * i] = __builtin_bit_cast(float, u << 16);       // a bf16 is the upper half of an fp32
            x[2 * i + 1] = __builtin_bit_cast(float, u & 0xffff0000u);
        }
    }
    __device__ __forceinline__ void round(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 p = {(__bf16)x[2 * i], (__bf16)x[2 * i + 1]};
            r[i] = __builtin_bit_cast(unsigned, p);
        }
    }
};

template <int D, bool HALVES> struct Vec<float, D, HALVES> {
    u32x4 a, b;
    __device__ __forceinline__ void load(const float* row, int l) {
        a = *(const u32x4*)(row + (HALVES ? 4 * l : 8 * l));
        b = *(const u32x4*)(row + (HALVES ? D / 2 + 4 * l : 8 * l + 4));
    }
    __device__ __forceinline__ void store(float* row, int l) const {
        *(u32x4*)(row + (HALVES ? 4 * l : 8 * l)) = a;
        *(u32x4*)(row + (HALVES ? D / 2 + 4 * l : 8 * l + 4)) = b;
    }
    __device__ __forceinline__ void stream(float* row, int l) const {
        __builtin_nontemporal_store(a, (u32x4*)(row + (HALVES ? 4 * l : 8 * l)));
        __builtin_nontemporal_store(b, (u32x4*)(row + (HALVES ? D / 2 + 4 * l : 8 * l + 4)));
    }
    __device__ __forceinline__ void widen(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned u = a[i], v = b[i];
            x[i] = __builtin_bit_cast(float, u);
            x[4 + i] = __builtin_bit_cast(float, v);
        }
    }
    __device__ __forceinline__ void round(const float (&x)[8]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = __builtin_bit_cast(unsigned, x[i]);
            b[i] = __builtin_bit_cast(unsigned, x[4 + i]);
        }
    }
};

// Where feature i of a lane's eight stands in the row.
template <int D, bool HALVES> __device__ __forceinline__ int feature(int l, int i) {
    if (HALVES) return (i < 4 ? 4 * l : D / 2 + 4 * l - 4) + i;
    return 8 * l + i;
}

// Cosines and sines of a lane's four pairs.
struct Turn {
    float c[4], s[4];
    __device__ __forceinline__ void load(const float* row, int l, float sign) {
        const float4 p = *(const float4*)(row + 8 * l), q = *(const float4*)(row + 8 * l + 4);
        c[0] = p.x; s[0] = sign * p.y; c[1] = p.z; s[1] = sign * p.w;
        c[2] = q.x; s[2] = sign * q.y; c[3] = q.z; s[3] = sign * q.w;
    }
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int i = 0; i < 4; ++i) { c[i] = 1.f; s[i] = 0.f; }
    }
    // A pair that is not turned keeps its features apart: an infinity or NaN of one is not in the other's result.
    template <bool HALVES> __device__ __forceinline__ void apply(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float& u = x[HALVES ? i : 2 * i];
            float& v = x[HALVES ? 4 + i : 2 * i + 1];
            const bool still = s[i] == 0.f;
            const float vs = still ? 0.f : v * s[i], us = still ? -0.f : u * s[i];
            const float a = u * c[i] - vs, b = us + v * c[i];
            u = a;
            v = b;
        }
    }
};

// Sum over the 8 or 16 neighbouring lanes of a head row; every one of them gets the same bits.
template <int CTRL> __device__ __forceinline__ float dpp(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
template <int LANES> __device__ __forceinline__ float row_sum(float x) {
    x += dpp<0xB1>(x);                          // quad_perm [1, 0, 3, 2]
    x += dpp<0x4E>(x);                          // quad_perm [2, 3, 0, 1]
    x += dpp<0x141>(x);                         // row_half_mirror
    if (LANES == 16) x += dpp<0x140>(x);        // row_mirror
    return x;
}

// 1 / sqrt(mean(x^2) + eps) of a row.  Where the squares leave fp32 the row is scaled by 2^-70 first, x with it, and
// `pre` says so: x * r is the normed row either way, pre * r the factor itself.
template <int D> __device__ __forceinline__ float inverse_rms(float (&x)[8], float eps, float& pre) {
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
    ss = row_sum<D / 8>(ss);
    pre = 1.f;
    if (ss > 3.4e38f) {
        pre = 0x1p-70f;
        ss = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] *= pre;
            ss = fmaf(x[i], x[i], ss);
        }
        ss = row_sum<D / 8>(ss);
        eps = eps * pre * pre;
    }
    return rsqrtf(fmaf(ss, 1.f / D, eps));
}

constexpr int kThreads = 256;
constexpr int kTableRows = 4;

}  // namespace

// Cosine and sine of 2 pi t, |t| <= 1/2, in 64 bits: t is taken to the nearest quarter turn, and what is left, at most pi / 4, goes through
// the Taylor series up to x^12 and x^13, whose next terms are below 4e-13 of a cosine and 2.1e-14 of a sine: fp32 is rounded
// to 3e-8.  (The library's own sine and cosine carry 53 bits: table of a video latent 7.3 us with them.)
__device__ __forceinline__ float2 cos_sin_turns(double t) {
    const double q = rint(4.0 * t), x = (t - 0.25 * q) * 6.283185307179586477, z = x * x;
    double s = fma(z, 1.0 / 6227020800.0, -1.0 / 39916800.0);
    s = fma(z, s, 1.0 / 362880.0);
    s = fma(z, s, -1.0 / 5040.0);
    s = fma(z, s, 1.0 / 120.0);
    s = fma(z, s, -1.0 / 6.0);
    const float sine = (float)fma(x * z, s, x);
    double c = fma(z, 1.0 / 479001600.0, -1.0 / 3628800.0);
    c = fma(z, c, 1.0 / 40320.0);
    c = fma(z, c, -1.0 / 720.0);
    c = fma(z, c, 1.0 / 24.0);
    c = fma(z, c, -0.5);
    const float cosine = (float)fma(z, c, 1.0);
    const int turn = (int)q;                                   // -2 .. 2
    const float u = turn & 1 ? sine : cosine, v = turn & 1 ? cosine : sine;
    // quarter turns 0: (c, s), 1: (-s, c), 2 and -2: (-c, -s), -1: (s, -c)
    return {turn == 1 || turn == 2 || turn == -2 ? -u : u, turn == -1 || turn == 2 || turn == -2 ? -v : v};
}

// ---- table: a thread keeps one pair and takes four rows at a time, whose positions are on their way together.
// angle / 2 pi = position * (theta^(-2j/d) / 2 pi) in 64 bits, its whole turns taken off before the cosine: the frequency's
// roundings are what counts, some 2^-49 of the angle with theta = 10000 (the logarithm, the exponent's product and quotient, 2^-53
// each of an exponent of up to 13).  Bound by its launch up to some 10 000 rows (6.8 us for 20536, host included), then by
// the table's bytes (200000 rows 31 us, 3.4 TB/s; 10^6 167 us, 3.1 TB/s).
__global__ __launch_bounds__(kThreads) void rope_table_kernel(RopeTableArgs a) {
    const int pair = threadIdx.x % a.half, per_pass = kThreads / a.half;
    int axis = 0, first = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < a.axes && pair >= a.pair_end[i]) { axis = i + 1; first = a.pair_end[i]; }
    const bool turned = axis < a.axes;
    double turns = 0.0;
    if (turned) {
        int end = a.pair_end[0];
#pragma unroll
        for (int i = 1; i < 4; ++i) end = axis == i ? a.pair_end[i] : end;
        turns = exp2(-a.log2_theta * (double)(pair - first) / (double)(end - first)) * 0.15915494309189533577;
    }
    constexpr int U = kTableRows;
    for (int64_t row0 = (int64_t)blockIdx.x * per_pass * U + threadIdx.x / a.half; row0 < a.n_rows; row0 += (int64_t)gridDim.x * per_pass * U) {
        float at[U];
#pragma unroll
        for (int u = 0; u < U; ++u) at[u] = turned && row0 + u * per_pass < a.n_rows ? a.positions[(row0 + u * per_pass) * a.axes + axis] : 0.f;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row0 + u * per_pass;
            if (row >= a.n_rows) break;
            const double t = (double)at[u] * turns;
            *(float2*)(a.table + (row * a.half + pair) * 2) = cos_sin_turns(t - rint(t));      // a pair that is not turned: (1, 0)
        }
    }
}

// ---- A workgroup's place: its number in the call is (b * chunks + chunk) * token_blocks + token block.
struct Place { int b, chunk, block; };
__device__ __forceinline__ Place place(unsigned first, int token_blocks, int chunks) {
    const unsigned p = first + blockIdx.x, bc = p / (unsigned)token_blocks;
    return {(int)(bc / (unsigned)chunks), (int)(bc % (unsigned)chunks), (int)(p - bc * (unsigned)token_blocks)};
}

template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(kThreads) void rotate_kernel(RotateArgs a, unsigned first, int token_blocks, int chunks, int per_chunk) {
    constexpr int L = D / 8;
    const Place p = place(first, token_blocks, chunks);
    const int64_t t = (int64_t)p.block * (kThreads / L) + threadIdx.x / L;
    const int l = threadIdx.x % L;
    if (t >= a.n_tokens) return;
    Turn turn;
    turn.load(a.table + p.b * a.table_stride_b + t * D, l, a.inverse ? -1.f : 1.f);
    const int h0 = p.chunk * per_chunk, h1 = h0 + per_chunk < a.heads ? h0 + per_chunk : a.heads;
    int64_t at = p.b * a.joint.b + h0 * a.joint.h + t * a.joint.n;
    const bool both = a.dst[1] != nullptr;
    for (int h = h0; h < h1; ++h, at += a.joint.h) {
        Vec<T, D, HALVES> q, k;
        q.load((const T*)a.src[0] + at, l);
        if (both) k.load((const T*)a.src[1] + at, l);
        float x[8];
        q.widen(x);
        turn.apply<HALVES>(x);
        q.round(x);
        q.store((T*)a.dst[0] + at, l);
        if (both) {
            k.widen(x);
            turn.apply<HALVES>(x);
            k.round(x);
            k.store((T*)a.dst[1] + at, l);
        }
    }
}

template <typename T, int D, bool HALVES>
__device__ __forceinline__ void load_weight(const void* w, int l, float (&x)[8]) {
    if (w && ((uintptr_t)w & 15) == 0) {
        Vec<T, D, HALVES> v;
        v.load((const T*)w, l);
        v.widen(x);
    } else if (w) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)((const T*)w)[feature<D, HALVES>(l, i)];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = 1.f;
    }
}

template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(kThreads) void norm_rotate_kernel(NormArgs a, unsigned first, int token_blocks, int chunks, int per_chunk) {
    constexpr int L = D / 8;
    const Place p = place(first, token_blocks, chunks);
    const int64_t t = (int64_t)p.block * (kThreads / L) + threadIdx.x / L;
    const int l = threadIdx.x % L;
    if (t >= a.n_tokens) return;
    const bool image = t >= a.stream[1].begin && t < (int64_t)a.stream[1].begin + a.stream[1].count;
    const NormStream& s = a.stream[image];
    Turn turn;
    if (a.table) turn.load(a.table + p.b * a.table_stride_b + t * D, l, 1.f); else turn.none();
    float wq[8], wk[8];
    load_weight<T, D, HALVES>(s.weight[0], l, wq);
    load_weight<T, D, HALVES>(s.weight[1], l, wk);
    const int h0 = p.chunk * per_chunk, h1 = h0 + per_chunk < a.heads ? h0 + per_chunk : a.heads;
    int64_t from = p.b * s.stride_b + (t - s.begin) * s.stride_n + h0 * s.stride_h;
    int64_t to = p.b * a.js.b + h0 * a.js.h + t * a.js.n;
    const bool copy = a.joint[2] != nullptr;
    for (int h = h0; h < h1; ++h, from += s.stride_h, to += a.js.h) {
        Vec<T, D, HALVES> q, k, v;
        q.load((const T*)s.src[0] + from, l);
        k.load((const T*)s.src[1] + from, l);
        if (copy) v.load((const T*)s.src[2] + from, l);
        auto norm = [&](Vec<T, D, HALVES>& row, const float (&w)[8], T* out) {
            float x[8], pre;
            row.widen(x);
            const float r = inverse_rms<D>(x, a.eps, pre);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * r * w[i];
            turn.apply<HALVES>(x);
            row.round(x);
            row.stream(out, l);
        };
        norm(q, wq, (T*)a.joint[0] + to);
        norm(k, wk, (T*)a.joint[1] + to);
        if (copy) v.stream((T*)a.joint[2] + to, l);
    }
}

// ---- Gradients.  A workgroup belongs to one stream and takes every blocks[stream]-th block of its (batch entry, heads, token)
// items, `per_item` heads each; each lane sums its features' weight gradients over all rows it meets, the workgroup's groups are added in LDS in
// the order of their numbers, and norm_weight_kernel adds the workgroups' sums: a fixed order throughout.
template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(kThreads) void norm_backward_kernel(NormArgs a) {
    constexpr int L = D / 8, G = kThreads / L;
    const bool image = (int)blockIdx.x >= a.blocks[0];
    const NormStream& s = a.stream[image];
    const NormGrad& d = a.grad[image];
    const int block = image ? (int)blockIdx.x - a.blocks[0] : (int)blockIdx.x, n_blocks = a.blocks[image];
    const int l = threadIdx.x % L, g = threadIdx.x / L;
    float wq[8], wk[8], sq[8], sk[8];
    load_weight<T, D, HALVES>(s.weight[0], l, wq);
    load_weight<T, D, HALVES>(s.weight[1], l, wk);
#pragma unroll
    for (int i = 0; i < 8; ++i) sq[i] = sk[i] = 0.f;
    const bool copy = a.joint[2] != nullptr && d.dst[2] != nullptr;
    const int per_item = a.per_item, chunks = (a.heads + per_item - 1) / per_item;
    const int64_t items = (int64_t)a.batch * chunks * s.count;
    for (int64_t item = (int64_t)block * G + g; item < items; item += (int64_t)n_blocks * G) {
        const int64_t bc = item / s.count, b = bc / chunks, t = item - bc * s.count;
        const int h0 = (int)(bc - b * chunks) * per_item, h1 = h0 + per_item < a.heads ? h0 + per_item : a.heads;
        Turn turn;
        if (a.table) turn.load(a.table + b * a.table_stride_b + (s.begin + t) * D, l, -1.f); else turn.none();
        int64_t from = b * s.stride_b + t * s.stride_n + h0 * s.stride_h, to = b * d.stride_b + t * d.stride_n + h0 * d.stride_h;
        int64_t at = b * a.js.b + (s.begin + t) * a.js.n + h0 * a.js.h;
        for (int h = h0; h < h1; ++h, from += s.stride_h, to += d.stride_h, at += a.js.h) {
            Vec<T, D, HALVES> q, k, gq, gk, gv;
            q.load((const T*)s.src[0] + from, l);
            gq.load((const T*)a.joint[0] + at, l);
            k.load((const T*)s.src[1] + from, l);
            gk.load((const T*)a.joint[1] + at, l);
            if (copy) gv.load((const T*)a.joint[2] + at, l);
            auto gradient = [&](Vec<T, D, HALVES>& row, const Vec<T, D, HALVES>& grad, const float (&w)[8], float (&sum)[8], T* out) {
                float x[8], y[8], pre;
                row.widen(x);
                grad.widen(y);
                turn.apply<HALVES>(y);
                const float r = inverse_rms<D>(x, a.eps, pre);
                float dot = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= r;                                  // the normed row
                    sum[i] = fmaf(y[i], x[i], sum[i]);
                    y[i] *= w[i];
                    dot = fmaf(y[i], x[i], dot);
                }
                dot = row_sum<L>(dot) * (1.f / D);
#pragma unroll
                for (int i = 0; i < 8; ++i) y[i] = pre * (r * (y[i] - x[i] * dot));
                row.round(y);
                row.stream(out, l);
            };
            gradient(q, gq, wq, sq, (T*)d.dst[0] + to);
            gradient(k, gk, wk, sk, (T*)d.dst[1] + to);
            if (copy) gv.stream((T*)d.dst[2] + to, l);
        }
    }
    if (!a.partial) return;
    __shared__ float sums[G][2][D];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        sums[g][0][feature<D, HALVES>(l, i)] = sq[i];
        sums[g][1][feature<D, HALVES>(l, i)] = sk[i];
    }
    __syncthreads();
    if (threadIdx.x < 2 * D) {
        const float* at = &sums[0][0][0] + threadIdx.x;
        float x = 0.f;
#pragma unroll
        for (int i = 0; i < G; ++i) x += at[i * 2 * D];
        a.partial[(int64_t)blockIdx.x * 2 * D + threadIdx.x] = x;
    }
}

// One workgroup per 16 columns of a (stream, q or k) pair: 64 threads a column, each every 64th workgroup's sum, eight of them
// in flight.
constexpr int kSlices = 64;
__global__ __launch_bounds__(16 * kSlices) void norm_weight_kernel(NormArgs a, int head_dim) {
    const int parts = head_dim / 16, which = blockIdx.x / parts, image = which >> 1, qk = which & 1;
    float* out = a.grad[image].weight[qk];
    if (!out || a.stream[image].count == 0) return;
    const int lane_col = threadIdx.x % 16, slice = threadIdx.x / 16, col = (blockIdx.x % parts) * 16 + lane_col;
    const int64_t row = 2 * head_dim;
    const float* at = a.partial + (image ? a.blocks[0] : 0) * row + qk * head_dim + col;
    float x = 0.f;
    for (int i = slice; i < a.blocks[image]; i += 8 * kSlices) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i + u * kSlices < a.blocks[image] ? at[(i + u * kSlices) * row] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) x += v[u];
    }
    __shared__ float part[kSlices][16];
    part[slice][lane_col] = x;
    __syncthreads();
#pragma unroll
    for (int half = kSlices / 2; half >= 1; half /= 2) {
        if (slice < half) part[slice][lane_col] += part[slice + half][lane_col];
        __syncthreads();
    }
    if (slice == 0) out[col] = part[0][lane_col];
}

// ---- launches

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream) {
    const int rows = kThreads / a.half * kTableRows;
    const int64_t blocks = ((int64_t)a.n_rows + rows - 1) / rows;
    rope_table_kernel<<<dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(kThreads), 0, stream>>>(a);
    return hipGetLastError();
}

namespace {

struct Split { int token_blocks, chunks, per_chunk; int64_t blocks; };
Split split(int64_t batch, int heads, int64_t n_tokens, int head_dim) {
    const int groups = kThreads / (head_dim / 8);
    const int64_t token_blocks = (n_tokens + groups - 1) / groups;
    int chunks = 1;
    while (chunks < heads && batch * token_blocks * chunks < 65536) ++chunks;
    const int per_chunk = (heads + chunks - 1) / chunks;
    chunks = (heads + per_chunk - 1) / per_chunk;
    return {(int)token_blocks, chunks, per_chunk, batch * token_blocks * chunks};
}

template <typename F> hipError_t by_kind(int dtype, int head_dim, bool halves, F&& f) {
    auto rows = [&](auto t, auto d) { halves ? f(t, d, std::true_type()) : f(t, d, std::false_type()); };
    auto type = [&](auto t) {
        if (head_dim == 128) rows(t, std::integral_constant<int, 128>());
        else rows(t, std::integral_constant<int, 64>());
    };
    if (dtype == DIFA_DTYPE_BF16) type((__bf16)0.f); else type(0.f);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, int dtype, int head_dim, bool halves, hipStream_t stream) {
    const Split sp = split(a.batch, a.heads, a.n_tokens, head_dim);
    if (sp.blocks > 0x7fffffff) return hipErrorInvalidValue;
    return in_slices(sp.blocks, [&](unsigned first, unsigned blocks) {
        return by_kind(dtype, head_dim, halves, [&](auto t, auto d, auto hv) {
            rotate_kernel<decltype(t), d.value, hv.value><<<dim3(blocks), dim3(kThreads), 0, stream>>>(
                a, first, sp.token_blocks, sp.chunks, sp.per_chunk);
        });
    });
}

hipError_t launch_norm_rotate(const NormArgs& a, int dtype, int head_dim, bool halves, hipStream_t stream) {
    const Split sp = split(a.batch, a.heads, a.n_tokens, head_dim);
    if (sp.blocks > 0x7fffffff) return hipErrorInvalidValue;
    return in_slices(sp.blocks, [&](unsigned first, unsigned blocks) {
        return by_kind(dtype, head_dim, halves, [&](auto t, auto d, auto hv) {
            norm_rotate_kernel<decltype(t), d.value, hv.value><<<dim3(blocks), dim3(kThreads), 0, stream>>>(
                a, first, sp.token_blocks, sp.chunks, sp.per_chunk);
        });
    });
}

// 768 workgroups, three to a compute unit, and items small enough that each takes some eight of them.  SD3-like 512 px, FLUX-like
// 1K and 2K layers: 19.2, 50.5 and 173 us with 768, 18.7, 51.0 and 176 with 1024, 18.7, 53.9 and 178 with 2048, whose
// sums the second kernel has to add; all heads in one item 28.2, 58.2 and 198.
void norm_backward_split(int64_t batch, int32_t heads, int32_t head_dim, int64_t n_text, int64_t n_img, int32_t (&blocks)[2], int32_t* per_item) {
    constexpr int64_t kMost = 768;
    const int groups = kThreads / (head_dim / 8);
    const int64_t n[2] = {batch * n_text, batch * n_img}, rows = (n[0] + n[1]) * heads;
    const int64_t per = rows / (groups * kMost * 8);
    *per_item = (int32_t)(per < 1 ? 1 : per < heads ? per : heads);
    const int64_t chunks = (heads + *per_item - 1) / *per_item;
    for (int i = 0; i < 2; ++i) {
        const int64_t all = (n[i] * chunks + groups - 1) / groups;
        int64_t share = rows > 0 ? (int64_t)((double)kMost * n[i] / (n[0] + n[1])) : 0;
        if (share < 1) share = 1;
        blocks[i] = (int32_t)(all < share ? all : share);
    }
}

hipError_t launch_norm_rotate_backward(const NormArgs& a, int dtype, int head_dim, bool halves, hipStream_t stream) {
    hipError_t e = by_kind(dtype, head_dim, halves, [&](auto t, auto d, auto hv) {
        norm_backward_kernel<decltype(t), d.value, hv.value>
            <<<dim3((unsigned)(a.blocks[0] + a.blocks[1])), dim3(kThreads), 0, stream>>>(a);
    });
    if (e != hipSuccess || !a.partial) return e;
    norm_weight_kernel<<<dim3((unsigned)(4 * head_dim / 16)), dim3(16 * kSlices), 0, stream>>>(a, head_dim);
    return hipGetLastError();
}

}  // namespace difa
