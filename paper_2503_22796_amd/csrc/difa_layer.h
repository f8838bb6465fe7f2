// Operators around the joint attention of a layer: what the host entries (difa_layer.cpp) and the kernels
// (difa_rope.hip, difa_linear.hip) share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <string>

#include "difa.h"

namespace difa {

// The plan object as these entries see it (defined beside it).
const difa_plan_desc_t& plan_desc(const difa_plan_t* plan);
difa_status_t plan_fail(difa_plan_t* plan, difa_status_t status, const std::string& msg) noexcept;

// Makes a device current and the earlier one again when it goes.
struct DeviceGuard {
    int prev = -1;
    bool switched = false;
    hipError_t enter(int dev) {
        hipError_t e = hipGetDevice(&prev);
        if (e != hipSuccess) return e;
        if (prev != dev) {
            e = hipSetDevice(dev);
            if (e != hipSuccess) return e;
            switched = true;
        }
        return hipSuccess;
    }
    ~DeviceGuard() {
        if (switched) (void)hipSetDevice(prev);
    }
};

// A grid of 2^32 work-items or more is no single launch: the runtime takes it and runs what its lowest 32 bits say.  So the
// workgroups of a call, of at most 512 threads each, go in slices, and a kernel counts its own from `first` on.
// A multiple of the 8 dies, so that workgroup first + i runs on the die that it would run on in one launch.
constexpr int64_t kSlice = 1 << 22;
template <class F> hipError_t in_slices(int64_t workgroups, F&& launch) {
    for (int64_t first = 0; first < workgroups; first += kSlice) {
        const hipError_t e = launch((unsigned)first, (unsigned)std::min(workgroups - first, kSlice));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

struct RopeTableArgs {
    const float* positions;
    float* table;
    int32_t n_rows, axes, half;      // half: pairs per row
    int32_t pair_end[4];             // first pair behind axis a's
    double log2_theta;
};

// A joint tensor in the plan's layout, in elements.
struct JointStrides { int64_t b, h, n; };

struct RotateArgs {
    const void* src[2];
    void* dst[2];                    // [1] NULL: queries only
    const float* table;
    int64_t table_stride_b;          // elements: 0 or n_tokens * head_dim
    JointStrides joint;
    int32_t batch, heads, n_tokens;
    int32_t inverse;
};

struct NormStream {
    const void* src[3];              // q, k, v
    const void* weight[2];           // q, k; NULL: ones
    int64_t stride_b, stride_n, stride_h;
    int32_t begin, count;            // its tokens of the joint sequence
};
struct NormGrad {
    void* dst[3];
    int64_t stride_b, stride_n, stride_h;
    float* weight[2];
};
struct NormArgs {
    NormStream stream[2];            // text, image
    NormGrad grad[2];
    void* joint[3];                  // forward: q_out, k_out, v_out (or NULL); backward: their gradients, read
    const float* table;              // NULL: no rotation
    int64_t table_stride_b;
    JointStrides js;
    float* partial;                  // backward: [block][q, k][head_dim] sums; NULL: no weight gradient wanted
    int32_t batch, heads, n_tokens;
    int32_t blocks[2];               // backward: workgroups of each stream, text's first
    int32_t per_item;                // ... and heads that a group of lanes walks over for one token
    float eps;
};
// Workgroups of the backward pass per stream and heads per item (they go by the sizes alone, so that the workspace and the
// sums' order do).
void norm_backward_split(int64_t batch, int32_t heads, int32_t head_dim, int64_t n_text, int64_t n_img, int32_t (&blocks)[2], int32_t* per_item);

struct LinearArgs {
    const void *x, *w, *bias, *gate, *residual;
    void* out;
    int64_t x_stride_b, x_stride_n, w_stride, out_stride_b, out_stride_n, res_stride_b, res_stride_n, gate_stride_b;
    int32_t batch, rows, m, n, k;    // m = batch * rows
    int32_t activation;
    void* workspace;                 // NULL: no split along k
    int64_t workspace_bytes;
};

hipError_t launch_rope_table(const RopeTableArgs& a, hipStream_t stream);
hipError_t launch_rotate(const RotateArgs& a, int dtype, int head_dim, bool halves, hipStream_t stream);
hipError_t launch_norm_rotate(const NormArgs& a, int dtype, int head_dim, bool halves, hipStream_t stream);
hipError_t launch_norm_rotate_backward(const NormArgs& a, int dtype, int head_dim, bool halves, hipStream_t stream);
hipError_t launch_linear(const LinearArgs& a, int dtype, hipStream_t stream);
int64_t linear_workspace_bytes(int dtype, int64_t m, int64_t n, int64_t k);

}  // namespace difa
