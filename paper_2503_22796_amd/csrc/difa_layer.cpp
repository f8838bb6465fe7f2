// Host side of the operators around a layer's joint attention: argument checks and launches.  None of them keeps state:
// a call is one launch (two with weight gradients) on the caller's stream.
#include <math.h>

#include <new>

#include "difa_layer.h"
#include "difa_testing.h"

using difa::plan_desc;

namespace {

difa_status_t invalid(difa_plan_t* p, const char* msg) { return difa::plan_fail(p, DIFA_ERR_INVALID_ARG, msg); }

// The launches of a call whose arguments are in order, with the plan's device current.
template <class F> difa_status_t launch(difa_plan_t* p, const char* what, F&& body) {
    difa::DeviceGuard guard;
    hipError_t e = guard.enter(plan_desc(p).device);
    if (e == hipSuccess) e = body();
    return e == hipSuccess ? DIFA_OK : difa::plan_fail(p, DIFA_ERR_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

// Runs an entry point's body; nothing it throws leaves the library.
template <class F> difa_status_t guarded(difa_plan_t* p, F&& body) noexcept {
    if (!p) return DIFA_ERR_INVALID_ARG;
    try {
        return body();
    } catch (const std::bad_alloc&) {
        return difa::plan_fail(p, DIFA_ERR_ALLOC, std::string());
    } catch (...) {
        return difa::plan_fail(p, DIFA_ERR_HIP, std::string());
    }
}

int64_t elem_size(const difa_plan_t* p) { return plan_desc(p).dtype == DIFA_DTYPE_BF16 ? 2 : 4; }

bool misaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }

// Two ranges of `bytes` that share some but not all of their bytes, or (same allowed = false) any.
bool overlap(const void* a, const void* b, int64_t bytes, bool same_allowed) {
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    if (!a || !b || (x == y && same_allowed)) return false;
    return x < y ? y - x < (uintptr_t)bytes : x - y < (uintptr_t)bytes;
}

difa::JointStrides joint_strides(const difa_plan_desc_t& d, int64_t n) {
    const int64_t D = d.head_dim, H = d.heads;
    if (d.layout == DIFA_LAYOUT_BHND) return {H * n * D, n * D, D};
    return {n * H * D, D, H * D};
}

int64_t joint_bytes(const difa_plan_t* p, int64_t n) {
    const difa_plan_desc_t& d = plan_desc(p);
    return (int64_t)d.batch * d.heads * n * d.head_dim * elem_size(p);
}

// The table of a call: NULL or a message.
const char* check_table(const difa_plan_desc_t& d, const float* table, int32_t table_batch) {
    if (misaligned(table, 16)) return "table must be 16-byte aligned";
    if (table_batch != 1 && table_batch != d.batch) return "table_batch must be 1 or the plan's batch";
    return nullptr;
}

}  // namespace

extern "C" difa_status_t difa_rope_table(difa_plan_t* p, const difa_rope_desc_t* desc, const float* positions, int32_t n_rows,
                                         float* table, void* stream) {
    return guarded(p, [&]() -> difa_status_t {
        if (!desc || !positions || !table) return invalid(p, "desc, positions and table must not be NULL");
        if (n_rows < 1) return invalid(p, "n_rows must be at least 1");
        if (misaligned(positions, 4) || misaligned(table, 16)) return invalid(p, "positions must be 4-byte and table 16-byte aligned");
        if (desc->axes < 1 || desc->axes > 4) return invalid(p, "axes must be in [1, 4]");
        if (!(desc->theta > 1.f) || isinf(desc->theta)) return invalid(p, "theta must be finite and above 1");
        difa::RopeTableArgs a{};
        const int32_t D = plan_desc(p).head_dim;
        int32_t sum = 0;
        for (int i = 0; i < desc->axes; ++i) {
            const int32_t d = desc->dims[i];
            if (d < 2 || d % 2 != 0 || d > D - sum) return invalid(p, "an axis's features must be even, at least 2 and together at most head_dim");
            sum += d;
            a.pair_end[i] = sum / 2;
        }
        a.positions = positions; a.table = table; a.n_rows = n_rows; a.axes = desc->axes; a.half = D / 2;
        a.log2_theta = log2((double)desc->theta);
        return launch(p, "rope-table launch", [&] { return difa::launch_rope_table(a, (hipStream_t)stream); });
    });
}

extern "C" difa_status_t difa_rotate(difa_plan_t* p, const void* q, const void* k, void* q_out, void* k_out, const float* table,
                                     int32_t table_batch, int32_t n_tokens, uint32_t flags, void* stream) {
    return guarded(p, [&]() -> difa_status_t {
        const difa_plan_desc_t& d = plan_desc(p);
        if (!q || !q_out || !table) return invalid(p, "q, q_out and table must not be NULL");
        if ((k == nullptr) != (k_out == nullptr)) return invalid(p, "k and k_out must both be given or both be NULL");
        if (n_tokens < 1 || n_tokens > d.max_tokens) return invalid(p, "n_tokens must be in [1, max_tokens]");
        if (flags & ~(uint32_t)(DIFA_ROPE_HALVES | DIFA_ROPE_INVERSE)) return invalid(p, "unknown flag bits");
        if (misaligned(q, 16) || misaligned(k, 16) || misaligned(q_out, 16) || misaligned(k_out, 16))
            return invalid(p, "q, k, q_out and k_out must be 16-byte aligned");
        if (const char* msg = check_table(d, table, table_batch)) return invalid(p, msg);
        const int64_t bytes = joint_bytes(p, n_tokens);
        if (overlap(q, q_out, bytes, true) || overlap(k, k_out, bytes, true) || overlap(q, k_out, bytes, false) ||
            overlap(k, q_out, bytes, false) || overlap(q_out, k_out, bytes, false))
            return invalid(p, "q_out may be q and k_out may be k; they must not overlap otherwise");
        difa::RotateArgs a{};
        a.src[0] = q; a.src[1] = k; a.dst[0] = q_out; a.dst[1] = k_out;
        a.table = table;
        a.table_stride_b = table_batch > 1 ? (int64_t)n_tokens * d.head_dim : 0;
        a.joint = joint_strides(d, n_tokens);
        a.batch = d.batch; a.heads = d.heads; a.n_tokens = n_tokens;
        a.inverse = (flags & DIFA_ROPE_INVERSE) != 0;
        return launch(p, "rotation launch", [&] { return difa::launch_rotate(a, d.dtype, d.head_dim, flags & DIFA_ROPE_HALVES, (hipStream_t)stream); });
    });
}

namespace {

// What the forward and the backward call check and fill in alike.  Returns DIFA_OK or the refusal.
difa_status_t norm_args(difa_plan_t* p, const difa_qkv_t* text, const difa_qkv_t* image, const float* table, int32_t table_batch,
                        float eps, uint32_t flags, difa::NormArgs* a) {
    const difa_plan_desc_t& d = plan_desc(p);
    const int64_t es = elem_size(p);
    const difa_qkv_t* in[2] = {text, image};
    int64_t n = 0;
    for (int i = 0; i < 2; ++i) {
        if (!in[i]) continue;
        if (in[i]->n_tokens < 0) return invalid(p, "n_tokens of a stream must not be negative");
        n += in[i]->n_tokens;
    }
    if (n < 1 || n > d.max_tokens) return invalid(p, "the streams' tokens together must be in [1, max_tokens]");
    if (!(eps > 0.f) || isinf(eps)) return invalid(p, "eps must be finite and above 0");
    if (flags & ~(uint32_t)DIFA_ROPE_HALVES) return invalid(p, "unknown flag bits");
    if (table)
        if (const char* msg = check_table(d, table, table_batch)) return invalid(p, msg);
    const bool image_first = (d.flags & DIFA_FLAG_IMAGE_FIRST) != 0;
    for (int i = 0; i < 2; ++i) {
        difa::NormStream& s = a->stream[i];
        s.count = in[i] ? in[i]->n_tokens : 0;
        if (s.count == 0) continue;
        const difa_qkv_t& x = *in[i];
        if (!x.q || !x.k) return invalid(p, "q and k of a stream with tokens must not be NULL");
        if (x.stride_b < 0 || x.stride_n < 0 || x.stride_h < 0) return invalid(p, "strides must not be negative");
        if (misaligned(x.q, 16) || misaligned(x.k, 16) || misaligned(x.v, 16) ||
            x.stride_b * es % 16 != 0 || x.stride_n * es % 16 != 0 || x.stride_h * es % 16 != 0)
            return invalid(p, "q, k and v and their strides must be multiples of 16 bytes");
        if (misaligned(x.q_weight, (uintptr_t)es) || misaligned(x.k_weight, (uintptr_t)es)) return invalid(p, "norm weights must be aligned to their elements");
        s.src[0] = x.q; s.src[1] = x.k; s.src[2] = x.v;
        s.weight[0] = x.q_weight; s.weight[1] = x.k_weight;
        s.stride_b = x.stride_b; s.stride_n = x.stride_n; s.stride_h = x.stride_h;
    }
    a->stream[0].begin = image_first ? a->stream[1].count : 0;
    a->stream[1].begin = image_first ? 0 : a->stream[0].count;
    a->table = table;
    a->table_stride_b = table && table_batch > 1 ? n * d.head_dim : 0;
    a->js = joint_strides(d, n);
    a->batch = d.batch; a->heads = d.heads; a->n_tokens = (int32_t)n;
    a->eps = eps;
    return DIFA_OK;
}

}  // namespace

extern "C" difa_status_t difa_qk_norm_rotate(difa_plan_t* p, const difa_qkv_t* text, const difa_qkv_t* image, const float* table,
                                             int32_t table_batch, float eps, uint32_t flags, void* q_out, void* k_out, void* v_out,
                                             void* stream) {
    return guarded(p, [&]() -> difa_status_t {
        const difa_plan_desc_t& d = plan_desc(p);
        difa::NormArgs a{};
        const difa_status_t st = norm_args(p, text, image, table, table_batch, eps, flags, &a);
        if (st != DIFA_OK) return st;
        if (!q_out || !k_out) return invalid(p, "q_out and k_out must not be NULL");
        if (misaligned(q_out, 16) || misaligned(k_out, 16) || misaligned(v_out, 16)) return invalid(p, "q_out, k_out and v_out must be 16-byte aligned");
        for (const difa::NormStream& s : a.stream)
            if (s.count > 0 && (s.src[2] == nullptr) != (v_out == nullptr)) return invalid(p, "v of every stream and v_out must all be given or all be NULL");
        void* outs[3] = {q_out, k_out, v_out};
        const int64_t bytes = joint_bytes(p, a.n_tokens);
        for (int i = 0; i < 3; ++i) {
            for (int j = i + 1; j < 3; ++j)
                if (overlap(outs[i], outs[j], bytes, false)) return invalid(p, "q_out, k_out and v_out must not overlap");
            for (const difa::NormStream& s : a.stream)
                for (const void* src : s.src)
                    if (outs[i] && s.count > 0 && src == outs[i]) return invalid(p, "q_out, k_out and v_out must not be an input");
            a.joint[i] = outs[i];
        }
        return launch(p, "norm-and-rotate launch", [&] { return difa::launch_norm_rotate(a, d.dtype, d.head_dim, flags & DIFA_ROPE_HALVES, (hipStream_t)stream); });
    });
}

extern "C" difa_status_t difa_qk_norm_rotate_workspace(difa_plan_t* p, int32_t n_text, int32_t n_img, int64_t* bytes_out) {
    return guarded(p, [&]() -> difa_status_t {
        const difa_plan_desc_t& d = plan_desc(p);
        if (!bytes_out) return invalid(p, "bytes_out must not be NULL");
        if (n_text < 0 || n_img < 0 || (int64_t)n_text + n_img < 1 || (int64_t)n_text + n_img > d.max_tokens)
            return invalid(p, "the streams' tokens together must be in [1, max_tokens]");
        int32_t blocks[2], per_item;
        difa::norm_backward_split(d.batch, d.heads, d.head_dim, n_text, n_img, blocks, &per_item);
        *bytes_out = (int64_t)(blocks[0] + blocks[1]) * 2 * d.head_dim * 4;
        return DIFA_OK;
    });
}

extern "C" difa_status_t difa_qk_norm_rotate_backward(difa_plan_t* p, const difa_qkv_t* text, const difa_qkv_t* image,
                                                      const float* table, int32_t table_batch, float eps, uint32_t flags,
                                                      const void* dq, const void* dk, const void* dv, const difa_qkv_grad_t* text_grad,
                                                      const difa_qkv_grad_t* image_grad, void* workspace, int64_t workspace_bytes,
                                                      void* stream) {
    return guarded(p, [&]() -> difa_status_t {
        const difa_plan_desc_t& d = plan_desc(p);
        const int64_t es = elem_size(p);
        difa::NormArgs a{};
        const difa_status_t st = norm_args(p, text, image, table, table_batch, eps, flags, &a);
        if (st != DIFA_OK) return st;
        if (!dq || !dk) return invalid(p, "dq and dk must not be NULL");
        if (misaligned(dq, 16) || misaligned(dk, 16) || misaligned(dv, 16)) return invalid(p, "dq, dk and dv must be 16-byte aligned");
        a.joint[0] = const_cast<void*>(dq); a.joint[1] = const_cast<void*>(dk); a.joint[2] = const_cast<void*>(dv);
        const difa_qkv_grad_t* grads[2] = {text_grad, image_grad};
        bool weights = false;
        for (int i = 0; i < 2; ++i) {
            if (a.stream[i].count == 0) continue;
            if (!grads[i] || !grads[i]->q || !grads[i]->k) return invalid(p, "a stream with tokens needs the q and k of its gradients");
            const difa_qkv_grad_t& g = *grads[i];
            // (a stride is of use only where there is more than one of its kind)
            const int64_t D = d.head_dim;
            if (g.stride_b < 0 || g.stride_n < 0 || g.stride_h < 0 || (d.batch > 1 && g.stride_b < D) ||
                (a.stream[i].count > 1 && g.stride_n < D) || (d.heads > 1 && g.stride_h < D))
                return invalid(p, "rows of a gradient must be at least head_dim apart");
            if (misaligned(g.q, 16) || misaligned(g.k, 16) || misaligned(g.v, 16) ||
                g.stride_b * es % 16 != 0 || g.stride_n * es % 16 != 0 || g.stride_h * es % 16 != 0)
                return invalid(p, "gradients of q, k and v and their strides must be multiples of 16 bytes");
            if (misaligned(g.q_weight, 4) || misaligned(g.k_weight, 4)) return invalid(p, "weight gradients must be 4-byte aligned");
            if (dv && !g.v) return invalid(p, "dv is given: every stream with tokens needs the v of its gradients");
            void* outs[3] = {g.q, g.k, g.v};
            for (int j = 0; j < 3; ++j) {
                for (int o = j + 1; o < 3; ++o)
                    if (outs[j] && outs[j] == outs[o]) return invalid(p, "the gradients of q, k and v must not overlap");
                for (const difa::NormStream& s : a.stream)
                    for (const void* src : s.src)
                        if (outs[j] && s.count > 0 && src == outs[j]) return invalid(p, "a gradient must not be an input");
                for (const void* joint : a.joint)
                    if (outs[j] && joint == outs[j]) return invalid(p, "a gradient must not be an input");
                a.grad[i].dst[j] = outs[j];
            }
            a.grad[i].stride_b = g.stride_b; a.grad[i].stride_n = g.stride_n; a.grad[i].stride_h = g.stride_h;
            a.grad[i].weight[0] = g.q_weight; a.grad[i].weight[1] = g.k_weight;
            weights |= g.q_weight || g.k_weight;
        }
        difa::norm_backward_split(d.batch, d.heads, d.head_dim, a.stream[0].count, a.stream[1].count, a.blocks, &a.per_item);
        if (weights) {
            const int64_t need = (int64_t)(a.blocks[0] + a.blocks[1]) * 2 * d.head_dim * 4;
            if (!workspace || misaligned(workspace, 16) || workspace_bytes < need)
                return invalid(p, "weight gradients need a 16-byte aligned workspace of difa_qk_norm_rotate_workspace() bytes");
            a.partial = (float*)workspace;
        }
        return launch(p, "norm-gradient launch", [&] { return difa::launch_norm_rotate_backward(a, d.dtype, d.head_dim, flags & DIFA_ROPE_HALVES, (hipStream_t)stream); });
    });
}

namespace {

// Room for a tile's overhang in 32-bit row and feature numbers.
constexpr int32_t kMostRows = 0x7fffffff - 512;
const char kSizes[] = "batch, rows, n and k must be at least 1; batch * rows, n and k at most 2^31 - 513";
bool sizes_fit(int32_t batch, int32_t rows, int32_t n, int32_t k) {
    return batch >= 1 && rows >= 1 && n >= 1 && k >= 1 && (int64_t)batch * rows <= kMostRows && n <= kMostRows && k <= kMostRows;
}

}  // namespace

extern "C" difa_status_t difa_linear_workspace(difa_plan_t* p, int32_t batch, int32_t rows, int32_t n, int32_t k, int64_t* bytes_out) {
    return guarded(p, [&]() -> difa_status_t {
        if (!bytes_out) return invalid(p, "bytes_out must not be NULL");
        if (!sizes_fit(batch, rows, n, k)) return invalid(p, kSizes);
        *bytes_out = difa::linear_workspace_bytes(plan_desc(p).dtype, (int64_t)batch * rows, n, k);
        return DIFA_OK;
    });
}

extern "C" difa_status_t difa_linear(difa_plan_t* p, const difa_linear_desc_t* desc, const void* x, const void* w, const void* bias,
                                     const void* gate, const void* residual, void* out, void* workspace, int64_t workspace_bytes,
                                     void* stream) {
    return guarded(p, [&]() -> difa_status_t {
        const uintptr_t es = (uintptr_t)elem_size(p);
        if (!desc || !x || !w || !out) return invalid(p, "desc, x, w and out must not be NULL");
        const difa_linear_desc_t& d = *desc;
        if (!sizes_fit(d.batch, d.rows, d.n, d.k)) return invalid(p, kSizes);
        if (d.activation < DIFA_ACT_NONE || d.activation > DIFA_ACT_SILU) return invalid(p, "unknown activation");
        if (d.x_stride_b < 0 || d.x_stride_n < 0 || d.residual_stride_b < 0 || d.residual_stride_n < 0 || d.gate_stride_b < 0)
            return invalid(p, "strides must not be negative");
        if (d.w_stride < d.k) return invalid(p, "w_stride must be at least k");
        // rows of the result may not overlap: batch entries inside rows' gaps are allowed, rows inside rows are not
        if ((d.rows > 1 && d.out_stride_n < d.n) || (d.batch > 1 && d.out_stride_b < d.n))
            return invalid(p, "rows of out must be at least n apart");
        if (misaligned(x, es) || misaligned(w, es) || misaligned(bias, es) || misaligned(gate, es) || misaligned(residual, es) || misaligned(out, es))
            return invalid(p, "tensors must be aligned to their elements");
        if (misaligned(workspace, 16) || workspace_bytes < 0) return invalid(p, "workspace must be 16-byte aligned and its size not negative");
        if (out == x || out == w || (bias && out == bias) || (gate && out == gate)) return invalid(p, "out must not be an input other than residual");
        if (residual == out && ((d.rows > 1 && d.residual_stride_n != d.out_stride_n) || (d.batch > 1 && d.residual_stride_b != d.out_stride_b)))
            return invalid(p, "a residual that is out must have out's strides");
        difa::LinearArgs a{};
        a.x = x; a.w = w; a.bias = bias; a.gate = gate; a.residual = residual; a.out = out;
        a.x_stride_b = d.x_stride_b; a.x_stride_n = d.x_stride_n; a.w_stride = d.w_stride;
        a.out_stride_b = d.out_stride_b; a.out_stride_n = d.out_stride_n;
        a.res_stride_b = d.residual_stride_b; a.res_stride_n = d.residual_stride_n; a.gate_stride_b = d.gate_stride_b;
        a.batch = d.batch; a.rows = d.rows; a.m = d.batch * d.rows; a.n = d.n; a.k = d.k;
        a.activation = d.activation;
        a.workspace = workspace; a.workspace_bytes = workspace ? workspace_bytes : 0;
        return launch(p, "matrix-product launch", [&] { return difa::launch_linear(a, plan_desc(p).dtype, (hipStream_t)stream); });
    });
}

// ---- a view for the library's tests (difa_testing.h)
extern "C" int32_t difa_testing_slices(int64_t workgroups, int64_t* first, int64_t* count, int32_t capacity) {
    int32_t n = 0;
    (void)difa::in_slices(workgroups, [&](unsigned f, unsigned c) {
        if (n < capacity) { first[n] = f; count[n] = c; }
        ++n;
        return hipSuccess;
    });
    return n;
}
