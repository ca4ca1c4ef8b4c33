// C entry points of include/rnngraph_layers.h: checks of the arguments, then the launches of rows.hip and attention.hip.
#include "../../include/rnngraph_layers.h"

#include <algorithm>
#include <cmath>
#include <cstdlib>
#include <initializer_list>
#include <new>

#include "layers.h"

using namespace rnng;

namespace {

int64_t align_up(int64_t v) { return (v + 255) / 256 * 256; }

// Nothing is thrown across the boundary.
template <class F>
auto guarded(F f) -> decltype(f()) {
    try {
        return f();
    } catch (const std::bad_alloc&) {
        return (decltype(f()))RNN_ERR_NO_MEMORY;
    } catch (...) {
        return (decltype(f()))RNN_ERR_DEVICE;
    }
}
int invalid(const std::string& why) { return set_error(RNN_ERR_INVALID_ARGUMENT, why); }
int done(hipError_t e, const char* what) { return e == hipSuccess ? RNN_OK : set_hip_error(e, what); }

int size_of(int dtype) { return dtype == RNN_F32 ? 4 : 2; }
bool misaligned(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)bytes != 0; }

int check_workspace(const void* ws, int64_t have, int64_t need) {
    if (need == 0) return RNN_OK;
    if (!ws) return set_error(RNN_ERR_WORKSPACE, "workspace is NULL");
    if (misaligned(ws, 256)) return set_error(RNN_ERR_WORKSPACE, "workspace is not 256-byte aligned");
    if (have < need) return set_error(RNN_ERR_WORKSPACE, "workspace too small: need " + std::to_string(need) + " bytes");
    return RNN_OK;
}

// ---- rows ---------------------------------------------------------------------------------
int check_rows(int64_t rows, int32_t dim, int32_t dtype, double p, const uint64_t* d_offset) {
    if (misaligned(d_offset, 8)) return invalid("the offset's pointer is not aligned to its type");
    if (rows < 0 || rows > 2147483647) return invalid("rows must lie in [0, 2^31 - 1]");
    if (dim < 1) return invalid("dim must be positive");
    if (dtype < RNN_F32 || dtype > RNN_F16) return invalid("unknown dtype " + std::to_string(dtype));
    if (!(p >= 0.0 && p <= 1.0)) return invalid("the dropout probability must lie in [0, 1]");
    return RNN_OK;
}
int check_row_tensor(const char* name, const void* p, int64_t ld, int64_t rows, int32_t dim, int bytes, bool needed) {
    if (!p) return needed && rows > 0 ? invalid(std::string(name) + " pointer is NULL") : RNN_OK;
    if (ld < dim) return invalid(std::string(name) + ": ld is less than dim");
    if (misaligned(p, bytes)) return invalid(std::string(name) + " is not aligned to its type");
    return RNN_OK;
}
// An output in an input's place is written row by row behind what is read: rows have to begin at the same places, and two outputs at different ones.
struct Place { const char* name; const void* p; int64_t ld; };
int check_places(int64_t rows, std::initializer_list<Place> outputs, std::initializer_list<Place> inputs, bool may_replace = true) {
    if (rows == 0) return RNN_OK;
    for (const Place& a : outputs) {
        if (!a.p) continue;
        for (const Place& b : outputs)
            if (&a != &b && a.p == b.p) return invalid(std::string(a.name) + " and " + b.name + " are one place");
        for (const Place& b : inputs)
            if (a.p == b.p && (!may_replace || (rows > 1 && a.ld != b.ld)))
                return invalid(std::string(a.name) + " may not be " + b.name + (may_replace ? " with another ld" : ""));
    }
    return RNN_OK;
}
int check_norm(const rnn_add_norm_desc* d) {
    if (!d) return invalid("descriptor is NULL");
    if (const int rc = check_rows(d->rows, d->dim, d->dtype, d->dropout, d->d_offset)) return rc;
    if (d->dim > NORM_MAX_DIM) return invalid("norm: dim exceeds " + std::to_string(NORM_MAX_DIM));
    if (!(d->eps >= 0.0f) || std::isinf(d->eps)) return invalid("norm: eps must be finite and not negative");
    return RNN_OK;
}

int add_norm(const rnn_add_norm_desc* d, const void* x, int64_t ld_x, const void* residual, int64_t ld_residual, const float* gain, void* h, int64_t ld_h,
             void* y, int64_t ld_y, float* scales, int group, float* rstd, hipStream_t s) {
    if (const int rc = check_norm(d)) return rc;
    const int b = size_of(d->dtype);
    int rc = check_row_tensor("x", x, ld_x, d->rows, d->dim, b, true);
    if (!rc) rc = check_row_tensor("residual", residual, ld_residual, d->rows, d->dim, b, false);
    if (!rc) rc = check_row_tensor("h", h, ld_h, d->rows, d->dim, b, false);
    if (!rc) rc = check_row_tensor("y", y, ld_y, d->rows, d->dim, scales ? 1 : b, true);
    if (!rc) rc = check_row_tensor("gain", gain, d->dim, 1, d->dim, 4, false);
    if (!rc) rc = check_row_tensor("rstd", rstd, d->dim, 1, d->dim, 4, false);
    if (!rc) rc = check_row_tensor("scales", scales, d->dim, 1, d->dim, 4, false);
    if (!rc) rc = check_places(d->rows, {{"h", h, ld_h}, {"y", y, ld_y}}, {{"x", x, ld_x}, {"residual", residual, ld_residual}});
    if (!rc && scales) rc = check_places(d->rows, {{"y in 8 bits", y, ld_y}}, {{"x", x, ld_x}, {"residual", residual, ld_residual}}, false);
    if (rc) return rc;
    AddNormArgs a = {};
    a.rows = d->rows; a.dim = d->dim; a.eps = d->eps; a.drop = dropout_args(d->dropout, d->seed, d->offset, d->d_offset);
    a.x = RowTensor{const_cast<void*>(x), ld_x}; a.residual = RowTensor{const_cast<void*>(residual), ld_residual};
    a.h = RowTensor{h, ld_h}; a.y = RowTensor{y, ld_y};
    a.gain = gain; a.rstd = rstd; a.scales = scales; a.group = group;
    return done(launch_add_norm(d->dtype, a, s), "norm launch");
}

// ---- linear attention -----------------------------------------------------------------------
int check_attention(const rnn_linear_attention_desc* d) {
    if (!d) return invalid("descriptor is NULL");
    if (d->T < 0 || d->N < 0 || (int64_t)d->T * d->N >= (int64_t(1) << 31)) return invalid("attention: T and N must not be negative and T * N below 2^31");
    if (d->T > (1 << 30)) return invalid("attention: T must not exceed 2^30");
    if (d->heads < 1 || d->kv_heads < 1 || d->heads % d->kv_heads != 0) return invalid("attention: heads must be a positive multiple of kv_heads");
    if ((int64_t)d->N * d->heads >= (int64_t(1) << 20)) return invalid("attention: N * heads must be below 2^20");
    if (d->dim_k < 1 || d->dim_k > ATTN_MAX_DIM || d->dim_v < 1 || d->dim_v > ATTN_MAX_DIM) return invalid("attention: dim_k and dim_v must lie in [1, " + std::to_string(ATTN_MAX_DIM) + "]");
    if (d->dtype != RNN_F32 && d->dtype != RNN_BF16) return invalid("attention: dtype must be RNN_F32 or RNN_BF16");
    if (!std::isfinite(d->scale)) return invalid("attention: scale must be finite");
    return RNN_OK;
}
int check_frames(const char* name, const rnn_frames* f, const rnn_linear_attention_desc* d, bool needed) {
    if (!f || !f->data) return needed && d->T > 0 && d->N > 0 ? invalid(std::string("attention: ") + name + " pointer is NULL") : RNN_OK;
    if (misaligned(f->data, size_of(d->dtype))) return invalid(std::string("attention: ") + name + " is not aligned to its type");
    return RNN_OK;
}
// An output, `heads` x `units` for a frame: two of its elements share a place where an axis steps, or two axes' steps differ, by less than a head's units.
int check_places(const char* name, const rnn_frames* f, const rnn_linear_attention_desc* d, int32_t heads, int32_t units) {
    if (!f || !f->data) return RNN_OK;
    typedef __int128 wide;
    const int32_t size[3] = {d->T, d->N, heads};
    const wide stride[3] = {f->stride_t, f->stride_n, f->stride_h};
    const auto small = [&](wide step) { return step > -units && step < units; };
    bool shared = false;
    for (int i = 0; i < 3; ++i) {
        shared = shared || (size[i] > 1 && small(stride[i]));
        for (int j = 0; j < i; ++j) shared = shared || (size[i] > 1 && size[j] > 1 && (small(stride[i] - stride[j]) || small(stride[i] + stride[j])));
    }
    return shared && d->T > 0 ? invalid(std::string("attention: elements of ") + name + " share places") : RNN_OK;
}
// Outputs begin where nothing else of the call does.
struct Start { const char* name; const void* p; };
Start start(const char* name, const rnn_frames* f) { return Start{name, f ? f->data : nullptr}; }
int check_apart(std::initializer_list<Start> outputs, std::initializer_list<Start> inputs) {
    for (const Start& a : outputs) {
        if (!a.p) continue;
        for (const Start& b : outputs)
            if (&a != &b && a.p == b.p) return invalid(std::string("attention: ") + a.name + " and " + b.name + " are one place");
        for (const Start& b : inputs)
            if (a.p == b.p) return invalid(std::string("attention: ") + a.name + " may not be " + b.name);
    }
    return RNN_OK;
}
int check_floats(const char* name, const void* p) { return misaligned(p, 4) ? invalid(std::string("attention: ") + name + " is not aligned to its type") : RNN_OK; }

AttnTensor tensor(const rnn_frames* f, int group) { return f ? AttnTensor{f->data, f->stride_t, f->stride_n, f->stride_h, group} : AttnTensor{nullptr, 0, 0, 0, group}; }
AttnOut output(const rnn_frames* f) { return f ? AttnOut{f->data, f->stride_t, f->stride_n, f->stride_h} : AttnOut{nullptr, 0, 0, 0}; }
AttnCall call_of(const rnn_linear_attention_desc* d, const float* log_decay, const int32_t* lengths) {
    return AttnCall{d->T, d->N, d->heads, d->dtype, log_decay, lengths};
}
AttnOp forward_op(const rnn_linear_attention_desc* d, const rnn_frames* q, const rnn_frames* k, const rnn_frames* v) {
    const int group = d->heads / d->kv_heads;
    AttnOp a = {};
    a.q = tensor(q, 1); a.k = tensor(k, group); a.v = tensor(v, group);
    a.dk = d->dim_k; a.dv = d->dim_v; a.si = d->dim_v; a.sj = 1;
    a.update = 1.0f; a.out = d->scale; a.early = true;
    return a;
}

// The operators of a backward call, without their outputs: 1 dq, 2 dv, 4 dk (bits of `which`).
int backward_ops(const rnn_linear_attention_desc* d, const AttnOp& f, const AttnTensor& t_do, int which, AttnOp* ops) {
    int n = 0;
    if (which & 1) {
        AttnOp a = f;
        a.q = t_do; a.k = f.v; a.v = f.k; a.dk = d->dim_v; a.dv = d->dim_k; a.si = 1; a.sj = d->dim_v;
        ops[n++] = a;
    }
    AttnOp r = f;
    r.reverse = true; r.early = false; r.update = d->scale; r.out = 1.0f; r.o_f32 = d->heads != d->kv_heads;
    if (which & 2) {
        AttnOp a = r;
        a.q = f.k; a.k = f.q; a.v = t_do;
        ops[n++] = a;
    }
    if (which & 4) {
        AttnOp a = r;
        a.q = f.v; a.k = t_do; a.v = f.q; a.dk = d->dim_v; a.dv = d->dim_k; a.si = 1; a.sj = d->dim_v;
        ops[n++] = a;
    }
    return n;
}

// Workspace of a call: the heads' own parts of dk and dv, where several share a key / value head, and the segments' states (as many as any
// choice of outputs takes).
struct AttnSpace { int64_t part_k = -1, part_v = -1, segments = 0, total = 0; };
AttnSpace space_of(const rnn_linear_attention_desc* d, bool backward) {
    AttnSpace w;
    if (backward && d->heads != d->kv_heads) {
        const int64_t heads = (int64_t)d->T * d->N * d->heads;
        w.part_k = w.total; w.total += align_up(heads * d->dim_k * 4);
        w.part_v = w.total; w.total += align_up(heads * d->dim_v * 4);
    }
    w.segments = w.total;
    const AttnCall c = call_of(d, nullptr, nullptr);
    const AttnOp f = forward_op(d, nullptr, nullptr, nullptr);
    int64_t most = 0;
    if (!backward) most = attention_space(c, &f, 1);
    else
        for (int which = 1; which < 8; ++which) {
            AttnOp ops[3];
            most = std::max(most, attention_space(c, ops, backward_ops(d, f, f.q, which, ops)));
        }
    w.total += align_up(most);
    return w;
}

}  // namespace

int64_t rnn_linear_attention_workspace_bytes(const rnn_linear_attention_desc* d, int32_t backward) {
    return guarded([&]() -> int64_t {
        if (const int rc = check_attention(d)) return rc;
        return space_of(d, backward != 0).total;
    });
}

int rnn_linear_attention_forward(const rnn_linear_attention_desc* d, const rnn_frames* q, const rnn_frames* k, const rnn_frames* v, const float* d_log_decay,
                                 const int32_t* d_lengths, const float* d_state_in, float* d_state_out, const rnn_frames* o, void* d_workspace,
                                 int64_t ws_bytes, void* hip_stream) {
    return guarded([&]() -> int {
        if (const int rc = check_attention(d)) return rc;
        const bool with_o = o && o->data;
        int rc = check_frames("q", q, d, with_o);
        if (!rc) rc = check_frames("k", k, d, true);
        if (!rc) rc = check_frames("v", v, d, true);
        if (!rc) rc = check_frames("o", o, d, false);
        if (!rc) rc = check_floats("state_in", d_state_in);
        if (!rc) rc = check_floats("state_out", d_state_out);
        if (!rc && !d_log_decay) rc = invalid("attention: log_decay pointer is NULL");
        if (!rc) rc = check_floats("log_decay", d_log_decay);
        if (!rc) rc = check_floats("lengths", d_lengths);
        if (!rc && !with_o && !d_state_out) rc = invalid("attention: neither o nor state_out is given");
        const AttnSpace w = space_of(d, false);
        if (!rc) rc = check_workspace(d_workspace, ws_bytes, w.total);
        if (rc || d->N == 0) return rc;
        if ((rc = check_places("o", o, d, d->heads, d->dim_v))) return rc;
        if (d->T > 0 && (rc = check_apart({start("o", o)}, {start("q", q), start("k", k), start("v", v)}))) return rc;
        AttnOp a = forward_op(d, q, k, v);
        if (with_o) a.o = output(o);
        a.s_in = d_state_in; a.s_out = d_state_out;
        return done(launch_attention(call_of(d, d_log_decay, d_lengths), &a, 1, reinterpret_cast<float*>(static_cast<char*>(d_workspace) + w.segments),
                                     static_cast<hipStream_t>(hip_stream)), "attention launch");
    });
}

int rnn_linear_attention_backward(const rnn_linear_attention_desc* d, const rnn_frames* q, const rnn_frames* k, const rnn_frames* v, const float* d_log_decay,
                                  const int32_t* d_lengths, const float* d_state_in, const rnn_frames* d_o, const float* d_dstate_out, const rnn_frames* dq,
                                  const rnn_frames* dk, const rnn_frames* dv, float* d_dstate_in, void* d_workspace, int64_t ws_bytes, void* hip_stream) {
    return guarded([&]() -> int {
        if (const int rc = check_attention(d)) return rc;
        const bool with_q = dq && dq->data, with_k = dk && dk->data, with_v = dv && dv->data;
        int rc = check_frames("q", q, d, true);
        if (!rc) rc = check_frames("k", k, d, true);
        if (!rc) rc = check_frames("v", v, d, true);
        if (!rc) rc = check_frames("do", d_o, d, true);
        if (!rc) rc = check_frames("dq", dq, d, false);
        if (!rc) rc = check_frames("dk", dk, d, false);
        if (!rc) rc = check_frames("dv", dv, d, false);
        if (!rc) rc = check_floats("state_in", d_state_in);
        if (!rc) rc = check_floats("dstate_out", d_dstate_out);
        if (!rc) rc = check_floats("dstate_in", d_dstate_in);
        if (!rc && !d_log_decay) rc = invalid("attention: log_decay pointer is NULL");
        if (!rc) rc = check_floats("log_decay", d_log_decay);
        if (!rc) rc = check_floats("lengths", d_lengths);
        if (!rc && d_dstate_in && d_dstate_in == d_dstate_out) rc = invalid("attention: dstate_in may not be dstate_out");
        const AttnSpace w = space_of(d, true);
        if (!rc) rc = check_workspace(d_workspace, ws_bytes, w.total);
        if (rc || d->N == 0) return rc;
        if ((rc = check_places("dq", dq, d, d->heads, d->dim_k))) return rc;
        if ((rc = check_places("dk", dk, d, d->kv_heads, d->dim_k))) return rc;
        if ((rc = check_places("dv", dv, d, d->kv_heads, d->dim_v))) return rc;
        if (d->T > 0 && (rc = check_apart({start("dq", dq), start("dk", dk), start("dv", dv)}, {start("q", q), start("k", k), start("v", v), start("do", d_o)}))) return rc;
        if (with_q && d_dstate_in && d_dstate_in == d_state_in) return invalid("attention: dstate_in may not be state_in, which dq is made from");
        hipStream_t s = static_cast<hipStream_t>(hip_stream);
        const int group = d->heads / d->kv_heads;
        const AttnCall call = call_of(d, d_log_decay, d_lengths);
        char* ws = static_cast<char*>(d_workspace);
        auto part = [&](int64_t off, int dim) { return AttnOut{ws + off, (int64_t)d->N * d->heads * dim, (int64_t)d->heads * dim, dim}; };
        const int which = (with_q ? 1 : 0) | (with_v || d_dstate_in ? 2 : 0) | (with_k ? 4 : 0);
        if (which == 0) return RNN_OK;
        AttnOp ops[3];
        const int n_ops = backward_ops(d, forward_op(d, q, k, v), tensor(d_o, 1), which, ops);
        AttnOp* a = ops;
        if (which & 1) { a->o = output(dq); a->s_in = d_state_in; ++a; }
        if (which & 2) {
            if (with_v) a->o = group > 1 ? part(w.part_v, d->dim_v) : output(dv);
            a->s_in = d_dstate_out; a->s_out = d_dstate_in; ++a;
        }
        if (which & 4) { a->o = group > 1 ? part(w.part_k, d->dim_k) : output(dk); a->s_in = d_dstate_out; }
        rc = done(launch_attention(call, ops, n_ops, reinterpret_cast<float*>(ws + w.segments), s), "attention gradient launch");
        if (!rc && group > 1 && d->T > 0) {
            if (with_k) rc = done(launch_attention_sum_heads(call, (const float*)(ws + w.part_k), output(dk), d->dim_k, group, s), "attention gradient sum");
            if (!rc && with_v) rc = done(launch_attention_sum_heads(call, (const float*)(ws + w.part_v), output(dv), d->dim_v, group, s), "attention gradient sum");
        }
        return rc;
    });
}

int rnn_add_norm_forward(const rnn_add_norm_desc* d, const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, const float* d_gain, void* d_h,
                         int64_t ld_h, void* d_y, int64_t ld_y, float* d_rstd, void* hip_stream) {
    return guarded([&]() -> int { return add_norm(d, d_x, ld_x, d_residual, ld_residual, d_gain, d_h, ld_h, d_y, ld_y, nullptr, 0, d_rstd, static_cast<hipStream_t>(hip_stream)); });
}

int rnn_add_norm_e4m3(const rnn_add_norm_desc* d, const void* d_x, int64_t ld_x, const void* d_residual, int64_t ld_residual, const float* d_gain, void* d_h,
                      int64_t ld_h, uint8_t* d_y8, int64_t ld_y8, float* d_scales, int32_t group, float* d_rstd, void* hip_stream) {
    return guarded([&]() -> int {
        if (const int rc = check_norm(d)) return rc;
        if (group != 0 && group != 128) return invalid("norm: group must be 0 (a scale for every row) or 128");
        if (!d_scales) return d->rows > 0 ? invalid("scales pointer is NULL") : RNN_OK;
        return add_norm(d, d_x, ld_x, d_residual, ld_residual, d_gain, d_h, ld_h, d_y8, ld_y8, d_scales, group, d_rstd, static_cast<hipStream_t>(hip_stream));
    });
}

int64_t rnn_add_norm_workspace_bytes(const rnn_add_norm_desc* d) {
    return guarded([&]() -> int64_t {
        if (const int rc = check_norm(d)) return rc;
        const int blocks = norm_grad_blocks(d->rows, d->dim);
        return blocks > 1 ? align_up((int64_t)blocks * d->dim * 4) : 0;
    });
}

int rnn_add_norm_backward(const rnn_add_norm_desc* d, const void* d_dy, int64_t ld_dy, const void* d_dh, int64_t ld_dh, const void* d_h, int64_t ld_h,
                          const float* d_rstd, const float* d_gain, void* d_dx, int64_t ld_dx, void* d_dresidual, int64_t ld_dresidual, float* d_dgain,
                          void* d_workspace, int64_t ws_bytes, void* hip_stream) {
    return guarded([&]() -> int {
        if (const int rc = check_norm(d)) return rc;
        const int b = size_of(d->dtype);
        int rc = check_row_tensor("dy", d_dy, ld_dy, d->rows, d->dim, b, true);
        if (!rc) rc = check_row_tensor("dh", d_dh, ld_dh, d->rows, d->dim, b, false);
        if (!rc) rc = check_row_tensor("h", d_h, ld_h, d->rows, d->dim, b, true);
        if (!rc) rc = check_row_tensor("dx", d_dx, ld_dx, d->rows, d->dim, b, false);
        if (!rc) rc = check_row_tensor("dresidual", d_dresidual, ld_dresidual, d->rows, d->dim, b, false);
        if (!rc) rc = check_row_tensor("rstd", d_rstd, d->dim, d->rows, d->dim, 4, true);
        if (!rc) rc = check_row_tensor("gain", d_gain, d->dim, 1, d->dim, 4, false);
        if (!rc) rc = check_row_tensor("dgain", d_dgain, d->dim, 1, d->dim, 4, false);
        if (!rc) rc = check_places(d->rows, {{"dx", d_dx, ld_dx}, {"dresidual", d_dresidual, ld_dresidual}}, {{"dy", d_dy, ld_dy}, {"dh", d_dh, ld_dh}, {"h", d_h, ld_h}});
        const int blocks = norm_grad_blocks(d->rows, d->dim);
        if (!rc && d_dgain && blocks > 1) rc = check_workspace(d_workspace, ws_bytes, align_up((int64_t)blocks * d->dim * 4));
        if (rc || (!d_dx && !d_dresidual && !d_dgain)) return rc;
        AddNormGradArgs a = {};
        a.rows = d->rows; a.dim = d->dim; a.drop = dropout_args(d->dropout, d->seed, d->offset, d->d_offset);
        a.dy = RowTensor{const_cast<void*>(d_dy), ld_dy}; a.dh = RowTensor{const_cast<void*>(d_dh), ld_dh}; a.h = RowTensor{const_cast<void*>(d_h), ld_h};
        a.dx = RowTensor{d_dx, ld_dx}; a.dresidual = RowTensor{d_dresidual, ld_dresidual};
        a.gain = d_gain; a.rstd = d_rstd; a.dgain = d_dgain; a.partial = static_cast<float*>(d_workspace); a.blocks = blocks;
        return done(launch_add_norm_grad(d->dtype, a, static_cast<hipStream_t>(hip_stream)), "norm gradient launch");
    });
}

int rnn_dropout(const rnn_dropout_desc* d, const void* d_x, int64_t ld_x, void* d_y, int64_t ld_y, void* hip_stream) {
    return guarded([&]() -> int {
        if (!d) return invalid("descriptor is NULL");
        if (const int rc = check_rows(d->rows, d->dim, d->dtype, d->p, d->d_offset)) return rc;
        const int b = size_of(d->dtype);
        int rc = check_row_tensor("x", d_x, ld_x, d->rows, d->dim, b, true);
        if (!rc) rc = check_row_tensor("y", d_y, ld_y, d->rows, d->dim, b, true);
        if (!rc) rc = check_places(d->rows, {{"y", d_y, ld_y}}, {{"x", d_x, ld_x}});
        if (rc) return rc;
        const DropoutRowsArgs a{d->rows, d->dim, dropout_args(d->p, d->seed, d->offset, d->d_offset), RowTensor{const_cast<void*>(d_x), ld_x}, RowTensor{d_y, ld_y}, 0, nullptr};
        return done(launch_dropout(d->dtype, a, static_cast<hipStream_t>(hip_stream)), "dropout launch");
    });
}
