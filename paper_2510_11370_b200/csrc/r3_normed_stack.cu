// Stacks of replayed MoE blocks with norms around every block, as the models of the paper have them:
//   h_l = RMSNorm(x_l) w_pre,l
//   x_{l+1} = residual_scale x_l + branch_scale gate_l RMSNorm(y_replay,l(h_l)) w_post,l
// forward, and forward plus the exact backward chain, with an optimiser step on a block's expert
// weights as soon as their gradients are there.  Between two blocks runs one r3_norm_residual (or its
// gradient), which ends block l - 1 and begins block l; the blocks are r3_replay_layer and
// r3_replay_layer_train.
#include "r3_common.cuh"
#include "r3_internal.h"

namespace r3 {

constexpr size_t kStatusBytes = 256;          // a status word of the call's own, and the alignment behind it

struct StackCall {
    const r3_shape* s;
    int32_t L;
    const r3_block_norms* n;
    const void *w_router, *idx, *w_gate, *w_up, *w_down;
    int32_t* dev_status;
    void* stream;

    size_t rows_bytes() const { return round_up((size_t)s->T * s->d * act_bytes(s), 256); }
    size_t router_bytes() const { return (size_t)s->E * s->d * (s->router_w_dtype == R3_BF16 ? 2 : 4); }
    size_t expert_bytes() const { return (size_t)s->E * s->F * s->d * act_bytes(s); }
    size_t record_bytes() const { return (size_t)s->T * s->K * idx_bytes(s); }
    static const void* at(const void* p, size_t off) { return static_cast<const char*>(p) + off; }
    const void* router(int l) const { return at(w_router, l * router_bytes()); }
    const void* record(int l) const { return at(idx, l * record_bytes()); }
    const void* gate_w(int l) const { return at(w_gate, l * expert_bytes()); }
    const void* up_w(int l) const { return at(w_up, l * expert_bytes()); }
    const void* down_w(int l) const { return at(w_down, l * expert_bytes()); }
    // a block's norm vector (null stays null) and its gradient
    const void* vec(const void* p, int l) const {
        return p ? at(p, (size_t)l * s->d * (n->w_dtype == R3_BF16 ? 2 : 4)) : nullptr;
    }
    float* grad(float* p, int l) const { return p ? p + (size_t)l * s->d : nullptr; }

    // The norm between block `before` (-1: none, in front of the stack) and the block behind it.
    r3_norm shape(int before) const {
        r3_norm q = {};
        q.T = s->T;
        q.d = s->d;
        q.act_dtype = s->act_dtype;
        q.w_dtype = n->w_dtype;
        q.gate_kind = before >= 0 && n->gate ? R3_GATE_CHANNEL : R3_GATE_NONE;
        q.eps = n->eps;
        q.residual_scale = n->residual_scale;
        q.branch_scale = n->branch_scale;
        return q;
    }
    // Ends block l - 1 (l > 0: x, y -> x_out) and begins block l (l < L: -> h).
    r3_status between(int l, const void* x, const void* y, void* x_out, void* h) const {
        const r3_norm q = shape(l - 1);
        return r3_norm_residual(&q, x, l > 0 ? y : nullptr, l > 0 ? vec(n->w_post, l - 1) : nullptr,
                                l > 0 ? vec(n->gate, l - 1) : nullptr, l < L ? vec(n->w_pre, l) : nullptr,
                                l > 0 ? x_out : nullptr, l < L ? h : nullptr, stream);
    }
    r3_status between_bwd(int l, const void* x_out, const void* y, const void* dx_out, const void* dh,
                          void* dx, void* dy, void* ws, size_t ws_bytes) const {
        const r3_norm q = shape(l - 1);
        return r3_norm_residual_bwd(&q, x_out, l > 0 ? y : nullptr, l > 0 ? vec(n->w_post, l - 1) : nullptr,
                                    l > 0 ? vec(n->gate, l - 1) : nullptr,
                                    l < L ? vec(n->w_pre, l) : nullptr, dx_out, l < L ? dh : nullptr, dx,
                                    l > 0 ? dy : nullptr, l > 0 ? grad(n->dw_post, l - 1) : nullptr,
                                    l > 0 ? grad(n->dgate, l - 1) : nullptr,
                                    l < L ? grad(n->dw_pre, l) : nullptr, ws, ws_bytes, stream);
    }
};

static r3_status check_stack(const r3_shape* shape, int32_t L, const r3_block_norms* n, bool train) {
    const r3_status st = check_shape(shape);
    if (st != R3_OK) return st;
    if (L <= 0 || !n || !n->w_pre) return R3_ERR_INVALID_ARG;
    if (train && (!n->dw_pre || (n->w_post != nullptr) != (n->dw_post != nullptr) ||
                  (n->gate != nullptr) != (n->dgate != nullptr)))
        return R3_ERR_INVALID_ARG;
    StackCall c = {};
    c.s = shape;
    c.n = n;
    const r3_norm q = c.shape(-1);
    if (!(q.eps > 0.f) || !(q.eps < 1e30f) || !(q.residual_scale > -1e30f && q.residual_scale < 1e30f) ||
        !(q.branch_scale > -1e30f && q.branch_scale < 1e30f) ||
        (q.w_dtype != R3_F32 && q.w_dtype != R3_BF16))
        return R3_ERR_INVALID_ARG;
    // every row of a vector [L, d] starts on a 16-byte boundary: d is a multiple of 8
    if (!aligned(n->w_pre, 16) || !aligned(n->w_post, 16) || !aligned(n->gate, 16) ||
        !aligned(n->dw_pre, 16) || !aligned(n->dw_post, 16) || !aligned(n->dgate, 16))
        return R3_ERR_INVALID_ARG;
    return r3_norm_residual_bwd_workspace_bytes(&q) == 0 && shape->T > 0 ? R3_ERR_UNSUPPORTED : R3_OK;
}

}  // namespace r3

extern "C" size_t r3_normed_stack_workspace_bytes(const r3_shape* shape) {
    if (r3::check_shape(shape) != R3_OK) return 0;
    const size_t xb = r3::round_up((size_t)shape->T * shape->d * r3::act_bytes(shape), 256);
    return 4 * xb + r3::round_up((size_t)shape->T * shape->E * 4, 256) + r3_replay_layer_workspace_bytes(shape);
}

extern "C" r3_status r3_normed_stack(const r3_shape* shape, int32_t L, const r3_block_norms* norms,
                                     const void* x0, const void* w_router, const void* idx,
                                     const void* w_gate, const void* w_up, const void* w_down,
                                     void* x_out, void* workspace, size_t ws_bytes,
                                     int32_t* dev_status, void* stream) {
    r3_status st = r3::check_stack(shape, L, norms, false);
    if (st != R3_OK) return st;
    if (shape->T == 0) return R3_OK;
    if (!x0 || !w_router || !idx || !w_gate || !w_up || !w_down || !x_out || !r3::aligned(x0, 16) ||
        !r3::aligned(x_out, 16))
        return R3_ERR_INVALID_ARG;
    if (!workspace || !r3::aligned(workspace, 256) || ws_bytes < r3_normed_stack_workspace_bytes(shape))
        return R3_ERR_WORKSPACE;
    const r3::StackCall c = {shape, L, norms, w_router, idx, w_gate, w_up, w_down, dev_status, stream};
    const size_t xb = c.rows_bytes(), lb = r3::round_up((size_t)shape->T * shape->E * 4, 256);
    char* ws = static_cast<char*>(workspace);
    void* ping[2] = {ws, ws + xb};
    void *h = ws + 2 * xb, *y = ws + 3 * xb;
    float* dlogits = reinterpret_cast<float*>(ws + 4 * xb);             // not wanted here
    void* inner = ws + 4 * xb + lb;
    const size_t inner_bytes = r3_replay_layer_workspace_bytes(shape);
    if ((st = c.between(0, x0, nullptr, nullptr, h)) != R3_OK) return st;
    const void* x = x0;
    for (int32_t l = 0; l < L; ++l) {
        // the layer also takes an upstream gradient: its own input will do
        st = r3_replay_layer(shape, h, c.router(l), c.record(l), c.gate_w(l), c.up_w(l), c.down_w(l), h, y,
                             dlogits, nullptr, inner, inner_bytes, dev_status, stream);
        if (st != R3_OK) return st;
        void* nxt = l == L - 1 ? x_out : ping[l & 1];
        if ((st = c.between(l + 1, x, y, nxt, h)) != R3_OK) return st;
        x = nxt;
    }
    return R3_OK;
}

extern "C" size_t r3_normed_stack_train_workspace_bytes(const r3_shape* shape, int32_t L) {
    if (r3::check_shape(shape) != R3_OK || shape->act_dtype != R3_BF16 || L <= 0) return 0;
    const size_t xb = r3::round_up((size_t)shape->T * shape->d * r3::act_bytes(shape), 256);
    r3_block_norms n = {};
    n.eps = 1.f;
    r3::StackCall c = {};
    c.s = shape;
    c.n = &n;
    const r3_norm q = c.shape(-1);
    return (3 * (size_t)L + 4) * xb + r3_norm_residual_bwd_workspace_bytes(&q) + r3::kStatusBytes +
           r3_replay_layer_train_workspace_bytes(shape);
}

extern "C" r3_status r3_normed_stack_train(const r3_shape* shape, int32_t L, const r3_block_norms* norms,
                                           const void* x0, const void* w_router, const void* idx,
                                           void* w_gate, void* w_up, void* w_down, const void* dy,
                                           void* x_out, float* dlogits, void* dx0, float* dw_router,
                                           float* dw_gate, float* dw_up, float* dw_down,
                                           const r3_adamw* adamw, const r3_adamw_tensor* expert_states,
                                           const float* grad_scale, const float* scalars,
                                           void* workspace, size_t ws_bytes, int32_t* dev_status,
                                           void* stream) {
    r3_status st = r3::check_stack(shape, L, norms, true);
    if (st != R3_OK) return st;
    if (shape->act_dtype != R3_BF16) return R3_ERR_UNSUPPORTED;
    const bool weights = dw_gate || dw_up || dw_down;
    if (weights && (!dw_gate || !dw_up || !dw_down)) return R3_ERR_INVALID_ARG;
    const r3::StackCall c = {shape, L, norms, w_router, idx, w_gate, w_up, w_down, dev_status, stream};
    const size_t per_block = (size_t)shape->E * shape->F * shape->d;
    // A block's three entries of the optimiser's list, with the gradients of this call.
    auto block_states = [&](int32_t l, r3_adamw_tensor* e) {
        const void* w[3] = {c.gate_w(l), c.up_w(l), c.down_w(l)};
        const float* g[3] = {dw_gate, dw_up, dw_down};
        for (int k = 0; k < 3; ++k) {
            e[k] = expert_states[3 * l + k];
            if (e[k].param != w[k] || e[k].n != (int64_t)per_block) return false;
            e[k].grad = g[k];
        }
        return true;
    };
    r3_adamw_tensor e[3];
    if (adamw) {
        if (!weights || !expert_states || adamw->param_dtype != R3_BF16 || adamw->grad_dtype != R3_F32)
            return R3_ERR_INVALID_ARG;
        for (int32_t l = 0; l < L; ++l) {
            if (!block_states(l, e)) return R3_ERR_INVALID_ARG;
            if ((st = r3::check_adamw_call(adamw, e, 3, grad_scale, scalars)) != R3_OK) return st;
        }
        const void* grads[3] = {dw_gate, dw_up, dw_down};
        st = r3::check_adamw_distinct(adamw, expert_states, 3 * L, grads, grad_scale, scalars);
        if (st != R3_OK) return st;
    }
    if (shape->T == 0) return R3_OK;
    if (!x0 || !w_router || !idx || !w_gate || !w_up || !w_down || !dy || !x_out || !dlogits || !dx0 ||
        !dw_router || x_out == x0 || x_out == dy || dx0 == x_out || !r3::aligned(x0, 16) ||
        !r3::aligned(dy, 16) || !r3::aligned(x_out, 16) || !r3::aligned(dx0, 16))
        return R3_ERR_INVALID_ARG;
    if (!workspace || !r3::aligned(workspace, 256) ||
        ws_bytes < r3_normed_stack_train_workspace_bytes(shape, L))
        return R3_ERR_WORKSPACE;
    const size_t xb = c.rows_bytes(), T = shape->T, E = shape->E;
    char* ws = static_cast<char*>(workspace);
    // kept for the backward pass: x_1 .. x_{L-1} (x_0 and x_L are the caller's), every h_l and y_l
    auto x_at = [&](int32_t l) {
        return l == 0 ? const_cast<void*>(x0) : l == L ? x_out : static_cast<void*>(ws + (size_t)(l - 1) * xb);
    };
    auto h_at = [&](int32_t l) { return static_cast<void*>(ws + ((size_t)L + l) * xb); };
    auto y_at = [&](int32_t l) { return static_cast<void*>(ws + (2 * (size_t)L + l) * xb); };
    char* rest = ws + 3 * (size_t)L * xb;
    void *dres[2] = {rest, rest + xb}, *dyb = rest + 2 * xb, *dh = rest + 3 * xb;
    const r3_norm q = c.shape(-1);
    void* norm_ws = rest + 4 * xb;
    const size_t norm_bytes = r3_norm_residual_bwd_workspace_bytes(&q);
    char* own_status = rest + 4 * xb + norm_bytes;
    void* inner = own_status + r3::kStatusBytes;
    const size_t fwd_bytes = r3_replay_layer_workspace_bytes(shape);
    const size_t train_bytes = r3_replay_layer_train_workspace_bytes(shape);

    cudaStream_t cs = static_cast<cudaStream_t>(stream);
    if (adamw && !dev_status) {
        // the steps look at what the blocks report, so that gradients which are not valid move no weight
        dev_status = reinterpret_cast<int32_t*>(own_status);
        if (cudaMemsetAsync(dev_status, 0, sizeof(int32_t), cs) != cudaSuccess) {
            cudaGetLastError();
            return R3_ERR_CUDA;
        }
    }
    if ((st = c.between(0, x0, nullptr, nullptr, h_at(0))) != R3_OK) return st;
    for (int32_t l = 0; l < L; ++l) {
        // the gradients that this call forms from dy are overwritten below
        st = r3_replay_layer(shape, h_at(l), c.router(l), c.record(l), c.gate_w(l), c.up_w(l), c.down_w(l), dy,
                             y_at(l), dlogits + (size_t)l * T * E, nullptr, inner, fwd_bytes, dev_status,
                             stream);
        if (st != R3_OK) return st;
        st = c.between(l + 1, x_at(l), y_at(l), x_at(l + 1), l + 1 < L ? h_at(l + 1) : nullptr);
        if (st != R3_OK) return st;
    }
    // `around`: the gradient at x_{l+1} past the block behind it; dh: the one at that block's input.
    // Together they give the gradients at x_l past block l (dres) and at y_l (dyb).
    const void* around = dy;
    for (int32_t l = L - 1; l >= 0; --l) {
        st = c.between_bwd(l + 1, x_at(l + 1), y_at(l), around, dh, dres[l & 1], dyb, norm_ws, norm_bytes);
        if (st != R3_OK) return st;
        around = dres[l & 1];
        const size_t off = adamw ? 0 : (size_t)l * per_block;      // with the optimiser: one block's gradients
        st = r3_replay_layer_train(shape, h_at(l), c.router(l), c.record(l), c.gate_w(l), c.up_w(l), c.down_w(l),
                                   dyb, y_at(l), dlogits + (size_t)l * T * E, dh,
                                   dw_router + (size_t)l * E * shape->d, weights ? dw_gate + off : nullptr,
                                   weights ? dw_up + off : nullptr, weights ? dw_down + off : nullptr, inner,
                                   train_bytes, dev_status, stream);
        if (st != R3_OK) return st;
        if (adamw) {
            // no later step reads block l's expert weights: they take their step while only this
            // block's gradients exist
            block_states(l, e);
            if ((st = r3::adamw_step(adamw, e, 3, grad_scale, scalars, dev_status, cs)) != R3_OK) return st;
        }
    }
    return c.between_bwd(0, x0, nullptr, around, dh, dx0, nullptr, norm_ws, norm_bytes);
}
