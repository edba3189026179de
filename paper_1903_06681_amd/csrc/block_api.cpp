// C entry points of a gated residual block: the gated product, the join of a branch with its
// residual stream, dropout.  No allocation, no state, no synchronisation.
#include <hip/hip_runtime.h>

#include "act_check.h"
#include "gate.h"
#include "join.h"

namespace dc {

// The draw of a tensor [N][C][H][W]; no drop: t = 0.
static dc_status drop_args(const dc_drop* d, const dc_view& v, int32_t C, DropArgs* a) {
    std::memset(a, 0, sizeof(*a));
    a->scale = 1.0f;
    if (!d) return DC_OK;
    if (!(d->p >= 0 && d->p < 1)) return DC_ERR_ARG;
    if (d->n0 < 0 || d->h0 < 0 || d->w0 < 0 || d->H < 0 || d->W < 0 || d->P < 0 || d->Q < 0) return DC_ERR_ARG;
    const int64_t P = std::max(d->P, 1), Q = std::max(d->Q, 1);
    const int64_t H = d->H ? d->H : d->h0 + P * v.H, W = d->W ? d->W : d->w0 + Q * v.W;
    if (v.N % (P * Q) || d->h0 + P * v.H > H || d->w0 + Q * v.W > W) return DC_ERR_SHAPE;
    a->groups = (C + 7) / 8;
    if ((double(d->n0) + v.N) * a->groups * double(H) * double(W) > 9e18) return DC_ERR_TOO_LARGE;
    if (misaligned(d->step, 8)) return DC_ERR_ALIGN;
    a->seed = d->seed;
    a->offset = d->offset;
    a->step = d->step;
    a->plane = H * W;
    a->cols = W;
    a->t = int32_t(std::min(std::nearbyint(65536 * d->p), 65535.0));
    a->scale = float(65536.0 / (65536 - a->t));
    a->n0 = d->n0;
    a->h0 = d->h0;
    a->w0 = d->w0;
    a->H = v.H;
    a->W = v.W;
    a->Q = int32_t(Q);
    a->per = fast_div(uint32_t(v.N / (P * Q)));
    a->dW = fast_div(uint32_t(v.W));
    a->dQ = fast_div(uint32_t(Q));
    return DC_OK;
}

static dc_status join_norm(const dc_norm* n, JoinNorm* k) {
    *k = JoinNorm{nullptr, nullptr, 0, DC_NORM_NONE};
    if (!n) return DC_OK;
    if (n->kind < DC_NORM_NONE || n->kind > DC_NORM_RMS) return DC_ERR_ARG;
    if (n->kind == DC_NORM_NONE) return DC_OK;
    if (!(n->eps >= 0) || std::isinf(n->eps)) return DC_ERR_ARG;
    if (misaligned(n->gamma) || misaligned(n->beta)) return DC_ERR_ALIGN;
    *k = JoinNorm{n->gamma, n->beta, n->eps, n->kind};
    return DC_OK;
}

}  // namespace dc

using namespace dc;

extern "C" {

dc_status dc_dropout(const dc_drop* drop, const dc_view* vx, const void* x, const dc_view* vy, void* y, void* stream) {
    if (!drop || !vx) return DC_ERR_NULL;
    dc_status st = check_tensor(vx, x, READ, false, *vx, vx->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vy, y, WRITE, false, *vx, vx->C)) != DC_OK) return st;
    DropoutArgs a;
    std::memset(&a, 0, sizeof(a));
    if ((st = drop_args(drop, *vx, vx->C, &a.d)) != DC_OK) return st;
    Together t;
    t.add(vx, x);
    t.add(vy, y);
    a.x = device_view(vx, x);
    a.y = device_view(vy, y);
    a.C = vx->C;
    a.rows = t.rows();
    a.HW = vx->H * vx->W;
    a.len = a.rows ? 1 : t.flat() ? a.HW : vx->W;
    a.per = dropout_chunk(a.x, a.y, a.rows, pixels_of(*vx), a.d.groups);
    a.cpr = (a.len - 1) / a.per + 1;
    a.chunks = vx->N * (a.HW / a.len) * a.cpr;
    a.dsample = fast_div(uint32_t(a.HW / a.len * a.cpr));
    a.dcpr = fast_div(uint32_t(a.cpr));
    (void)hipGetLastError();
    return launched(launch_dropout(a, static_cast<hipStream_t>(stream)));
}

dc_status dc_gate_fwd(const dc_view* vx, const void* x, const void* w, const float* bias, int32_t act, const dc_drop* drop,
                      const dc_view* vz, void* zg, void* zu, const dc_view* vh, void* h, void* stream) {
    if (!vx || !vh) return DC_ERR_NULL;
    dc_status st = check_tensor(vx, x, READ, false, *vx, vx->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vh, h, WRITE, false, *vx, vh->C)) != DC_OK) return st;
    if (zg || zu) {
        if ((st = check_tensor(vz, zg, WRITE, true, *vx, vh->C)) != DC_OK) return st;
        if ((st = check_tensor(vz, zu, WRITE, true, *vx, vh->C)) != DC_OK) return st;
    }
    if (!known_act(act)) return DC_ERR_ARG;
    if (!w) return DC_ERR_NULL;
    if (misaligned(w) || misaligned(bias)) return DC_ERR_ALIGN;
    GateArgs g;
    std::memset(&g, 0, sizeof(g));
    if ((st = drop_args(drop, *vh, vh->C, &g.drop)) != DC_OK) return st;
    LinearArgs& a = g.l;
    const bool f32 = vx->dtype == DC_F32;
    Together t;
    t.add(vx, x);
    t.add(vh, h);
    t.add(vz, zg);
    a.cl = channel_rows(*vx);
    if ((st = slots_for(*vx, t.flat(), a.cl, f32 ? 4 : 2, &a.s)) != DC_OK) return st;
    if ((st = block_limits(2 * int64_t(vh->C), vx->C, a.s)) != DC_OK) return st;
    a.a.p = static_cast<const char*>(w);
    a.a.ld = vx->C;
    a.a.end = 2 * int64_t(vh->C) * vx->C;
    a.b = pixel_operand(*vx, x);
    a.a.rows = a.rows = vh->C;
    a.a.red = a.b.red = vx->C;
    a.direct = direct_pixels(*vx, x, a.cl, a.s.len) && vx->C % (f32 ? 4 : 8) == 0;
    a.bias = bias;
    a.res.dt = a.h.dt = -1;
    a.z = device_view(vz, zg);
    g.zu = device_view(vz, zu);
    a.out = device_view(vh, h);
    a.qm = map_of(*vh, vh->C);
    a.act = act_code(act, vh->dtype == DC_F32);
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launched(gate_few(g, false, f32) ? launch_gate_few(g, false, f32, s) : launch_gate_fwd(g, f32, s));
}

dc_status dc_gate_bwd_data(const dc_view* vdy, const void* dy, const void* w, int32_t act, const dc_drop* drop,
                           const dc_view* vz, const void* zg, const void* zu, const dc_view* vh, void* h,
                           const dc_view* vdz, void* dz, void* stream) {
    if (!vdy || !vz || !vdz) return DC_ERR_NULL;
    dc_status st = check_tensor(vdy, dy, READ, false, *vdy, vdy->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vz, zg, READ, true, *vdy, vz->C)) != DC_OK) return st;
    if ((st = check_tensor(vz, zu, READ, true, *vdy, vz->C)) != DC_OK) return st;
    if (vz->C > kMaxChannels / 2) return DC_ERR_TOO_LARGE;
    if ((st = check_tensor(vdz, dz, WRITE, false, *vdy, 2 * vz->C)) != DC_OK) return st;
    if (h && (st = check_tensor(vh, h, WRITE, false, *vdy, vz->C)) != DC_OK) return st;
    if (!known_act(act)) return DC_ERR_ARG;
    if (!w) return DC_ERR_NULL;
    if (misaligned(w)) return DC_ERR_ALIGN;
    GateArgs g;
    std::memset(&g, 0, sizeof(g));
    if ((st = drop_args(drop, *vz, vz->C, &g.drop)) != DC_OK) return st;
    LinearArgs& a = g.l;
    const bool f32 = vdy->dtype == DC_F32;
    Together t;
    t.add(vdy, dy);
    t.add(vdz, dz);
    t.add(vz, zg);
    t.add(vh, h);
    a.cl = channel_rows(*vdy);
    if ((st = slots_for(*vdy, t.flat(), a.cl, f32 ? 4 : 2, &a.s)) != DC_OK) return st;
    if ((st = block_limits(vdy->C, vz->C, a.s)) != DC_OK) return st;
    a.a.p = static_cast<const char*>(w);
    a.a.ld = vz->C;
    a.a.end = int64_t(vdy->C) * vz->C;
    a.b = pixel_operand(*vdy, dy);
    a.a.rows = a.rows = vz->C;
    a.a.red = a.b.red = vdy->C;
    a.direct = direct_pixels(*vdy, dy, a.cl, a.s.len) && vz->C % (f32 ? 4 : 8) == 0;
    a.res.dt = -1;
    a.z = device_view(vz, zg);
    g.zu = device_view(vz, zu);
    a.h = device_view(vh, h);
    a.out = device_view(vdz, dz);
    a.qm = map_of(*vz, vz->C);
    a.act = act_code(act, vdz->dtype == DC_F32 || (h && vh->dtype == DC_F32));
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launched(gate_few(g, true, f32) ? launch_gate_few(g, true, f32, s) : launch_gate_bwd(g, f32, s));
}

dc_status dc_join_fwd(const dc_view* vy, const void* y, const dc_norm* post, const float* scale, const float* gate,
                      const dc_drop* drop, const dc_view* vx, const void* x, const dc_norm* pre, const dc_view* vo, void* o,
                      const dc_view* vu, void* u, float* stat, void* ckpt, void* stream) {
    if (!vy) return DC_ERR_NULL;
    dc_status st = check_tensor(vy, y, READ, false, *vy, vy->C);
    if (st != DC_OK) return st;
    if (x && (st = check_tensor(vx, x, READ, false, *vy, vy->C)) != DC_OK) return st;
    if ((st = check_tensor(vo, o, WRITE, false, *vy, vy->C)) != DC_OK) return st;
    JoinArgs a;
    std::memset(&a, 0, sizeof(a));
    if ((st = join_norm(post, &a.post)) != DC_OK) return st;
    if ((st = join_norm(pre, &a.pre)) != DC_OK) return st;
    if (a.pre.kind && (st = check_tensor(vu, u, WRITE, false, *vy, vy->C)) != DC_OK) return st;
    if (!a.pre.kind && u) return DC_ERR_ARG;
    if (misaligned(scale) || misaligned(gate) || misaligned(stat) || misaligned(ckpt)) return DC_ERR_ALIGN;
    if ((st = drop_args(drop, *vy, vy->C, &a.drop)) != DC_OK) return st;
    Together t;
    t.add(vy, y);
    t.add(vx, x);
    t.add(vo, o);
    t.add(vu, u);
    a.y = device_view(vy, y);
    a.x = device_view(vx, x);
    a.o = device_view(vo, o);
    a.u = device_view(vu, u);
    a.q = static_cast<char*>(ckpt);
    a.qm = map_of(*vy, vy->C);
    a.px = pixels_for(*vy, t.flat());
    a.scale = scale;
    a.gate = gate;
    a.stat = stat;
    a.C = vy->C;
    a.cl = t.rows();
    join_plan(a, false);
    (void)hipGetLastError();
    return launched(launch_join_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t dc_join_bwd_workspace_bytes(const dc_view* vdy, int32_t gate) {
    if (check_view(vdy, READ, false) != DC_OK) return 0;
    return join_bwd_part_bytes(vdy->N, vdy->H * vdy->W, vdy->C, gate != 0);
}

dc_status dc_join_bwd(const dc_view* vdu, const void* du, const dc_view* vdo, const void* d_o, const dc_view* vy, const void* y,
                      const dc_view* vx, const void* x, const dc_view* vo, const void* o, const float* stat, const dc_norm* post, const float* scale,
                      const float* gate, const dc_drop* drop, const dc_norm* pre, const dc_view* vdx, void* dx,
                      const dc_view* vdy, void* dy, const dc_join_grads* grads, int32_t accumulate, void* workspace,
                      size_t workspace_bytes, void* stream) {
    if (!vdy) return DC_ERR_NULL;
    dc_status st = check_tensor(vdy, dy, WRITE, false, *vdy, vdy->C);
    if (st != DC_OK) return st;
    if (!du && !d_o) return DC_ERR_NULL;
    if (du && (st = check_tensor(vdu, du, READ, false, *vdy, vdy->C)) != DC_OK) return st;
    if (d_o && (st = check_tensor(vdo, d_o, READ, false, *vdy, vdy->C)) != DC_OK) return st;
    if (dx && (st = check_tensor(vdx, dx, WRITE, false, *vdy, vdy->C)) != DC_OK) return st;
    JoinArgs a;
    std::memset(&a, 0, sizeof(a));
    if ((st = join_norm(post, &a.post)) != DC_OK) return st;
    if ((st = join_norm(du ? pre : nullptr, &a.pre)) != DC_OK) return st;    // without du none: its parameters are not read
    if (du && !a.pre.kind) return DC_ERR_ARG;
    static const dc_join_grads none = {};
    const dc_join_grads& g = grads ? *grads : none;
    // parameters that the call has not: nothing to write a gradient for
    if ((g.gate && !gate) || (!du && (g.gamma_pre || g.beta_pre)) || (!a.post.kind && (g.gamma_post || g.beta_post)))
        return DC_ERR_ARG;
    if (accumulate != 0 && accumulate != 1) return DC_ERR_ARG;
    const bool form_o = du && !o, need_y = a.post.kind || g.scale || g.gate || form_o;
    if (need_y && (st = check_tensor(vy, y, READ, true, *vdy, vdy->C)) != DC_OK) return st;
    if (du && o && (st = check_tensor(vo, o, READ, true, *vdy, vdy->C)) != DC_OK) return st;
    if (form_o && x && (st = check_tensor(vx, x, READ, true, *vdy, vdy->C)) != DC_OK) return st;
    if ((du || a.post.kind) && !stat) return DC_ERR_NULL;
    if (misaligned(stat) || misaligned(scale) || misaligned(gate) || misaligned(g.scale) || misaligned(g.gate) ||
        misaligned(g.gamma_post) || misaligned(g.beta_post) || misaligned(g.gamma_pre) || misaligned(g.beta_pre))
        return DC_ERR_ALIGN;
    if ((st = drop_args(drop, *vdy, vdy->C, &a.drop)) != DC_OK) return st;
    if (g.scale || g.gate || g.gamma_post || g.beta_post || g.gamma_pre || g.beta_pre) {
        if (!workspace || workspace_bytes < dc_join_bwd_workspace_bytes(vdy, gate != nullptr)) return DC_ERR_WORKSPACE;
        if (misaligned(workspace)) return DC_ERR_ALIGN;
    }
    Together t;
    t.add(vdu, du);
    t.add(vdo, d_o);
    if (need_y) t.add(vy, y);
    if (du && o) t.add(vo, o);
    if (form_o) t.add(vx, x);
    t.add(vdx, dx);
    t.add(vdy, dy);
    a.du = device_view(vdu, du);
    a.dr = device_view(vdo, d_o);
    a.y = device_view(need_y ? vy : nullptr, y);
    a.form_o = form_o;
    a.x = form_o ? device_view(vx, x) : device_view(du ? vo : nullptr, o);
    a.dx = device_view(vdx, dx);
    a.dy = device_view(vdy, dy);
    a.qm = map_of(*vdy, vdy->C);
    a.px = pixels_for(*vdy, t.flat());
    a.scale = scale;
    a.gate = gate;
    a.stat = const_cast<float*>(stat);
    a.C = vdy->C;
    a.cl = t.rows();
    a.dscale = g.scale;
    a.dgate = g.gate;
    a.dgpost = g.gamma_post;
    a.dbpost = g.beta_post;
    a.dgpre = g.gamma_pre;
    a.dbpre = g.beta_pre;
    a.part = static_cast<float*>(workspace);
    a.accumulate = accumulate;
    join_plan(a, true);
    (void)hipGetLastError();
    return launched(launch_join_bwd(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
