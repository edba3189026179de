// C entry points of norm, pointwise products and 8-bit checkpoints: validation,
// dispatch.  No allocation, no state, no synchronisation.
#include <hip/hip_runtime.h>

#include "act_check.h"

namespace dc {

static dc_status wgrad_args(const dc_view* vx, const dc_view* vdy, const void* x, const void* dy, LinWgradArgs* a) {
    std::memset(a, 0, sizeof(*a));
    Together t;
    t.add(vx, x);
    t.add(vdy, dy);
    const bool f32 = vx->dtype == DC_F32;
    a->cl = channel_rows(*vx) && channel_rows(*vdy);
    dc_status st = slots_for(*vx, t.flat(), a->cl, f32 ? 4 : 2, &a->s);
    if (st != DC_OK) return st;
    a->K = vdy->C;
    a->C = vx->C;
    if ((st = block_limits(a->K, a->C, a->s)) != DC_OK) return st;
    a->a = pixel_operand(*vdy, dy);
    a->b = pixel_operand(*vx, x);
    a->a.rows = a->K;
    a->b.rows = a->C;
    a->direct = direct_pixels(*vx, x, a->cl, a->s.len) && direct_pixels(*vdy, dy, a->cl, a->s.len);
    linear_wgrad_plan(*a, f32);
    return DC_OK;
}

// the views of a weight gradient; *need = workspace bytes
static dc_status wgrad_views(const dc_view* vx, const dc_view* vdy) {
    dc_status st = check_view(vx, READ, false);
    if (st != DC_OK) return st;
    if ((st = check_view(vdy, READ, false)) != DC_OK) return st;
    if (vx->N != vdy->N || vx->H != vdy->H || vx->W != vdy->W) return DC_ERR_SHAPE;
    return vx->dtype == vdy->dtype ? DC_OK : DC_ERR_DTYPE;
}

}  // namespace dc

using namespace dc;

extern "C" {

int64_t dc_ckpt_bytes(const dc_view* vq) {
    if (check_view(vq, READ, true) != DC_OK) return -1;
    const int64_t blocks = int64_t((vq->C + 31) / 32) * pixels_of(*vq);
    return (blocks * 33 + 15) / 16 * 16;
}

static dc_status ckpt_common(const dc_view* vx, const void* x, const void* q, int32_t act, bool save, void* stream) {
    if (!q) return DC_ERR_NULL;
    if (misaligned(q)) return DC_ERR_ALIGN;
    CkptArgs a{};
    Together t;
    t.add(vx, x);
    a.x = device_view(vx, x);
    a.q = static_cast<char*>(const_cast<void*>(q));
    a.qm = map_of(*vx, vx->C);
    a.px = pixels_for(*vx, t.flat());
    a.C = vx->C;
    a.act = act;
    a.cl = t.rows();
    (void)hipGetLastError();
    return launched(launch_ckpt(a, save, static_cast<hipStream_t>(stream)));
}

dc_status dc_ckpt_save(const dc_view* vx, const void* x, void* q, void* stream) {
    const dc_status st = vx ? check_tensor(vx, x, READ, false, *vx, vx->C) : DC_ERR_NULL;
    return st != DC_OK ? st : ckpt_common(vx, x, q, DC_ACT_NONE, true, stream);
}

dc_status dc_ckpt_load(const dc_view* vq, const void* q, int32_t act, const dc_view* vy, void* y, void* stream) {
    dc_status st = check_view(vq, READ, true);
    if (st != DC_OK) return st;
    if (vq->dtype != DC_Q8) return DC_ERR_DTYPE;
    if (!known_act(act)) return DC_ERR_ARG;
    if ((st = check_tensor(vy, y, WRITE, false, *vq, vq->C)) != DC_OK) return st;
    return ckpt_common(vy, y, q, act, false, stream);
}

dc_status dc_norm_fwd(const dc_view* vx, const void* x, const float* gamma, const float* beta, float eps,
                      const dc_view* vu, void* u, float* stat, void* ckpt, void* stream) {
    if (!vx) return DC_ERR_NULL;
    dc_status st = check_tensor(vx, x, READ, false, *vx, vx->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vu, u, WRITE, false, *vx, vx->C)) != DC_OK) return st;
    if (!(eps >= 0) || std::isinf(eps)) return DC_ERR_ARG;
    if (misaligned(gamma) || misaligned(beta) || misaligned(stat) || misaligned(ckpt)) return DC_ERR_ALIGN;
    NormArgs a{};
    Together t;
    t.add(vx, x);
    t.add(vu, u);
    a.x = device_view(vx, x);
    a.u = device_view(vu, u);
    a.q = static_cast<char*>(ckpt);
    a.qm = map_of(*vx, vx->C);
    a.px = pixels_for(*vx, t.flat());
    a.gamma = gamma;
    a.beta = beta;
    a.stat = stat;
    a.eps = eps;
    a.C = vx->C;
    a.cl = t.rows();
    norm_plan(a, false);
    (void)hipGetLastError();
    return launched(launch_norm_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t dc_norm_bwd_workspace_bytes(const dc_view* vdu) {
    if (check_view(vdu, READ, false) != DC_OK) return 0;
    return norm_bwd_part_bytes(int(pixels_of(*vdu)), vdu->C);
}

dc_status dc_norm_bwd(const dc_view* vdu, const void* du, const dc_view* vx, const void* x, const float* stat,
                      const float* gamma, const float* beta, const dc_view* vres, const void* res,
                      const dc_view* vu, void* u, const dc_view* vdx, void* dx, float* dgamma, float* dbeta,
                      int32_t accumulate, void* workspace, size_t workspace_bytes, void* stream) {
    if (!vdu) return DC_ERR_NULL;
    dc_status st = check_tensor(vdu, du, READ, false, *vdu, vdu->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vx, x, READ, true, *vdu, vdu->C)) != DC_OK) return st;
    if ((st = check_tensor(vdx, dx, WRITE, false, *vdu, vdu->C)) != DC_OK) return st;
    if (res && (st = check_tensor(vres, res, READ, false, *vdu, vdu->C)) != DC_OK) return st;
    if (u && (st = check_tensor(vu, u, WRITE, false, *vdu, vdu->C)) != DC_OK) return st;
    if (accumulate != 0 && accumulate != 1) return DC_ERR_ARG;
    if (!stat) return DC_ERR_NULL;
    if (misaligned(stat) || misaligned(gamma) || misaligned(beta) || misaligned(dgamma) || misaligned(dbeta))
        return DC_ERR_ALIGN;
    if (dgamma || dbeta) {
        if (!workspace || workspace_bytes < dc_norm_bwd_workspace_bytes(vdu)) return DC_ERR_WORKSPACE;
        if (misaligned(workspace)) return DC_ERR_ALIGN;
    }
    NormArgs a{};
    Together t;
    t.add(vdu, du);
    t.add(vx, x);
    t.add(vdx, dx);
    t.add(vres, res);
    t.add(vu, u);
    a.du = device_view(vdu, du);
    a.x = device_view(vx, x);
    a.res = device_view(vres, res);
    a.u = device_view(vu, u);
    a.dx = device_view(vdx, dx);
    a.q = vx->dtype == DC_Q8 ? a.x.p : nullptr;
    a.qm = map_of(*vdu, vdu->C);
    a.px = pixels_for(*vdu, t.flat());
    a.gamma = gamma;
    a.beta = beta;
    a.stat = const_cast<float*>(stat);
    a.dgamma = dgamma;
    a.dbeta = dbeta;
    a.part = static_cast<float*>(workspace);
    a.C = vdu->C;
    a.accumulate = accumulate;
    a.cl = t.rows();
    norm_plan(a, true);
    (void)hipGetLastError();
    return launched(launch_norm_bwd(a, static_cast<hipStream_t>(stream)));
}

dc_status dc_linear_fwd(const dc_view* vx, const void* x, const void* w, const float* bias, int32_t act,
                        const dc_view* vres, const void* res, const dc_view* vz, void* z,
                        const dc_view* vy, void* y, void* stream) {
    if (!vx || !vy) return DC_ERR_NULL;
    dc_status st = check_tensor(vx, x, READ, false, *vx, vx->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vy, y, WRITE, false, *vx, vy->C)) != DC_OK) return st;
    if (res && (st = check_tensor(vres, res, READ, false, *vx, vy->C)) != DC_OK) return st;
    if (z && (st = check_tensor(vz, z, WRITE, true, *vx, vy->C)) != DC_OK) return st;
    if (!known_act(act)) return DC_ERR_ARG;
    if (!w) return DC_ERR_NULL;
    if (misaligned(w) || misaligned(bias)) return DC_ERR_ALIGN;
    const bool f32 = vx->dtype == DC_F32;
    LinearArgs a;
    std::memset(&a, 0, sizeof(a));
    Together t;
    t.add(vx, x);
    t.add(vy, y);
    t.add(vres, res);
    t.add(vz, z);
    a.cl = channel_rows(*vx);
    if ((st = slots_for(*vx, t.flat(), a.cl, f32 ? 4 : 2, &a.s)) != DC_OK) return st;
    if ((st = block_limits(vy->C, vx->C, a.s)) != DC_OK) return st;
    a.a.p = static_cast<const char*>(w);
    a.a.ld = vx->C;
    a.a.end = int64_t(vy->C) * vx->C;
    a.b = pixel_operand(*vx, x);
    a.a.rows = a.rows = vy->C;
    a.a.red = a.b.red = vx->C;
    a.direct = direct_pixels(*vx, x, a.cl, a.s.len) && vx->C % (f32 ? 4 : 8) == 0;
    a.bias = bias;
    a.res = device_view(vres, res);
    a.z = device_view(vz, z);
    a.h.dt = -1;
    a.out = device_view(vy, y);
    a.qm = map_of(*vy, vy->C);
    a.act = act_code(act, vy->dtype == DC_F32);
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launched(linear_few(a, false, f32) ? launch_linear_few(a, false, f32, s) : launch_linear_fwd(a, f32, s));
}

dc_status dc_linear_bwd_data(const dc_view* vdy, const void* dy, const void* w, int32_t act,
                             const dc_view* vz, const void* z, const dc_view* vh, void* h,
                             const dc_view* vdx, void* dx, void* stream) {
    if (!vdy || !vdx) return DC_ERR_NULL;
    dc_status st = check_tensor(vdy, dy, READ, false, *vdy, vdy->C);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vdx, dx, WRITE, false, *vdy, vdx->C)) != DC_OK) return st;
    if (!known_act(act)) return DC_ERR_ARG;
    if (act == DC_ACT_NONE) {
        if (z || h) return DC_ERR_ARG;
    } else {
        if ((st = check_tensor(vz, z, READ, true, *vdy, vdx->C)) != DC_OK) return st;
        if (h && (st = check_tensor(vh, h, WRITE, false, *vdy, vdx->C)) != DC_OK) return st;
    }
    if (!w) return DC_ERR_NULL;
    if (misaligned(w)) return DC_ERR_ALIGN;
    const bool f32 = vdy->dtype == DC_F32;
    LinearArgs a;
    std::memset(&a, 0, sizeof(a));
    Together t;
    t.add(vdy, dy);
    t.add(vdx, dx);
    t.add(vz, z);
    t.add(vh, h);
    a.cl = channel_rows(*vdy);
    if ((st = slots_for(*vdy, t.flat(), a.cl, f32 ? 4 : 2, &a.s)) != DC_OK) return st;
    if ((st = block_limits(vdy->C, vdx->C, a.s)) != DC_OK) return st;
    a.a.p = static_cast<const char*>(w);
    a.a.ld = vdx->C;
    a.a.end = int64_t(vdy->C) * vdx->C;
    a.b = pixel_operand(*vdy, dy);
    a.a.rows = a.rows = vdx->C;
    a.a.red = a.b.red = vdy->C;
    a.direct = direct_pixels(*vdy, dy, a.cl, a.s.len) && vdx->C % (f32 ? 4 : 8) == 0;
    a.res.dt = -1;
    a.z = device_view(vz, z);
    a.h = device_view(vh, h);
    a.out = device_view(vdx, dx);
    a.qm = map_of(*vdx, vdx->C);
    a.act = act_code(act, vdx->dtype == DC_F32 || (h && vh->dtype == DC_F32));
    (void)hipGetLastError();
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launched(linear_few(a, true, f32) ? launch_linear_few(a, true, f32, s) : launch_linear_bwd(a, f32, s));
}

size_t dc_linear_bwd_filter_workspace_bytes(const dc_view* vx, const dc_view* vdy) {
    LinWgradArgs a;
    // the pointers do not matter to the plan, but count as present
    if (wgrad_views(vx, vdy) != DC_OK || wgrad_args(vx, vdy, vx, vdy, &a) != DC_OK) return 0;
    return linear_wgrad_part_bytes(a);
}

dc_status dc_linear_bwd_filter(const dc_view* vx, const void* x, const dc_view* vdy, const void* dy,
                               float* dw, float* db, int32_t accumulate, void* workspace,
                               size_t workspace_bytes, void* stream) {
    dc_status st = wgrad_views(vx, vdy);
    if (st != DC_OK) return st;
    if ((st = check_tensor(vx, x, READ, false, *vx, vx->C)) != DC_OK) return st;
    if ((st = check_tensor(vdy, dy, READ, false, *vx, vdy->C)) != DC_OK) return st;
    if (accumulate != 0 && accumulate != 1) return DC_ERR_ARG;
    if (!dw) return DC_ERR_NULL;
    if (misaligned(dw) || misaligned(db)) return DC_ERR_ALIGN;
    LinWgradArgs a;
    if ((st = wgrad_args(vx, vdy, x, dy, &a)) != DC_OK) return st;
    const size_t need = linear_wgrad_part_bytes(a);
    if (need && (!workspace || workspace_bytes < need)) return DC_ERR_WORKSPACE;
    if (need && misaligned(workspace)) return DC_ERR_ALIGN;
    a.dw = dw;
    a.db = db;
    a.part = static_cast<float*>(workspace);
    a.accumulate = accumulate;
    (void)hipGetLastError();
    return launched(launch_linear_wgrad(a, vx->dtype == DC_F32, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
