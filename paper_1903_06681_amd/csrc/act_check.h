// What the entry points of the operators between two convolutions share: validation of
// views, device views, pixel numbering.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "act_kernels.h"
#include "dc.h"

namespace dc {

static const int64_t kMaxPixels = (int64_t(1) << 31) - (int64_t(1) << 16);   // a block past the end still counts in 32 bits
static const int32_t kMaxChannels = 1 << 20;
static const int64_t kMaxBlocks = int64_t(1) << 22;   // of 128 x 128; threads are counted in 32 bits

// Results of the products from this size on are stored non-temporally: they leave the
// caches to the operands.  Outputs that change from call to call: 32 to 128 channels on
// 512 x 512 pixels (fp32, 134 MB) 46 us against 55, 64 to 256 on 100352 with z in 8 bits
// (51 MB) 29 against 35 and its gradient 34 against 42; at 6 MB 13.1 against 12.7.
static const int64_t kStreamed = int64_t(32) << 20;

inline bool misaligned(const void* p, size_t to = 16) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
inline dc_status launched(hipError_t e) { return e == hipSuccess ? DC_OK : DC_ERR_HIP; }
inline int64_t pixels_of(const dc_view& v) { return int64_t(v.N) * v.H * v.W; }
inline int esize(const dc_view& v) { return v.dtype == DC_F32 ? 4 : v.dtype == DC_BF16 ? 2 : 1; }

enum Use { READ, WRITE };

inline dc_status check_view(const dc_view* v, Use use, bool q8) {
    if (!v) return DC_ERR_NULL;
    if (v->N < 1 || v->C < 1 || v->H < 1 || v->W < 1) return DC_ERR_SHAPE;
    if (v->dtype != DC_F32 && v->dtype != DC_BF16 && !(q8 && v->dtype == DC_Q8)) return DC_ERR_DTYPE;
    if (v->C > kMaxChannels || double(v->N) * v->H * v->W > double(kMaxPixels)) return DC_ERR_TOO_LARGE;
    if (v->dtype == DC_Q8) return DC_OK;
    struct Dim { int64_t n, s; } d[4] = {{v->W, 1}, {v->H, v->sh}, {v->C, v->sc}, {v->N, v->sn}};
    double end = 0;
    for (const Dim& k : d) {
        if (k.n > 1 && k.s < 0) return DC_ERR_SHAPE;
        if (k.n > 1) end += double(k.n - 1) * double(k.s);
    }
    if (end > 4e18) return DC_ERR_TOO_LARGE;
    if (use == WRITE) {        // nested: a dimension's step lies past the last element of those inside it
        std::sort(d, d + 4, [](const Dim& a, const Dim& b) { return a.s < b.s || (a.s == b.s && a.n < b.n); });
        int64_t next = 1;
        for (const Dim& k : d) {
            if (k.n == 1) continue;
            if (k.s < next) return DC_ERR_SHAPE;
            next += (k.n - 1) * k.s;
        }
    }
    return DC_OK;
}

// A view that must hold N, C, H, W of another's pixels, with its pointer.
inline dc_status check_tensor(const dc_view* v, const void* p, Use use, bool q8, const dc_view& like, int32_t C) {
    dc_status st = check_view(v, use, q8);
    if (st != DC_OK) return st;
    if (v->N != like.N || v->H != like.H || v->W != like.W || v->C != C) return DC_ERR_SHAPE;
    if (!p) return DC_ERR_NULL;
    if (misaligned(p, v->dtype == DC_Q8 ? 16 : size_t(esize(*v)))) return DC_ERR_ALIGN;
    return DC_OK;
}

inline View device_view(const dc_view* v, const void* p) {
    View r{};
    r.dt = -1;
    if (!v || !p) return r;
    r.p = static_cast<char*>(const_cast<void*>(p));
    r.sn = v->N > 1 ? v->sn : 0;
    r.sc = v->sc;
    r.sh = v->H > 1 ? v->sh : 0;
    r.dt = v->dtype;
    r.big = int64_t(pixels_of(*v)) * v->C * esize(*v) >= kStreamed;
    return r;
}

// The tensors of a call whose pixels are numbered alike.
struct Together {
    const dc_view* v[6];
    const void* p[6];
    int n = 0;
    void add(const dc_view* view, const void* ptr) {
        if (!view || !ptr || view->dtype == DC_Q8) return;
        v[n] = view;
        p[n++] = ptr;
    }
    // rows follow each other without a gap in all of them: an image is one row
    bool flat() const {
        for (int i = 0; i < n; ++i)
            if (v[i]->H > 1 && v[i]->sh != v[i]->W) return false;
        return true;
    }
    // rows of channels
    bool rows() const {
        for (int i = 0; i < n; ++i)
            if (v[i]->W != 1 || v[i]->sc != 1) return false;
        return n > 0;
    }
};

inline Pixels pixels_for(const dc_view& v, bool flat) {
    Pixels x{};
    x.HW = v.H * v.W;
    x.M = v.N * x.HW;
    x.len = flat ? x.HW : v.W;
    x.dHW = fast_div(uint32_t(x.HW));
    x.dlen = fast_div(uint32_t(x.len));
    return x;
}

inline Q8Map map_of(const dc_view& v, int32_t C) { return q8_map(v.N, C, int64_t(v.H) * v.W); }

// ---- products

inline bool channel_rows(const dc_view& v) { return v.W == 1 && v.sc == 1; }

inline dc_status slots_for(const dc_view& v, bool flat, bool cl, int es, Slots* s) {
    const int64_t hw = int64_t(v.H) * v.W;
    s->per = cl ? 1 : 16 / es;
    s->len = cl ? 1 : int32_t(flat ? hw : v.W);
    s->cpr = (s->len + s->per - 1) / s->per;
    const int64_t sample = hw / s->len * s->cpr;
    if (double(sample) * v.N * s->per > double(kMaxPixels)) return DC_ERR_TOO_LARGE;
    s->chunks = int32_t(sample * v.N);
    s->dsample = fast_div(uint32_t(sample));
    s->dcpr = fast_div(uint32_t(s->cpr));
    return DC_OK;
}

inline Operand pixel_operand(const dc_view& v, const void* p) {
    Operand o{};
    const View d = device_view(&v, p);
    o.p = d.p;
    o.sn = d.sn;
    o.sc = d.sc;
    o.sh = d.sh;
    o.end = (v.N - 1) * d.sn + (v.C - 1) * d.sc + (v.H - 1) * d.sh + v.W;
    return o;
}

// Whether every chunk that holds elements of a pixel operand is an aligned 16-byte vector
// whose elements lie between the view's first and last: rows start on 16-byte
// boundaries, and either end there or are not the view's last.
inline bool direct_pixels(const dc_view& v, const void* p, bool cl, int64_t row) {
    const int e = 16 / esize(v);
    if (misaligned(p)) return false;
    if ((v.N > 1 && v.sn % e) || (v.H > 1 && v.sh % e && row == v.W)) return false;
    if (cl) return v.C % e == 0 && (v.H == 1 || v.sh % e == 0);
    return v.sc % e == 0 && row % e == 0;
}

inline dc_status block_limits(int64_t K, int64_t C, const Slots& s) {
    if (K * C > (int64_t(1) << 31) - 1) return DC_ERR_TOO_LARGE;
    const int64_t slots = int64_t(s.chunks) * s.per, rows = std::max(K, C);
    return (rows + 127) / 128 * ((slots + 127) / 128) > kMaxBlocks ? DC_ERR_TOO_LARGE : DC_OK;
}

inline bool known_act(int32_t act) { return act >= DC_ACT_NONE && act <= DC_ACT_SILU; }

}  // namespace dc
