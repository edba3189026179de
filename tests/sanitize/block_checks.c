/* Host code of a gated residual block's operators over seeded random views: every valid call
 * plans and launches within the limits that the stub HIP runtime checks, every broken one is
 * refused without a launch.  Run under ASan and UBSan. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include "dc.h"

extern long stub_launches;
static uint64_t state = 88172645463325252ull;
static uint64_t rnd(void) { state ^= state << 13; state ^= state >> 7; state ^= state << 17; return state; }
static int pick(int lo, int hi) { return lo + (int)(rnd() % (uint64_t)(hi - lo + 1)); }
static int spread(int hi) { int b = pick(0, 30), v = 1 << b; v += (int)(rnd() % (uint64_t)v); return v > hi ? pick(1, hi) : v; }

#define CHECK(c) do { if (!(c)) { fprintf(stderr, "line %d: %s\n", __LINE__, #c); abort(); } } while (0)

/* dense, padded, or rows of channels */
static dc_view view(int N, int C, int H, int W, int dtype)
{
    dc_view v = {N, C, H, W, 0, 0, 0, dtype};
    if (W == 1 && pick(0, 1)) {
        v.sc = 1; v.sh = C; v.sn = (int64_t)C * H;
    } else {
        const int pad = pick(0, 2) ? 0 : pick(1, 5);
        v.sh = W + pad; v.sc = v.sh * (H + pad); v.sn = v.sc * C + pad;
    }
    return v;
}

int main(void)
{
    /* addresses that are only looked at */
    char* const A = (char*)0x100000;
    float* const F = (float*)0x200000;
    long calls = 0;
    for (int i = 0; i < 20000; ++i) {
        const int rows = pick(0, 3) == 0;
        const int N = rows ? spread(1 << 16) : spread(64), H = rows ? spread(4096) : spread(2048), W = rows ? 1 : spread(2048);
        const int C = spread(pick(0, 9) ? 4096 : 20000), K = spread(4096);
        if ((double)N * H * W > 1.5e9) continue;
        const int f = pick(0, 1), act = pick(0, 3);
        dc_view x = view(N, C, H, W, f), h = view(N, K, H, W, pick(0, 1)), z = view(N, K, H, W, pick(0, 1));
        dc_view zq = {N, K, H, W, 0, 0, 0, DC_Q8}, q = {N, C, H, W, 0, 0, 0, DC_Q8};
        dc_view y = view(N, C, H, W, pick(0, 1)), o = view(N, C, H, W, pick(0, 1)), u = view(N, C, H, W, pick(0, 1));
        dc_view dz = view(N, 2 * K, H, W, pick(0, 1));
        dc_drop d = {pick(0, 999) / 1000.0, rnd(), rnd(), pick(0, 1) ? (uint64_t*)A : NULL, pick(0, 5), pick(0, 99), pick(0, 99), 0, 0, 0, 0};
        if (N % 4 == 0 && pick(0, 1)) d.P = pick(0, 1) ? 2 : 4, d.Q = d.P == 2 ? 2 : 1;
        dc_drop* dp = pick(0, 1) ? &d : NULL;
        long before = stub_launches;
        dc_status st = dc_dropout(&d, &x, A, &y, A, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK)); before = stub_launches;
        const dc_view* kept = pick(0, 1) ? &z : &zq;
        void* keep = pick(0, 2) ? A : NULL;
        st = dc_gate_fwd(&x, A, A, pick(0, 1) ? F : NULL, act, dp, kept, keep, keep, &h, A, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK)); before = stub_launches;
        st = dc_gate_bwd_data(&x, A, A, act, dp, kept, A, A, &h, pick(0, 1) ? A : NULL, &dz, A, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK)); before = stub_launches;
        dc_norm post = {pick(0, 2), 1e-5f, F, NULL}, pre = {pick(0, 2), 1e-5f, NULL, F};
        float* gate = pick(0, 1) ? F : NULL;
        st = dc_join_fwd(&y, A, &post, F, gate, dp, &x, pick(0, 1) ? A : NULL, &pre, &o, A, &u, pre.kind ? A : NULL, F, pick(0, 1) ? A : NULL, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK)); before = stub_launches;
        const size_t need = dc_join_bwd_workspace_bytes(&y, gate != NULL);
        CHECK(need > 0 && need % 16 == 0);
        dc_join_grads g = {F, gate, post.kind ? F : NULL, NULL, pre.kind ? F : NULL, NULL};
        const int grads = pick(0, 1);
        void* whole = pick(0, 1) ? A : NULL;
        st = dc_join_bwd(&u, pre.kind ? A : NULL, &o, A, pick(0, 1) ? &y : &q, A, pick(0, 1) ? &x : &q, A, &o, whole, F, &post, F, gate, dp, &pre,
                         &x, A, &y, A, grads ? &g : NULL, pick(0, 1), A, need, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK ? 1 + grads : 0)); before = stub_launches;
        if (grads)
            CHECK(dc_join_bwd(NULL, NULL, &o, A, &y, A, NULL, NULL, NULL, NULL, F, &post, F, gate, NULL, NULL, NULL, NULL, &y, A, &g, 0, A, need - 1,
                              NULL) != DC_OK);
        /* broken in one respect: no launch */
        dc_view b = x;
        switch (pick(0, 5)) {
            case 0: b.N = 0; break;
            case 1: b.dtype = pick(2, 9); break;
            case 2: b.C = -C; break;
            case 3: b.sc = -1 - (int64_t)pick(0, 99); if (C == 1) b.H = 0; break;
            case 4: b.W = INT32_MAX; b.H = INT32_MAX; break;
            default: b.sn = INT64_MAX / 2; if (N < 4) b.N = -1; break;
        }
        CHECK(dc_dropout(&d, &b, A, &y, A, NULL) != DC_OK && dc_gate_fwd(&b, A, A, NULL, 0, NULL, NULL, NULL, NULL, &h, A, NULL) != DC_OK);
        CHECK(dc_join_fwd(&b, A, NULL, NULL, NULL, NULL, NULL, NULL, NULL, &o, A, NULL, NULL, NULL, NULL, NULL) != DC_OK);
        CHECK(dc_gate_bwd_data(&b, A, A, 0, NULL, &z, A, A, NULL, NULL, &dz, A, NULL) != DC_OK && dc_join_bwd_workspace_bytes(&b, 1) == 0);
        d.p = pick(0, 2) ? 1.0 : NAN;
        CHECK(dc_dropout(&d, &x, A, &y, A, NULL) == DC_ERR_ARG);
        CHECK(stub_launches == before);
        ++calls;
    }
    printf("%ld rounds, %ld launches\n", calls, stub_launches);
    return 0;
}
