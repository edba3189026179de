/* Host code of the operators between two convolutions over seeded random views: every
 * valid call plans and launches within the limits that the stub HIP runtime checks, every
 * broken one is refused without a launch.  Run under ASan and UBSan. */
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
        const int N = rows ? spread(1 << 20) : spread(64), H = rows ? 1 : spread(2048), W = rows ? 1 : spread(2048);
        const int C = spread(4096), K = spread(4096);
        if ((double)N * H * W > 1.5e9) continue;
        const int f = pick(0, 1), act = pick(0, 3);
        dc_view x = view(N, C, H, W, f), y = view(N, K, H, W, pick(0, 1)), r = view(N, K, H, W, pick(0, 1));
        dc_view q = {N, K, H, W, 0, 0, 0, DC_Q8}, qc = {N, C, H, W, 0, 0, 0, DC_Q8};
        dc_view u = view(N, C, H, W, pick(0, 1)), dy = view(N, K, H, W, f);
        long before = stub_launches;
        dc_status st = dc_linear_fwd(&x, A, A, pick(0, 1) ? F : NULL, act, &r, pick(0, 1) ? A : NULL,
                                     pick(0, 1) ? &q : &r, pick(0, 1) ? A : NULL, &y, A, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK)); before = stub_launches;
        dc_view dx = view(N, C, H, W, pick(0, 1));
        st = dc_linear_bwd_data(&dy, A, A, act, &qc, act ? A : NULL, &u, act && pick(0, 1) ? A : NULL, &dx, A, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK)); before = stub_launches;
        const size_t need = dc_linear_bwd_filter_workspace_bytes(&x, &dy);
        st = dc_linear_bwd_filter(&x, A, &dy, A, F, pick(0, 1) ? F : NULL, pick(0, 1), A, need, NULL);
        CHECK(st == DC_OK || st == DC_ERR_TOO_LARGE);
        CHECK(stub_launches == before + (st == DC_OK ? need ? 2 : 1 : 0)); before = stub_launches;
        if (need) CHECK(dc_linear_bwd_filter(&x, A, &dy, A, F, NULL, 0, A, need - 1, NULL) == DC_ERR_WORKSPACE);
        CHECK(dc_norm_fwd(&x, A, F, F, 1e-5f, &u, A, F, pick(0, 1) ? A : NULL, NULL) == DC_OK);
        CHECK(stub_launches == before + 1); before = stub_launches;
        const size_t nw = dc_norm_bwd_workspace_bytes(&u);
        CHECK(nw > 0 && nw % 16 == 0);
        const int grads = pick(0, 1);
        CHECK(dc_norm_bwd(&u, A, pick(0, 1) ? &x : &qc, A, F, F, NULL, &dx, pick(0, 1) ? A : NULL, &u, pick(0, 1) ? A : NULL,
                          &dx, A, grads ? F : NULL, grads ? F : NULL, 0, A, nw, NULL) == DC_OK);
        CHECK(stub_launches == before + 1 + grads); before = stub_launches;
        CHECK(dc_ckpt_bytes(&qc) >= (int64_t)N * C * H * W);
        CHECK(dc_ckpt_save(&x, A, A, NULL) == DC_OK && dc_ckpt_load(&qc, A, act, &u, A, NULL) == DC_OK);
        CHECK(stub_launches == before + 2); before = stub_launches;
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
        CHECK(dc_ckpt_save(&b, A, A, NULL) != DC_OK && dc_linear_fwd(&b, A, A, NULL, 0, NULL, NULL, NULL, NULL, &y, A, NULL) != DC_OK);
        CHECK(dc_norm_fwd(&b, A, F, F, 1e-5f, &u, A, F, NULL, NULL) != DC_OK && dc_linear_bwd_filter_workspace_bytes(&b, &dy) == 0);
        CHECK(stub_launches == before);
        ++calls;
    }
    printf("%ld rounds, %ld launches\n", calls, stub_launches);
    return 0;
}
