/* What the join's plan says of sizes: "N HW C rows gate" a line; pixels a wave, eights a lane,
 * workgroups and units of the backward pass, bytes of its workspace. */
#include <hip/hip_runtime.h>

#include <cstdio>

#include "join.h"

int main()
{
    static const float some = 0;
    int N, HW, C, rows, gate;
    while (std::scanf("%d %d %d %d %d", &N, &HW, &C, &rows, &gate) == 5) {
        dc::JoinArgs a{};
        a.px.M = N * HW;
        a.px.HW = HW;
        a.C = C;
        a.cl = rows;
        a.gate = gate ? &some : nullptr;
        dc::join_plan(a, true);
        std::printf("%d %d %d %d %zu\n", a.lpx, a.held, a.grid, a.units, dc::join_bwd_part_bytes(N, HW, C, gate));
    }
}
