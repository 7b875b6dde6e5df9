// Prints what runs a product in 8 bits, for tests on the CPU.  A line "rows width channels gated" from standard input gives a line
// "shape splits per steps": the tile shape (-1: the few-row kernels), the parts that K is cut into, the steps of a part, all steps.
// Rows start at multiples of 16 bytes.  Built host-only against the library, whose own estimate this is.
#include <stdio.h>

#include "nm_q8_internal.h"

int main()
{
    nm::Q8Linear p{};
    while (scanf("%d %d %d %d", &p.rows, &p.width, &p.channels, &p.gated) == 4) {
        p.ldq = (p.width + 15) / 16 * 16;
        p.outs = p.gated ? p.channels / 2 : p.channels;
        p.groups = (p.channels + 63) / 64;
        p.kblocks = (p.width + 127) / 128 * 2;
        const nm::Q8Plan plan = nm::q8_plan(p);
        if (plan.rows_bytes || (plan.splits > 1) != (plan.part_bytes > 0)) return 1;
        printf("%d %d %d %d\n", plan.shape, plan.splits, plan.per, p.kblocks / 2);
    }
    return 0;
}
