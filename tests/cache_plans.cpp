// How attention calls on caches are launched.  Reads a problem a line, B Hq Hk Lq Lp Lk d W causal dtype store (Lp 0: no prefix), and prints
// whether an item's workgroups take the prefix too, blocks of 16 rows of a workgroup, parts of the own keys' walk and of the prefix's, whether the longest walks come first,
// workgroups of either side, and the estimated cost.
#include "ska_cache_plan.h"

#include <cstdio>

int main()
{
    CaProblem p;
    while (std::scanf("%d %d %d %d %d %d %d %d %d %d %d", &p.B, &p.Hq, &p.Hk, &p.Lq, &p.Lp, &p.Lk, &p.d, &p.W, &p.causal, &p.dtype, &p.store) == 11) {
        const CaPlan l = ca_plan(p);
        CaPlan x;
        std::printf("%d %d %d %d %d %ld %ld %.1f %.1f\n", l.both, l.nq, l.own.parts, l.front.units ? l.front.parts : 0, l.own.order == CA_LAST_FIRST, l.own.units * l.own.parts,
                    l.front.units * l.front.parts, ca_plan(p, 2, x), ca_plan(p, 4, x));
    }
    return 0;
}
