// Prints what the channel products choose, a call a line of the input: dtype act x_is_8bit m k n ldg ldx ldw, and whether
// g, x and W start on 16-byte boundaries.  For each product (y, dx, dw): kernel, splits, contraction of a split, whether
// a copy of either operand is made, and the strides of the rows that the kernel reads.
#include "../paper_2204_03643_amd/csrc/tv_linear_plan.hpp"
#include <cstdio>

using namespace tvl;

static void print(const Plan &p, int64_t lda, int64_t ldb)
{
    printf("%d %d %d %d %d %lld %lld ", (int)p.c.kind, p.c.splits, p.c.k_per, (int)p.copy_a, (int)p.copy_b, (long long)lda, (long long)ldb);
}

int main()
{
    int dtype, act, x8, ag, ax, aw;
    long long m, k, n, ldg, ldx, ldw;
    while (scanf("%d %d %d %lld %lld %lld %lld %lld %lld %d %d %d", &dtype, &act, &x8, &m, &k, &n, &ldg, &ldx, &ldw, &ag, &ax, &aw) == 12) {
        const tv_linear_desc d = {m, k, n, ldx, ldw, n, ldg, dtype, act};
        char *const base = (char *)0x10000;
        const size_t off = elem_bytes(dtype);
        const bool dg = direct({base + (ag ? 0 : off), ldg, m, n}), dx = direct({base + (ax ? 0 : off), ldx, m, k}), dw = direct({base + (aw ? 0 : off), ldw, n, k});
        const FwdPlan f = fwd_plan(d, dx, dw);
        const BwdPlan b = bwd_plan(d, x8 != 0, dg, dx, dw, {true, true, true});
        const int64_t ldz = b.own_dz ? b.ldz : ldg;
        print(f.product, f.product.copy_a ? up(k, 8) : ldx, f.product.copy_b ? up(k, 8) : ldw);
        print(b.dx, ldz, b.dx.copy_b ? up(k, 8) : ldw);
        print(b.dw, ldz, x8 || b.dw.copy_b ? up(k, 8) : ldx);
        printf("%zu %zu\n", f.bytes, b.bytes);
    }
    return 0;
}
