// The host side of the attention calls' schedule, for tests/test_attn_schedule.py: no GPU is used.
//   schedule shares                                              check first_unit and cta_of
//   schedule decode BATCH HEADS KV_HEADS D MAX_KV PREFIX SMS [UNSPLIT]  print "unsplit joined ctas bytes limit_ns"
//   schedule prefill HEADS KV_HEADS D SMS POS0 N [POS0 N ...]    print "unsplit joined groups units n_split"
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "attn_walk.cuh"

using namespace hs;
using namespace hs::attn;

// every CTA's run against its definition, units * c / ctas in 64 bits, and the CTA of the units at its ends
static int shares()
{
    const int edge = 1 << 22;
    const int sizes[] = {1, 2, 151, 320, 12345, edge - 1, edge, edge + 1, 2 * edge + 77, 8400000, 33600001,
                         INT_MAX / 320, INT_MAX / 320 + 1, 1 << 30, INT_MAX - 1, INT_MAX};
    const int counts[] = {1, 2, 3, 151, 152, 303, 304, 319, 320};
    long checks = 0;
    for (int units : sizes)
        for (int ctas : counts) {
            if (ctas > units)
                continue;
            for (int c = 0; c <= ctas; ++c) {
                const int64_t want = (int64_t)units * c / ctas;
                if (first_unit(units, ctas, c) != want)
                    return std::printf("first_unit %d %d %d\n", units, ctas, c), 1;
                if (c == ctas)
                    break;
                const int64_t end = (int64_t)units * (c + 1) / ctas;
                const int64_t at[] = {want, want + (end - want) / 2, end - 1};
                for (int64_t u : at)
                    if (cta_of(units, ctas, (int)u) != c)
                        return std::printf("cta_of %d %d %lld: %d\n", units, ctas, (long long)u,
                                           cta_of(units, ctas, (int)u)), 1;
                checks += 4;
            }
        }
    std::printf("%ld\n", checks);
    return 0;
}

int main(int argc, char **argv)
{
    if (argc == 2 && !std::strcmp(argv[1], "shares"))
        return shares();
    if ((argc == 9 || argc == 10) && !std::strcmp(argv[1], "decode")) {
        int a[7];
        for (int i = 0; i < 7; ++i)
            a[i] = std::atoi(argv[2 + i]);
        AttnParams p;
        std::memset(&p, 0, sizeof p);
        p.batch = a[0];
        p.n_heads = a[1];
        p.n_kv = a[2];
        p.group = a[1] / a[2];
        p.by_group.set(p.group);
        p.by_kv.set(p.n_kv);
        p.max_kv = a[4];
        p.prefix_len = a[5];
        p.unsplit = argc == 10 ? std::atoi(argv[9]) : 0;
        const int64_t bytes = plan_attn_decode(p, a[3], a[6]);
        std::printf("%d %d %d %lld %llu\n", p.unsplit, p.joined, p.ctas, (long long)bytes,
                    (unsigned long long)p.limit_ns);
        return 0;
    }
    if (argc >= 8 && argc % 2 == 0 && !std::strcmp(argv[1], "prefill")) {
        static PrefillPlan plan;
        AttnParams p;
        std::memset(&p, 0, sizeof p);
        p.batch = (argc - 6) / 2;
        p.n_heads = std::atoi(argv[2]);
        p.n_kv = std::atoi(argv[3]);
        p.group = p.n_heads / p.n_kv;
        p.by_group.set(p.group);
        p.by_kv.set(p.n_kv);
        for (int b = 0; b < p.batch; ++b) {
            plan.req[b].pos0 = std::atoi(argv[6 + 2 * b]);
            plan.req[b].n = std::atoi(argv[7 + 2 * b]);
        }
        plan_attn_prefill(p, plan, std::atoi(argv[4]), std::atoi(argv[5]));
        std::printf("%d %d %d %d %d\n", p.unsplit, p.joined, p.groups, p.units, p.n_split);
        return 0;
    }
    return 2;
}
