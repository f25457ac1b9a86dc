// Host-side probe of how the masked attention cuts its work (test infrastructure): one
// call per line from stdin, its plan printed, with the library's own functions.
//
//   fwd <B> <T> <kT> <H> <Hk> <dh> <causal> -> fwd <groups> <splits> <workgroups> <workspace>
//   bwd <B> <T> <kT> <H> <Hk> <dh> <causal> -> bwd <parts over keys> <parts over queries>
//       <workgroups> <workspace beyond the sums>
//   work <B> <T> <kT> <H> <Hk> <dh> <causal> <parts> <blocks> <resident> -> work <fold> <group>,
//       then <part> <block> <unit> of every workgroup, in the order of their numbers
#include "../paper_2607_08526_amd/csrc/attn.h"

#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>

int main()
{
    using namespace qlk;
    std::string line, kind;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        SeqAttn s{};
        in >> kind >> s.B >> s.T >> s.KT >> s.H >> s.Hk >> s.dh >> s.causal;
        s.cus = current_cus();
        if (kind == "fwd") {
            const SeqAttnPlan p = seq_attn_plan(s);
            std::printf("fwd %d %d %lld %lld\n", p.groups, p.splits,
                        (long long)seq_attn_workgroups(s, p), (long long)seq_attn_bytes(s, p));
        } else if (kind == "bwd") {
            const SeqAttnGradPlan p = seq_attn_grad_plan(s, true);
            std::printf("bwd %d %d %lld %lld\n", p.qparts, p.kparts,
                        (long long)seq_attn_grad_workgroups(s, p),
                        (long long)seq_attn_grad_bytes(s, p));
        } else if (kind == "work") {
            int parts, blocks, resident;
            in >> parts >> blocks >> resident;
            order_work(s, (int64_t)parts * blocks, resident);
            const int grid = s.B * s.Hk * parts * blocks;
            std::printf("work %d %d", s.fold, s.group);
            for (int p = 0; p < grid; ++p) {
                const Work w = work_of(s, p, grid, parts, blocks);
                std::printf(" %d %d %d", w.part, w.blk, w.unit);
            }
            std::printf("\n");
        } else {
            return 1;
        }
    }
    return 0;
}
