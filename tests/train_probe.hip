// Host-side probe of how the masked attention cuts its work (test infrastructure): one
// call per line from stdin, its plan printed, with the library's own functions.
//
//   fwd <B> <T> <kT> <H> <Hk> <dh> <causal> -> fwd <groups> <splits> <workgroups> <workspace>
//   bwd <B> <T> <kT> <H> <Hk> <dh> <causal> -> bwd <parts over keys> <parts over queries>
//       <workgroups> <workspace beyond the sums>
#include "../paper_2607_08526_amd/csrc/internal.h"

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
        } else {
            return 1;
        }
    }
    return 0;
}
