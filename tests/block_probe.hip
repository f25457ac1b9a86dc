// Host-side probe of which kernels the operators of include/qlinear_block.h take
// (test infrastructure): one call per line from stdin, its plan printed, with the
// library's own functions.
//
//   rows <fmt> <fp32 X> <gated> <max M> <M> <N> <K>  -> rows any | rows kgm <shape>
//       <tile rows> <tile columns> | rows tile <tile rows>
//   mx4 <epi> <act> <M> <N> <K>          -> mx4 few | mx4 tile <tile rows>
//   grad <fmt> <M> <N> <K> <address of the scales> -> grad <direct> <dX rows> <dX parts>
//       <dX workgroups> <dW rows> <dW parts> <dW workgroups>
#include "../paper_2607_08526_amd/csrc/internal.h"

#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>

int main()
{
    using namespace qlk;
    const int cus = current_cus();
    std::string line, kind;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        int64_t fmt, M, N, K;
        in >> kind;
        if (kind == "rows") {
            int xf32, gated, shape;
            int64_t maxM;
            in >> fmt >> xf32 >> gated >> maxM >> M >> N >> K;
            const RowsKernel k = choose_rows((int)fmt, xf32, gated, maxM, M, N, K, cus, &shape);
            if (k == ROWS_KGM) {
                const KgTile t = kgm_tile_shape((int)fmt, xf32, gated, maxM, shape);
                std::printf("rows kgm %d %d %d\n", shape, t.m, t.n);
            } else if (k == ROWS_TILE) {
                std::printf("rows tile %d\n", shape);
            } else {
                std::printf("rows any\n");
            }
        } else if (kind == "mx4") {
            int epi, act;
            in >> epi >> act >> M >> N >> K;
            Mx4Args a{};
            a.ep.bias = epi ? reinterpret_cast<const float *>(16) : nullptr;
            a.ep.act = act;
            a.M = (int)M;
            a.N = (int)N;
            a.K = (int)K;
            if (mx4_takes(a) && mx4_wins(a, cus))
                std::printf("mx4 tile %d\n", mx4_rows(a, cus));
            else
                std::printf("mx4 few\n");
        } else {
            uintptr_t at;
            in >> fmt >> M >> N >> K >> at;
            const void *const s = reinterpret_cast<const void *>(at);
            const GradPlan g = grad_plan((int)fmt, M, N, K, s, s, true, true, cus);
            std::printf("grad %d %d %d %lld %d %d %lld\n", g.direct, g.xrows, g.xparts,
                        (long long)(gemm_tiles(g.xrows, M, K) * g.xparts), g.wrows, g.wparts,
                        (long long)(gemm_tiles(g.wrows, N, K) * 2 * g.wparts));
        }
    }
    return 0;
}
