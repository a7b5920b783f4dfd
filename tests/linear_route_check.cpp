// Host-only: which launches a linear layer's call is, asked of the library's own rules.  Built with g++ and the sanitizers by
// tests/test_linear_routes.py.  One call a line on standard input:
//   pass (f forward, b backward with both gradients, x or w with the input's or the weights' alone)  tokens n k  bf16 param_bf16  direct (identity without dropout)  bias  x_address x_stride  dy_address dy_stride
#include <cinttypes>
#include <cstdio>
#include <string>

#include "psgd_linear_rules.h"

using namespace psgd;

// one launch of k_product: operands (how they come, along or across the contraction), side of the tiles, whether the contraction is divided
struct Operands {
    Way way;
    bool a_along, b_along, b_fp32;
};
static std::string sources(const Operands& o) {
    return o.way == kInFp32 ? "fp32" : o.way != kByRegisters ? "straight" : o.b_fp32 ? "registers-fp32" : "registers";
}
static std::string sides(const Operands& o) { return std::string(o.a_along ? "along" : "across") + "-" + (o.b_along ? "along" : "across"); }
static std::string tiles(const Choice& c) { return std::string(c.kind == 0 ? "256" : c.kind == 1 ? "128" : "64") + (c.splits > 1 ? "/split" : ""); }

static std::string product(const Operands& o, int64_t M, int64_t N, int64_t K) {
    const ProductRoute r = product_route(o.way, o.a_along, M, N, K);
    const std::string what = sources(o) + ":" + sides(o) + ":";
    if (!r.over) return " product:" + what + tiles(r.whole);
    if (r.one_launch) return " rest:" + what + tiles(r.main);
    const int64_t m = r.rows ? M - r.over : M, n = r.rows ? N : N - r.over;
    return std::string(r.rows ? " rows" : " columns") + product(o, m, n, K) + product(o, r.rows ? r.over : M, r.rows ? N : r.over, K);
}

int main() {
    char pass;
    int64_t T, n, k, x_ld, dy_ld;
    uint64_t x, dy;
    int bf16, param_bf16, direct, bias;
    while (std::scanf(" %c %" SCNd64 " %" SCNd64 " %" SCNd64 " %d %d %d %d %" SCNu64 " %" SCNd64 " %" SCNu64 " %" SCNd64, &pass, &T, &n, &k, &bf16, &param_bf16,
                      &direct, &bias, &x, &x_ld, &dy, &dy_ld) == 12) {
        LinearCall c{};
        c.T = T, c.n = n, c.k = k, c.bf16 = bf16, c.param_bf16 = param_bf16;
        c.x = reinterpret_cast<const void*>(x), c.x_ld = x_ld, c.dy = reinterpret_cast<const void*>(dy), c.dy_ld = dy_ld;
        std::string out;
        const bool w_fp32 = bf16 && !param_bf16;
        if (pass == 'f') {
            if (few_tokens(c)) {
                std::printf("few\n");
                continue;
            }
            const Comes w0 = weights_come(c, true), in0 = input_comes(c, false, true);
            const Comes w = weights_come(c, in0.ready || in0.lay), in = input_comes(c, false, w0.ready || w0.lay);
            if (w.lay) out += " lay:w";
            if (in.lay) out += " lay:x";
            out += product({way_by(bf16, in.ready || in.lay, w.ready || w.lay, true), true, true, w_fp32 && !w.lay}, T, n, k);
        } else {
            char some;
            c.act = direct ? PSGD_ACT_IDENTITY : PSGD_ACT_GELU;
            c.dx = pass == 'w' ? nullptr : &some;
            c.dw = pass == 'x' ? nullptr : &some;
            const Comes dz = dz_comes(c);
            const bool a = dz.ready || dz.lay;
            const Comes w = weights_come(c, a), in = input_comes(c, true, a);
            if (dz.lay && direct) out += " lay:dy";
            if (w.lay && pass != 'w') out += " lay:w";
            if (in.lay && pass != 'x') out += " lay:x";
            const Operands ox{way_by(bf16, a, w.ready || w.lay, false), true, false, w_fp32 && !w.lay}, ow{way_by(bf16, a, in.ready || in.lay, false), false, false, false};
            const int64_t sums = !dz.lay && bias ? (n + 255) / 256 * ((T + kSumRows - 1) / kSumRows) : 0;
            const BackwardRoute r = backward_route({ox.way, T, k, n}, {ow.way, n, k, T}, sums);
            if (pass == 'x') out += product(ox, T, k, n);
            else if (pass == 'w') out += product(ow, n, k, T);
            else if (r.kind == BackwardRoute::kLarge) out += std::string(" large:") + (r.x_first ? "x" : "w");
            else if (r.kind == BackwardRoute::kTogether)
                out += " two:" + (ox.way >= kStraightAcross && ow.way >= kStraightAcross ? "straight" : bf16 ? sources({kByRegisters, true, false, ox.b_fp32}) : "fp32") + ":" + tiles(r.x).substr(0, r.x.kind == 1 ? 3 : 2);
            else out += product(ox, T, k, n) + product(ow, n, k, T);
        }
        std::printf("%s\n", out.c_str() + 1);
    }
    return 0;
}
