// Which launches a linear layer's call is: the rules, on the host and without HIP, so that they can be asked by themselves.
#ifndef PSGD_LINEAR_RULES_H
#define PSGD_LINEAR_RULES_H

#include <algorithm>

#include "psgd_operators.h"

namespace psgd {

constexpr int kCUs = 256;

// The tiles, and what they take: us a step with a unit full, of one tile by itself, and for first loads and epilogue; tiles that a
// unit holds at once.  Fitted to products of one to four rounds, 128 .. 8192 of the contraction; bf16 both operands straight to LDS along
// the contraction, and all others (reads across it, loads through registers).  Over 39 bf16 products and every division that was timed the
// choice takes 1.1 % more than the best one on average, 21 % at most (128 x 2048 x 2048, 14.3 and 11.8 us); over 39 fp32 ones 0.8 and 5 %.
struct TileKind {
    int side;
    int at_once;
    double full, alone, ends;
};
constexpr int lanes_of(int kind) { return kind == 0 ? 512 : 256; }
constexpr TileKind kTilesAlong[] = {{256, 1, 1.2, 1.2, 9}, {128, 2, 0.41, 0.42, 5.7}, {64, 4, 0.138, 0.204, 3.5}};
constexpr TileKind kTilesAcross[] = {{256, 1, 1.36, 1.36, 8.5}, {128, 2, 0.465, 0.735, 4.4}, {64, 4, 0.163, 0.46, 2.9}};
constexpr TileKind kTilesFp32[] = {{256, 1, 0, 0, 0}, {128, 2, 1.9, 2.4, 5}, {64, 4, 0.5, 0.8, 3}};   // none of 256
// How a product's operands come
enum Way { kInFp32, kByRegisters, kStraightAcross, kStraightAlong };
inline const TileKind& tile_kind(Way way, int kind) { return (way == kInFp32 ? kTilesFp32 : way == kStraightAlong ? kTilesAlong : kTilesAcross)[kind]; }

// A split takes four steps at least, and there are no more tiles and splits than the units hold at a time, so that the sums
// take at most 64 MiB whatever the sizes.
constexpr int64_t kMostSplits = 32, kLeastSteps = 4, kMostPartial = int64_t(kCUs) * 256 * 256 * 4;

struct Choice {
    int kind;          // of the tiles
    int64_t splits, steps_each, tiles_m, tiles_n;
    double us;         // expected
};

// The tile and the division of the contraction with the least expected time: steps of a tile one after the other, as many tiles
// at a time as the units hold, and the sums of the splits written and read again.  One launch takes the tiles: those of 64 where they are few
// enough, and those of 128 of any product of up to kLinMaxElems outputs.
inline Choice choose(Way way, int64_t M, int64_t N, int64_t K, int only = -1) {
    const int64_t step = way == kInFp32 ? 32 : 64, steps = (K + step - 1) / step;
    const bool small_fit = ((M + 63) / 64) * ((N + 63) / 64) <= most_groups(lanes_of(2));
    Choice best{-1, 0, 0, 0, 0, 0};
    for (int kind = 0; kind < 3; ++kind) {
        const TileKind& t = tile_kind(way, kind);
        if ((kind == 0 && way < kStraightAcross) || (only >= 0 && kind != only)) continue;
        if (only < 0 && t.side > 64 && (M <= t.side / 2 || N <= t.side / 2) && small_fit) continue;   // more than half of every tile outside
        const int64_t tm = (M + t.side - 1) / t.side, tn = (N + t.side - 1) / t.side, tiles = tm * tn;
        if (only < 0 && kind == 2 && !small_fit) continue;
        for (int64_t splits = 1; splits <= (kind == 0 ? 1 : kMostSplits) && (splits == 1 || (splits <= steps / kLeastSteps && tiles * splits <= kCUs * t.at_once)); ++splits) {
            const int64_t each = std::max<int64_t>(1, (steps + splits - 1) / splits), parts = std::max<int64_t>(1, (steps + each - 1) / each);
            if (parts != splits) continue;
            // tiles a unit works off: full loads, and what is left, which does not spread evenly
            const int64_t n = tiles * splits, batches = n / (kCUs * t.at_once), rest = n % (kCUs * t.at_once);
            const double left = rest == 0 ? 0 : std::max<double>((double)((rest + kCUs - 1) / kCUs), batches ? 0.8 * t.at_once : 0);
            const double work = batches * t.at_once + left;
            double us = each * std::max(t.alone, work * t.full) + t.ends * std::max<double>(1, work / std::min(t.at_once, 2));
            if (splits > 1) us += 4.2 + 1.6e-6 * splits * M * N;
            if (best.kind < 0 || us < best.us) best = Choice{kind, splits, each, tm, tn, us};
        }
    }
    return best;
}

// Rows (`rows`) or columns beyond the last full tile that are better a product of their own, 0 if none are, and the expected time
struct Rest {
    int64_t count;
    bool rows;
    double us;
};
inline Rest rest_of(Way way, int64_t M, int64_t N, int64_t K, double whole_us, bool columns_only) {
    Rest best{0, false, whole_us};
    for (int64_t side : {128, 256})
        for (bool rows : {true, false}) {
            const int64_t all = rows ? M : N, r = all % side;
            if ((rows && columns_only) || r == 0 || r > side / 2 || all < side) continue;
            const int64_t m = rows ? M - r : M, n = rows ? N : N - r;
            double us = choose(way, m, n, K).us;
            if (rows) us = rest_of(way, m, n, K, us, true).us;
            us += 2 + choose(way, rows ? r : M, rows ? N : r, K).us;
            if (us < 0.9 * whole_us && us < best.us) best = Rest{r, rows, us};
        }
    return best;
}

// Expected time of a product as launch_product runs it
inline double product_us(Way way, int64_t M, int64_t N, int64_t K) {
    const double us = choose(way, M, N, K).us;
    return us > 30 ? rest_of(way, M, N, K, us, false).us : us;
}

// Expected time of two products in the largest tiles in one launch, the one with the longer tiles first: units that are through with theirs
// (some one round earlier than others) take the other one's in turn
inline double two_large_us(const Choice& a, const Choice& b) {
    const TileKind& t = kTilesAcross[0];
    const double ta = a.steps_each * t.full + t.ends, tb = b.steps_each * t.full + t.ends;
    const int64_t na = a.tiles_m * a.tiles_n, late = na % kCUs;
    int64_t nb = b.tiles_m * b.tiles_n;
    double late_at = ((na + kCUs - 1) / kCUs) * ta, early_at = (na / kCUs) * ta;
    const int64_t rounds = std::max<int64_t>(0, nb / kCUs - 2 - (int64_t)(ta / tb));   // of all units
    late_at += rounds * tb, early_at += rounds * tb, nb -= rounds * kCUs;
    while (nb > 0) {
        if (late == 0 || early_at <= late_at) early_at += tb, nb -= kCUs - late;
        else late_at += tb, nb -= late;
    }
    return std::max(late ? late_at : 0, early_at);
}

// ---- one product ----------------------------------------------------------------------------------------------------

// How launch_product runs M x N x K: in one launch (`whole`), or, where `over` is not 0, that many rows (`rows`) or columns beyond the last full
// tile as a product of their own: in the same launch, `main` in the tiles of its choice and `rest` in those of 64, or one after the other.
struct ProductRoute {
    Choice whole;
    int64_t over;
    bool rows, one_launch;
    Choice main, rest;
};
inline ProductRoute product_route(Way way, bool a_along, int64_t M, int64_t N, int64_t K) {
    ProductRoute r{choose(way, M, N, K), 0, false, false, {}, {}};
    // Rows or columns beyond the last full tile cost a row of tiles, which may be the one too many for the last round: a product of
    // their own, in small tiles, where that is expected to be faster by a tenth.  4099 x 2048 x 8192 bf16 205 us without.
    if (r.whole.us <= 30) return r;
    const Rest over = rest_of(way, M, N, K, r.whole.us, false);
    r.over = over.count;
    r.rows = over.rows;
    if (!over.count || !over.rows || way < kStraightAcross || !a_along) return r;
    // rows: in the same launch where the main product is one undivided launch of the larger tiles and they fill no more than one round
    r.main = choose(way, M - over.count, N, K);
    if (r.main.kind == 2 || r.main.splits > 1 || (r.main.us > 30 && rest_of(way, M - over.count, N, K, r.main.us, false).count)) return r;
    const int64_t wide = r.main.kind == 0 ? 128 : 64, steps = (K + 63) / 64, tm = (over.count + 63) / 64, tn = (N + wide - 1) / wide;
    const int64_t splits = std::min({kCUs * (int64_t)kTilesAlong[r.main.kind].at_once / (tm * tn), steps / kLeastSteps, kMostSplits});
    if (splits < 2 || r.main.tiles_m * r.main.tiles_n + tm * tn * splits > most_groups(lanes_of(r.main.kind))) return r;
    const int64_t each = (steps + splits - 1) / splits;
    r.rest = Choice{2, (steps + each - 1) / each, each, tm, tn, 0};
    r.one_launch = true;
    return r;
}

// ---- the two products of a backward pass ----------------------------------------------------------------------------

struct Extent {
    Way way;
    int64_t M, N, K;
};
// kLarge: one launch in the largest tiles, the input gradient's first (`x_first`) or the weight gradient's; kTogether: one launch of smaller
// tiles, with the columns' sums; kApart: each as product_route says
struct BackwardRoute {
    enum { kApart, kTogether, kLarge } kind;
    Choice x, w;
    bool x_first;
};
inline BackwardRoute backward_route(const Extent& x, const Extent& w, int64_t sum_blocks) {
    BackwardRoute r{BackwardRoute::kApart, {}, {}, false};
    // Large ones in one launch where that is expected to be faster than each by itself: 4096 x 2048 x 8192, 128 tiles of twice the length, and
    // 8192 x 2048 x 4096, 256 tiles, 241 us one after the other and 217 together
    if (x.way >= kStraightAcross && w.way >= kStraightAcross) {
        r.x = choose(x.way, x.M, x.N, x.K, 0);
        r.w = choose(w.way, w.M, w.N, w.K, 0);
        r.x_first = r.x.steps_each >= r.w.steps_each;
        const int64_t all = r.x.tiles_m * r.x.tiles_n + r.w.tiles_m * r.w.tiles_n;
        const double apart = product_us(x.way, x.M, x.N, x.K) + product_us(w.way, w.M, w.N, w.K);
        if (apart > 60 && all <= most_groups(lanes_of(0)) && two_large_us(r.x_first ? r.x : r.w, r.x_first ? r.w : r.x) < 0.95 * apart) {
            r.kind = BackwardRoute::kLarge;
            return r;
        }
    }
    // Small ones where both take the same tiles: worth a tile that is not each one's best if what that costs is less than the launch
    r.x = choose(x.way, x.M, x.N, x.K);
    r.w = choose(w.way, w.M, w.N, w.K);
    if (r.x.us + r.w.us < 150 && (r.x.kind != r.w.kind || r.x.kind == 0)) {
        double least = r.x.us + r.w.us + 4;
        for (int kind : {1, 2}) {
            const Choice tx = choose(x.way, x.M, x.N, x.K, kind), tw = choose(w.way, w.M, w.N, w.K, kind);
            if (tx.us + tw.us < least) least = tx.us + tw.us, r.x = tx, r.w = tw;
        }
    }
    const int64_t blocks = r.x.tiles_m * r.x.tiles_n * r.x.splits + r.w.tiles_m * r.w.tiles_n * r.w.splits + sum_blocks;
    if (r.x.kind == r.w.kind && r.x.kind > 0 && r.x.us + r.w.us < 150 && blocks <= most_groups(lanes_of(r.x.kind))) r.kind = BackwardRoute::kTogether;
    return r;
}

constexpr int kSumRows = 64;   // rows of a block of the columns' sums

// ---- how the operands of a call come --------------------------------------------------------------------------------

inline int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }
inline bool vec_aligned(const void* p, int64_t ld) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld % 8 == 0; }   // bf16

inline Way way_by(bool bf16, bool a_ready, bool b_ready, bool along) {
    return !bf16 ? kInFp32 : !a_ready || !b_ready ? kByRegisters : along ? kStraightAlong : kStraightAcross;
}

// Whether operands of a bf16 product that cannot go straight to LDS are laid out for it first: a pass over them against slower
// loads in every tile.  us, laid out / in place: forward, fp32 weights of 8192 x 2048, 300 tokens 34 / 27, 700 44 / 41, 1500 63 / 70, 4000
// 119 / 165; 50304 x 2048 700 270 / 229, 1500 380 / 444; 4096 x 4095 bf16, both operands, 300 48 / 41, 700 54 / 68, 4000 124 / 196; 2600 x 650
// bf16 1500 25 / 16, 4000 39 / 32.  The weight gradient, which reads the input alone in another place: 1000 x 1001, 4000 tokens 34 / 31, 2600 x
// 650 700 14 / 13, 1500 23 / 25, 4000 47 / 64; 4096 x 4095 300 30 / 31, 4000 121 / 192.
inline bool large_enough(const LinearCall& c, bool weight_gradient) {
    const double work = (double)c.T * (double)c.n * (double)c.k;
    return weight_gradient ? work >= 2e9 : c.T >= (c.param_bf16 ? 640 : 1000) && work >= 1e10;
}
inline bool lay_out_pays(const LinearCall& c, int64_t rows, int64_t ld, bool weight_gradient) {
    return large_enough(c, weight_gradient) && (rows * (ld / 8) + kBlock - 1) / kBlock <= most_groups(kBlock);   // one launch takes 64 GiB
}

// Which operands of a bf16 product can go straight to LDS where they are (`ready`), and which are laid out for it first (`lay`).  For bf16 operands that
// is of use only if the product's other operand comes that way too; fp32 weights are rounded once instead of in every tile (the input gradient of 1500 x
// 4095 x 2000 through registers 83 us in place, 75 laid out; of 8192 x 50257 x 2048 3208 and 2218).
struct Comes {
    bool ready, lay;
};
inline Comes weights_come(const LinearCall& c, bool other_ready) {
    const bool ready = !c.bf16 || (c.param_bf16 && c.k % 8 == 0);
    return Comes{ready, !ready && (other_ready || !c.param_bf16) && lay_out_pays(c, c.n, up(c.k, 8), false)};
}
inline Comes input_comes(const LinearCall& c, bool weight_gradient, bool other_ready) {
    const bool ready = !c.bf16 || (vec_aligned(c.x, c.x_ld) && c.k % 8 == 0);
    return Comes{ready, !ready && other_ready && lay_out_pays(c, c.T, up(c.k, 8), weight_gradient)};
}
// dz: where it is dy itself, it can be read in place; otherwise it is written for the products anyway, in padded rows.  That is done with dy too (`lay`)
// where its rows do not begin on multiples of sixteen bytes and the products are large enough; in place, its products go through registers.  us, in place / laid
// out, n x k, tokens: both gradients 1001 x 1000 1500 33 / 32, with fp32 weights 35 / 40, 8192 82 / 73 and 80 / 87; 4095 x 4096 300 60 / 65, 700
// 117 / 88, 4000 424 / 263, fp32 441 / 280; 650 x 2601 4000 80 / 97, 8192 135 / 127; 50257 x 2048 300 302 / 251, 8192 4329 / 3717, fp32 4552 /
// 3853.  The input gradient alone: 650 x 2601 8192 62 / 66; 4095 x 4096 700 50 / 53, 1500 88 / 77.  The weight gradient alone: 1001 x 1000 300
// 15 / 15, 700 22 / 19; 4095 x 4096 4000 242 / 133; 650 x 2601, where the input is laid out too, 1500 37 / 40, 4000 74 / 64.
inline Comes dz_comes(const LinearCall& c) {
    if (c.act != PSGD_ACT_IDENTITY || c.drop.below) return Comes{false, true};
    if (!c.bf16 || (vec_aligned(c.dy, c.dy_ld) && c.n % 8 == 0)) return Comes{true, false};
    const double work = (double)c.T * (double)c.n * (double)c.k, least = !c.dw ? 2e10 : c.dx ? 1e10 : input_comes(c, true, true).ready ? 1e9 : 4e9;
    return Comes{false, work >= least && (c.n + 255) / 256 * ((c.T + kSumRows - 1) / kSumRows) <= most_groups(kBlock)};
}

// ---- the forward product of a few tokens ----------------------------------------------------------------------------

// At most kFewTokens tokens, without scratch and whatever the operands' types and alignment.
constexpr int64_t kFewTokens = 32;
// Where this takes less time than the tiles of the other products, which read x once for 64 rows of W and divide the contraction
// over the chip: us, this / tiles, one, 16 and 32 tokens, n x k, called again and again, so that weights of up to some 200 MB come from the caches.
//   fp32: 650 x 650 4.3 / 9.7, 4.6 / 9.8, 6.4 / 10.1; 8192 x 2048 12.9 / 24.9, 16.9 / 25.3, 18.4 / 26.2; 50304 x 2048 82 / 137, 107 / 137, 119 / 138;
//   2048 x 8192, short of workgroups, 20.5 / 25.9, 30.4 / 26.3, 44.5 / 26.8; 512 x 8192 19.6 / 13.3.
//   bf16: 512 x 512 2.9 / 4.6, 3.3 / 4.7, 3.7 / 5.0; 2048 x 2048 4.4 / 6.6, 5.8 / 7.0, 7.5 / 7.6; 8192 x 2048 6.6 / 9.9, 7.9 / 16.1, 9.8 / 16.6; beyond
//   2^24 weights it loses: 8192 x 4096 16.3 / 15.0, 16.4 / 15.7, 17.9 / 16.5; 50304 x 2048 39 / 31, 44 / 32, 52 / 34; and where n is small or
//   rows of odd length begin between words: 2048 x 8192 11.6 / 10.6, 16.6 / 12.1, 23.6 / 13.0; 1000 x 1001 6.5 / 7.2, 8.7 / 7.9, 11.5 / 8.1; 4096 x
//   4095 18.7 / 11.5, 30.3 / 13.0, 43.4 / 13.7.
//   bf16, fp32 weights: 512 x 512 3.4 / 6.0, 4.1 / 6.0, 5.0 / 6.5; 1000 x 1001 4.8 / 7.4, 6.6 / 8.0, 9.4 / 8.2; 2048 x 2048 6.9 / 7.5, 9.5 / 8.0, 13.0 / 8.6;
//   8192 x 2048 12.5 / 15.1, 16.8 / 15.9, 18.9 / 16.6; 50304 x 2048 69 / 103, 97 / 105, 109 / 108.
// With the weights from memory, as a model of more layers than the caches hold reads them, both take longer and this one loses later: fp32 8192 x 2048 16.1 /
// 26.8, 19.7 / 27.2, 19.7 / 27.8; 2048 x 8192 25.9 / 28.3, 31.6 / 29.3, 48.1 / 29.7; bf16 2048 x 2048 5.2 / 9.4, 6.6 / 10.2, 9.2 / 11.0; 8192 x 2048 9.6 / 13.6,
// 10.6 / 25.3, 12.4 / 25.6; 8192 x 4096 18.7 / 19.3, 19.3 / 19.9, 21.9 / 20.7; 50304 x 2048 41.4 / 48.8, 54.7 / 49.4, 66.4 / 51.5; 2048 x 8192 13.7 / 14.2, 17.5
// / 14.6, 27.3 / 15.1; bf16, fp32 weights 8192 x 2048 14.1 / 17.6, 17.8 / 18.0, 19.9 / 19.1; 50304 x 2048 70.1 / 99.0, 99.1 / 100.5, 111.1 / 102.6; and on
// the other side of the lines on n, small layers with a longer contraction: fp32 158 x 700 4.4 / 10.2 for one token.
inline bool few_tokens(const LinearCall& c) {
    if (c.T > kFewTokens) return false;
    const int64_t weights = c.n * c.k;
    const bool one = c.T <= 4, some = c.T <= 16;
    if (!c.bf16) return 2 * c.n >= c.k || (one && 4 * c.n >= c.k);
    if (2 * c.n < c.k) return false;
    if (!c.param_bf16) return one || weights <= (some ? 1 << 20 : 1 << 19);
    return c.k % 2 ? one && weights <= 1 << 21 : weights <= 1 << 24;
}

}  // namespace psgd

#endif
