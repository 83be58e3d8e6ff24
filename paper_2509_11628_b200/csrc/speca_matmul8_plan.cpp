// Which kernel a product in 8 bits takes, and in what tiles and shares of k: rules on sizes, types and alignment alone. Host only, and nothing but arithmetic.
#include <algorithm>
#include <cmath>

#include "speca_layer_internal.h"

namespace speca {
namespace {

constexpr int kTile = 128;  // rows of a tile of one SM, features of a tile for few rows

// Shares of k, of four stages of 128 at least: as many as run at once. Two blocks share an SM, and a cluster's SMs lie together, so that only 66 clusters of
// four fit 148 SMs (72 took 14.4 us for 4 rows x 9216 x 4096, where two shares take 10.7); eight are worth it one to an SM (15 clusters): 4 rows x
// 1152 x 4096 5.2 us, 6.3 with four; 4096 x 4096 as 256 blocks of eight 8.2, as 128 of four 7.7.
int ranks_few(int64_t tiles, int k_blocks, int sm_count) {
    int ranks = 1;
    for (const double room : {2.0, 1.8, 0.82}) {
        if (2 * ranks * tiles > room * sm_count || k_blocks < 8 * ranks) break;
        ranks *= 2;
    }
    return ranks;
}

// Smaller tiles start and end sooner but read the weights more often, out of L2; blocks that share an SM share its way to L2. Fitted to 21 sizes of
// each, within some 10 %: 211 rows x 333 x 1155 5.8 us in tiles of 16 rows, 10.4 in tiles of 128; 128 x 4096 x 4096 10.4 of 64, 10.8 of 128,
// 12.0 of 32; 256 x 1152 x 4608 9.5 of 64, 11.4 of 128.
FewPlan plan_few(const Matmul8Params& p, int shares, int sm_count) {
    const int k_blocks = (p.k + kBlock8 - 1) / kBlock8;
    FewPlan best{0, 0, 0.0};
    for (const int rows : {16, 32, 64, 128}) {
        if (rows > 16 && rows / 2 >= p.m) break;
        const int64_t m_tiles = (p.m + rows - 1) / rows, tiles = (static_cast<int64_t>(p.n) + kTile - 1) / kTile * m_tiles;
        const int ranks = std::max(ranks_few(tiles, k_blocks, sm_count), shares);
        const double blocks = static_cast<double>(tiles) * ranks, sms = sm_count;
        const double together = blocks <= sms ? 1.0 : blocks <= 2 * sms ? std::max(ranks > 2 ? 1.7 : 1.0, blocks / sms) : 2 * std::ceil(blocks / (2 * sms));
        const double weights = static_cast<double>(p.n) * p.k / 6.5e6 * (0.75 + 0.25 * static_cast<double>(m_tiles));
        const double steps = together * ((k_blocks + ranks - 1) / ranks) * (0.137 + 0.0013 * rows);
        const double start = rows == 16 ? 6.0 : rows == 32 ? 6.4 : rows == 64 ? 7.3 : 9.1;
        const double us = start + std::max(weights, steps) + 1.5 * (together - 1);
        if (best.rows == 0 || us < best.us) best = FewPlan{rows, ranks, us};
    }
    return best;
}

// The three kernels' times in us, as fits to what they measured over 1 to 4096 rows, 1152 to 14336 features and elements of k
// (largest error 25 %; what matters is where they cross). A start, then rounds of tiles over the SMs, each with a step for 128 elements of
// k and an end, longer where rows do not start on 16 bytes; all read the weights at 6.5 TB/s at best. In us, rows x features x k, few / one SM / a pair:
// 1 x 4096 x 4096 8.5 / 12.6 / 15.6;  512 x 4096 x 4096 17.7 / 13.3 / 16.6;  384 x 4096 x 14336 34 / 40 / 41;  1024 x 4096 x 14336 63 / 73 / 48;
// 64 x 4608 x 1152 6.2 / 6.9 / 8.8;  4096 x 1152 x 4608 30 / 27 / 30;  4096 x 14336 x 4096 307 / 252 / 180.
// A mask, which only the device knows, is taken to leave three rows of four where tiles of one SM and of a pair are compared: of 16 samples of 256 rows, 11
// of them active, x 1152 x 4608 a pair's tiles fill one round in place of two (23.7 us, 31.4). In a graph the pair then takes 18.2 us with one sample active, 20.1 with 8 to
// 14 and 29.9 with all 16, where tiles of one SM take 23.7. These two add in the same order, so a row's
// bits do not depend on the mask; shares of k add in another, so few rows are told apart without it.
Matmul8Kernel choose(const Matmul8Params& p, const FewPlan& few, int sm_count) {
    const int64_t kb = (p.k + kBlock8 - 1) / kBlock8;
    auto tiles = [&](int64_t m, int64_t rows, int64_t features) { return (m + rows - 1) / rows * ((p.n + features - 1) / features); };
    auto rounds = [](int64_t n, int64_t places) { return static_cast<double>((n + places - 1) / places); };
    // (tiles of one SM with 16 rows or fewer took half as long again: 22 us for 14336 x 4096, 15.4 from 32 rows on)
    auto one = [&](int64_t m) { return 4.2 + rounds(tiles(m, kTile, 128), sm_count) * (0.7 + (p.m <= 16 ? 0.45 : 0.27) * kb); };
    auto pair = [&](int64_t m) { return 4.5 + rounds(tiles(m, 2 * kTile, 256), sm_count / 2) * (1.0 + 0.34 * kb); };
    const double least = static_cast<double>(p.n) * p.k / 6.5e6 + (p.m <= 64 ? 8.0 : 6.9), odd = p.vectors ? 0.0 : 3.0;
    if (few.us <= std::max(std::min(one(p.m), pair(p.m)) + odd, least)) return kFew;
    const int64_t m = p.dev_mask != nullptr ? p.m - p.m / 4 : p.m;
    return one(m) <= pair(m) ? kOne : kPair;
}

// The tensor cores cut what they add to a sum, each step of 32 products, at about 2^-25 of the largest of the step's terms and the sum, so that a sum over all of k
// comes out short: of normal values by 2.2e-7 of its size at k = 4096 and 5.0e-7 at 8192 (twice that in rows with a value 20 times the others), of uniform positive
// ones by 9.4e-7 and 2.7e-6. At worst, of s terms next to a large one, each just below 2^-25 of it, s 2^-25 of the sum are lost (half of them were, where tried).
// bf16 and 8 bits see that where it passes half a rounding, 2^-10: so at most 32768 elements are summed at once. Outputs in fp32 with more than 8192
// elements take shares of 4096 (k / 8 beyond 32768): 2304 x 4096 x 16384 is 3.7e-7 off in place of 1.9e-6, for 193 us in place of 101. At 8192 the pair's 9e-7 stay
// (58 us; shares would take 134). Shares of k are added up with rounding, by the kernel for few rows.
int shares_of(const Matmul8Params& p, int dtype) {
    const int64_t kb = (p.k + kBlock8 - 1) / kBlock8;
    const bool exact = dtype == SPECA_F32 && p.out != nullptr;
    if (kb <= (exact ? 64 : 256)) return 1;
    int shares = 2;
    while (shares < kFewRanks && shares * (exact ? 32 : 256) < kb) shares *= 2;
    return shares;
}
static_assert(SPECA_MAX_K8 <= kFewRanks * 32768, "no share is longer");

}  // namespace

Matmul8Plan plan_matmul8(const Matmul8Params& p, int dtype, int sm_count) {
    const int shares = shares_of(p, dtype);
    const FewPlan few = plan_few(p, shares, sm_count);
    return Matmul8Plan{shares > 1 ? kFew : choose(p, few, sm_count), few};
}

}  // namespace speca
