// How the attention kernels cut their work, on the host: the units in front of a tile against the steps of the tiles, one by one.
#include "attention_shared.cuh"

namespace {

template <typename C>
int differs(const tiga::AttnParams& p, const tiga::Segment& g) {
    const int tiles = C::tiles(p, g);
    long long sum = 0;
    for (int t = 0; t <= tiles; ++t) {
        if (C::before(p, g, t) != sum) return 1 + t;
        if (t == tiles) break;
        const int n = C::steps(p, g, t);
        if (n < 1) return 1 + t;
        // the steps cover what the tile's rows read, and none of them is empty where there is anything
        for (int r = t * C::TILE; r < C::rows(p, g) && r < (t + 1) * C::TILE; ++r) {
            if (C::KEYS) {
                const long long first = p.causal ? (long long)r - (g.length - g.nq) : 0, packed = (long long)g.nq * p.group;
                if (first < g.nq && (first > 0 ? first : 0) * p.group < (long long)C::skipped(p, g, t) * C::STEP) return -1 - t;
                if ((long long)(C::skipped(p, g, t) + n) * C::STEP < packed) return -1 - t;
            } else if ((long long)n * C::STEP < tiga::keys_of_row(p, g, r / p.group)) return -1 - t;
        }
        sum += n;
    }
    return C::units(p, g) == sum ? 0 : 1 << 30;
}

}  // namespace

// 0: all alike; otherwise which tile is not
extern "C" int run_cut(int keys, int causal, int group, int nq, int nk, int length) {
    tiga::AttnParams p{};
    p.group = group;
    p.causal = causal;
    const tiga::Segment g{0, nq, 0, nk, length};
    return keys ? differs<tiga::Cut<128, 128, true, tiga::CUT_COSTS>>(p, g) : differs<tiga::Cut<256, 128, false, tiga::CUT_COSTS>>(p, g) | differs<tiga::Cut<128, 128, false, tiga::CUT_COSTS>>(p, g);
}
extern "C" long long run_lattice(long long n, long long a, long long b, long long m) { return tiga::lattice_points(n, a, b, m); }
