// How the attention kernels deal out their work, on the host.
#include "attention_shared.cuh"

// blocks that prepare the gradients, of a device of `sms`
extern "C" long long run_prepare_blocks(int causal, int n_seg, long long rows, int heads, int lanes, int sms) {
    tiga::AttnParams p{};
    p.causal = causal;
    p.n_seg = n_seg;
    p.heads = heads;
    return tiga::prepare_blocks(p, rows * heads, lanes, sms);
}

#include <vector>

namespace {

using namespace tiga;

// 0, or what is wrong when `grid` blocks share the line: 1 a tile's place, 2 a step that is not done once, 3 parts of a tile that do not follow one another,
// 4 what a block says of the tile that it ends, 5 what is looked up for any tile, 6 two partial states of a block in one place, 7 units
template <typename C>
int differs(AttnParams p, const Segment* line, int grid) {
    std::vector<long long> unit_start(p.n_seg + 1, 0);
    struct Tile { std::vector<int> owner; };
    std::vector<std::vector<Tile>> tiles(p.n_seg);          // [segment][kv head * tiles + tile]
    for (int s = 0; s < p.n_seg; ++s) {
        const Segment g = C::segment(p, s);
        if (line && (g.nq != line[s].nq || g.nk != line[s].nk || g.length != line[s].length)) return 1;
        const int n = C::tiles(p, g);
        long long sum = 0;
        for (int t = 0; t < n; ++t) {
            if (C::before(p, g, t) != sum) return 1;
            sum += (long long)C::steps(p, g, t) * C::step_cost(p, g) + C::item_cost(p);
        }
        if (C::units(p, g) != sum) return 7;
        unit_start[s + 1] = unit_start[s] + sum * p.kv_heads;
        tiles[s].resize((size_t)n * p.kv_heads);
        for (int h = 0; h < p.kv_heads; ++h) for (int t = 0; t < n; ++t) tiles[s][(size_t)h * n + t].owner.assign(C::steps(p, g, t), -1);
    }
    struct End { int s, at, first, parts, block; };
    std::vector<End> ends;
    for (int block = 0; block < grid; ++block) {
        Walker<C> w{};
        w.begin_alone(p, unit_start.data(), block, grid);
        bool used[2] = {false, false};
        int item = 0;
        for (bool more = w.here; more; more = w.next(p), ++item) {
            const int n = C::tiles(p, w.g), at = w.h * n + w.t;
            if (w.s < 0 || w.s >= p.n_seg || w.h < 0 || w.h >= p.kv_heads || w.t < 0 || w.t >= n) return 1;
            std::vector<int>& owner = tiles[w.s][at].owner;
            if (w.steps != (int)owner.size() || w.i0 < 0 || w.i1 > w.steps || w.i1 <= w.i0) return 2;
            for (int i = w.i0; i < w.i1; ++i) {
                if (owner[i] != -1) return 2;
                owner[i] = block;
            }
            if (w.i1 - w.i0 < w.steps) {                    // a partial state
                bool& place = used[w.i0 == 0];
                if (place) return 6;
                place = true;
            }
            if (item == 0 && w.i0 > 0 && w.i1 == w.steps) {
                const int first = w.first_block(p, block);
                ends.push_back({w.s, at, first, block - first + 1, block});
            } else if (w.i0 > 0 && w.i1 == w.steps) return 3;          // (only a block's first item ends a tile that another one began)
        }
    }
    long long shared = 0;
    for (int s = 0; s < p.n_seg; ++s)
        for (size_t at = 0; at < tiles[s].size(); ++at) {
            const Segment g = C::segment(p, s);
            const std::vector<int>& owner = tiles[s][at].owner;
            for (size_t i = 0; i < owner.size(); ++i) {
                if (owner[i] < 0) return 2;
                if (i && owner[i] != owner[i - 1] && owner[i] != owner[i - 1] + 1) return 3;
            }
            shared += owner.front() != owner.back();
            const int n = C::tiles(p, g);
            const auto had = Walker<C>::blocks_of_tile(p, g, unit_start[s], (int)at / n, (int)at % n, unit_start[p.n_seg], Walker<C>::pieces(p, unit_start[p.n_seg], grid));
            if (had.first != owner.front() || had.parts != owner.back() - owner.front() + 1) return 5;
        }
    for (const End& e : ends) {
        const std::vector<int>& owner = tiles[e.s][e.at].owner;
        if (e.first != owner.front() || e.block != owner.back() || e.parts != owner.back() - owner.front() + 1) return 4;
    }
    return shared == (long long)ends.size() ? 0 : 4;
}

}  // namespace

// kind: 0 rows stay, equal steps (dense blocks, chunks over a cache); 1 the same, 2 keys stay; 3, 4, 5 with costs: rows stay by 256, by 128, keys
// stay; 6 a line of shared prefixes; 7 weights.  lengths: nq, nk, length of every segment.
extern "C" int run_pieces(int kind, int causal, int item_cost, int group, int kv_heads, int n_seg, const int* lengths, int grid) {
    std::vector<Segment> line;
    std::vector<int32_t> q_start{0}, kv_start{0}, kv_len;
    for (int s = 0; s < n_seg; ++s) {
        const int nq = lengths[3 * s], nk = lengths[3 * s + 1], length = lengths[3 * s + 2];
        line.push_back({q_start.back(), nq, kind == 6 ? 0 : kv_start.back(), nk, length});
        q_start.push_back(q_start.back() + nq);
        kv_start.push_back(kv_start.back() + nk);
        kv_len.push_back(length);
    }
    tiga::AttnParams p{};
    p.causal = causal;
    p.group = group;
    p.kv_heads = kv_heads;
    p.heads = group * kv_heads;
    p.n_seg = n_seg;
    p.n_q = q_start.back();
    p.n_kv = kv_start.back();
    p.q_start = q_start.data();
    p.kv_start = kv_start.data();
    p.item_cost = item_cost;
    p.line = kind == 6 ? line.data() : nullptr;
    p.uneven = kind == 6;
    const int32_t none = -1;
    if (kind == 7) {                // a paged cache: keys end where the table does, which is as long as all sequences here
        p.table = &none;
        p.kv_len = kv_len.data();
        p.max_pages = 1 << 20;
        p.page_size = 16;
    }
    switch (kind) {
        case 0: return differs<Cut<256, 128, false, CUT_STEPS>>(p, line.data(), grid);
        case 1: return differs<Cut<128, 128, false, CUT_STEPS>>(p, line.data(), grid);
        case 2: return differs<Cut<128, 128, true, CUT_STEPS>>(p, line.data(), grid);
        case 3: return differs<Cut<256, 128, false, CUT_COSTS>>(p, line.data(), grid);
        case 4: return differs<Cut<128, 128, false, CUT_COSTS>>(p, line.data(), grid);
        case 5: return differs<Cut<128, 128, true, CUT_COSTS>>(p, line.data(), grid);
        case 6: return differs<Cut<256, 128, false, CUT_LINE>>(p, line.data(), grid);
        default: return differs<WtCut>(p, line.data(), grid);
    }
}
