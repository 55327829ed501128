// Host checks of how the shared-prefix attention divides its work (csrc/shared_attention.cuh); no GPU takes part.
// Drawn batches: the tiles' key blocks are each taken exactly once, the spans cover the line without gap or overlap, what a span leaves for the merge
// is what the merge looks for.  And the bound on a call's key blocks: what it lets through stays below 2^31.
#include "shared_attention.cuh"

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <vector>

using namespace ctcsd;

#define CHECK(x)                                                             \
    do {                                                                     \
        if (!(x)) { printf("line %d: %s\n", __LINE__, #x); exit(1); }        \
    } while (0)

struct Batch {
    std::vector<int> n, row_off, own_cum, own_len, kv, pre, edge, tile_cum;
    SharedPlan p;
    // n nodes, L cached rows, P rows of the prefix of each sequence
    Batch(const std::vector<int>& nodes, const std::vector<int>& L, const std::vector<int>& P, int grp, int TR, int KB)
        : n(nodes), row_off(n.size() + 1), own_cum(n.size() + 1), own_len(n.size()), kv(n.size()), pre(n.size()), edge(2) {
        const int B = (int)n.size();
        edge[0] = 0x7fffffff;
        for (int b = 0; b < B; ++b) {
            own_len[b] = n[b] ? L[b] + n[b] : 0;
            kv[b] = n[b] ? L[b] : 0;
            pre[b] = n[b] ? P[b] : 0;
            row_off[b + 1] = row_off[b] + n[b] * grp;
            own_cum[b + 1] = own_cum[b] + (own_len[b] + KB - 1) / KB;
            if (n[b]) { edge[0] = std::min(edge[0], P[b]); edge[1] = std::max(edge[1], P[b]); }
        }
        edge[0] = std::min(edge[0], edge[1]);
        p.row_off = row_off.data(); p.own_cum = own_cum.data(); p.own_len = own_len.data(); p.kv = kv.data(); p.pre = pre.data(); p.edge = edge.data();
        p.rows = row_off[B];
        p.tiles = (p.rows + TR - 1) / TR;
        tile_cum.resize(p.tiles + 1);
        for (int t = 0; t < p.tiles; ++t) {
            const int blocks = plan_tile_blocks(p, plan_tile(p, B, TR, t), KB);
            CHECK(blocks > 0);
            tile_cum[t + 1] = tile_cum[t] + blocks;
        }
        p.tile_cum = tile_cum.data();
    }
};

static void drawn_batches() {
    std::mt19937 rng(1);
    auto upto = [&](int k) { return (int)(rng() % (unsigned)(k + 1)); };
    for (int trial = 0; trial < 2000; ++trial) {
        const int B = 1 + upto(39), max_nodes = 2 + upto(62), grp = 1 + upto(8), Hkv = 1 + upto(7);
        const int TR = upto(1) ? kTcRows : kSimpleRows, KB = TR == kTcRows ? kTcKeys : kSimpleKeys;
        const int spans = 1 + upto(299), min_blocks = 1 + upto(4), long_span = upto(29), alike = upto(1);
        std::vector<int> n(B), L(B), P(B);
        for (int b = 0; b < B; ++b) {
            n[b] = upto(3) == 0 ? 0 : upto(max_nodes);
            L[b] = upto(2) ? upto(699) : 0;
            P[b] = alike ? 500 : (upto(2) ? upto(999) : 0);
        }
        const Batch x(n, L, P, grp, TR, KB);
        const SharedPlan& p = x.p;
        CHECK(plan_fits(B, max_nodes, grp, TR, KB, 1000, 700 + max_nodes));
        CHECK(x.tile_cum[p.tiles] <= plan_most_blocks(B, max_nodes, grp, TR, KB, 1000, 700 + max_nodes));
        const SpanMap sp = span_map(x.tile_cum[p.tiles], p.tiles, Hkv, spans, min_blocks, long_span);
        CHECK(sp.spans >= 1 && sp.spans <= spans);
        if (sp.total == 0) continue;
        CHECK(sp.start(0) == 0 && sp.start(sp.spans) == sp.total);
        std::map<std::pair<int, int>, std::set<std::pair<int, int>>> taken;      // (kv head, tile) -> (source, first key)
        for (int c = 0; c < sp.spans; ++c) {
            long long at = sp.start(c);
            std::set<int> slots;
            SpanWalk w;
            for (bool more = w.init(p, sp, c); more; more = w.next(p)) {
                CHECK(at < sp.start(c + 1) && sp.span_of(at) == c);
                CHECK(w.g < Hkv && w.t < p.tiles && w.blk1 > w.blk0);
                const TileInfo ti = plan_tile(p, B, TR, w.t);
                int pmax = 0, pmin = 0x7fffffff;
                for (int b = ti.b0; b <= ti.b1; ++b)
                    if (x.own_len[b]) { pmax = std::max(pmax, x.pre[b]); pmin = std::min(pmin, x.pre[b]); }
                CHECK(pmax == ti.pmax && pmin == ti.pmin);
                CHECK((long long)w.g * sp.per_head + x.tile_cum[w.t] + w.blk0 == at);
                at += w.blk1 - w.blk0;
                // the merge's view: first and last span of the tile; only the first part may begin it (slot 1)
                const long long xs = (long long)w.g * sp.per_head + x.tile_cum[w.t], xe = (long long)w.g * sp.per_head + x.tile_cum[w.t + 1];
                CHECK((sp.span_of(xs) == sp.span_of(xe - 1)) == w.whole());
                if (!w.whole()) {
                    CHECK(slots.insert(w.slot()).second);
                    CHECK((c == sp.span_of(xs) ? 1 : 0) == w.slot() && c <= sp.span_of(xe - 1));
                }
                BlockIter it;
                it.init(p, ti, KB, w.blk0);
                for (int blk = w.blk0; blk < w.blk1; ++blk) {
                    if (it.seq < 0) CHECK(it.key0 < ti.pmax && it.len == ti.pmax);
                    else CHECK(it.seq >= ti.b0 && it.seq <= ti.b1 && it.key0 < x.own_len[it.seq] && it.len == x.own_len[it.seq]);
                    CHECK(taken[std::make_pair(w.g, w.t)].insert(std::make_pair(it.seq, it.key0)).second);
                    if (blk + 1 < w.blk1) it.next(p, ti, KB);
                }
            }
            CHECK(at == sp.start(c + 1));
        }
        for (int g = 0; g < Hkv; ++g)
            for (int t = 0; t < p.tiles; ++t) {
                const TileInfo ti = plan_tile(p, B, TR, t);
                size_t want = (ti.pmax + KB - 1) / KB;
                for (int r = ti.row0; r < ti.row0 + ti.nrows; ++r) {
                    const int b = plan_seq_of_row(p, B, r);
                    CHECK(x.row_off[b] <= r && r < x.row_off[b + 1] && b >= ti.b0 && b <= ti.b1);
                }
                for (int b = ti.b0; b <= ti.b1; ++b) want += (x.own_len[b] + KB - 1) / KB;
                CHECK(taken[std::make_pair(g, t)].size() == want);
            }
    }
}

// Lines of more than 2^31 blocks: the long division.
static void long_lines() {
    for (int spans : {1, 7, 148, 296})
        for (int per_head : {40000000, 2147483647})
            for (int Hkv : {1, 60, 2048}) {
                const SpanMap m = span_map_n(per_head, Hkv, spans);
                CHECK(m.start(0) == 0 && m.start(spans) == (long long)per_head * Hkv);
                for (int c = 0; c < spans; ++c) {
                    CHECK(m.start(c + 1) - m.start(c) == m.each + (c < m.extra ? 1 : 0));
                    CHECK(m.span_of(m.start(c)) == c && m.span_of(m.start(c + 1) - 1) == c);
                }
            }
}

// The most rows a call may have, behind long prefixes and caches: what passes the bound adds up below 2^31.
static void bound_on_blocks() {
    int fits = 0, refused = 0;
    for (int TR : {kTcRows, kSimpleRows})
        for (int B : {1, 100, 1024})
            for (int max_nodes : {2, 64, 256})
                for (int rows : {kSharedMaxRows, 5000})
                    for (long long pre = 128; pre <= 2147483000ll; pre *= 4)
                        for (long long own : {100ll, 70000ll, 300000000ll}) {
                            const int KB = TR == kTcRows ? kTcKeys : kSimpleKeys, grp = rows / (B * max_nodes);
                            if (grp < 1) continue;
                            // every node live, every cache full: Σ over tiles of (prefix blocks + own blocks of its sequences)
                            long long sum = 0;
                            const int per_seq = max_nodes * grp, total = B * per_seq;
                            for (int r = 0; r < total; r += TR) {
                                const int b0 = r / per_seq, b1 = (std::min(r + TR, total) - 1) / per_seq;
                                sum += (pre + KB - 1) / KB + (b1 - b0 + 1) * ((own + KB - 1) / KB);
                            }
                            CHECK(sum <= plan_most_blocks(B, max_nodes, grp, TR, KB, (int)pre, (int)own));
                            if (plan_fits(B, max_nodes, grp, TR, KB, (int)pre, (int)own)) { ++fits; CHECK(sum < (1ll << 31)); }
                            else ++refused;
                        }
    CHECK(fits > 0 && refused > 0);
    CHECK(plan_fits(1024, 256, 2, kTcRows, kTcKeys, 1 << 20, 1 << 20));          // a million rows each way
}

int main() {
    drawn_batches();
    long_lines();
    bound_on_blocks();
    puts("ok");
    return 0;
}
