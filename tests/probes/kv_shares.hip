// The work list of the attention over the 4-bit cache, without a GPU: what the host chooses for a batch, and the items and shares
// that the kernels' own functions make of its lengths.
//
//   kv_shares random < batches
//
// First the batches of the standard input, one a line, then `random` made-up ones:
//   heads R D G page window sinks max_len entries n len new [len new ..]     (entries: of a table's row)
// For every tile of rows: its shares have the items that it owns, together they are its steps once each, the steps hold every key
// that a row sees, and no item is past the list.  Prints one line: the batches, those that are cut, the tiles of those, and the faults.
#include <stdio.h>
#include <stdlib.h>

#include <cmath>
#include <random>
#include <sstream>
#include <string>
#include <vector>

#include "tpq_kv_items.h"

using namespace tpq;

struct Batch {
    int heads, R, D, G, page, window, sinks, max_len, entries;
    std::vector<int> len, n;
};

static int64_t g_cut, g_tiles, g_bad;

static void fault(const Batch &b, const char *what, int seq, int rt, const KvShare &s, int cuts, int items)
{
    if (g_bad++ >= 10) return;
    fprintf(stderr, "%s: heads %d R %d D %d G %d page %d window %d sinks %d max_len %d entries %d sequences %zu (%d of %d tokens..): sequence %d (%d of %d) "
                    "tile %d: steps %d share %d live %d of %d, item %lld of %d\n",
            what, b.heads, b.R, b.D, b.G, b.page, b.window, b.sinks, b.max_len, b.entries, b.len.size(), b.n[0], b.len[0], seq, b.n[seq], b.len[seq], rt,
            s.span.tiles, s.share, s.live, cuts, static_cast<long long>(s.item0), items);
}

static int log2_of(int v)
{
    int lg = 0;
    while ((1 << lg) < v) ++lg;
    return lg;
}

template <int TOK>
static void look(const Batch &b, const KvArgs &a, const KvAttendArgs &p, const KvChoice &c)
{
    std::vector<KvSeq> q(a.n_seqs);
    uint64_t work = 0;
    uint32_t tiles = 0;
    for (int i = 0; i < a.n_seqs; ++i) {
        q[i] = kv_seq<TOK>(a, p, c.rows, i);
        work += kv_work(q[i]);
        tiles += q[i].row_tiles;
    }
    const bool even = kv_even(a, p);
    const uint32_t step = even ? 0 : kv_step(p, work, tiles, 0, [](uint32_t n) { return n; }, [&](uint32_t by) {
        uint32_t n = 0;
        for (const KvSeq &x : q) n += kv_items(x, by);
        return n;
    });
    if (c.splits > 1) ++g_cut;
    int64_t first = 0;
    for (int i = 0; i < a.n_seqs; ++i) {
        const int cuts = even ? p.splits : static_cast<int>(std::max((q[i].most + step - 1) / step, 1u));
        if (even && a.n_seqs > 1) first = i;
        for (int rt = 0; rt < q[i].row_tiles; ++rt) {
            KvShare s;
            s.rt = rt;
            kv_tile_share<TOK>(a, p, c.rows, q[i], cuts, static_cast<int>(first), s);
            if (c.splits > 1) ++g_tiles;
            if (s.live < 1 || s.live > cuts) fault(b, "more shares than items", i, rt, s, cuts, p.items);
            if (static_cast<int64_t>(s.share) * s.live < s.span.tiles || (s.live > 1 && static_cast<int64_t>(s.share) * (s.live - 1) >= s.span.tiles))
                fault(b, "shares are not the steps", i, rt, s, cuts, p.items);
            if (s.item0 < first || s.item0 + s.live > p.items) fault(b, "past the list", i, rt, s, cuts, p.items);
            // the keys that the tile's rows see are between the first row's window and the last row's position, and the first tokens
            const int end = std::min({s.hi + 1, s.len, b.entries * b.page});
            const auto has = [&](int key) {
                const int t = key / TOK;
                return t < s.span.first || (t >= s.span.start && t < s.span.start + (s.span.tiles - s.span.first));
            };
            const int low = p.window > 0 ? std::max(s.lo - p.window + 1, 0) : 0;
            bool all = true;
            for (int key = low; key < end; key += key + TOK < end ? TOK : std::max(end - 1 - key, 1)) all &= has(key);
            for (int key = 0; p.window > 0 && key < std::min(p.sinks, end); ++key) all &= has(key);
            if (!all || s.span.start < s.span.first) fault(b, "keys without a step", i, rt, s, cuts, p.items);
        }
        first += static_cast<int64_t>(q[i].row_tiles) * cuts;
    }
    if (static_cast<uint64_t>(c.items) * a.heads * c.rows > choose(a, b.D, b.R, b.max_len, 256).partial_rows && c.splits > 1)
        fault(b, "no room", 0, 0, KvShare{}, 0, p.items);
}

static void look(const Batch &b)
{
    std::vector<int32_t> starts(1, 0);
    KvArgs a = {};
    a.n_seqs = static_cast<int>(b.len.size());
    for (int i = 0; i < a.n_seqs; ++i) {
        starts.push_back(starts.back() + b.n[i]);
        a.max_new = std::max(a.max_new, std::max(b.n[i], 1));
    }
    const bool single = starts.back() == a.n_seqs && a.max_new == 1;
    a.rows = starts.back();
    a.lens = b.len.data();
    a.starts = single ? nullptr : starts.data();
    a.ld_table = b.entries;
    a.heads = b.heads;
    a.lg_page = log2_of(b.page);
    a.ng = b.D / b.G;
    KvAttendArgs p = {};
    p.R = b.R;
    p.window = b.window;
    p.sinks = b.sinks;
    const KvChoice c = choose(a, b.D, b.R, reach_of(a, p, b.max_len), 256);
    if (c.items * a.heads > kKvMaxItems) return;
    take_choice(a, c, p);
    if (c.many && b.D <= 128) look<64>(b, a, p, c);
    else look<32>(b, a, p, c);
}

int main(int argc, char **argv)
{
    int64_t batches = 0;
    char *line = nullptr;
    size_t room = 0;
    while (getline(&line, &room, stdin) > 0) {
        std::istringstream in(line);
        Batch b;
        size_t n;
        if (!(in >> b.heads >> b.R >> b.D >> b.G >> b.page >> b.window >> b.sinks >> b.max_len >> b.entries >> n)) continue;
        b.len.resize(n);
        b.n.resize(n);
        for (size_t i = 0; i < n; ++i) in >> b.len[i] >> b.n[i];
        look(b);
        ++batches;
    }
    free(line);

    std::mt19937_64 g(1);
    const auto upto = [&](int n) { return static_cast<int>(g() % static_cast<uint64_t>(n)); };  // 0 .. n - 1
    const auto spread = [&](double lo, double hi) { return static_cast<int>(lo * std::pow(hi / lo, (g() >> 11) * 0x1p-53)); };
    for (int i = argc > 1 ? atoi(argv[1]) : 0; i > 0; --i, ++batches) {
        Batch b;
        b.D = 64 << upto(3);
        b.G = 32 << upto(log2_of(b.D / 32) + 1);
        b.page = 16 << upto(5);
        b.heads = upto(3) ? 1 << upto(6) : spread(1, 257);
        b.R = upto(2) ? 1 << upto(5) : spread(1, 17);
        b.window = upto(4) ? spread(1, 8000) : 0;
        b.sinks = b.window && upto(2) ? spread(1, 300) : 0;
        const int n = upto(3) ? spread(1, 20) : spread(1, 200), new_ = upto(3) ? spread(1, 64) : spread(1, 2000), most = spread(16, 40000 / std::sqrt(n));
        for (int k = 0; k < n; ++k) {
            b.len.push_back(upto(4) ? most : 1 + upto(most));
            b.n.push_back(upto(2) ? new_ : upto(new_ + 1));
            if (upto(8)) b.n.back() = std::min(b.n.back(), b.len.back());
        }
        b.entries = std::max((most + b.page - 1) / b.page - (upto(5) == 0 ? 1 : 0), 1);
        b.max_len = upto(3) ? std::min(most, b.entries * b.page) : b.entries * b.page;
        if (upto(6) == 0) b.max_len = std::max(b.max_len / 3, 1);
        look(b);
    }
    printf("%lld batches, %lld cut, %lld tiles, %lld faults\n", static_cast<long long>(batches), static_cast<long long>(g_cut), static_cast<long long>(g_tiles),
           static_cast<long long>(g_bad));
    return 0;
}
