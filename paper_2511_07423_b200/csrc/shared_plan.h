// The host planner of attention over shared prefixes (no device): which keys which query tokens meet together, cut into work
// items of equal time, and where the items' partial results lie.
//
// Requests next to each other in the batch whose page tables begin with the same pages, all of them full and cached for either,
// share those keys.  The common pages of neighbours form a tree: a run of requests, its common prefix, and within the run
// shorter runs that have more in common.  Every node is one set of (tokens of the run) x (keys beyond the parent's); a leaf
// is a request with what only it sees, its chunk among that.  A token's keys are those of its path from the root, each once.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <vector>

namespace syn {

constexpr int SHARED_STAGE = 128;        // keys of a stage
constexpr int SHARED_TILE_ROWS = 128;    // rows (token, query head of the kv head) of a tile; an item has one tile or two
constexpr int SHARED_NO_LIMIT = 0x3FFFFFFF;   // q_pos0 of an item whose rows see all of its keys

struct SharedItem {
    int q_tok, n_tok;        // query tokens
    int kvh, req;            // kv head; the request whose page table names the keys
    int kv_begin, kv_end;    // keys (the first a multiple of 16)
    int q_pos0;              // token j sees keys <= q_pos0 + j
    int base;                // its first row of partial results: row (j, g) at base + j * G + g
    int mode;                // who works on it, SharedMode
    int pad0, pad1, pad2;
};

// The kernel has two groups of warps.  One tile of rows and few stages: the whole item is one group's, while the other has another
// item.  One tile and many stages: the groups take alternate stages, and the second's partial results lie n_tok * G rows behind
// the first's.  Two tiles: a tile each, over every stage.
enum SharedMode { SHARED_GROUP0 = 0, SHARED_GROUP1 = 1, SHARED_TILES = 2, SHARED_STAGES = 3 };
constexpr int SHARED_SOLO_STAGES = 4;    // most stages of an item that one group takes alone

// Cycles of an item by its stages, and of a launch with its merge: where requests share keys, besides for each partial row, which
// deeply nested prefixes leave many of.
struct SharedCost {
    int tiles_stage, tiles_item;     // two tiles
    int stages_stage, stages_item;   // one tile, both groups
    int solo_stage, solo_item;       // one tile, one group; the other group's items run beside it
    int fixed;                       // nothing is shared
    int fixed_shared, row_256;       // (of 256 rows)
    int64_t of(int tiles, int stages) const {
        return tiles == 2 ? (int64_t)stages * tiles_stage + tiles_item
                          : stages <= SHARED_SOLO_STAGES ? (int64_t)stages * solo_stage + solo_item : (int64_t)stages * stages_stage + stages_item;
    }
    // most stages whose item takes no more than `room`
    int fit(int tiles, int64_t room) const {
        if (tiles == 2) return (int)std::max<int64_t>(0, (room - tiles_item) / tiles_stage);
        const int64_t n = (room - stages_item) / stages_stage;
        return n > SHARED_SOLO_STAGES ? (int)n : (int)std::min<int64_t>(SHARED_SOLO_STAGES, std::max<int64_t>(0, (room - solo_item) / solo_stage));
    }
};

struct SharedPlan {
    bool shares = false;                 // some keys are met by several requests' tokens
    int n_cta = 0;
    int64_t rows = 0;                    // rows of partial results
    int64_t estimate = 0;                // cycles
    int64_t kv_keys = 0;                 // keys read, each node's once (per kv head)
    std::vector<SharedItem> items;       // by CTA
    std::vector<int> cta_begin;
    // where a token's partial results are: segment of the token; of (segment, kv head) the rows of the segment's first token
    std::vector<int> seg_of_token, seg_first, list_begin, list;
};

struct SharedNode { int a, b, from, to; };   // requests [a, b), pages [from, to); to < 0: the leaf of request a

// The tree, as the list of its nodes; least: pages from which on a common prefix is worth a node.
inline std::vector<SharedNode> shared_tree(int n_req, const int* page_tables, int max_pages, const int* ctx_lens, int page_size, int least) {
    std::vector<int> common(n_req, 0);       // pages that i and i + 1 share
    for (int i = 0; i + 1 < n_req; ++i) {
        const int most = std::min(ctx_lens[i], ctx_lens[i + 1]) / page_size;
        const int *p = page_tables + (size_t)i * max_pages, *q = p + max_pages;
        int k = 0;
        while (k < most && p[k] == q[k]) ++k;
        common[i] = k;
    }
    std::vector<SharedNode> nodes;
    struct Run { int a, b, from; };
    std::vector<Run> todo = {{0, n_req, 0}};
    while (!todo.empty()) {
        const Run r = todo.back();
        todo.pop_back();
        if (r.b - r.a == 1) {
            nodes.push_back({r.a, r.b, r.from, -1});
            continue;
        }
        const int s = *std::min_element(common.begin() + r.a, common.begin() + r.b - 1);
        int from = r.from;
        if (s - from >= least) {
            nodes.push_back({r.a, r.b, from, s});
            from = s;
        }
        int end = r.b;                        // pushed back to front: taken front to back
        for (int i = r.b - 2; i >= r.a; --i)
            if (common[i] == s) {
                todo.push_back({i + 1, end, from});
                end = i + 1;
            }
        todo.push_back({r.a, end, from});
    }
    return nodes;
}

// Most rows of partial results of a plan.  A node leaves one for every token and query head of its run, so deeply nested prefixes would
// leave as many as there are levels, at (4 head_dim + 8) bytes each (512 requests of 8 tokens and 32 heads of 128, each sharing 128 keys more with the next:
// 33.7 M rows, 17.6 GB, for an output of 34 MB).  Eight rows an output row are more than two or three levels and the cuts between CTAs
// ask for; half a million (273 MB with heads of 128) leave room for the parts of few rows on very many keys.
inline int64_t shared_most_rows(int64_t out_rows) { return std::max<int64_t>((int64_t)1 << 19, 8 * out_rows); }

inline void shared_cut(const std::vector<SharedNode>& nodes, int n_req, const int* chunk_offsets, const int* ctx_lens, int page_size,
                       int group, int n_kv_heads, int n_sm, const SharedCost& cost, SharedPlan& sp) {
    const int T = chunk_offsets[n_req], tile_tokens = SHARED_TILE_ROWS / group;
    // units: a node's tokens in items of at most two tiles
    struct Unit { int q_tok, n_tok, req, kv_begin, kv_end, q_pos0, tiles, stages; int64_t time; };
    std::vector<Unit> units;
    std::vector<int> cuts = {0, T};
    for (const SharedNode& nd : nodes) {
        const bool leaf = nd.to < 0;
        const int t0 = chunk_offsets[nd.a], t1 = chunk_offsets[nd.b];
        const int kv0 = nd.from * page_size, kv1 = leaf ? ctx_lens[nd.a] + (t1 - t0) : nd.to * page_size;
        sp.shares = sp.shares || !leaf;
        sp.kv_keys += kv1 - kv0;
        for (int t = t0; t < t1; t += 2 * tile_tokens) {
            const int n = std::min(2 * tile_tokens, t1 - t);
            // a leaf's tokens see keys up to their own position; those of its first tiles need not read what only later ones see
            const int end = leaf ? ctx_lens[nd.a] + (t - t0) + n : kv1;
            Unit u = {t, n, nd.a, kv0, end, leaf ? ctx_lens[nd.a] + (t - t0) : SHARED_NO_LIMIT, n > tile_tokens ? 2 : 1, (end - kv0 + SHARED_STAGE - 1) / SHARED_STAGE, 0};
            u.time = cost.of(u.tiles, u.stages);
            units.push_back(u);
            cuts.push_back(t);
            cuts.push_back(t + n);
        }
    }
    std::stable_sort(units.begin(), units.end(), [](const Unit& x, const Unit& y) { return x.time > y.time; });
    int64_t total = 0, longest = 0;
    for (const Unit& u : units) {
        total += u.time * n_kv_heads;
        longest = std::max(longest, u.time);
    }
    // The units one after the other, longest first, each CTA filled up to `limit`; what does not fit goes on in the next CTA.
    auto fill = [&](int64_t limit, auto&& emit) {
        int cta = 0;
        int64_t load = 0;
        for (const Unit& u : units)
            for (int h = 0; h < n_kv_heads; ++h)
                for (int at = 0; at < u.stages;) {
                    int take = std::min(u.stages - at, cost.fit(u.tiles, limit - load));
                    if (take < u.stages - at && take < 2) take = 0;      // no slivers
                    if (take == 0 && load == 0) return false;
                    if (take) {
                        emit(u, h, at, at + take, cta);
                        load += cost.of(u.tiles, take);
                        at += take;
                    }
                    if (at < u.stages) {
                        load = 0;
                        if (++cta >= n_sm) return false;
                    }
                }
        return true;
    };
    auto nothing = [](const Unit&, int, int, int, int) {};
    int64_t lo = total / n_sm, hi = std::max(lo, longest);
    while (!fill(hi, nothing)) hi += hi / 4;
    while (hi - lo > 64 + lo / 128) {
        const int64_t mid = (lo + hi) / 2;
        if (fill(mid, nothing)) hi = mid; else lo = mid;
    }
    std::vector<int> owner, solo(n_sm, 0);   // (a CTA's items of one group: the groups in turn)
    // parts of (unit, head), for the lists below
    struct Part { int unit, h, base, second; };
    std::vector<Part> parts;
    fill(hi, [&](const Unit& u, int h, int s0, int s1, int cta) {
        const int mode = u.tiles == 2 ? SHARED_TILES : s1 - s0 > SHARED_SOLO_STAGES ? SHARED_STAGES : solo[cta]++ & 1;
        const int rows = u.n_tok * group, copies = mode == SHARED_STAGES ? 2 : 1;
        sp.items.push_back({u.q_tok, u.n_tok, h, u.req, u.kv_begin + s0 * SHARED_STAGE, std::min(u.kv_end, u.kv_begin + s1 * SHARED_STAGE), u.q_pos0,
                            (int)sp.rows, mode, 0, 0, 0});
        parts.push_back({(int)(&u - units.data()), h, (int)sp.rows, copies == 2 ? (int)sp.rows + rows : -1});
        sp.rows += (int64_t)rows * copies;
        owner.push_back(cta);
    });
    sp.estimate = hi + (sp.shares ? cost.fixed_shared + sp.rows * cost.row_256 / 256 : cost.fixed);
    sp.n_cta = owner.back() + 1;
    sp.cta_begin.assign(sp.n_cta + 1, 0);
    for (int k : owner) sp.cta_begin[k + 1]++;
    for (int k = 0; k < sp.n_cta; ++k) sp.cta_begin[k + 1] += sp.cta_begin[k];
    // segments: tokens between two cuts belong to the same units
    std::sort(cuts.begin(), cuts.end());
    cuts.erase(std::unique(cuts.begin(), cuts.end()), cuts.end());
    const int n_seg = (int)cuts.size() - 1;
    sp.seg_of_token.resize(T);
    sp.seg_first.assign(cuts.begin(), cuts.end() - 1);
    for (int s = 0; s < n_seg; ++s)
        for (int t = cuts[s]; t < cuts[s + 1]; ++t) sp.seg_of_token[t] = s;
    sp.list_begin.assign((size_t)n_seg * n_kv_heads + 1, 0);
    auto each = [&](auto&& f) {
        for (const Part& p : parts) {
            const Unit& u = units[p.unit];
            for (int s = sp.seg_of_token[u.q_tok]; s < n_seg && cuts[s] < u.q_tok + u.n_tok; ++s) f(p, u, s);
        }
    };
    each([&](const Part& p, const Unit&, int s) { sp.list_begin[(size_t)s * n_kv_heads + p.h + 1] += p.second >= 0 ? 2 : 1; });
    for (size_t k = 0; k + 1 < sp.list_begin.size(); ++k) sp.list_begin[k + 1] += sp.list_begin[k];
    sp.list.resize(sp.list_begin.back());
    std::vector<int> at(sp.list_begin.begin(), sp.list_begin.end() - 1);
    each([&](const Part& p, const Unit& u, int s) {
        const int off = (cuts[s] - u.q_tok) * group;
        int& k = at[(size_t)s * n_kv_heads + p.h];
        sp.list[k++] = p.base + off;
        if (p.second >= 0) sp.list[k++] = p.second + off;
    });
}

// Where the tree of all common prefixes would leave too many rows, a common prefix has to be twice as long to be worth a node, and so
// on: in the end nothing is shared.
inline void shared_plan(int n_req, const int* chunk_offsets, const int* page_tables, int max_pages, const int* ctx_lens, int page_size,
                        int group, int n_kv_heads, int n_sm, const SharedCost& cost, SharedPlan& sp) {
    const int64_t heads = (int64_t)group * n_kv_heads, most = shared_most_rows(heads * chunk_offsets[n_req]);
    for (int64_t least = SHARED_STAGE / page_size;; least *= 2) {
        const std::vector<SharedNode> nodes = shared_tree(n_req, page_tables, max_pages, ctx_lens, page_size, (int)least);
        const bool leaves_alone = nodes.size() == (size_t)n_req;
        int64_t rows = 0;   // of one item a node and tile
        for (const SharedNode& nd : nodes) rows += heads * (chunk_offsets[nd.b] - chunk_offsets[nd.a]);
        if (rows > most && !leaves_alone) continue;
        sp = SharedPlan();
        shared_cut(nodes, n_req, chunk_offsets, ctx_lens, page_size, group, n_kv_heads, n_sm, cost, sp);
        if (sp.rows <= most || leaves_alone) return;
    }
}

}  // namespace syn
