// How an attention launch divides its work (host only).
//
// A unit of work is one or two tiles of 128 query rows over the key tiles that they see.  Units go to thread blocks
// whole, the longest first to the block with the least (no joins); or they are cut along their keys, and the parts of a
// unit are joined by a second kernel: whole as long as they fit into an even share, the rest cut to fill the blocks up,
// or, where less than a quarter of the work is in units that fit so, all in order with the boundaries between the blocks
// falling where the costs are even.  The whole and the cut layout are made with one and with two tiles a unit, and the
// cheapest by the model below is kept.  The model counts time on the SMs and no bytes: where HBM bounds the launch (few
// rows, long keys) it is too low, which is why the two ways of cutting are told apart by the quarter and not by it.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <numeric>
#include <queue>
#include <vector>

#include "geocache.h"
#include "geocache_internal.h"

namespace {

using geocache::AttentionItem;
using geocache::AttentionJoin;
constexpr int kRows = geocache::kAttentionRows, kKeys = geocache::kAttentionKeys;

// Nanoseconds, measured with 152 equal pieces of 1 to 64 key tiles and runs of short pieces: a key tile for two query
// tiles, for one; a piece's start and end, and that of each of its full tiles of rows; a launch that joins, and its
// reading a tile's part (times D).
struct Cost {
    double two, one, piece, tile, join, join_slot;
};

Cost cost_of(int D) {
    if (D > 64) return {1450.0, 1020.0, 1200.0, 10.0 * D, 4000.0, 0.06};
    return {1140.0, 960.0, 900.0, 10.0 * D, 4000.0, 0.06};
}

struct Unit {
    int seq, head, kv_head;
    int token;        // first token of the sequence's queries
    int n_tok[2];
    int n_kv[2];      // key tiles each sees
    int most() const { return std::max(n_kv[0], n_kv[1]); }
    // cost of a piece beside its key tiles: its rows' queries and output
    double start(const Cost& c, int pack) const { return c.piece + c.tile * (n_tok[0] + n_tok[1]) * pack / kRows; }
    // cost of the key tiles [a, b)
    double cost(const Cost& c, int a, int b) const {
        const int both = std::min(n_tok[1] ? std::min(n_kv[0], n_kv[1]) : 0, b);
        const int pairs = std::max(0, both - a);
        return pairs * c.two + (b - a - pairs) * c.one;
    }
};

struct Piece {
    int unit, from, to;
};

struct Layout {
    int tiles = 0;
    std::vector<Unit> units;
    std::vector<std::vector<Piece>> of_cta;
    double cost = 0.0;
};

struct Problem {
    const int32_t *q, *k;
    int n_seq, Hq, Hk, D, causal, n_ctas, pack;
};

std::vector<Unit> make_units(const Problem& p, int tiles) {
    const int tok = kRows / p.pack, groups = p.Hq / p.Hk / p.pack;
    std::vector<Unit> units;
    // heads inside of tokens where one row of tiles has all tokens: their units may be divided together (assign_even)
    auto add = [&](int s, int hk, int g, long long t) {
        Unit u{s, hk * (p.Hq / p.Hk) + g * p.pack, hk, (int)t, {0, 0}, {0, 0}};
        for (int i = 0; i < tiles; ++i) {
            const long long first = t + (long long)i * tok;
            u.n_tok[i] = (int)std::max(0LL, std::min<long long>(tok, p.q[s] - first));
            if (!u.n_tok[i]) continue;
            long long sees = p.k[s];
            if (p.causal) sees = std::max(0LL, first + u.n_tok[i] + p.k[s] - p.q[s]);
            u.n_kv[i] = (int)((sees + kKeys - 1) / kKeys);
        }
        units.push_back(u);
    };
    for (int s = 0; s < p.n_seq; ++s) {
        const long long step = (long long)tok * tiles;
        if (p.q[s] <= step) {
            for (int hk = 0; hk < p.Hk && p.q[s] > 0; ++hk)
                for (int g = 0; g < groups; ++g) add(s, hk, g, 0);
        } else {
            for (int hk = 0; hk < p.Hk; ++hk)
                for (int g = 0; g < groups; ++g)
                    for (long long t = 0; t < p.q[s]; t += step) add(s, hk, g, t);
        }
    }
    return units;
}

// Whole units, the longest first, each to the block with the least: blocks that run at the same time have units of the
// same heads, whose keys stay in the L2 (24,576 tokens x 16 heads of 128: 2.90 ms, 2.72 with `fill`; 3.63 with the units in
// order over the blocks, all heads at once).  With `fill`, only those that an even share has room for; the others are cut along their
// keys, over the blocks' rests.
void assign_whole(const Problem& p, const Cost& c, Layout& l, bool fill) {
    std::vector<double> cost(l.units.size());
    double total = 0.0, start = 0.0;
    for (size_t i = 0; i < cost.size(); ++i) {
        total += cost[i] = l.units[i].start(c, p.pack) + l.units[i].cost(c, 0, l.units[i].most());
        start = std::max(start, l.units[i].start(c, p.pack));
    }
    const double share = (total + (p.n_ctas - 1) * start) / p.n_ctas;
    std::vector<int> order(l.units.size()), rest;
    std::iota(order.begin(), order.end(), 0);
    std::stable_sort(order.begin(), order.end(), [&](int a, int b) { return cost[a] > cost[b]; });
    using Load = std::pair<double, int>;
    std::priority_queue<Load, std::vector<Load>, std::greater<Load>> least;
    std::vector<double> load(p.n_ctas, 0.0);
    for (int i = 0; i < p.n_ctas; ++i) least.push({0.0, i});
    l.of_cta.assign(p.n_ctas, {});
    for (int i : order) {
        Load x = least.top();
        if (fill && x.first + cost[i] > share) {
            rest.push_back(i);
            continue;
        }
        least.pop();
        l.of_cta[x.second].push_back({i, 0, l.units[i].most()});
        x.first += cost[i];
        load[x.second] = x.first;
        least.push(x);
    }
    int cta = 0;
    double slots = 0.0, room = share - load[0], spent = 0.0;  // of the blocks up to `cta` (roundings do not add up)
    for (int i : rest) {
        const Unit& u = l.units[i];
        const int n = u.most();
        const double own = u.start(c, p.pack);
        int at = 0;
        do {
            const bool final = cta == p.n_ctas - 1;
            const double left = room - spent - own;
            int take = n - at;
            if (!final && u.cost(c, at, n) > left) {
                int fit = 0;
                double sum = 0.0;
                while (at + fit < n) {
                    const double next = u.cost(c, at + fit, at + fit + 1);
                    if (sum + 0.5 * next > left) break;
                    sum += next;
                    ++fit;
                }
                if (u.cost(c, at + fit, n) > 0.5 * own) take = fit;
            }
            if (take > 0 || n == at) {
                l.of_cta[cta].push_back({i, at, at + take});
                load[cta] += own + u.cost(c, at, at + take);
                spent += own + u.cost(c, at, at + take);
                if (take < n) slots += (u.n_tok[0] + u.n_tok[1]) * (double)p.pack / kRows;
                at += take;
            }
            if (at < n && !final) room += share - load[++cta];
        } while (at < n);
    }
    for (double x : load) l.cost = std::max(l.cost, x);
    if (slots > 0.0) l.cost += c.join + slots * c.join_slot * p.D;
}

// Units in order, cut where the blocks' costs are even.  Where a head's row is not whole 128-byte lines, units longer than
// a block's share are taken in ranges of their keys, the same range of all heads of a sequence before the next one: blocks
// that run at the same time then read the two heads of a line (22 rows over 98,304 keys of 72: 266 -> 218 us).  Whole
// lines have nothing to share, and the ranges cost pieces (32 single tokens over 298,000 keys of 128: 99 -> 102 us).
void assign_even(const Problem& p, const Cost& c, Layout& l) {
    double total = 0.0, starts = 0.0, start = 0.0;
    for (const Unit& u : l.units) {
        total += u.cost(c, 0, u.most());
        starts += u.start(c, p.pack);
        start = std::max(start, u.start(c, p.pack));
    }
    l.of_cta.assign(p.n_ctas, {});
    double share = (total + starts + (p.n_ctas - 1) * start) / p.n_ctas;
    std::vector<Piece> order;
    for (size_t i = 0; i < l.units.size();) {
        // the units of one sequence and one row of tiles, whatever their heads
        size_t end = i;
        while (end < l.units.size() && l.units[end].seq == l.units[i].seq && l.units[end].token == l.units[i].token) ++end;
        const int n = l.units[i].most();
        const int ranges = p.D % 64 ? std::max(1, std::min(n, (int)std::ceil(l.units[i].cost(c, 0, n) / share))) : 1;
        for (int r = 0; r < ranges; ++r)
            for (size_t j = i; j < end; ++j) {
                if (r) starts += l.units[j].start(c, p.pack);
                order.push_back({(int)j, (int)((long long)n * r / ranges), (int)((long long)n * (r + 1) / ranges)});
            }
        i = end;
    }
    share = (total + starts + (p.n_ctas - 1) * start) / p.n_ctas;
    int cta = 0;
    double load = 0.0, spent = 0.0, slots = 0.0;
    for (const Piece& whole : order) {
        const Unit& u = l.units[whole.unit];
        const int n = whole.to;
        const double own = u.start(c, p.pack);
        int at = whole.from;
        do {
            int take = n - at;
            const double left = share * (cta + 1) - spent - own;  // (not the block's own: roundings do not add up)
            if (cta < p.n_ctas - 1 && u.cost(c, at, n) > left) {
                // the key tiles that fit, to the nearest; a rest of under half a piece's start stays here
                int fit = 0;
                double sum = 0.0;
                while (at + fit < n) {
                    const double next = u.cost(c, at + fit, at + fit + 1);
                    if (sum + 0.5 * next > left) break;
                    sum += next;
                    ++fit;
                }
                if (u.cost(c, at + fit, n) > 0.5 * own) take = load == 0.0 ? std::max(fit, 1) : fit;
            }
            if (take > 0 || n == at) {
                l.of_cta[cta].push_back({whole.unit, at, at + take});
                load += own + u.cost(c, at, at + take);
                spent += own + u.cost(c, at, at + take);
                l.cost = std::max(l.cost, load);
                if (take < u.most()) slots += (u.n_tok[0] + u.n_tok[1]) * (double)p.pack / kRows;
                at += take;
            }
            if (at < n || (spent >= share * (cta + 1) - 0.5 * own && cta < p.n_ctas - 1)) {
                ++cta;
                load = 0.0;
            }
        } while (at < n);
    }
    if (slots > 0.0) l.cost += c.join + slots * c.join_slot * p.D;
}

// the query heads of a key/value head that share a tile: the divisor of their number with the fewest tiles
int choose_pack(const int32_t* q, int n_seq, int group) {
    int best = 1;
    long long least = -1;
    for (int p = 1; p <= group && p <= kRows; ++p) {
        if (group % p) continue;
        const int tok = kRows / p;
        long long tiles = 0;
        for (int s = 0; s < n_seq; ++s) tiles += (q[s] + (long long)tok - 1) / tok;
        tiles *= group / p;
        if (least < 0 || tiles <= least) { least = tiles; best = p; }
    }
    return best;
}

int plan(const Problem& prob, geocache_attention_plan* out, char* schedule, int64_t schedule_bytes) {
    Problem p = prob;
    p.pack = choose_pack(p.q, p.n_seq, p.Hq / p.Hk);
    const Cost c = cost_of(p.D);
    const int tok = kRows / p.pack;
    long long n_units = 0;
    for (int s = 0; s < p.n_seq; ++s) n_units += (p.q[s] + 2LL * tok - 1) / (2 * tok);
    n_units *= p.Hq / p.pack;
    if (n_units > (1LL << 24)) return geocache::set_error(GEOCACHE_ESHAPE, "geocache_plan_attention: over 2^24 pieces of work");
    Layout best;
    for (int tiles = 2; tiles >= 1; --tiles) {
        if (tiles == 1 && n_units > 4LL * p.n_ctas) continue;  // every block has its share of pairs
        Layout l;
        l.tiles = tiles;
        l.units = make_units(p, tiles);
        // Cut what is left over where a good part of the work is in units that fit into a share, else cut all in order.
        // Measured on both sides: continued prompts with a third of it 42.6 us in order and 39.7 so, 32 single tokens with a
        // seventh 99.6 in order and 102.6 so; the quarter lies between.
        double total = 0.0, fitting = 0.0;
        for (const Unit& u : l.units) total += u.start(c, p.pack) + u.cost(c, 0, u.most());
        for (const Unit& u : l.units) {
            const double cost = u.start(c, p.pack) + u.cost(c, 0, u.most());
            if (cost <= total / p.n_ctas) fitting += cost;
        }
        for (int way = 0; way < 2; ++way) {
            Layout x = l;
            if (way == 0 || fitting >= 0.25 * total)
                assign_whole(p, c, x, way == 1);
            else
                assign_even(p, c, x);
            if (!best.tiles || x.cost < best.cost) best = std::move(x);
        }
    }
    // parts of a unit in the order of their keys: tile t takes part in those that begin before the end of what it sees
    std::vector<int> parts[2], slot[2], seen(best.units.size(), 0);
    for (int t = 0; t < 2; ++t) {
        parts[t].assign(best.units.size(), 0);
        slot[t].assign(best.units.size(), -1);
    }
    size_t n_items = 0;
    for (const auto& list : best.of_cta)
        for (const Piece& x : list) {
            const Unit& u = best.units[x.unit];
            ++n_items;
            for (int t = 0; t < 2; ++t)
                if (u.n_tok[t] && (x.from == 0 || x.from < u.n_kv[t])) ++parts[t][x.unit];
        }
    long long n_slots = 0;
    size_t n_joins = 0;
    for (size_t i = 0; i < best.units.size(); ++i)
        for (int t = 0; t < 2; ++t)
            if (parts[t][i] > 1) {
                slot[t][i] = (int)n_slots;
                n_slots += parts[t][i];
                ++n_joins;
            }
    const int64_t bytes = geocache::attention_items_at(p.n_ctas) + 64LL * n_items + 32LL * n_joins;
    if (n_items > (1u << 26) || n_slots > (1LL << 26))
        return geocache::set_error(GEOCACHE_ESHAPE, "geocache_plan_attention: over 2^26 pieces of work");
    out->Hq = p.Hq; out->Hk = p.Hk; out->D = p.D; out->causal = p.causal;
    out->n_ctas = p.n_ctas;
    out->n_items = (int)n_items;
    out->n_joins = (int)n_joins;
    out->pack = p.pack;
    out->q_tokens = std::accumulate(p.q, p.q + p.n_seq, 0LL);
    out->k_tokens = std::accumulate(p.k, p.k + p.n_seq, 0LL);
    out->schedule_bytes = bytes;
    out->workspace_bytes = n_slots * geocache::attention_slot_bytes(p.D);
    if (!schedule) return GEOCACHE_OK;
    if (schedule_bytes < bytes)
        return geocache::set_error(GEOCACHE_EINVAL, "geocache_plan_attention: the schedule takes %lld bytes", (long long)bytes);

    std::vector<long long> q_at(p.n_seq + 1, 0), k_at(p.n_seq + 1, 0);
    for (int s = 0; s < p.n_seq; ++s) {
        q_at[s + 1] = q_at[s] + p.q[s];
        k_at[s + 1] = k_at[s] + p.k[s];
    }
    std::memset(schedule, 0, (size_t)bytes);
    int32_t* ptr = reinterpret_cast<int32_t*>(schedule);
    AttentionItem* item = reinterpret_cast<AttentionItem*>(schedule + geocache::attention_items_at(p.n_ctas));
    AttentionJoin* join = reinterpret_cast<AttentionJoin*>(item + n_items);
    // a unit's pieces come in the order of their keys, block by block: each way fills the blocks one after the other, and
    // ranges of keys come in their order, with other units' pieces between them
    std::vector<int> next[2] = {slot[0], slot[1]};
    int n = 0;
    for (int cta = 0; cta < p.n_ctas; ++cta) {
        ptr[cta] = n;
        for (const Piece& x : best.of_cta[cta]) {
            const Unit& u = best.units[x.unit];
            AttentionItem& o = item[n++];
            const long long key = (long long)x.from * kKeys;
            o.q_row = (int32_t)(q_at[u.seq] + u.token);
            o.head = u.head;
            o.kv_head = u.kv_head;
            o.kv_row = (int32_t)(k_at[u.seq] + key);
            o.n_keys = (int32_t)(p.k[u.seq] - std::min<long long>(key, p.k[u.seq]));
            o.sees = p.causal ? (int32_t)(u.token + 1LL + p.k[u.seq] - p.q[u.seq] - key) : o.n_keys;
            for (int t = 0; t < 2; ++t) {
                o.slot[t] = -1;
                if (!u.n_tok[t] || !(x.from == 0 || x.from < u.n_kv[t])) continue;
                o.n_tok[t] = u.n_tok[t];
                o.n_kv[t] = std::max(0, std::min(x.to, u.n_kv[t]) - x.from);
                if (slot[t][x.unit] >= 0) o.slot[t] = next[t][x.unit]++;
            }
        }
    }
    ptr[p.n_ctas] = n;
    for (size_t i = 0; i < best.units.size(); ++i)
        for (int t = 0; t < 2; ++t)
            if (slot[t][i] >= 0) {
                const Unit& u = best.units[i];
                *join++ = {(int32_t)(q_at[u.seq] + u.token + t * tok), u.n_tok[t], u.head, slot[t][i], parts[t][i], {0, 0, 0}};
            }
    return GEOCACHE_OK;
}

}  // namespace

extern "C" int geocache_plan_attention(const int32_t* q_lens, const int32_t* k_lens, int n_seq, int Hq, int Hk, int D,
                                       int causal, int n_ctas, geocache_attention_plan* out, void* schedule,
                                       int64_t schedule_bytes) {
    const char* fn = "geocache_plan_attention";
    if (!out || (n_seq > 0 && (!q_lens || !k_lens)))
        return geocache::set_error(GEOCACHE_EINVAL, "%s: q_lens, k_lens and plan are required", fn);
    if ((uintptr_t)schedule & 15) return geocache::set_error(GEOCACHE_EINVAL, "%s: schedule must be 16-byte aligned", fn);
    if (n_seq < 0 || Hk < 1 || Hq < Hk || Hq > 65536 || Hq % Hk)
        return geocache::set_error(GEOCACHE_ESHAPE, "%s: n_seq=%d, Hq=%d, Hk=%d out of range", fn, n_seq, Hq, Hk);
    if (D < 8 || D > 128 || D % 8) return geocache::set_error(GEOCACHE_ESHAPE, "%s: D=%d must be a multiple of 8 in [8, 128]", fn, D);
    if (n_ctas < 0 || n_ctas > 65536) return geocache::set_error(GEOCACHE_ESHAPE, "%s: n_ctas=%d out of range", fn, n_ctas);
    long long sum[2] = {0, 0};
    for (int s = 0; s < n_seq; ++s) {
        if (q_lens[s] < 0 || k_lens[s] < 0)
            return geocache::set_error(GEOCACHE_ESHAPE, "%s: sequence %d has a negative length", fn, s);
        sum[0] += q_lens[s];
        sum[1] += k_lens[s];
    }
    if (sum[0] > geocache::kAttentionTokens || sum[1] > geocache::kAttentionTokens)
        return geocache::set_error(GEOCACHE_ESHAPE, "%s: over %lld tokens", fn, geocache::kAttentionTokens);
    if (n_ctas == 0) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&n_ctas, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n_ctas < 1) {
            cudaGetLastError();
            return geocache::set_error(GEOCACHE_EDEVICE, "%s: no device to ask for its SMs (give n_ctas)", fn);
        }
    }
    try {
        geocache_attention_plan p{};
        const int st = plan({q_lens, k_lens, n_seq, Hq, Hk, D, causal != 0, n_ctas, 1}, &p, static_cast<char*>(schedule), schedule_bytes);
        if (p.n_ctas) *out = p;  // the sizes are there when only the schedule did not fit
        if (st) return st;
    } catch (const std::exception&) {
        return geocache::set_error(GEOCACHE_ESHAPE, "%s: the work does not fit in host memory", fn);
    }
    return GEOCACHE_OK;
}
