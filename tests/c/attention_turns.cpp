// Every interleaving of the attention kernel's two issuing warps over sequences of pieces, by the rules of
// csrc/geocache_attention_turns.h.  A barrier is what the hardware has: a phase count of which a wait sees the parity.
// Exits 0 when no wait can stop for good and none can pass early; else prints the pieces and exits 1.
#include <cstdio>
#include <vector>

#include "geocache_attention_turns.h"

struct Op {
    bool wait;
    int bar;  // turn[bar]
};

// What warp t does with the barriers over the pieces (goes of tile 0, goes of tile 1).
static std::vector<Op> program(const std::vector<std::pair<int, int>>& pieces, int t) {
    std::vector<Op> ops;
    bool first = true;
    for (const auto& p : pieces) {
        const int n = t ? p.second : p.first, n_other = t ? p.first : p.second;
        for (int j = 0; j < n; ++j) {
            if (geocache::turn_taken(t, j, n_other, first)) ops.push_back({true, t});
            if (geocache::turn_given(t, j, n_other)) ops.push_back({false, t ^ 1});
        }
        if (n > 0 && n_other > 0) first = false;
    }
    return ops;
}

// Walks all states (place of warp 0, place of warp 1).
static bool sound(const std::vector<std::pair<int, int>>& pieces) {
    const std::vector<Op> ops[2] = {program(pieces, 0), program(pieces, 1)};
    // waits on and arrivals at turn[t] before place i: turn[t] is waited for by warp t and arrived at by the other
    std::vector<int> waits[2], given[2];
    for (int t = 0; t < 2; ++t) {
        int w = 0, g = 0;
        for (const Op& o : ops[t]) {
            waits[t].push_back(w);
            given[t].push_back(g);
            (o.wait ? w : g) += 1;
        }
        waits[t].push_back(w);
        given[t].push_back(g);
    }
    const size_t n0 = ops[0].size(), n1 = ops[1].size();
    std::vector<char> seen((n0 + 1) * (n1 + 1), 0);
    std::vector<std::pair<size_t, size_t>> todo{{0, 0}};
    seen[0] = 1;
    while (!todo.empty()) {
        const auto at = todo.back();
        todo.pop_back();
        const size_t place[2] = {at.first, at.second};
        bool moved = false;
        for (int t = 0; t < 2; ++t) {
            if (place[t] == ops[t].size()) continue;
            const Op& o = ops[t][place[t]];
            if (o.wait) {
                const int k = waits[t][place[t]], phase = given[t ^ 1][place[t ^ 1]];
                const bool passes = ((phase ^ k) & 1) != 0;  // the phase of parity k is not the current one
                if (passes && phase < k + 1) return false;   // before its turn was given
                if (phase > k + 1) return false;             // two turns ahead: the parity says the wrong thing
                if (!passes) continue;
            }
            moved = true;
            const size_t a = place[0] + (t == 0), b = place[1] + (t == 1);
            if (!seen[a * (n1 + 1) + b]) {
                seen[a * (n1 + 1) + b] = 1;
                todo.push_back({a, b});
            }
        }
        if (!moved && (place[0] < n0 || place[1] < n1)) return false;  // nobody can go on
    }
    return true;
}

int main() {
    // pieces by their goes: two tiles (tile 0 has no more than tile 1), one tile, none
    const std::pair<int, int> kinds[] = {{1, 1}, {2, 2}, {3, 3}, {1, 2}, {1, 3}, {2, 3}, {0, 2}, {2, 0}, {0, 0}};
    const int n = sizeof(kinds) / sizeof(kinds[0]);
    for (int a = 0; a < n; ++a)
        for (int b = 0; b < n; ++b)
            for (int c = 0; c < n; ++c)
                for (int d = 0; d < n; ++d) {
                    const std::vector<std::pair<int, int>> pieces{kinds[a], kinds[b], kinds[c], kinds[d]};
                    if (sound(pieces)) continue;
                    for (const auto& p : pieces) std::printf("(%d, %d) ", p.first, p.second);
                    std::printf("\n");
                    return 1;
                }
    return 0;
}
