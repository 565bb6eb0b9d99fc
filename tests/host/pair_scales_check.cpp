// Host-only check of the hand-over of scale words inside a pair of CTAs: every order of steps is walked through, for lines of 0 to 14 blocks.
// Four writing warps in turn, the passing warps and the issuer, with barriers that are waited for by parity as on the GPU.  Every order has to
// end with all blocks multiplied, each with its own words, behind a fence of the warp that passed them on; a rule that forgets the half-full
// group at the end, a fence, or the issuer's hold on a stage has to be found out.
#include <cstdio>
#include <set>
#include <string>
#include <vector>

#include "pair_scales.h"

struct Rule {
    bool flush = true, fence = true, hold = true;
};

constexpr int S = uoe::kPairStages, W = uoe::kPassWarps, WRITERS = 4;

struct State {
    signed char writer[WRITERS];        // next block of each writing warp
    signed char pass[W];                // next block that each passing warp waits for
    signed char sent[W];                // arrivals it still owes: blocks [pass - sent, pass)
    signed char issued = 0;             // blocks multiplied
    signed char ready[S], full[S];      // completed phases of the barriers
    signed char words[S], fenced[S];    // block whose words lie in the stage; block that a passing warp's fence stands behind
    std::string key() const { return std::string((const char*)this, sizeof(*this)); }
};

struct Walk {
    Rule rule;
    int N;
    std::set<std::string> seen;
    int bad = 0;

    static bool passes(int completed, int use) { return (completed & 1) != (use & 1); }       // a wait by parity for the use-th phase
    int next_of(int w, int b) const {                                                         // first block >= b of passing warp w
        while (b < N && uoe::pass_warp(b % S) != w) ++b;
        return b;
    }
    void go(const State& s) {
        if (bad || !seen.insert(s.key()).second) return;
        bool moved = false, done = s.issued == N;
        for (int i = 0; i < WRITERS; ++i) {
            const int b = s.writer[i], st = b % S, use = b / S;
            if (b >= N) continue;
            done = false;
            // the stage's last use has been multiplied: phases of `empty` are issued blocks of this stage
            const int emptied = (s.issued + S - 1 - st) / S;
            if (rule.hold && !passes(emptied, use - 1 < 0 ? 1 : use - 1) && use > 0) continue;
            if (rule.hold && use > 0 && emptied < use) { bad = 1; return; }
            if (s.words[st] >= 0 && s.words[st] >= s.issued) { bad = 2; return; }              // written over before it was read
            State t = s;
            t.words[st] = (signed char)b;
            ++t.ready[st];
            t.writer[i] = (signed char)(b + WRITERS);
            moved = true;
            go(t);
        }
        for (int w = 0; w < W; ++w) {
            if (s.sent[w] > 0) {
                done = false;
                State t = s;
                const int b = s.pass[w] - 1, q = uoe::pass_first(b % S) + (b % S - uoe::pass_first(b % S) + 1 - s.sent[w]);
                ++t.full[q];
                --t.sent[w];
                moved = true;
                if (t.sent[w] == 0) t.pass[w] = (signed char)next_of(w, s.pass[w]);
                go(t);
                continue;
            }
            const int b = s.pass[w], st = b % S;
            if (b >= N) continue;
            done = false;
            if (!passes(s.ready[st], b / S)) continue;
            if (s.ready[st] != b / S + 1) { bad = 3; return; }                                // looked a whole turn too late
            State t = s;
            moved = true;
            t.pass[w] = (signed char)(b + 1);
            if (uoe::pass_now(st, rule.flush && b == N - 1)) {
                t.sent[w] = (signed char)(st - uoe::pass_first(st) + 1);
                for (int q = uoe::pass_first(st); q <= st; ++q)
                    if (rule.fence) t.fenced[q] = (signed char)(b - (st - q));
            } else {
                t.pass[w] = (signed char)next_of(w, b + 1);
            }
            go(t);
        }
        if (s.issued < N) {
            const int b = s.issued, st = b % S;
            if (passes(s.full[st], b / S)) {
                if (s.full[st] != b / S + 1) { bad = 4; return; }
                if (s.words[st] != b || s.fenced[st] != b) { bad = 5; return; }
                State t = s;
                ++t.issued;
                moved = true;
                go(t);
            }
        }
        if (!done && !moved) bad = 6;
    }
    int run(int blocks) {
        N = blocks;
        bad = 0;
        seen.clear();
        State s = {};
        for (int i = 0; i < WRITERS; ++i) s.writer[i] = (signed char)i;
        for (int i = 0; i < S; ++i) s.words[i] = s.fenced[i] = -1;
        for (int w = 0; w < W; ++w) s.pass[w] = (signed char)next_of(w, 0);
        go(s);
        return bad;
    }
};

int main() {
    Walk v;
    size_t states = 0;
    for (int n = 0; n <= 14; ++n) {
        if (const int bad = v.run(n)) { std::printf("%d blocks: %d\n", n, bad); return 1; }
        states += v.seen.size();
    }
    std::printf("%zu states\n", states);
    v.rule = Rule{false, true, true};
    if (v.run(7) != 6) return 2;
    v.rule = Rule{true, false, true};
    if (v.run(4) != 5) return 3;
    v.rule = Rule{true, true, false};
    if (!v.run(9)) return 4;
    std::printf("ok\n");
    return 0;
}
