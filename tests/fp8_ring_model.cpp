// The barriers of the 8-bit layer's kernels (csrc/fwd_fp8.cu) as one CTA or pair uses them, in a model that runs its warps in many orders; what a
// loader waits for behind its last request is the kernels' own (csrc/fp8_ring.h).
//
// A wait by parity passes where the phase it asks for, or one that differs from it by an even number, has ended; the model knows which
// phase is meant.  Copies land in any order.  MMAs complete in the order of their issue; each commit behind them is an arrival of its own, in
// each CTA of a pair, that comes at any time after.  Errors: a warp that passes before its phase, all warps waiting, and copies or arrivals still to
// come when the last warp has ended (the CTA's shared memory is then another CTA's).
//   With `withheld` >= 0 the copies of that group do not land, and a wait gives up when nothing else can happen: then all the others have to end too
// (what was started is given time at the CTA's end).
//
// Usage: fp8_ring_model <pair 0 | 1> <places> <buffers> <groups of a buffer> <groups> <tiles> <withheld> <seeds>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2410_09615_b200/csrc/fp8_ring.h"

namespace {

using namespace slim;

struct Barrier {
    int count = 0, pending = 0, bytes = 0, phases = 0;
    void init(int n) { count = pending = n; }
    void settle() { if (pending == 0 && bytes == 0) { ++phases; pending = count; } }
    bool passes(int phase) const { return (phases & 1) != (phase & 1); }
};

struct Shape { int pair, places, buffers, batch, groups, tiles, withheld; };
int ctas(const Shape& s) { return s.pair ? 2 : 1; }

// Where a warp goes on behind a wait that gave up: SKIP: the next operation, GIVE_UP: its end (loaders).
enum Kind { WAIT, ARRIVE, EXPECT, COPY, COMMIT };
enum Failing { SKIP, GIVE_UP };
struct Op { Kind kind; int cta, bar, n; Failing failing; int group; };

struct Warp {
    std::vector<Op> ops;
    size_t at = 0;
    int cta = 0, requested = 0;         // groups a loader has asked for
    bool loader = false, drains = false;
    void add(Kind k, int to, int bar, int n, Failing f = SKIP, int group = -1) { ops.push_back({k, to, bar, n, f, group}); }
};

int full(const Shape&, int g_place) { return g_place; }
int empty(const Shape& s, int place) { return s.places + place; }
int acc_full(const Shape& s, int buf) { return 2 * s.places + buf; }
int acc_empty(const Shape& s, int buf) { return 2 * s.places + s.buffers + buf; }

std::vector<Warp> warps_of(const Shape& s) {
    const int total = s.tiles * s.groups;
    std::vector<Warp> all;
    for (int cta = 0; cta < ctas(s); ++cta) {
        for (int tokens = 0; tokens < 2; ++tokens) {             // loaders; the announcement is the even CTA's tokens' (single CTAs: one of the two)
            Warp w;
            w.cta = cta; w.loader = true;
            for (int g = 0; g < total; ++g) {
                if (g >= s.places) w.add(WAIT, cta, empty(s, g % s.places), g / s.places - 1, GIVE_UP);
                if (tokens && cta == 0) w.add(EXPECT, 0, full(s, g % s.places), 2 * ctas(s));
                w.add(COPY, 0, full(s, g % s.places), 1, SKIP, g);
            }
            all.push_back(w);
        }
        for (int warp = 0; warp < 4; ++warp) {                   // accumulation
            Warp w;
            w.cta = cta;
            for (int t = 0, n = 0; t < s.tiles; ++t)
                for (int g = 0; g < s.groups; g += s.batch, ++n) {
                    w.add(WAIT, cta, acc_full(s, n % s.buffers), n / s.buffers);
                    w.add(ARRIVE, 0, acc_empty(s, n % s.buffers), 1);
                }
            all.push_back(w);
        }
    }
    Warp mma;
    for (int t = 0, n = 0, at = 0; t < s.tiles; ++t)
        for (int g = 0; g < s.groups; ++g, ++at) {
            if (g % s.batch == 0 && n >= s.buffers) mma.add(WAIT, 0, acc_empty(s, n % s.buffers), n / s.buffers - 1);
            mma.add(WAIT, 0, full(s, at % s.places), at / s.places);
            if (g % s.batch + 1 == s.batch || g + 1 == s.groups) { mma.add(COMMIT, 0, acc_full(s, n % s.buffers), 1); ++n; }
            mma.add(COMMIT, 0, empty(s, at % s.places), 1);
        }
    all.push_back(mma);
    return all;
}

// Returns nullptr, or what went wrong.
const char* run(const Shape& s, const std::vector<Warp>& program, unsigned seed) {
    std::mt19937 rng(seed);
    std::vector<Warp> warps = program;
    std::vector<Barrier> bars[2];
    for (int cta = 0; cta < 2; ++cta) {
        bars[cta].resize(2 * s.places + 2 * s.buffers);
        for (int i = 0; i < s.places; ++i) { bars[cta][full(s, i)].init(1); bars[cta][empty(s, i)].init(1); }
        for (int i = 0; i < s.buffers; ++i) { bars[cta][acc_full(s, i)].init(1); bars[cta][acc_empty(s, i)].init(4 * ctas(s)); }
    }
    struct Event { int cta, bar; bool copy, held; };
    std::vector<Event> coming;
    bool aborted = false;
    std::vector<unsigned> prio(warps.size() + 1);
    for (auto& p : prio) p = rng();
    // A loader that has made its last request goes on to its last waits.
    auto drain = [&](Warp& w) {
        w.drains = true;
        w.ops.clear(); w.at = 0;
        for (int g = ring_tail(w.requested, s.places); g < w.requested; ++g) w.add(WAIT, w.cta, empty(s, g % s.places), g / s.places, GIVE_UP);
    };
    for (;;) {
        int best = -1;
        bool left = false;
        for (size_t i = 0; i < warps.size(); ++i) {
            Warp& w = warps[i];
            if (w.at == w.ops.size() && w.loader && !w.drains) drain(w);
            if (w.at == w.ops.size()) continue;
            left = true;
            const Op& o = w.ops[w.at];
            const bool can = o.kind != WAIT || bars[o.cta][o.bar].passes(o.n) || aborted;
            if (can && (best < 0 || prio[i] > prio[best])) best = (int)i;
        }
        std::vector<size_t> ready;
        for (size_t i = 0; i < coming.size(); ++i) if (!coming[i].held) ready.push_back(i);
        if (!left) return coming.empty() || aborted ? nullptr : "in flight when the last warp has ended";
        if (!ready.empty() && (best < 0 || prio.back() > prio[best])) best = (int)warps.size();
        if (best < 0) {                                          // nothing can happen: a wait gives up
            if (s.withheld < 0) return "all wait";
            aborted = true;
            continue;
        }
        if (rng() % 16 == 0) prio[best] = rng();
        if (best == (int)warps.size()) {
            const size_t i = ready[rng() % ready.size()];
            Barrier& b = bars[coming[i].cta][coming[i].bar];
            if (coming[i].copy) --b.bytes; else --b.pending;
            b.settle();
            coming.erase(coming.begin() + i);
            if (b.pending < 0 && !aborted) return "an arrival too many";
            continue;
        }
        Warp& w = warps[best];
        const Op o = w.ops[w.at++];
        Barrier& b = bars[o.cta][o.bar];
        switch (o.kind) {
        case WAIT:
            if (!b.passes(o.n)) {                                // gave up
                if (o.failing == GIVE_UP) w.at = w.ops.size();
            } else if (!aborted && b.phases <= o.n) return "passed before the phase";
            break;
        case ARRIVE: --b.pending; b.settle(); break;
        case EXPECT: b.bytes += o.n; --b.pending; b.settle(); break;
        case COPY: ++w.requested; coming.push_back({o.cta, o.bar, true, o.group == s.withheld}); break;
        case COMMIT: for (int cta = 0; cta < ctas(s); ++cta) coming.push_back({cta, o.bar, false, false}); break;
        }
        if (b.pending < 0 && !aborted) return "an arrival too many";
    }
}

}  // namespace

int main(int argc, char** argv) {
    if (argc != 9) { fprintf(stderr, "usage: %s pair places buffers groups_of_a_buffer groups tiles withheld seeds\n", argv[0]); return 2; }
    auto arg = [&](int i) { return atoi(argv[i]); };
    const Shape s{arg(1), arg(2), arg(3), arg(4), arg(5), arg(6), arg(7)};
    const std::vector<Warp> program = warps_of(s);
    for (unsigned seed = 1; seed <= (unsigned)arg(8); ++seed)
        if (const char* what = run(s, program, seed)) { printf("seed %u: %s\n", seed, what); return 1; }
    printf("ok\n");
    return 0;
}
