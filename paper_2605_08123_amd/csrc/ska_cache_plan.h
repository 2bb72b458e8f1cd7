// How the attention on caches is launched: arithmetic on sizes, without anything of the GPU.
#pragma once
#include <algorithm>
#include <cmath>

#include "sinkhorn_attn_cache.h"

namespace {

constexpr int CA_WAVES = 8;   // of a workgroup: they share their rows and split the keys
// Order of the workgroups.  Blocks of the same keys next to each other and a contiguous piece of them per XCD (workgroups go to the XCDs
// in turn): few blocks, a prefix, a band.  Many blocks that walk over most of the keys: those with the longest walks first, problems fastest
// (4096 tokens of 2 items, 8 heads on 2, causal, e4m3, d = 64: 78 us, and 100 as neighbours; 16 heads on 2, int8, d = 128: 178 and 258).
enum CaOrder { CA_NEIGHBOURS, CA_LAST_FIRST };
inline bool scaled(int store) { return store == SKA_E4M3 || store == SKA_INT8; }
// Most blocks of rows of a wavefront: what it has registers for, and two in fp32, whose products take the time of all rows however they are
// dealt (64 items behind 60000, d = 64: 52 us, with four 53)
constexpr int ca_most(bool wide_store, int d) { return wide_store || d == 128 ? 2 : 4; }
struct CaProblem {
    int B, Hq, Hk, Lq, Lp, Lk, d, W, causal, dtype, store;   // Lp 0: no prefix
    int G() const { return Hq / Hk; }
    long R() const { return (long)Lq * G(); }
    long rows() const { return (long)B * Hk * R(); }
};
// How one side is launched: blocks of a problem's rows, those of all problems, tiles that a block reaches at most, parts of a walk, the
// workgroups' order
struct CaGrid { long blocks, units, tiles; int parts, order; };
inline int ca_tile(const CaProblem &p) { return p.store == SKA_F32 ? 16 : 32; }
// Workgroups at a time, one on each CU (a token of 8 items, 4 key heads of d = 128 on 32768 in int8: 60 us, with half of them 79, with twice
// as many 64; eight wavefronts each, and not 16 with half the parts: short caches would wait for the join, 3000 tokens 11.2 us and 12.8)
constexpr long CA_ROOM = 256;
// Keys that a block of an item's rows reaches at most
inline long ca_reach(const CaProblem &p, int nq)
{
    return std::min((long)p.Lk, std::min(16L * nq / p.G() + 1, (long)p.Lq) + (p.causal ? 1L : 2L) * p.W);
}
// Whether an item's workgroups take the prefix too: one launch and nothing to join, but the prefix is read by each.  Few rows, all workgroups
// at a time, and a walk of five tiles a wavefront at most (4 heads on each key head, together and apart; 30 items, 2 key heads: e4m3, d = 64,
// 30 tokens behind 500 7.9 and 11.5 us, 100 behind 1000 9.1 and 11.5; int8, d = 128, 100 behind 2000 19.6 and 16.8; fp32, d = 128, 30 behind
// 500 16.7 and 19.4; one item, 1 key head: 7.3 and 8.9, 8.5 and 9.6, 18.8 and 13.5, 15.8 and 13.2).  Where the items' workgroups fill the CUs
// by themselves, the prefix's would be a second round: eight tiles of a prefix, and any number behind it (2000 behind 1000, 4 key heads, together
// and apart; 64 items: e4m3, d = 64, 19.9 and 24.4, int8, d = 128, 31.8 and 39.1, bf16, d = 64, 27 and 35; 40 items: 16.0 and 15.5, 26.9 and
// 22.8, 23.0 and 20.3)
inline bool ca_together(const CaProblem &p)
{
    if (!p.Lp || p.R() > 16 || (long)p.B * p.Hk > CA_ROOM) return false;
    const long turn = (long)ca_tile(p) * CA_WAVES, front = std::min(p.Lp, p.W);
    return front + ca_reach(p, 1) <= 5 * turn || (8L * p.B * p.Hk >= 7 * CA_ROOM && front <= 8 * turn);
}
// One side of a launch without its parts
inline CaGrid ca_grid(const CaProblem &p, int nq, bool prefix)
{
    const long rows = prefix ? p.R() * p.B : p.R(), L = prefix ? p.Lp : p.Lk, reach = prefix ? std::min(L, (long)p.W) : ca_reach(p, nq);
    CaGrid g;
    g.blocks = (rows + 16 * nq - 1) / (16 * nq);
    g.units = g.blocks * (prefix ? p.Hk : (long)p.B * p.Hk);
    g.tiles = (reach + ca_tile(p) - 1) / ca_tile(p);
    g.order = prefix || g.blocks <= 8 || reach < L / 2 ? CA_NEIGHBOURS : CA_LAST_FIRST;
    g.parts = 1;
    return g;
}
// How a problem is launched
struct CaPlan {
    int nq;             // blocks of rows of a workgroup
    bool both;          // ca_together
    CaGrid own, front;  // front: of the prefix, where it has workgroups of its own
    int parts;          // of both sides
    long wgs() const { return own.units * own.parts + 7 + front.units * front.parts + 7; }   // with both sides' rounding up to 8
    // Fewer than 2^32 threads: a launch is accepted with more, and runs their number modulo 2^32
    bool fits() const { return wgs() * 64 * CA_WAVES < 1L << 32; }
};
// ... with workgroups of nq blocks of rows, and what it costs: in us nearly, a tile of a wavefront, a workgroup's start and end, a join.  Only
// comparisons of these count; the constants are fits to measured calls.  From rounds of few tiles (400 tokens of 16 items behind 300, 8 heads on
// 2; 32 rows and 64): e4m3, d = 64, 99 and 85 us, of 12.5 and 6.25 rounds, less the tiles 5.7 and 10 a round; from rounds of many (512
// tokens of 16 items behind 16384, 4 and 2 rounds of the prefix): e4m3 902 and 701, bf16 1031 and 805, fp32 results of int8 1911 and 1530.  At
// d = 32 two workgroups of 32 rows fit a CU, so that one begins and ends beside the other's tiles: int8 59 and 71, 651 and 626, bf16 54 and
// 64, 570 and 624.  (Only where there is a prefix: without one 32 rows and 64 at d = 32 are within 12 %.)  Few rows of an item leave
// blocks without a row, whose products are passed over (0.7).
inline double ca_plan(const CaProblem &p, int nq, CaPlan &l)
{
    l = {};
    l.nq = nq;
    l.own = ca_grid(p, nq, false);
    const bool wide = nq == 4, small = p.Lp && p.d == 32;
    const double twice = !wide ? 1 : small ? (scaled(p.store) && p.dtype == SKA_BF16 ? 1.75 : 2.05) : scaled(p.store) ? 1.65 : 1.3;
    const double tile = (scaled(p.store) ? (p.dtype == SKA_F32 ? 1.9 : 1) : 1.7) * twice, ends = wide ? 8 : 5, join = 4;
    const auto walk = [&](const CaGrid &g, long n) { return (&g == &l.own && p.R() <= 16 ? 0.7 : 1) * tile * g.tiles / (double)(n * CA_WAVES) + ends; };
    if (!p.Lp) {
        // Parts: rounds of CA_ROOM workgroups, two tiles to a wavefront at least (one part and the best: 132 problems of 16000 tokens, e4m3, d = 64, 61
        // and 57 us, int8, d = 32, 44 and 33; 320 of 12000, int8, d = 128, 227 and 194; 1500 tokens of 8 heads on 6000, int8, d = 128, 85 and 89).
        // Of the numbers with the same rounds the largest is taken; 16 rounds more than the least are as even as it gets.
        // Causal walks of different lengths, the longest first, fill their rounds: they count as much as they are.
        const long most = std::min(l.own.tiles / (2 * CA_WAVES), 256L), least = (l.own.units + CA_ROOM - 1) / CA_ROOM;
        const double uneven = p.causal && l.own.order == CA_LAST_FIRST ? std::min(1., p.Lq / (double)p.Lk) : 0;
        const auto rounds_of = [&](long n) {
            const double full = l.own.units * n / (double)CA_ROOM, whole = std::ceil(full);
            return std::max(1., whole - (whole - full) * uneven);
        };
        double best = rounds_of(1) * walk(l.own, 1);
        for (long rounds = least; rounds <= least + 16 && ends * rounds < best; ++rounds) {
            const long n = std::min(CA_ROOM * rounds / l.own.units, most);
            const double cost = rounds_of(n) * walk(l.own, n) + join;
            if (n > 1 && cost < best) best = cost, l.own.parts = (int)n;
        }
        l.parts = l.own.parts;
        return best;
    }
    // Two tiles to a wavefront at least; four for an item's keys beside a prefix's workgroups: more parts only have to be joined (32 tokens of 1024
    // behind 65536, bf16: 29 us, 31 with two).  The prefix takes the room that the items' own workgroups leave, unless these take more than half of it
    // and its walk there would be longer than one in all of the room and an item's before it (64 tokens of 2048 behind 16384, 4 key heads, int8,
    // d = 128: 55 us in turn with the items', 64 with half of the room; 33 of 1000 behind 10000: 35 in turn, 26 beside them); more workgroups than
    // places would take a prefix's blocks apart, which read its keys together (94 items behind 97725, int8, d = 128: 68 us, 88).
    l.front = ca_grid(p, nq, true);
    l.own.parts = (int)std::max(1L, std::min({CA_ROOM / l.own.units, l.own.tiles / (4 * CA_WAVES), 256L}));
    const long own = l.own.units * l.own.parts, rest = CA_ROOM - own;
    const auto parts = [&](long space) { return std::max(1L, std::min({space / l.front.units, l.front.tiles / (2 * CA_WAVES), 256L})); };
    // Of more workgroups than places some begin while others end: as many rounds as they fill
    const auto rounds = [&](long wgs, long room, const CaGrid &g, long n) {
        const double full = std::max(1., wgs / (double)room);
        return full * walk(g, n) - (small && !wide ? 4.5 * (full - 1) : 0);
    };
    // in turn with the items' in all of the room
    long n = parts(CA_ROOM);
    double best = rounds(l.front.units * n, CA_ROOM, l.front, n) + rounds(own, CA_ROOM, l.own, l.own.parts);
    if (rest >= (own > CA_ROOM / 2 ? l.front.units : 1)) {   // beside them
        const long m = parts(rest);
        const double cost = std::max(rounds(l.front.units * m, rest, l.front, m), walk(l.own, l.own.parts));
        if (own <= CA_ROOM / 2 || cost <= best) best = cost, n = m;
    }
    l.front.parts = (int)n;
    l.parts = l.own.parts + l.front.parts;
    return best + join;
}
// Workgroups of 32 rows or of 64, whose wavefronts turn a key's codes into operands once for twice the rows, but begin and end later (8 problems of 48
// rows on 2500 keys, e4m3, d = 64: 12.7 us and 15.4; of 400 on 30000 61 and 54; 2048 tokens of 8 heads on 2 on 16384 119 and 96; 128 rows of 32 items behind
// 60000, bf16: 26 and 22; 2048 of 16 items on 4096 behind 16384, e4m3: 3580 and 2740; 128 of 64 items behind 65536: 3280 and 2480).  One
// block in workgroups of its own registers gains nothing (a token of 4 items on 65536 keys: 20.2 us, 20.8 with two).
inline CaPlan ca_plan(const CaProblem &p)
{
    CaPlan l{};
    if (ca_together(p)) {
        l.nq = 1;
        l.both = true;
        l.own = ca_grid(p, 1, false);
        l.parts = 1;
        return l;
    }
    const double cost = ca_plan(p, 2, l);
    CaPlan wide;
    if (ca_most(p.store == SKA_F32, p.d) == 4 && (p.Lp ? p.R() * p.B : p.R()) > 32 && (ca_plan(p, 4, wide) < cost || !l.fits())) return wide;
    return l;
}
// Launches of the join of a call's parts: d / 4 threads a row for each slice of the parts, as many slices as there are parts, or threads.
struct CaJoin {
    static constexpr int THREADS = 256;   // of a workgroup
    int slices;
    long per;                             // rows of a workgroup
    CaJoin(int parts, int d) : slices(1)
    {
        while (slices * 2 <= parts && slices * 2 * (d / 4) <= THREADS) slices *= 2;
        per = THREADS / (d / 4) / slices;
    }
    // Rows of a launch, which has 2^31 threads at most: one of 2^32 would be accepted, and run their number modulo 2^32
    long most() const { return per << 23; }
};

}  // namespace
