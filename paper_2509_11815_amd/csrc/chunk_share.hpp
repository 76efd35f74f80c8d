// How the attention of token chunks is divided among workgroups.  Usable on the host as well, so that it can be checked without a GPU.
#pragma once
#include <math.h>
#include <stdint.h>

#include "lengths.hpp"

#ifdef __HIPCC__
#define SPECVLM_SHARE_FN __device__ __forceinline__
#else
#define SPECVLM_SHARE_FN inline
#endif

namespace specvlm {

constexpr int kChunkKeys = 32;               // keys per tile
constexpr int kMostParts = 128;              // parts of one (request, KV head, row block)

// A value that all lanes agree about, in a scalar register where the compiler does not see that they do.
SPECVLM_SHARE_FN int u(int x) {
#ifdef __HIPCC__
    return __builtin_amdgcn_readfirstlane(x);
#else
    return x;
#endif
}

SPECVLM_SHARE_FN float reciprocal(float x) {
#ifdef __HIPCC__
    return __builtin_amdgcn_rcpf(x);
#else
    return 1.f / x;
#endif
}

// n / d for n * d < 2^31, with m = ceil(2^31 / d).
SPECVLM_SHARE_FN int quotient(uint32_t n, uint32_t m) { return static_cast<int>((static_cast<uint64_t>(2 * n) * m) >> 32); }

// Whether n new tokens behind a prefix of P lie inside the cache, or the bit of the error word (2: the number, 4: the length).
SPECVLM_SHARE_FN int chunk_length_error(int n, int P, int N_max, int capacity) { return n < 0 || n > N_max ? 2 : P < 0 || P > capacity - n ? 4 : 0; }

// A segment of a workgroup's share of the call: steps `from` .. `to` (excluded) of the `steps` of (request b, KV head hk, row block rb).
// Where that is not all of them, part `part` of `parts` of its result; `first`: the workgroup that has part 0.
struct Item { int b, hk, rb, n, P, from, to, steps, part, parts, first; };

// ---- the division of a call ------------------------------------------------------------------
// The host does not know the lengths, the device does.  What an item is; ROWS: rows of a block.
template <typename Params, int ROWS>
struct Work {
    static SPECVLM_SHARE_FN int blocks(const Params& p, int n) { return static_cast<int>((static_cast<uint32_t>(p.group) * n + ROWS - 1) / ROWS); }
    // Rounds of four key streams: 128 keys
    static SPECVLM_SHARE_FN int rounds(int P, int n) { return static_cast<int>((static_cast<uint32_t>(P + n - 1) + kSharesRound) / kSharesRound); }
    static SPECVLM_SHARE_FN int last_token(const Params& p, int n, int rb) {
        const int last = quotient((rb + 1) * ROWS - 1, p.magic_group);
        return last < n - 1 ? last : n - 1;
    }
    // Shared tiles: a step is a tile of 32 keys.  Weight of an item: its steps and what it costs beside them (first loads, the result), in units
    // of 1 / (32 group) tiles, the last block's full: whole numbers, sums of which stay below 2^53 (at most kMostPairs items).
    static constexpr int kFixed = 4;
    static SPECVLM_SHARE_FN int steps(const Params& p, int n, int P, int rb) { return (P + last_token(p, n, rb)) / kChunkKeys + 1; }
    static SPECVLM_SHARE_FN double weight(const Params& p, int n, int P, int rb) {
        return (static_cast<double>(P) + kFixed * kChunkKeys) * p.group + static_cast<double>(ROWS) * (rb + 1);
    }
    static SPECVLM_SHARE_FN double before(const Params& p, int n, int P, int rb) {       // of a head's blocks 0 .. rb - 1
        return ((static_cast<double>(P) + kFixed * kChunkKeys) * p.group + 0.5 * ROWS * (rb + 1)) * rb;
    }
};

// Shared tiles.  All (request, KV head, row block) items, one after another, are a line of weights; every workgroup has an equal stretch of
// it, cut at whole steps, and works out from the lengths which items that is: all of them the same cuts.  An item that a cut goes through has several
// parts, whose results meet in the workspace.  Or, where that is estimated to be faster, a workgroup has an item, or half of one.

// Where a workgroup is in its share; in LDS while its wavefronts work on a segment.
struct ShareState {
    double base, per;
    float inv_per;
    int workgroups, mine, b, hk, rb, n, P, blocks, skip, whole, done;
};

// A workgroup's share, item by item.  The first wavefront works it out.
template <typename Params, int ROWS, bool HALVES>
struct Share {
    using W = Work<Params, ROWS>;
    static constexpr float kLeast = 12.f;                  // steps of a stretch at least, so that two cuts of an item lie a step apart or more
    static constexpr int kNear = 6, kHalved = 24;          // steps from an end at which a cut is moved there; of an item that is halved at least
    const Params& p;
    double per;                                            // weight of a stretch
    float inv_per;
    int workgroups, mine;                                  // stretches; this one's number
    int b, hk, rb, n, P, blocks;                           // item the share is at
    double base;                                           // where its request begins
    int skip;                                              // its first step
    bool whole;                                            // an item, or half of one, a workgroup (skip: 1, 2 which; mine: who has the first)
    bool done;

    SPECVLM_SHARE_FN Share(const Params& p_) : p(p_) {}
    SPECVLM_SHARE_FN void keep(ShareState& s) const { s = ShareState{base, per, inv_per, workgroups, mine, b, hk, rb, n, P, blocks, skip, whole, done}; }
    SPECVLM_SHARE_FN void take(const ShareState& s) {
        base = s.base; per = s.per; inv_per = s.inv_per;
        workgroups = u(s.workgroups); mine = u(s.mine); b = u(s.b); hk = u(s.hk); rb = u(s.rb); n = u(s.n); P = u(s.P);
        blocks = u(s.blocks); skip = u(s.skip); whole = u(s.whole); done = u(s.done);
    }
    // Stretch w begins here
    SPECVLM_SHARE_FN double cut(int w) const { return per * w; }
    // Steps per weight of an item: all that matters of it is that every workgroup finds the same.
    static SPECVLM_SHARE_FN float rate_of(double weight, int steps) { return steps * reciprocal(static_cast<float>(weight)); }
    // Where in an item that begins at `begin` stretch w's cut is, in steps; near an end it is moved there
    SPECVLM_SHARE_FN int step_at(int w, double begin, float rate, int steps) const {
        const int t = static_cast<int>(static_cast<float>(cut(w) - begin) * rate + 0.5f);
        return t < kNear ? 0 : t > steps - kNear ? steps : t;
    }
    // The first stretch that begins at x or behind it
    SPECVLM_SHARE_FN int stretch_from(double x) const {
        int w = static_cast<int>(static_cast<float>(x) * inv_per);
        w = w < 0 ? 0 : w > workgroups ? workgroups : w;
        while (w > 0 && cut(w - 1) >= x) --w;
        while (w < workgroups && cut(w) < x) ++w;
        return u(w);
    }
    SPECVLM_SHARE_FN bool request(int which, int new_tokens, int prefix) {
        b = which;
        n = chunk_length_error(new_tokens, prefix, p.N_max, p.g.capacity) ? 0 : new_tokens;
        P = prefix;
        blocks = n ? W::blocks(p, n) : 0;
        return n > 0;
    }
    SPECVLM_SHARE_FN bool lengths(int which) { return request(which, p.num_new ? u(p.num_new[which]) : p.N_max, u(p.prefix_len[which])); }
    // The number of stretches: as many as workgroups fit the chip, but none shorter than kLeast steps, and one each where there are fewer items
    // than that; at most kMostParts of the heaviest item.
    SPECVLM_SHARE_FN void divide_line(double line, int items, float heaviest) {
        const float total = static_cast<float>(line), least = kLeast * kChunkKeys * p.group;
        const float parts = total * reciprocal(heaviest) * (0.9999f * (kMostParts - 2));
        float most = floorf(total * reciprocal(least) * 0.9999f);
        most = most > items ? most : items;
        most = most < p.target ? most : p.target;
        most = most < parts ? most : parts;
        workgroups = u(most < 1.f ? 1 : static_cast<int>(most));
        per = line * static_cast<double>(reciprocal(static_cast<float>(workgroups)));
        inv_per = reciprocal(static_cast<float>(per));
    }
    // Whether an item a workgroup is expected to take less time.  The costs of a cut (128 KB of partial results to memory and back, one more segment's
    // first loads) are about 25 tiles' time: 3008 tokens of 32 heads 92 us undivided, 118 divided; 1024, 1024 and 333 tokens over 4096, 7001 and 5120
    // keys of 8 heads 419 undivided, 258 divided.  Undivided: one round of items takes as long as the longest, more of them about as long as
    // the mean where they begin in the order of their lengths (requests of one length), and up to half an item longer otherwise.
    SPECVLM_SHARE_FN float undivided_time(double line, int items, float heaviest, bool even) const {
        const float mean = static_cast<float>(line) * (1.f / 256);
        const float undivided = items <= 256 ? heaviest : even ? 1.08f * mean : mean + 0.4f * heaviest;
        return undivided > heaviest ? undivided : heaviest;
    }
    SPECVLM_SHARE_FN bool undivided_is_faster(double line, int items, float heaviest, bool even) const {
        return undivided_time(line, items, heaviest, even) < static_cast<float>(per) + 25.f * (kChunkKeys * p.group);
    }
    // HALVES: equal stretches (-1), or an item a workgroup with the last k blocks of every head in halves.  A half, whose workgroup has nothing else to
    // begin, costs about 12 tiles' time: 1024 tokens of 32 heads 37.8 -> 32.0 us, 1536 51.9 -> 40.0; only while all are under way at once, for otherwise
    // halves take the compute units that other items need (2048 tokens 66 -> 73).  bf16 caches only: with the same code the e4m3 kernel of paged caches
    // keeps fewer of its scalars in registers (1024 tokens 42 -> 36.6, but 4096 154 -> 164 and chunks of 1024, 1024 and 333 248 -> 260).
    SPECVLM_SHARE_FN int choose(double line, int items, float heaviest, bool even) const {
        const float unit = kChunkKeys * p.group, part = 0.5f * heaviest + 12.f * unit;
        float time = undivided_time(line, items, heaviest, even);
        int halved = 0;
        const int pairs = p.B * p.H_kv;
        for (int k = 1; items + k * pairs <= 256 && 2 * k * pairs <= p.target && k <= p.row_blocks; ++k) {
            const float rest = heaviest - static_cast<float>(ROWS) * k, t = rest > part ? rest : part;
            if (t < time) {
                time = t;
                halved = k;
            }
        }
        return u(time < static_cast<float>(per) + 25.f * unit ? halved : -1);
    }
    // An item a workgroup, every head's longest first, the first `halved` of them in halves.
    SPECVLM_SHARE_FN bool whole_item(uint32_t workgroup, int halved) {
        const uint32_t pairs = static_cast<uint32_t>(p.B) * p.H_kv, halves = 2 * halved * pairs;
        uint32_t level, pair;
        whole = true;
        skip = 0;
        if (workgroup < halves) {
            level = workgroup / (2 * pairs);
            pair = (workgroup - level * 2 * pairs) >> 1;
            skip = u(1 + (workgroup & 1));
            mine = u(workgroup & ~1u);
        } else {
            level = (workgroup - halves) / pairs;
            pair = workgroup - halves - level * pairs;
            level += halved;
        }
        b = u(pair / static_cast<uint32_t>(p.H_kv));
        hk = u(pair - b * p.H_kv);
        if (!lengths(b)) return false;
        rb = u(blocks - 1 - static_cast<int>(level));
        return rb >= 0;
    }
    // Stretch number of a workgroup, -1: it has none.  Every XCD has contiguous ones, so that the row blocks of a head's keys share an L2.
    SPECVLM_SHARE_FN int stretch_of(int workgroup) const {
        const int xcd = workgroup & 7, place = workgroup >> 3, share = workgroups >> 3, more = workgroups & 7;
        return place >= share + (xcd < more) ? -1 : xcd * share + (xcd < more ? xcd : more) + place;
    }
    // The item that stretch `mine` begins in, given its request (lengths()) and that one's place in the line.
    SPECVLM_SHARE_FN void find_block(double request_base) {
        base = request_base;
        const double at = cut(mine), head = W::before(p, n, P, blocks);
        int heads = static_cast<int>(static_cast<float>(at - base) * reciprocal(static_cast<float>(head)));
        heads = heads < p.H_kv - 1 ? heads : p.H_kv - 1;
        while (heads > 0 && heads * head > at - base) --heads;
        while (heads < p.H_kv - 1 && (heads + 1) * head <= at - base) ++heads;
        hk = u(heads);
        const double in_head = at - base - hk * head;
        int lo = 0, hi = blocks - 1;                       // the last block that begins at in_head or before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (W::before(p, n, P, mid) <= in_head) lo = mid;
            else hi = mid - 1;
        }
        rb = u(lo);
        const int steps = W::steps(p, n, P, rb);
        skip = u(step_at(mine, base + hk * head + W::before(p, n, P, rb), rate_of(W::weight(p, n, P, rb), steps), steps));
        if (skip == steps) {
            skip = 0;
            advance();
        }
    }
    SPECVLM_SHARE_FN void advance() {
        if (++rb < blocks) return;
        rb = 0;
        if (++hk < p.H_kv) return;
        hk = 0;
        base += W::before(p, n, P, blocks) * p.H_kv;
        for (;;) {
            if (++b >= p.B) { done = true; return; }
            if (lengths(b)) return;
        }
    }
    // The next segment of the share; false: there is none.
    SPECVLM_SHARE_FN bool next(Item& it) {
        for (;;) {
            if (done) return false;
            it.b = b; it.hk = hk; it.rb = rb; it.n = n; it.P = P;
            it.steps = u(W::steps(p, n, P, rb));
            it.from = skip;
            it.to = it.steps;
            it.part = 0;
            it.parts = 1;
            it.first = 0;
            if (whole) {
                done = true;
                if constexpr (HALVES) {
                    it.from = 0;
                    if (skip && it.steps < kHalved) return skip == 1;
                    if (skip) {
                        it.part = u(skip - 1);
                        it.parts = 2;
                        it.first = mine;
                        if (it.part) it.from = it.steps >> 1;
                        else it.to = it.steps >> 1;
                    }
                }
                return true;
            }
            const double weight = W::weight(p, n, P, rb);
            const double start = base + hk * W::before(p, n, P, blocks) + W::before(p, n, P, rb), stop = start + weight;
            const float rate = rate_of(weight, it.steps);
            // Stretch w of a cut in [start, stop) begins at step_at(w) of this item; all of its steps: at the next item
            bool ends = false;
            if (mine + 1 < workgroups && cut(mine + 1) < stop) {
                it.to = u(cut(mine + 1) < start ? 0 : step_at(mine + 1, start, rate, it.steps));
                ends = it.to < it.steps;
            }
            const bool divided = it.from > 0 || it.to < it.steps;
            if (divided && it.from < it.to) {
                int first = stretch_from(start) - 1;       // begins before this item, or at its first step:
                while (first + 1 < workgroups && cut(first + 1) < stop && step_at(first + 1, start, rate, it.steps) == 0) ++first;
                int last = stretch_from(stop) - 1;
                while (last > first && step_at(last, start, rate, it.steps) == it.steps) --last;
                it.first = u(first);
                it.part = u(mine - first);
                it.parts = u(last - first + 1);
            }
            const bool some = it.from < it.to;
            skip = 0;
            if (ends) done = true;
            else advance();
            if (some) return true;
        }
    }
};

// Where part i of an item is: a workgroup has room for two, one of an item that it begins and one of an item that another began.
SPECVLM_SHARE_FN int64_t part_at(const Item& it, int i, int bytes) { return static_cast<int64_t>(2 * (it.first + i) + (i == 0)) * bytes; }

}  // namespace specvlm
