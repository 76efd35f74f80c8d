"""How the attention of token chunks is divided among workgroups (csrc/chunk_share.hpp), compiled for the host: every step of every item
belongs to one segment of one workgroup, and the parts of an item are numbered as the merge expects them."""
import os
import random
import subprocess

import pytest

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "chunk_share.hpp"
using namespace specvlm;
struct Cap { int capacity; };
struct Params { int B, N_max, H_kv, group, target, row_blocks; uint32_t magic_group; Cap g; const int32_t *num_new, *prefix_len; };
void show(const char* what, int workgroups, int mine, const Item& it) {
    printf("%s %d %d %d %d %d %d %d %d %d %d %d %lld\n", what, workgroups, mine, it.b, it.hk, it.rb, it.from, it.to, it.steps, it.part, it.parts, it.first, (long long)part_at(it, it.part, 1));
}
constexpr int ROWS = 256;
void run(const Params& p) {
    using S = Share<Params, ROWS, true>;
    using W = S::W;
    S probe(p);
    double line = 0, heaviest = 0, lightest = 1e300;
    int items = 0;
    for (int b = 0; b < p.B; ++b) if (probe.lengths(b)) {
        items += probe.blocks * p.H_kv;
        line += W::before(p, probe.n, probe.P, probe.blocks) * p.H_kv;
        const double w = W::weight(p, probe.n, probe.P, probe.blocks - 1);
        heaviest = w > heaviest ? w : heaviest;
        lightest = w < lightest ? w : lightest;
    }
    printf("items %d\n", items);
    for (int b = 0; b < p.B; ++b) if (probe.lengths(b))
        for (int rb = 0; rb < probe.blocks; ++rb) printf("steps %d %d %d\n", b, rb, W::steps(p, probe.n, probe.P, rb));
    if (!items) return;
    probe.divide_line(line, items, (float)heaviest);
    const int pairs = p.B * p.H_kv, most = p.target / (2 * pairs), chosen = probe.choose(line, items, (float)heaviest, heaviest == lightest);
    printf("chosen %d\n", chosen);
    const int halves[3] = {0, chosen, most < p.row_blocks ? most : p.row_blocks};
    const char* const names[3] = {"whole", "half", "most"};
    for (int way = 0; way < 3; ++way)
        for (int wg = 0, halved = halves[way]; halved >= 0 && wg < (std::max(p.target, pairs * p.row_blocks + p.target / 2) + 7) / 8 * 8; ++wg) {
            S s(p);
            s.done = false;
            s.skip = 0;
            Item it;
            if (s.whole_item(wg, halved) && s.next(it)) {
                show(names[way], p.target, wg, it);
                if (s.next(it)) printf("again\n");
            }
        }
    for (int wg = 0; wg < (p.target + 7) / 8 * 8; ++wg) {
        S s(p);
        s.done = s.whole = false;
        s.skip = 0;
        s.divide_line(line, items, (float)heaviest);
        s.mine = s.stretch_of(wg);
        if (s.mine < 0) continue;
        const double at = s.cut(s.mine);
        double past = 0;
        for (int b = 0; b < p.B; ++b) {
            if (!s.lengths(b)) continue;
            const double w = W::before(p, s.n, s.P, s.blocks) * p.H_kv;
            if (past + w > at) break;
            past += w;
        }
        s.find_block(past);
        Item it;
        ShareState kept;
        while (!s.done && s.next(it)) {
            show("seg", s.workgroups, s.mine, it);
            s.keep(kept);
            S again(p);
            again.take(kept);
            s.done = again.done; s.skip = again.skip;
        }
    }
}
int main() {
    int B;
    Params p;
    while (scanf("%d %d %d %d %d %d", &B, &p.N_max, &p.H_kv, &p.group, &p.target, &p.g.capacity) == 6) {
        std::vector<int32_t> n(B), P(B);
        for (auto& x : n) if (scanf("%d", &x) != 1) return 1;
        for (auto& x : P) if (scanf("%d", &x) != 1) return 1;
        p.B = B; p.num_new = n.data(); p.prefix_len = P.data();
        p.magic_group = (0x80000000u + p.group - 1) / p.group;
        p.row_blocks = (int)(((int64_t)p.group * p.N_max + ROWS - 1) / ROWS);
        run(p);
        printf("end\n");
    }
}
"""
ROWS = 256
MOST_PARTS = 128


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2509_11815_amd import build
    d = tmp_path_factory.mktemp("share")
    (d / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I" + build.CSRC, "-o", str(d / "share"), str(d / "main.cpp")], check=True)
    return str(d / "share")


def ask(program, cases):
    text = "".join(f"{len(c['n'])} {c['N']} {c['G']} {c['group']} {c['target']} {c['capacity']} {' '.join(map(str, c['n']))} {' '.join(map(str, c['P']))}\n"
                   for c in cases)
    out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=300).stdout
    answers = out.split("end\n")[:-1]
    assert len(answers) == len(cases)
    return answers


def check(case, answer):
    """Equal stretches, an item a workgroup, and the chosen and the greatest number of blocks in halves: the steps each workgroup has of the first."""
    valid = {b for b, (n, P) in enumerate(zip(case["n"], case["P"])) if 0 < n <= case["N"] and 0 <= P <= case["capacity"] - n}
    steps, ways, load, chosen = {}, {}, {}, -1
    for line in answer.splitlines():
        w, *x = line.split()
        x = [int(v) for v in x]
        if w == "steps":
            steps[(x[0], x[1])] = x[2]
        elif w == "chosen":
            chosen = x[0]
        elif w in ("seg", "whole", "half", "most"):
            workgroups, mine, b, hk, rb, lo, hi, of, part, parts, first, place = x
            assert of == steps[(b, rb)] and 0 <= lo < hi <= of
            ways.setdefault(w, {}).setdefault((b, hk, rb), []).append((lo, hi, part, parts, first, mine, place))
            if w == "seg":
                load[mine] = load.get(mine, 0) + hi - lo
                assert 1 <= workgroups <= case["target"] and 0 <= mine < workgroups
        else:
            assert w == "items"
    assert {b for b, _ in steps} == valid
    assert not valid or {"seg", "whole"} <= set(ways)
    assert chosen * 2 * len(case["n"]) * case["G"] <= case["target"]
    for w, segments in ways.items():
        assert set(segments) == {(b, hk, rb) for b, rb in steps for hk in range(case["G"])}
        places = set()
        for (b, hk, rb), of in segments.items():
            of.sort()
            assert [s[0] for s in of] == [0] + [s[1] for s in of[:-1]] and of[-1][1] == steps[(b, rb)]
            if len(of) == 1:
                assert of[0][2:4] == (0, 1)
                continue
            assert len(of) <= {"seg": MOST_PARTS, "whole": 1}.get(w, 2)
            for i, (lo, hi, part, parts, first, mine, place) in enumerate(of):
                assert part == i and parts == len(of) and first + i == mine, (b, hk, rb, of)
                assert 0 <= place < 2 * case["target"] and place not in places
                places.add(place)
    return load


def random_case(r):
    group = r.choice([1, 1, 2, 3, 4, 5, 7, 8, 16])
    N = r.choice([r.randint(1, 400), r.randint(100, 3000)])
    B = r.choice([1, 1, 2, 3, 4, 8, 16, 64, 65, 130])
    G = r.choice([1, 2, 5, 8, 32, 40])
    while B * G * -(-group * N // ROWS) > 4096:
        if B > 1:
            B //= 2
        elif G > 1:
            G //= 2
        else:
            N = max(1, N // 2)
    longest = r.choice([0, 3, 130, 1000, 9000, 40000, 200000])
    P = [r.randint(0, longest) if r.random() < 0.7 else longest for _ in range(B)]
    n = [N if r.random() < 0.6 else r.randint(0, N) for _ in range(B)]
    if r.random() < 0.2:
        n[r.randrange(B)] = r.choice([-1, N + 1, -2 ** 31, 2 ** 31 - 1])
        P[r.randrange(B)] = r.choice([-1, 2 ** 31 - 1, -2 ** 31])
    return dict(N=N, G=G, group=group, target=r.choice([256, 256, 251, 8, 9, 100]), capacity=longest + N + r.randint(0, 40), n=n, P=P)


def test_every_step_once(program):
    r = random.Random(5)
    cases = [random_case(r) for _ in range(600)]
    for case, answer in zip(cases, ask(program, cases)):
        check(case, answer)


def test_all_steps_of_one_length(program):
    """Cuts that fall on the ends of items, and items of one to a few steps."""
    cases = []
    for N in (1, 300, 1000):
        for G in (1, 3, 8, 64):
            for B in (1, 2, 7, 16):
                for P in (0, 100, 127, 128, 255, 256, 383, 511, 1000, 4096):
                    cases.append(dict(N=N, G=G, group=1, target=256, capacity=P + N, n=[N] * B, P=[P] * B))
    for case, answer in zip(cases, ask(program, cases)):
        check(case, answer)


def test_shares_are_even(program):
    """Requests of different lengths: no workgroup has much more than the mean."""
    case = dict(N=1024, G=8, group=4, target=251, capacity=9000, n=[1024, 1024, 0, 333], P=[4096, 7001, 3264, 5120])
    load = check(case, ask(program, [case])[0])
    assert max(load.values()) <= 1.1 * sum(load.values()) / 251


def test_longest_lengths(program):
    top = 2 ** 31 - 1
    cases = [dict(N=64, G=1, group=1, target=256, capacity=top, n=[1, 64], P=[top - 1, top - 64])]
    for case, answer in zip(cases, ask(program, cases)):
        check(case, answer)
