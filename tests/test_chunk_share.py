"""How the attention of token chunks is divided among workgroups (csrc/chunk_share.hpp), compiled for the host: every step of every item
belongs to one segment of one workgroup, and the parts of an item are numbered as the merge expects them."""
import os
import random
import subprocess

import pytest

PROGRAM = r"""
#include <cstdio>
#include <vector>
#include "chunk_share.hpp"
using namespace specvlm;
struct Cap { int capacity; };
struct Params { int B, N_max, H_kv, group, target; uint32_t magic_group; Cap g; const int32_t *num_new, *prefix_len; };
template <int ROWS, bool TILES> void run(const Params& p) {
    using S = Share<Params, ROWS, TILES>;
    using W = typename S::W;
    S probe(p);
    double line = 0, heaviest = 0;
    int items = 0;
    for (int b = 0; b < p.B; ++b) if (probe.lengths(b)) {
        items += probe.blocks * p.H_kv;
        line += W::before(p, probe.n, probe.P, probe.blocks) * p.H_kv;
        const double w = W::weight(p, probe.n, probe.P, probe.blocks - 1);
        heaviest = w > heaviest ? w : heaviest;
    }
    printf("items %d\n", items);
    for (int b = 0; b < p.B; ++b) if (probe.lengths(b))
        for (int rb = 0; rb < probe.blocks; ++rb) printf("steps %d %d %d\n", b, rb, W::steps(p, probe.n, probe.P, rb));
    if (!items) return;
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
            printf("seg %d %d %d %d %d %d %d %d %d %d %d %lld\n", s.workgroups, s.mine, it.b, it.hk, it.rb, it.from, it.to, it.steps, it.part, it.parts, it.first, (long long)part_at(it, it.part, 1));
            s.keep(kept);
            S again(p);
            again.take(kept);
            s.done = again.done; s.skip = again.skip;
        }
    }
}
int main() {
    int kind, B;
    Params p;
    while (scanf("%d %d %d %d %d %d %d", &kind, &B, &p.N_max, &p.H_kv, &p.group, &p.target, &p.g.capacity) == 7) {
        std::vector<int32_t> n(B), P(B);
        for (auto& x : n) if (scanf("%d", &x) != 1) return 1;
        for (auto& x : P) if (scanf("%d", &x) != 1) return 1;
        p.B = B; p.num_new = n.data(); p.prefix_len = P.data();
        p.magic_group = (0x80000000u + p.group - 1) / p.group;
        if (kind == 0) run<32, false>(p); else if (kind == 1) run<64, false>(p); else run<256, true>(p);
        printf("end\n");
    }
}
"""
ROWS = {0: 32, 1: 64, 2: 256}
MOST_PARTS = 128


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    from paper_2509_11815_amd import build
    d = tmp_path_factory.mktemp("share")
    (d / "main.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I" + build.CSRC, "-o", str(d / "share"), str(d / "main.cpp")], check=True)
    return str(d / "share")


def ask(program, cases):
    text = "".join(f"{c['kind']} {len(c['n'])} {c['N']} {c['G']} {c['group']} {c['target']} {c['capacity']} {' '.join(map(str, c['n']))} {' '.join(map(str, c['P']))}\n"
                   for c in cases)
    out = subprocess.run([program], input=text, capture_output=True, text=True, check=True, timeout=300).stdout
    answers = out.split("end\n")[:-1]
    assert len(answers) == len(cases)
    return answers


def check(case, answer):
    valid = {b for b, (n, P) in enumerate(zip(case["n"], case["P"])) if 0 < n <= case["N"] and 0 <= P <= case["capacity"] - n}
    steps, segments, load = {}, {}, {}
    for line in answer.splitlines():
        w, *x = line.split()
        x = [int(v) for v in x]
        if w == "steps":
            steps[(x[0], x[1])] = x[2]
        elif w == "seg":
            workgroups, mine, b, hk, rb, lo, hi, of, part, parts, first, place = x
            assert of == steps[(b, rb)] and 0 <= lo < hi <= of
            segments.setdefault((b, hk, rb), []).append((lo, hi, part, parts, first, mine, place))
            load[mine] = load.get(mine, 0) + hi - lo
            assert 1 <= workgroups <= case["target"] and 0 <= mine < workgroups
    assert {b for b, _ in steps} == valid
    assert set(segments) == {(b, hk, rb) for b, rb in steps for hk in range(case["G"])}
    places = set()
    for (b, hk, rb), of in segments.items():
        of.sort()
        assert [s[0] for s in of] == [0] + [s[1] for s in of[:-1]] and of[-1][1] == steps[(b, rb)]
        if len(of) == 1:
            assert of[0][2:4] == (0, 1)
            continue
        assert len(of) <= MOST_PARTS
        for i, (lo, hi, part, parts, first, mine, place) in enumerate(of):
            assert part == i and parts == len(of) and first + i == mine, (b, hk, rb, of)
            assert 0 <= place < 2 * case["target"] and place not in places
            places.add(place)
    return load


def random_case(r):
    kind = r.randrange(3)
    group = r.choice([1, 1, 2, 3, 4, 5, 7, 8, 16])
    rows = ROWS[kind]
    N = {0: max(1, 32 // group), 1: max(1, r.randint(33, 128) // group), 2: r.choice([r.randint(1, 400), r.randint(100, 3000)])}[kind]
    B = r.choice([1, 1, 2, 3, 4, 8, 16, 64, 65, 130])
    G = r.choice([1, 2, 5, 8, 32, 40])
    while B * G * -(-group * N // rows) > 4096:
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
    return dict(kind=kind, N=N, G=G, group=group, target=r.choice([512, 256, 251, 8, 9, 100]), capacity=longest + N + r.randint(0, 40), n=n, P=P)


def test_every_step_once(program):
    r = random.Random(5)
    cases = [random_case(r) for _ in range(600)]
    for case, answer in zip(cases, ask(program, cases)):
        check(case, answer)


def test_all_steps_of_one_length(program):
    """Cuts that fall on the ends of items, and items of one to a few steps."""
    cases = []
    for kind in (0, 1, 2):
        for G in (1, 3, 8, 64):
            for B in (1, 2, 7, 16):
                for P in (0, 100, 127, 128, 255, 256, 383, 511, 1000, 4096):
                    cases.append(dict(kind=kind, N=1, G=G, group=1, target=512 if kind == 0 else 256, capacity=P + 1, n=[1] * B, P=[P] * B))
    for case, answer in zip(cases, ask(program, cases)):
        check(case, answer)


def test_shares_are_even(program):
    """One long request beside short ones: no workgroup has much more than the mean."""
    case = dict(kind=0, N=1, G=8, group=4, target=512, capacity=20000, n=[1] * 16, P=[16383] + [500] * 15)
    load = check(case, ask(program, [case])[0])
    assert max(load.values()) <= 1.5 * sum(load.values()) / len(load) + 2
    case = dict(kind=2, N=1024, G=8, group=4, target=251, capacity=9000, n=[1024, 1024, 0, 333], P=[4096, 7001, 3264, 5120])
    load = check(case, ask(program, [case])[0])
    assert max(load.values()) <= 1.1 * sum(load.values()) / 251


def test_longest_lengths(program):
    top = 2 ** 31 - 1
    cases = [dict(kind=kind, N=64, G=1, group=1, target=256, capacity=top, n=[1, 64], P=[top - 1, top - 64]) for kind in (0, 1, 2)]
    for case, answer in zip(cases, ask(program, cases)):
        check(case, answer)
