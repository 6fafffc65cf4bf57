"""Models of the barrier traffic of k_cache_attn and k_cache_attn_few (a CTA each), run in random order on the CPU as those of the other kernels are: every agent
ends, nobody reads or overwrites what another one still needs, and when the last agent has ended no asynchronous arrival is under way any more."""
import os
import random
import re
import subprocess

import pytest

from .test_barrier_protocols import CSRC, Barrier, Clock, play, some, until

RING = 16
MANY = {64: (5, 3), 128: (2, 3), 256: (2, 4)}             # units of K (and V) in shared memory, buffers of S, by head_dim
FEW = {64: (3, 4), 128: (3, 4), 256: (3, 4)}


class Committer:
    """tcgen05.commit: arrives behind the MMAs issued before it, and when it arrives beyond that nothing says, later commits' arrivals on other barriers included."""

    def __init__(self, clock, late=()):
        self.clock, self.late, self.last = clock, late, 0.0

    def __call__(self, *barriers):
        self.last = max(self.last, self.clock.now) + self.clock.rng.uniform(0.05, 0.6)
        for b in barriers:
            self.clock.at(self.last + self.clock.rng.uniform(0, 10 if b in self.late else 1), b.arrive)


def closing_waits(path):
    """Whether the kernel waits at its end for the arrivals that nothing else waits for, as its source has it."""
    return bool(re.search(r"// the last O [^\n]*\n[^}]*?\(o_done \+", open(os.path.join(CSRC, path)).read()))


def clears_behind_o():
    """Whether k_cache_attn clears values that are nobody's behind the O that left their stage, as its source has it."""
    return "mbar_wait(o_done + (g - STAGES) % SB, (uint32_t)((g - STAGES) / SB) & 1u, abort_flag)" in open(os.path.join(CSRC, "cache_attn.cuh")).read()


def bars(n, count=1):
    return [Barrier(count) for _ in range(n)]


def step(i, ph, n):
    return (i + 1, ph) if i + 1 < n else (0, ph ^ 1)


def producer(which, segments, full, empty, seg_full, held, ring, stages):
    st, ph, g = 0, 1, 0
    for i, n in enumerate(segments + [0]):
        if which == "k":
            ring["seg"][i % RING] = (i, n)
            seg_full[i % RING].arrive()
            yield
        for _ in range(n):
            yield from until(lambda: empty[st].done(ph))
            if which == "k":
                ring["mask"][g % RING] = g
            held[which][st] = g
            full[st].load(held["clock"], 2)
            st, ph = step(st, ph, stages)
            g += 1
    for _ in range(stages):
        yield from until(lambda: empty[st].done(ph))
        st, ph = step(st, ph, stages)


def segment(i, seg_full):
    return until(lambda: seg_full[i % RING].done(i // RING & 1))


def many(hd, segments, seed, closing=True, behind_o=True):
    stages, SB = MANY[hd]
    rng = random.Random(seed)
    clock = Clock(rng)
    k_full, k_empty, v_full, v_empty = bars(stages), bars(stages), bars(stages), bars(stages)
    s_full, p_full, o_done, q_full, o_free, seg_full = bars(SB), bars(SB, 16), bars(SB), bars(1)[0], bars(1, 16)[0], bars(RING)
    held = dict(clock=clock, k=[None] * stages, v=[None] * stages, s=[None] * SB, p=[[None] * 16 for _ in range(SB)], o=-1, q=-1)
    ring = dict(seg=[None] * RING, mask=[None] * RING)

    def s_issuer():
        commit = Committer(clock)
        ks = sb = kph = g = 0
        sph = 1
        for seg in range(len(segments) + 1):
            yield from segment(seg, seg_full)
            i, n = ring["seg"][seg % RING]
            assert i == seg
            if not n:
                break
            held["q"] = seg
            q_full.load(clock, 2)
            yield from until(lambda: q_full.done(seg & 1))
            for _ in range(n):
                yield from until(lambda: o_done[sb].done(sph) and k_full[ks].done(kph))
                assert held["k"][ks] == g and held["q"] == seg and held["o"] >= g - SB
                held["s"][sb] = g
                commit(k_empty[ks], s_full[sb])
                ks, kph = step(ks, kph, stages)
                sb, sph = step(sb, sph, SB)
                g += 1
            yield from until(lambda: s_full[(g - 1) % SB].done((g - 1) // SB & 1))
        for _ in range(SB if closing else 0):
            yield from until(lambda: o_done[sb].done(sph))
            sb, sph = step(sb, sph, SB)

    def o_issuer():
        commit = Committer(clock, o_done)
        vs = vph = sb = pph = g = 0
        for seg in range(len(segments) + 1):
            yield from segment(seg, seg_full)
            i, n = ring["seg"][seg % RING]
            assert i == seg
            if not n:
                break
            if seg:
                yield from until(lambda: o_free.done(seg - 1 & 1))
            for _ in range(n):
                yield from until(lambda: v_full[vs].done(vph) and p_full[sb].done(pph))
                assert held["v"][vs] == g and held["p"][sb] == [g] * 16
                commit(v_empty[vs], o_done[sb])
                held["o"] = g
                vs, vph = step(vs, vph, stages)
                sb, pph = step(sb, pph, SB)
                g += 1

    votes = [dict(n=0, round=0) for _ in range(8)]              # the barrier of a pair

    def meet(pair):
        v = votes[pair]
        at = v["round"]
        v["n"] += 1
        if v["n"] == 2:
            v["n"], v["round"] = 0, at + 1
        yield from until(lambda: v["round"] > at)

    def softmax(w):
        g = sb = sph = 0
        moves = random.Random(seed * 8 + w % 8)                 # the same in both of a pair
        for seg in range(len(segments) + 1):
            yield from segment(seg, seg_full)
            i, n = ring["seg"][seg % RING]
            assert i == seg
            yield from meet(w % 8)
            if not n:
                break
            for u in range(n):
                yield from until(lambda: s_full[sb].done(sph))
                assert held["s"][sb] == g and ring["mask"][g % RING] == g
                if rng.random() < 0.3:                          # values that are cleared
                    if stages < SB and g >= stages and behind_o:
                        yield from until(lambda: o_done[(g - stages) % SB].done((g - stages) // SB & 1))
                    yield from until(lambda: v_full[g % stages].done(g // stages & 1))
                    assert held["v"][g % stages] == g and v_full[g % stages].phase == g // stages + 1
                yield from meet(w % 8)
                if moves.random() < 0.3:
                    yield from meet(w % 8)
                    if u:
                        yield from until(lambda: o_done[(g - 1) % SB].done((g - 1) // SB & 1))
                        assert held["o"] == g - 1
                held["p"][sb][w] = g
                yield from some(rng, 3)
                assert ring["seg"][seg % RING][0] == seg
                p_full[sb].arrive()
                sb, sph = step(sb, sph, SB)
                g += 1
            yield from meet(w % 8)
            yield from some(rng, 3)
            assert ring["seg"][seg % RING][0] == seg            # what the epilogue looks at
            yield from until(lambda: o_done[(g - 1) % SB].done((g - 1) // SB & 1))
            assert held["o"] == g - 1
            yield from some(rng, 3)
            assert held["o"] == g - 1
            o_free.arrive()

    return play(clock, [producer("k", segments, k_full, k_empty, seg_full, held, ring, stages), producer("v", segments, v_full, v_empty, None, held, ring, stages),
                        s_issuer(), o_issuer()] + [softmax(w) for w in range(16)])


def few(hd, segments, seed, closing=True):
    stages, SB = FEW[hd]
    rng = random.Random(seed)
    clock = Clock(rng)
    k_full, k_empty, v_full, v_empty = bars(stages), bars(stages), bars(stages), bars(stages)
    s_full, s_empty, p_full, o_done, o_free, q_full, q_empty = bars(SB), bars(SB, 4), bars(2, 4), bars(2), bars(2, 4), bars(2), bars(2)
    seg_full = bars(RING)
    held = dict(clock=clock, k=[None] * stages, v=[None] * stages, s=[None] * SB, p=[[None] * 4 for _ in range(2)], o=[-1, -1], q=[-1, -1])
    ring = dict(seg=[None] * RING, mask=[None] * RING)
    first = [sum(segments[:i]) for i in range(len(segments))]

    def s_issuer():
        commit = Committer(clock)
        st = ph = sb = g = 0
        sph = 1

        def fetch(seg):
            yield from segment(seg, seg_full)
            if not ring["seg"][seg % RING][1]:
                return
            yield from until(lambda: q_empty[seg & 1].done((seg >> 1 & 1) ^ 1))
            held["q"][seg & 1] = seg
            q_full[seg & 1].load(clock, 2)

        yield from fetch(0)
        seg = 0
        while True:
            yield from segment(seg, seg_full)
            i, n = ring["seg"][seg % RING]
            assert i == seg
            if not n:
                break
            ahead = False
            yield from until(lambda: q_full[seg & 1].done(seg >> 1 & 1))
            for u in range(n):
                yield from until(lambda: s_empty[sb].done(sph) and k_full[st].done(ph))
                assert held["k"][st] == g and held["q"][seg & 1] == seg
                held["s"][sb] = g
                commit(k_empty[st], s_full[sb])
                if u == n - 1:
                    commit(q_empty[seg & 1])
                st, ph = step(st, ph, stages)
                sb, sph = step(sb, sph, SB)
                g += 1
                nx = seg + 1
                if not ahead and (u == n - 1 or (seg_full[nx % RING].done(nx // RING & 1) and q_empty[nx & 1].done((nx >> 1 & 1) ^ 1))):
                    ahead = True
                    yield from fetch(nx)
            seg += 1
        for _ in range(2 if closing else 0):
            yield from until(lambda: q_empty[seg & 1].done((seg >> 1 & 1) ^ 1))
            seg += 1

    def o_issuer():
        commit = Committer(clock, o_done)
        st = ph = g = 0
        for seg in range(len(segments) + 1):
            yield from segment(seg, seg_full)
            n = ring["seg"][seg % RING][1]
            if not n:
                break
            if seg > 1:
                yield from until(lambda: o_free[seg & 1].done((seg >> 1) - 1 & 1))
            for _ in range(n):
                yield from until(lambda: v_full[st].done(ph) and p_full[g & 1].done(g >> 1 & 1))
                assert held["v"][st] == g and held["p"][g & 1] == [g] * 4
                commit(v_empty[st], o_done[g & 1])
                held["o"][seg & 1] = g
                st, ph = step(st, ph, stages)
                g += 1

    vote = dict(n=0, round=0)

    def meet():
        at = vote["round"]
        vote["n"] += 1
        if vote["n"] == 4:
            vote["n"], vote["round"] = 0, at + 1
        yield from until(lambda: vote["round"] > at)

    def softmax(w):
        g = sb = sph = 0
        moves = random.Random(seed)
        for seg in range(len(segments) + 1):
            yield from segment(seg, seg_full)
            i, n = ring["seg"][seg % RING]
            assert i == seg
            yield from meet()
            if not n:
                break
            for u in range(n):
                pb = g & 1
                yield from until(lambda: s_full[sb].done(sph) and (g < 2 or o_done[pb].done((g >> 1) - 1 & 1)))
                assert held["s"][sb] == g and ring["mask"][g % RING] == g
                yield from some(rng, 2)
                s_empty[sb].arrive()
                sb, sph = step(sb, sph, SB)
                yield from meet()
                if moves.random() < 0.3:
                    yield from meet()
                    if u:
                        yield from until(lambda: o_done[(g - 1) & 1].done((g - 1) >> 1 & 1))
                        assert held["o"][seg & 1] == g - 1
                held["p"][pb][w] = g
                if rng.random() < 0.3:
                    yield from until(lambda: v_full[g % stages].done(g // stages & 1))
                    assert held["v"][g % stages] == g and v_full[g % stages].phase == g // stages + 1
                yield from some(rng, 3)
                p_full[pb].arrive()
                g += 1
            yield from meet()
            assert ring["seg"][seg % RING][0] == seg
            yield from until(lambda: o_done[(g - 1) & 1].done((g - 1) >> 1 & 1))
            assert held["o"][seg & 1] == first[seg] + n - 1
            yield from some(rng, 2)
            assert held["o"][seg & 1] == first[seg] + n - 1
            o_free[seg & 1].arrive()
            yield from meet()
        if closing and g > 1:
            yield from until(lambda: o_done[g & 1].done((g - 2) >> 1 & 1))

    return play(clock, [producer("k", segments, k_full, k_empty, seg_full, held, ring, stages), producer("v", segments, v_full, v_empty, None, held, ring, stages),
                        s_issuer(), o_issuer()] + [softmax(w) for w in range(4)])


SEGMENTS = [[], [1], [2], [3], [4], [5], [9], [1, 1], [3, 1, 2], [1] * 20, [1, 7, 1, 4], [2] * 18 + [5]]


@pytest.mark.parametrize("hd", [64, 128, 256])
def test_values_are_cleared_where_they_have_come(hd):
    for segments in SEGMENTS:
        for seed in range(12, 36):
            many(hd, list(segments), seed, behind_o=clears_behind_o())


def test_values_cleared_by_their_barrier_alone():
    with pytest.raises(AssertionError):
        for segments in SEGMENTS:
            for seed in range(12, 36):
                many(256, list(segments), seed, behind_o=False)


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("model,path", [(many, "cache_attn.cuh"), (few, "cache_few.cuh")])
def test_every_agent_ends_and_nothing_is_under_way(model, path, hd):
    closing = closing_waits(path)               # as the kernel has it
    for segments in SEGMENTS:
        for seed in range(12):
            assert model(hd, list(segments), seed, closing) == 0


@pytest.mark.parametrize("model", [many, few])
def test_without_the_closing_waits(model):
    assert any(model(256, list(segments), seed, closing=False) for segments in SEGMENTS for seed in range(12))


def test_shapes(tmp_path):
    """The depths above are those of the kernels."""
    lines = ["#include <cstddef>", "#include <cstdio>"]
    for path, name in (("cache_attn.cuh", "CaShape"), ("cache_few.cuh", "CfShape")):
        src = open(os.path.join(CSRC, path)).read()
        lines += re.findall(r"^#define C[AF]_(?:N|S|ENTRIES) .*$", src, re.M)
        body = src[src.index("template <int HD> struct " + name):]
        lines.append(body[:body.index("\n};") + 3])
    ring = re.search(r"^#define CA_RING (\d+)", open(os.path.join(CSRC, "cache_work.cuh")).read(), re.M)
    assert int(ring.group(1)) == RING
    lines.append("int main() {")
    for hd in MANY:
        lines.append('  printf("%%d %%d %%d %%d\\n", CaShape<%d>::STAGES, CaShape<%d>::S_BUFS, CfShape<%d>::STAGES, CF_S);' % (hd, hd, hd))
    (tmp_path / "shape.cpp").write_text("\n".join(lines + ["}"]))
    subprocess.run(["g++", "-std=c++17", "-o", str(tmp_path / "shape"), str(tmp_path / "shape.cpp")], check=True)
    out = subprocess.run([str(tmp_path / "shape")], check=True, capture_output=True, text=True).stdout.split("\n")
    assert [tuple(map(int, line.split())) for line in out if line] == [MANY[hd] + FEW[hd] for hd in MANY]
