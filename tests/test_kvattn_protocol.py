"""A model of the barrier protocol of kv_attention_tc_kernel
(csrc/kvattn_tc.cu), run under random and starving interleavings of its
roles, for runs of several units with one or two row tiles.

The warp that brings the codes, the warps that convert keys and values, the
MMA warp and the two softmax streams communicate only through mbarriers
whose waits name a phase parity. The model replays each role's waits and
arrivals in the kernel's order and numbering and checks that

- no schedule deadlocks;
- a wait never meets a barrier that has gone on to a later phase (its parity
  would be that of the phase before: the wait would last for ever);
- descriptions, tiles of codes, fp16 tiles, scores, weights and the queries'
  memory are overwritten only after their readers are done with them.

A stream's four warps are one role, and so are the keys' and the values'
converting warps. MMAs complete in issue order, so a commit is modelled at
the issuing point."""

import random

import pytest

INFOS, K_STAGES, V_STAGES, CK_STAGES, CV_STAGES = 4, 1, 1, 3, 2


class Bar:
    def __init__(self, count):
        self.count, self.arrived, self.phases = count, 0, 0

    def arrive(self):
        self.arrived += 1
        if self.arrived == self.count:
            self.arrived = 0
            self.phases += 1


def run(segments, seed, prefer=None, moves=0.3, drop=None):
    """segments: (key tiles, shared) of each unit's part. moves: how often a
    stream's maximum moves (the accumulators are rescaled after a wait for
    the product before). drop: a wait to leave out."""
    count = sum(n for n, _ in segments)
    rng = random.Random(seed)
    bars = {}
    counts = {"q_full": 2, "meet": 2}                 # both streams arrive

    def bar(name):
        return bars.setdefault(name, Bar(counts.get(name if isinstance(name, str) else name[0], 1)))

    W = lambda name, want: ("wait", name, want)
    A = lambda name: ("arrive", name)
    info = {}                                         # slot -> [tile, readers left]
    codes = {"k": {}, "v": {}}                        # stage -> tile whose codes are there and unread
    tiles = {"k": {}, "v": {}}                        # stage -> [tile, products left]
    scores = [None, None]                             # per stream: ("s" scores, "p" weights, None free)
    q_busy = [0]                                      # products with the segment's queries still to come
    of = []                                           # tile -> (shared, products a tile takes part in)
    for n, shared in segments:
        of += [shared] * n

    def bring():
        for it in range(count):
            slot = it % INFOS
            yield W(("info_empty", slot), it // INFOS)
            assert info.get(slot, [0, 0])[1] == 0, "description overwritten before its readers were done"
            info[slot] = [it, 2 + (2 if of[it] else 1)]              # both conversions, the streams
            yield A(("info", slot))
            for kind, stages in (("k", CK_STAGES), ("v", CV_STAGES)):
                st = it % stages
                yield W((kind + "codes_empty", st), it // stages)
                assert codes[kind].get(st) is None, "codes overwritten before they were converted"
                codes[kind][st] = it
                yield A((kind + "codes_full", st))
        for slot in range(min(INFOS, count)):
            yield W(("info_empty", slot), (count - slot + INFOS - 1) // INFOS)

    def read_info(it):
        assert info[it % INFOS][0] == it, "a description was read after it was overwritten"
        info[it % INFOS][1] -= 1

    def convert(kind):
        stages, cstages = (K_STAGES, CK_STAGES) if kind == "k" else (V_STAGES, CV_STAGES)
        for it in range(count):
            st, cs = it % stages, it % cstages
            yield W(("info", it % INFOS), it // INFOS + 1)
            yield W((kind + "codes_full", cs), it // cstages + 1)
            read_info(it)
            assert codes[kind][cs] == it
            if drop != kind + "_empty":
                yield W((kind + "_empty", st), it // stages)
            assert tiles[kind].get(st, [0, 0])[1] == 0, "tile overwritten before its products"
            tiles[kind][st] = [it, 2 if of[it] else 1]
            codes[kind][cs] = None
            yield A((kind + "codes_empty", cs))
            yield A((kind + "_full", st))
        for st in range(min(stages, count)):
            yield W((kind + "_empty", st), (count - st + stages - 1) // stages)

    def mma():
        tile0, steps = 0, [0, 0]
        for seg, (n, shared) in enumerate(segments):
            items = 2 * n if shared else n
            yield W("q_full", seg + 1)

            def qk(u):
                kt, s = tile0 + (u >> 1 if shared else u), u & 1
                yield W(("k_full", kt % K_STAGES), kt // K_STAGES + 1)
                assert scores[s] is None, "scores written over weights that were not used"
                t = tiles["k"][kt % K_STAGES]
                assert t[0] == kt
                t[1] -= 1
                q_busy[0] -= 1
                scores[s] = "s"
                if not shared or s == 1:
                    yield A(("k_empty", kt % K_STAGES))
                yield A(("s_full", s))

            for u in range(min(2, items)):
                yield from qk(u)
            for u in range(items):
                kt, s, step = tile0 + (u >> 1 if shared else u), u & 1, u >> 1
                yield W(("v_full", kt % V_STAGES), kt // V_STAGES + 1)
                if drop != "p_full":
                    yield W(("p_full", s), steps[s] + step + 1)
                assert scores[s] == "p", "product taken before the weights were there"
                t = tiles["v"][kt % V_STAGES]
                assert t[0] == kt
                t[1] -= 1
                scores[s] = None
                if not shared or s == 1:
                    yield A(("v_empty", kt % V_STAGES))
                    yield A(("info_empty", kt % INFOS))
                yield A(("pv_done", s))
                if u + 2 < items:
                    yield from qk(u + 2)
            steps[0] += (items + 1) // 2
            steps[1] += items // 2
            tile0 += n

    def softmax(s):
        tile0 = steps = meets = 0
        for n, shared in segments:
            mine = n if shared else (n - s + 1) // 2
            if shared or s == 0:                      # the queries' tile
                assert q_busy[0] <= 0 or s == 1, "queries overwritten before their products"
                if s == 0:
                    q_busy[0] = 2 * n if shared else n
            yield A("q_full")
            for step in range(mine):
                kt = tile0 + (step if shared else 2 * step + s)
                yield W(("s_full", s), steps + step + 1)
                yield W(("info", kt % INFOS), kt // INFOS + 1)
                assert scores[s] == "s"
                if step > 0 and rng.random() < moves:
                    yield W(("pv_done", s), steps + step)
                read_info(kt)
                scores[s] = "p"
                yield A(("p_full", s))
            steps += mine
            if mine > 0:
                yield W(("pv_done", s), steps)

            def meet():
                nonlocal meets
                meets += 1
                yield A("meet")
                yield W("meet", meets)
            if not shared:
                yield from meet()
                assert q_busy[0] == 0, "the join area is the queries' memory"
                yield from meet()
            yield from meet()
            tile0 += n

    roles = {"bring": bring(), "k": convert("k"), "v": convert("v"), "mma": mma(), "s0": softmax(0), "s1": softmax(1)}
    cur = {k: next(v, None) for k, v in roles.items()}
    ready = lambda step: step[0] == "arrive" or bar(step[1]).phases >= step[2]
    while any(c is not None for c in cur.values()):
        for k, c in cur.items():                      # also of a role that is not scheduled yet
            assert c is None or c[0] == "arrive" or bar(c[1]).phases <= c[2], \
                f"{k} waits for phase {c[2] - 1} of {c[1]}, which has gone on to {bar(c[1]).phases}"
        live = [k for k, c in cur.items() if c is not None and ready(c)]
        assert live, f"deadlock at {cur}"
        k = next((r for r in prefer or () if r in live), None) or rng.choice(live)
        if cur[k][0] == "arrive":
            bar(cur[k][1]).arrive()
        cur[k] = next(roles[k], None)


ORDERS = (None, ("bring", "k", "v", "mma"), ("mma", "s0"), ("mma", "s1"), ("s0", "s1"), ("s0", "mma", "k", "v", "bring"),
          ("s1", "v", "bring"), ("k", "bring", "s0"), ("v", "k", "mma"))


@pytest.mark.parametrize("segments", [
    [(1, False)], [(1, True)], [(2, False)], [(3, True)], [(7, False)], [(9, True)],
    [(1, False), (1, False), (1, False)], [(1, True), (2, False), (5, True)], [(4, False), (1, True), (1, False)],
    [(13, False), (2, True), (6, False), (1, False)], [(20, True), (21, False)]])
def test_cache_attention_barrier_protocol(segments):
    for prefer in ORDERS:
        for moves in (0.0, 0.3, 1.0):
            for seed in range(4):
                run(segments, seed, prefer, moves)


@pytest.mark.parametrize("drop,prefer", [
    ("k_empty", ("bring", "k")), ("v_empty", ("bring", "v")), ("p_full", ("mma",))])
def test_model_catches_a_missing_wait(drop, prefer):
    """The model is not vacuous: each of these waits left out trips it. (The
    wait for info_empty would be implied by the others with two stages of
    the values' codes.)"""
    for segments in ([(12, False)], [(12, True)]):
        run(segments, 0, prefer)
        with pytest.raises(AssertionError):
            run(segments, 0, prefer, drop=drop)
