"""The order of waits of the tcgen05 paged-attention kernel (wq_attn_paged_tc.cu), as a model on the CPU: the warp that plans,
the MMA warp, the converting warps (as one) and the two softmax streams run their programs' waits and arrivals over every mix
of blocks, in orders that a scheduler may choose at random, and must come to their ends; a stage is only written when all that
reads it is done.  Barriers are mbarriers: a wait names the parity of a phase.
"""
import random

import pytest


class Bar:
    def __init__(self, count):
        self.count, self.here, self.phase = count, 0, 0

    def arrive(self):
        self.here += 1
        assert self.here <= self.count
        if self.here == self.count:
            self.here = 0
            self.phase += 1

    def passed(self, parity):
        return self.phase & 1 != parity


def bars(stages):
    ring = lambda k, n: [Bar(n) for _ in range(k)]  # noqa: E731
    return dict(q_full=Bar(1), q_empty=Bar(1), k_full=ring(stages, 1), k_empty=ring(stages, 1),
                v_full=ring(stages, 1), v_empty=ring(stages, 1), s_full=ring(3, 1), p_full=ring(3, 1), o_full=[ring(2, 1), ring(2, 1)], run_full=ring(4, 1), run_empty=ring(4, 4))


def plan(runs, B, state):
    for turn in range(len(runs) + 1):
        if turn >= 4:
            yield B["run_empty"][turn & 3], (turn >> 2) + 1 & 1
        state["run"][turn & 3] = runs[turn] if turn < len(runs) else None
        B["run_full"][turn & 3].arrive()


def each_run(B, state):
    """The runs as a role reads them: (wait) or (None, run)."""
    turn = 0
    while True:
        yield B["run_full"][turn & 3], turn >> 2 & 1
        if state["run"][turn & 3] is None:
            return
        yield None, state["run"][turn & 3]
        assert state["run"][turn & 3] is not None
        B["run_empty"][turn & 3].arrive()
        turn += 1


def conv(B, bf16, stages, state):
    T = seg = 0
    for got, run in each_run(B, state):
        if got is not None:
            yield got, run
            continue
        n, split = run
        if n == 0:
            continue
        if seg > 0:
            yield B["q_empty"], (seg - 1) & 1
        assert state["q"] == 0, "queries overwritten"
        state["q"] = n if split else 2 * n
        B["q_full"].arrive()
        for ti in range(n):
            st, last = (T + ti) % stages, (T + ti - 1) % stages
            for x in "kv":
                if T + ti >= stages:
                    yield B[x + "_empty"][st], (T + ti) // stages + 1 & 1
                assert state[x][st] == 0, "a stage overwritten"
                state[x][st] = 1 if split else 2
                state["scales"] = T + ti
                if not bf16:
                    B[x + "_full"][st].arrive()
                elif ti > 0:  # (the copies of the tile before have landed)
                    B[x + "_full"][last].arrive()
        if bf16:
            B["k_full"][(T + n - 1) % stages].arrive()
            B["v_full"][(T + n - 1) % stages].arrive()
        T += n
        seg += 1


def mma(B, stages, bufs, state):
    T = seg = K = 0

    def k_full(k, split):
        x = T + (k if split else k // 2)
        return B["k_full"][x % stages], x // stages & 1

    def scores(k, steps, split):
        x, s, buf = T + (k if split else k // 2), k % 2, (K + k) % bufs
        st = x % stages
        assert B["k_full"][st].phase * stages + st > x, "K is not there"
        assert state["k"][st] > 0 and state["s"][buf] == state["p"][buf] == 0
        state["k"][st] -= 1
        state["q"] -= 1
        state["s"][buf] = 1
        B["s_full"][buf].arrive()
        if split or s == 1:
            B["k_empty"][st].arrive()
        if k == steps - 1:
            B["q_empty"].arrive()

    for got, run in each_run(B, state):
        if got is not None:
            yield got, run
            continue
        n, split = run
        steps, ahead = (n, 2) if split else (2 * n, bufs)
        if n > 0:
            yield B["q_full"], seg & 1
        for k in range(min(ahead, steps)):
            yield k_full(k, split)
            scores(k, steps, split)
        for k in range(steps):
            x, s, buf = T + (k if split else k // 2), k % 2, (K + k) % bufs
            st = x % stages
            if not split and k + ahead < steps:
                yield k_full(k + ahead, split)
            yield B["v_full"][st], x // stages & 1
            yield B["p_full"][buf], (K + k) // bufs & 1
            assert state["v"][st] > 0 and state["p"][buf] == 1
            state["v"][st] -= 1
            state["p"][buf] = 0
            if bufs > 2 or k + ahead >= steps:
                B["o_full"][s][state["o"][s] & 1 if bufs > 2 else 0].arrive()
            state["o"][s] += 1
            if split or s == 1:
                B["v_empty"][st].arrive()
            if k + ahead < steps:
                if split:
                    yield k_full(k + ahead, split)
                scores(k + ahead, steps, split)
        K += steps
        T += n
        seg += n > 0


def softmax(s, B, bufs, state, meet, rng):
    cs = os = K = T = blocks = 0
    for got, run in each_run(B, state):
        if got is not None:
            yield got, run
            continue
        n, split = run
        if n == 0:
            continue
        first = s if split else 0
        for ti in range(first, n, 2 if split else 1):
            k = K + (ti if split else 2 * ti + s)
            buf = k % bufs
            yield B["s_full"][buf], k // bufs & 1
            cs += 1
            assert state["s"][buf] == 1
            if ti != first and rng.random() < 0.3:  # a maximum is raised: O of the tiles before is rescaled
                if bufs > 2:
                    yield B["o_full"][s][cs & 1], (cs - 2) >> 1 & 1
                assert state["o"][s] == cs - 1
            assert state["scales"] < T + ti + 8  # (whose scales take the place of this tile's)
            state["s"][buf], state["p"][buf] = 0, 1
            B["p_full"][buf].arrive()
        if first < n:
            yield (B["o_full"][s][cs - 1 & 1], (cs - 1) >> 1 & 1) if bufs > 2 else (B["o_full"][s][0], os & 1)
            assert state["o"][s] == cs
            os += 1
        T += n
        K += n if split else 2 * n
        blocks += 1
        meet[s] = blocks  # the barrier of both streams at a block's end
        yield None, blocks


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("stages,bufs", [(2, 2), (4, 3)])
@pytest.mark.parametrize("seed", range(40))
def test_every_role_comes_to_its_end(bf16, stages, bufs, seed):
    rng = random.Random(seed)
    runs = [(rng.choice([0, 1, 1, 2, 3, 4, 5, 6, 7, 12, 31]), rng.random() < 0.5) for _ in range(rng.choice([1, 2, 5, 12]))]
    for _ in range(5):
        B, meet = bars(stages), [0, 0]
        state = dict(q=0, k=[0] * stages, v=[0] * stages, s=[0] * 3, p=[0] * 3, o=[0, 0], scales=-1, run=[None] * 4)
        roles = [plan(runs, B, state), conv(B, bf16, stages, state), mma(B, stages, bufs, state),
                 softmax(0, B, bufs, state, meet, rng), softmax(1, B, bufs, state, meet, rng)]
        waits = {i: next(g, "end") for i, g in enumerate(roles)}
        while any(w != "end" for w in waits.values()):
            ready = [i for i, w in waits.items() if w != "end" and (min(meet) >= w[1] if w[0] is None else w[0].passed(w[1]))]
            assert ready, f"stuck: {runs}"
            i = rng.choice(ready)
            waits[i] = next(roles[i], "end")
        assert state["q"] == 0 and state["k"] == state["v"] == [0] * stages and state["s"] == state["p"] == [0] * 3
