"""The order of waits of the tcgen05 paged-attention kernel (wq_attn_paged_tc.cu), as a model on the CPU: the MMA warp,
the converting warps (as one) and the two softmax streams run their programs' waits and arrivals over every mix of blocks,
in all orders that a scheduler may choose at random, and must come to their ends; a stage is only written when all that reads
it is done.  Barriers are mbarriers: a wait names the parity of a phase.
"""
import random

import pytest


class Bar:
    def __init__(self, count):
        self.count, self.here, self.phase = count, 0, 0

    def arrive(self):
        self.here += 1
        if self.here == self.count:
            self.here = 0
            self.phase += 1

    def passed(self, parity):
        return self.phase & 1 != parity


def bars():
    two = lambda n: [Bar(n), Bar(n)]  # noqa: E731
    return dict(q_full=Bar(1), q_empty=Bar(1), k_full=two(1), k_empty=two(1), v_full=two(1), v_empty=two(1),
                s_full=[two(1), two(1)], p_full=[two(1), two(1)], o_full=two(1))


def conv(runs, B, bf16, state):
    T = seg = 0
    for n, split in runs:
        if seg > 0:
            yield B["q_empty"], (seg - 1) & 1
        B["q_full"].arrive()
        for ti in range(n):
            st = (T + ti) & 1
            if T + ti >= 2:
                yield B["k_empty"][st], ((T + ti) >> 1) + 1 & 1
            assert state["k"][st] == 0, "K overwritten"
            state["k"][st] = 1 if split else 2
            if bf16 and ti > 0:
                B["v_full"][st ^ 1].arrive()
            B["k_full"][st].arrive()
            if T + ti >= 2:
                yield B["v_empty"][st], ((T + ti) >> 1) + 1 & 1
            assert state["v"][st] == 0, "V overwritten"
            state["v"][st] = 1 if split else 2
            if not bf16:
                B["v_full"][st].arrive()
        if bf16:
            B["v_full"][(T + n - 1) & 1].arrive()
        T += n
        seg += 1


def mma(runs, B, state):
    T, seg, cs = 0, 0, [0, 0]
    for n, split in runs:
        step = 2 if split else 1

        def scores(s, t, hh):
            yield B["k_full"][(T + t) & 1], (T + t) >> 1 & 1
            B["s_full"][s][hh].arrive()
            if hh == 1:
                state["k"][(T + t) & 1] -= 1
            if hh == 1 and (split or s == 1):
                B["k_empty"][(T + t) & 1].arrive()
                if t == n - 1:
                    B["q_empty"].arrive()

        yield B["q_full"], seg & 1
        for i in range(4):
            s, hh = (i // 2, i % 2) if split else (i % 2, i // 2)
            t = s if split else 0
            if t < n:
                yield from scores(s, t, hh)
        for t in range(0, n, step):
            for i in range(4):
                s, hh = (i // 2, i % 2) if split else (i % 2, i // 2)
                mine = t + s if split else t
                if mine >= n:
                    continue
                st = (T + mine) & 1
                yield B["v_full"][st], (T + mine) >> 1 & 1
                yield B["p_full"][s][hh], cs[s] & 1
                cs[s] += hh
                if hh == 1:
                    state["v"][st] -= 1
                if hh == 1 and (split or s == 1):
                    B["v_empty"][st].arrive()
                if mine + step < n:
                    yield from scores(s, mine + step, hh)
                elif hh == 1:
                    B["o_full"][s].arrive()
        T += n
        seg += 1


def softmax(s, runs, B, meet):
    cs = os = 0
    for r, (n, split) in enumerate(runs):
        for ti in range(s if split else 0, n, 2 if split else 1):
            for hh in range(2):
                yield B["s_full"][s][hh], cs & 1
                cs += hh
                B["p_full"][s][hh].arrive()
        if (s if split else 0) < n:
            yield B["o_full"][s], os & 1
            os += 1
        meet[s] = r + 1  # the barrier of both streams at a block's end
        yield None, r + 1


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("seed", range(40))
def test_every_role_comes_to_its_end(bf16, seed):
    rng = random.Random(seed)
    runs = [(rng.choice([1, 1, 2, 3, 4, 5, 6, 7, 12, 31]), rng.random() < 0.5) for _ in range(rng.choice([1, 2, 5, 12]))]
    for _ in range(5):
        B, meet, state = bars(), [0, 0], dict(k=[0, 0], v=[0, 0])
        roles = [conv(runs, B, bf16, state), mma(runs, B, state), softmax(0, runs, B, meet), softmax(1, runs, B, meet)]
        waits = {i: next(g, "end") for i, g in enumerate(roles)}
        while any(w != "end" for w in waits.values()):
            ready = [i for i, w in waits.items() if w != "end" and (min(meet) >= w[1] if w[0] is None else w[0].passed(w[1]))]
            assert ready, f"stuck: {runs}"
            i = rng.choice(ready)
            waits[i] = next(roles[i], "end")
