"""The barriers between the loading thread, the decoding teams and the tensor operations of the attention over a 4-bit cache, played
through on the CPU in random order (as the kernel for many query rows has them: `tree_attn_tc.cu`).

A wait asks for a parity, so it is right only while the waiter is at most one phase away; the model gives every wait the phase it means and
checks that it passes no sooner, that no stage is overwritten before it was read, that every reader finds its own tile, and that
everything comes to an end."""
import random

import pytest


class Barrier:
    def __init__(self, count):
        self.count = self.left = count
        self.phase = 0

    def arrive(self):
        assert self.left > 0
        self.left -= 1
        if self.left == 0:
            self.phase, self.left = self.phase + 1, self.count


class Wrong(Exception):
    pass


def play(seed, slots=3, told=6, teams=2, stages=4, scores=3, warps=2):
    rnd = random.Random(seed)
    full, empty = [Barrier(warps) for _ in range(stages)], [Barrier(1) for _ in range(stages)]
    s_full, p_ready, pv_done = ([Barrier(1) for _ in range(scores)] for _ in range(3))
    filled, free = [Barrier(1) for _ in range(told)], [Barrier(warps) for _ in range(slots)]
    u_full, u_empty, q_free = ([Barrier(n) for _ in range(2)] for n in (1, 4, 1))
    o_full, o_free = Barrier(1), Barrier(1)
    units = [rnd.choice([1, 1, 2, 3, 4, 5, 8, 13]) for _ in range(rnd.choice([1, 2, 6, 12]))]
    tree = [rnd.random() < 0.7 for _ in units]
    job, stage, copies, products = [None] * slots, [None] * stages, [], []
    k_pos, v_pos = (lambda t: t if t < 2 else 2 * t - 2), (lambda t: 2 * t + 3)

    def loader():
        n, kt, vt, behind = 0, 0, 0, []

        def post(is_tree, pos):
            nonlocal n
            if n >= slots:
                yield free[n % slots], n // slots - 1
            job[n % slots] = (n, pos, is_tree)
            bar = filled[n % told]
            n += 1
            if pos >= 0 and not is_tree and rnd.random() < 0.8:        # (codes arrive when they arrive; a page that is not there at once)
                copies.append(bar.arrive)
            else:
                bar.arrive()
        for u, tiles in enumerate(units):
            if u >= 2:
                yield u_empty[u % 2], u // 2 - 1
            u_full[u % 2].arrive()
            if u >= 2:
                yield q_free[u % 2], u // 2 - 1
            for it in range(tiles):
                is_tree = tree[u] and it == tiles - 1
                yield from post(is_tree, k_pos(kt))
                kt += 1
                if len(behind) == 2:
                    yield from post(behind.pop(0), v_pos(vt))
                    vt += 1
                behind.append(is_tree)
        while behind:
            yield from post(behind.pop(0), v_pos(vt))
            vt += 1
        for _ in range(teams):
            yield from post(False, -1)

    def decoder(team, warp):
        n = team
        while True:
            yield filled[n % told], n // told
            number, pos, is_tree = job[n % slots]
            if number != n:
                raise Wrong("a slot holds another job")
            if pos < 0:
                return
            if pos >= stages:
                yield empty[pos % stages], pos // stages - 1
            yield None
            if warp == 0:
                if stage[pos % stages] and not stage[pos % stages][1]:
                    raise Wrong("a stage is overwritten before it was read")
                stage[pos % stages] = [pos, False]
            (copies.append if is_tree and warp == 0 else lambda f: f())(full[pos % stages].arrive)
            free[n % slots].arrive()
            n += teams

    def read(pos):
        if stage[pos % stages][0] != pos:
            raise Wrong("a stage holds another tile")
        stage[pos % stages][1] = True

    def score():
        t = 0
        for u, tiles in enumerate(units):
            yield u_full[u % 2], u // 2
            u_empty[u % 2].arrive()
            for _ in range(tiles):
                if t >= scores:
                    yield pv_done[t % scores], t // scores - 1
                yield full[k_pos(t) % stages], k_pos(t) // stages
                read(k_pos(t))
                products.append((s_full[t % scores], empty[k_pos(t) % stages]))
                t += 1
            products.append((q_free[u % 2],))

    def softmax():
        t = 0
        for u, tiles in enumerate(units):
            yield u_full[u % 2], u // 2
            u_empty[u % 2].arrive()
            for _ in range(tiles):
                yield s_full[t % scores], t // scores
                yield None
                p_ready[t % scores].arrive()
                t += 1

    def output_of(first):
        t = 0
        for u, tiles in enumerate(units):
            yield u_full[u % 2], u // 2
            u_empty[u % 2].arrive()
            if first:
                yield o_full, u
                yield None
                o_free.arrive()
                continue
            if u:
                yield o_free, u - 1
            for j in range(tiles):
                yield p_ready[t % scores], t // scores
                yield full[v_pos(t) % stages], v_pos(t) // stages
                read(v_pos(t))
                products.append((empty[v_pos(t) % stages], pv_done[t % scores]) + ((o_full,) if j == tiles - 1 else ()))
                t += 1

    agents = {"load": loader(), "S": score(), "softmax": softmax(), "PV": output_of(False), "out": output_of(True)}
    agents |= {(t, w): decoder(t, w) for t in range(teams) for w in range(warps)}
    waits, pace = dict.fromkeys(agents), {k: rnd.choice([1, 1, 3, 10]) for k in agents}
    while agents:
        ready = []
        for k in agents:
            if waits[k] is None:
                ready.append(k)
            elif waits[k][0].phase % 2 != waits[k][1] % 2:             # what a wait for a parity sees
                if waits[k][0].phase <= waits[k][1]:
                    raise Wrong("a wait passes too soon")
                ready.append(k)
        ready += ["copy"] * bool(copies) + ["product"] * bool(products)
        if not ready:
            raise Wrong("nothing can go on")
        k = rnd.choices(ready, [pace.get(r, 2) for r in ready])[0]
        if k == "copy":
            copies.pop(rnd.randrange(len(copies)))()
        elif k == "product":
            for bar in products.pop(0):
                bar.arrive()
        else:
            try:
                waits[k] = next(agents[k])
            except StopIteration:
                del agents[k], waits[k]


def test_the_queue_of_the_decoding_teams_comes_to_its_end():
    for seed in range(1200):
        play(seed)


@pytest.mark.parametrize("change", [dict(told=3), dict(slots=6, teams=3)])
def test_the_model_finds_what_would_be_wrong(change):
    """One barrier a slot where the slots are odd, so that a team waits for every other phase of it; and three teams, so that a stage's
    jobs are not one team's."""
    with pytest.raises(Wrong):
        for seed in range(3000):
            play(seed, **change)
