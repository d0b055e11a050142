"""The rings between the warps of the products on the tensor cores, played through on the CPU with the kernels' own numbers of stages and barriers.

A barrier counts the phases that have ended; a wait for phase p looks at one bit of that count, so it also ends where phase p - 1 has not ended yet.  Copies may arrive in any order: each play has some that come only when
nothing else can go on.  What a team of warps takes from a stage has to be its block's, in every play."""
import ctypes
import random

import pytest

WIDTHS = (32, 64, 128, 256)


def rings(width, dtype, gated):
    from paper_2608_18147_gb300 import native
    to = (ctypes.c_int32 * 7)()
    assert native.lib().ecasq_project_rings(width, {"f32": native.F32, "bf16": native.BF16}[dtype], gated, to) == native.OK
    return dict(zip(("teams", "code_stages", "code_bars", "x_stages", "levels", "parts", "buffers"), to))


def passes(ended, phase):
    """A wait for phase number `phase` of a barrier with `ended` phases behind it."""
    return (ended & 1) != (phase & 1)


def play(r, total, late_codes, late_x, rng):
    """None, or (what, block, the block found in its place)."""
    T, C, B, X, A = r["teams"], r["code_stages"], r["code_bars"], r["x_stages"], r["levels"]
    c_full, c_empty, x_full, x_empty, a_full, a_empty = [0] * B, [0] * C, [0] * X, [0] * X, [0] * A, [0] * A
    codes, xs = [None] * C, [None] * X  # the block that lies in each stage
    asked = {"c": 0, "x": 0}
    flying = {"c": set(), "x": set()}
    team = [(t, "first") for t in range(T)]  # block, and what comes next for it
    issued = done = 0
    wrong = []

    def fetch(i):
        if not passes(c_full[i % B], i // B):
            return False
        if codes[i % C] != i:
            wrong.append(("codes", i, codes[i % C]))
        c_empty[i % C] += 1
        return True

    def step_team(t):
        i, at = team[t]
        if i >= total:
            return False
        if at == "first":
            if not fetch(i):
                return False
            team[t] = (i, "levels")
        elif at == "levels":
            if not passes(a_empty[i % A], i // A - 1):
                return False
            team[t] = (i, "x")
        elif at == "x":
            if not passes(x_full[i % X], i // X):
                return False
            if xs[i % X] != i:
                wrong.append(("x", i, xs[i % X]))
            team[t] = (i, "next")
        else:
            if i + T < total and not fetch(i + T):
                return False
            a_full[i % A] += 1
            team[t] = (i + T, "levels")
        return True

    def ask(kind, empty, n):
        i = asked[kind]
        if i >= total or not passes(empty[i % n], i // n - 1):
            return False
        asked[kind] += 1
        flying[kind].add(i)
        return True

    def land(kind, i):
        flying[kind].remove(i)
        if kind == "c":
            codes[i % C] = i
            c_full[i % B] += 1
        else:
            xs[i % X] = i
            x_full[i % X] += 1

    while done < total and not wrong:
        moved = False
        actions = ["c", "x", "issue", "done"] + list(range(T))
        rng.shuffle(actions)
        for a in actions:
            if a == "c":
                moved |= ask("c", c_empty, C)
            elif a == "x":
                moved |= ask("x", x_empty, X)
            elif a == "issue":
                if issued < total and passes(a_full[issued % A], issued // A):
                    issued += 1
                    moved = True
            elif a == "done":
                if done < issued:
                    a_empty[done % A] += 1
                    x_empty[done % X] += 1
                    done += 1
                    moved = True
            else:
                moved |= step_team(a)
        for kind, late in (("c", late_codes), ("x", late_x)):
            for i in sorted(flying[kind] - late):
                if rng.random() < 0.7:
                    land(kind, i)
                moved = True
        if not moved:  # only now the late ones
            waiting = [(kind, i) for kind in "cx" for i in flying[kind]]
            if not waiting:
                return ("nothing can go on", done, None)
            land(*rng.choice(waiting))
    return wrong[0] if wrong else None


def plays(r):
    rng, total = random.Random(1), 2 * r["code_stages"] * r["teams"] + 6
    for i in range(total):
        for late in (({i}, set()), (set(), {i}), ({i, i + 1}, set()), ({i}, {i + 1}), ({i, i + 3}, {i})):
            for _ in range(3):
                found = play(r, total, *late, rng)
                if found:
                    return found
    for _ in range(200):
        found = play(r, total, {i for i in range(total) if rng.random() < 0.3}, {i for i in range(total) if rng.random() < 0.3}, rng)
        if found:
            return found
    return None


@pytest.mark.parametrize("gated", [0, 1])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_each_team_takes_its_own_block(width, dtype, gated):
    assert plays(rings(width, dtype, gated)) is None


def test_the_plays_find_what_they_look_for():
    """One barrier a stage of codes, where two teams take turns at three stages; a stage of x that comes round before it is known to have been there."""
    good = dict(teams=2, code_stages=3, code_bars=6, x_stages=3, levels=2, parts=1, buffers=3)
    assert plays(good) is None
    assert plays(dict(good, code_bars=3))[0] == "codes"
    assert plays(dict(good, code_stages=2, code_bars=2)) is None and plays(dict(good, code_stages=5, code_bars=5)) is None
    assert plays(dict(good, x_stages=1, levels=4))[0] in ("x", "codes", "nothing can go on")


def test_refusals():
    from paper_2608_18147_gb300 import native
    to = (ctypes.c_int32 * 7)()
    L = native.lib()
    assert all(L.ecasq_project_rings(*bad) == native.EINVAL for bad in ((0, 1, 0, to), (96, 1, 0, to), (128, 3, 0, to), (128, -1, 0, to), (128, 1, 0, None)))


@pytest.mark.gpu
@pytest.mark.parametrize("n,k,b,group,gated", [(9762, 4, 539, 64, 1), (4000, 70, 1030, 128, 0), (6000, 300, 257, 32, 1)])
def test_codes_that_come_late(n, k, b, group, gated):
    """Tiles of 128 rows of x, few blocks of columns, codes that nothing has read before: the same results as with codes in the caches."""
    torch = pytest.importorskip("torch")
    import paper_2608_18147_gb300 as E
    from test_gpu_project_tiles import check, inputs, plan, sums
    assert plan(n, k, b, group, "f16", gated)["width"] == 128
    for seed in range(10):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        x, codes, levels, scales, w = inputs(n, k, b, group, "f16", gated, 16, gen)
        p, dp = sums(x, w, k, "f16")
        for turn in range(10):
            fresh = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")[turn * 4096:][:codes.numel()].view(codes.shape)
            fresh.copy_(codes)
            torch.empty(200 << 20, dtype=torch.uint8, device="cuda").zero_()  # (nothing of it is in the caches)
            if gated:
                y = E.ecasq_gated(x, fresh, levels, scales, group, activation=None)
                (g, u), (dg, du) = p.chunk(2, dim=1), dp.chunk(2, dim=1)
                check(y, g * u, dg * u.abs() + g.abs() * du + dg * du + 2.0 ** -23 * (g * u).abs(), "f16")
            else:
                check(E.ecasq_project(x, fresh, levels, scales, group), p, dp, "f16")
