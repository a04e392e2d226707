"""How the loss over a vocabulary cuts its work, on the host: every tile once, every step of a cut contraction once, pieces' results
within their room, launches large enough for any number of tokens that have a target."""
import ctypes as C
import math
import os
import random
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def L(tmp_path_factory):
    lib = str(tmp_path_factory.mktemp("vocab_plan") / "vocab_plan.so")
    subprocess.run(["g++", "-O1", "-std=c++17", "-Wall", "-shared", "-fPIC", os.path.join(HERE, "vocab_plan_shim.cpp"), "-o", lib], check=True)
    L = C.CDLL(lib)
    L.room.restype = C.c_longlong
    for f, n in ((L.dx_tile, 3), (L.dw_tile, 3), (L.dx, 4), (L.dw, 4)):
        f.argtypes = [C.c_int] * n + [C.c_longlong] + ([C.c_void_p] if n == 4 else [])
    L.grid_dx.argtypes = [C.c_int] * 3 + [C.c_longlong]
    L.slots.argtypes = [C.c_int, C.c_longlong]
    L.step.argtypes, L.power.restype = [C.c_float], C.c_float
    return L


def numbers(f, *args, n=6):
    out = (C.c_int * n)()
    f(*args, out)
    return list(out)


def check_items(L, plan, grid, slots):
    GM, GN, full, rest, pieces, steps = plan
    out = (C.c_int * (4 * max(grid, 1)))()
    n = L.items((C.c_int * 6)(*plan), grid, out)
    seen, places = {}, set()
    for i in range(n):
        unit, lo, hi, slot = out[4 * i:4 * i + 4]
        assert 0 <= unit < GM * GN and 0 <= lo <= hi <= steps
        seen.setdefault(unit, []).append((lo, hi))
        if slot >= 0:
            assert slot < slots and slot not in places
            places.add(slot)
            assert slot == (unit - full) * pieces + [x for x in range(pieces) if steps * x // pieces == lo and steps * (x + 1) // pieces == hi][0]
        else:
            assert (lo, hi) == (0, steps)
    assert sorted(seen) == list(range(GM * GN)) and full + rest == GM * GN
    for unit, parts in seen.items():
        parts.sort()
        assert parts[0][0] == 0 and parts[-1][1] == steps and all(a[1] == b[0] for a, b in zip(parts, parts[1:]))
        assert len(parts) == (1 if unit < full or pieces == 1 else pieces)


def cases():
    rng = random.Random(1)
    out = [(1, 64, 1), (64, 64, 1), (777, 768, 32003), (8192, 2048, 50272), (4096, 4096, 50272), (8192, 512, 700), (256, 32768, 500), (65536, 64, 30)]
    for _ in range(60):
        out.append((round(2 ** rng.uniform(0, 13.5)), 64 * round(2 ** rng.uniform(0, 7)), round(2 ** rng.uniform(0, 17))))
    return out


def test_gradients_are_cut_into_every_step_once(L):
    rng = random.Random(2)
    for T, d, V in cases():
        rows = L.rows(T, V, 1, 0)
        room = C.c_longlong()
        L.room(rows, T, d, V, 1, 1, 0, C.byref(room))
        count = min(T, rows)
        for share in (room.value, 0):
            dx, dw = L.dx_tile(count, d, V, share), L.dw_tile(count, d, V, share)
            grid = L.grid_dx(dx, count, d, share)
            for n in {0, 1, count, rng.randint(0, count), rng.randint(0, count), count // 2}:
                plan = numbers(L.dx, dx, n, d, V, share)
                assert plan[5] == -(-V // 64)
                check_items(L, plan, grid, L.slots(dx, share))
                # cut units are within the launch that adds them
                tm, tn = numbers(L.tile_size, dx, n=2)
                units = -(-count // tm) * -(-d // tn)
                assert plan[4] == 1 or plan[3] <= min(units, L.slots(dx, share) // 2)
            whole = numbers(L.dw, dw, count, d, V, share)
            dw_share = share if whole[4] > 1 else 0
            for n in (0, 1, count, count // 2):
                plan = numbers(L.dw, dw, n, d, V, dw_share)
                check_items(L, plan, (whole[0] * whole[1] + 7) // 8 * 8 + (L.slots(dw, dw_share) + 7) // 8 * 8, L.slots(dw, dw_share))
                assert plan[4] == 1 or plan[3] == whole[3]


def test_tiles_once(L):
    for GM, GN in ((1, 1), (1, 197), (3, 126), (20, 197), (32, 3), (33, 5), (4, 8), (7, 1)):
        out = (C.c_int * (2 * GM * GN))()
        assert L.tiles(GM, GN, out) == GM * GN
        assert {(out[2 * i], out[2 * i + 1]) for i in range(GM * GN)} == {(m, n) for m in range(GM) for n in range(GN)}


def test_tiles_suit_the_sizes(L):
    wide, tokens = 0, lambda *a: numbers(L.tile_size, L.logits_tile(*a), n=2)[0]  # noqa: E731
    assert L.logits_tile(8192, 2048, 50272) == L.dx_tile(8192, 2048, 50272, 1 << 26) == L.dw_tile(8192, 2048, 50272, 1 << 26) == wide
    assert tokens(1, 2048, 50272) == tokens(64, 4096, 32000) == 64 and tokens(100, 2048, 50272) == 128


def test_pieces(L):
    for T in (1, 255, 256, 257, 8192, 100000, 1 << 20):
        for V in (1, 700, 50272, 1 << 20):
            for grads, f32 in ((0, 0), (1, 0), (1, 1)):
                rows = L.rows(T, V, grads, f32)
                assert rows % 256 == 0 and 256 <= rows <= 65536
                wide = -(-V // 256) * 256
                if grads and rows > 256:
                    assert rows * wide * (4 if f32 else 2) <= (1 << 30)
                assert rows - T < 256 or T <= 256


def test_tokens_by_tile_have_room(L):
    """Of each tile's tokens, filled up to the next 64 behind those of smaller targets and 64 for each tile before: no two places the same, and all within."""
    rng = random.Random(4)
    for T, d, V in list(cases()) + [(300, 64, 1), (5000, 64, 300)]:
        rows = L.rows(T, V, 1, 0)
        n = min(T, rows)
        out = (C.c_longlong * 2)()
        L.lacks_room(rows, T, d, V, 1, out)
        spread = [rng.randrange(V) for _ in range(n)]
        for targets in (spread, [V - 1] * n, [t // 128 * 128 for t in spread], [0]):
            for width in (128, 256):
                at, below = 0, 0
                counts = {}
                for t in targets:
                    counts[t // width] = counts.get(t // width, 0) + 1
                for tile in sorted(counts):
                    start = below + 64 * tile
                    assert start >= at
                    at = start + -(-counts[tile] // 64) * 64
                    below += counts[tile]
                # (the next step's tokens are read ahead)
                assert at * width * 2 <= out[1] and (at + 64) * 4 <= out[0]


def test_exponentials_as_steps(L):
    """Relative errors of exponentials that are kept as steps of their logarithm: those of half precision over 79 powers of two, 2^-9 over all that
    bfloat16 holds as normal numbers; beyond, and in masked places, 0."""
    assert L.step(0.0) == 65535 and L.power(65535) == 0.0 and L.step(-math.inf) == 0 and L.power(0) == -math.inf and 0 <= L.step(math.nan) <= 65535
    rng, last = random.Random(3), 65536
    for i in range(40000):
        y = C.c_float(-87.3 * (i + rng.random()) / 40000).value
        s = L.step(y)
        assert 0 < s <= last
        last = s
        off = abs(math.expm1(L.power(s) * math.log(2) - y))
        # (half a step, and the roundings of a 32-bit product and of its sum with 2^23 .. 2^24, and back)
        assert off <= (2.0 ** -11 if y > -54.8 else 2.0 ** -9), (y, s, off)
    assert L.step(-88.5) == L.step(-1000.0) == L.step(-3e38) == 0
    assert all(L.power(s) < L.power(s + 1) for s in range(65535))


def test_plans_do_not_hang_on_fused_arithmetic(L, tmp_path):
    """Host and device, which fuses products with sums where it may, and each kernel for itself make the same plans: their costs are the same bits by a
    build that fuses and by one that cannot."""
    clang = "/opt/rocm/llvm/bin/clang++"
    if not os.path.exists(clang) or " fma " not in open("/proc/cpuinfo").read():
        pytest.skip("no compiler or processor that fuses")
    lib = str(tmp_path / "fused.so")
    subprocess.run([clang, "-O2", "-std=c++17", "-mfma", "-ffp-contract=fast-honor-pragmas", "-shared", "-fPIC", os.path.join(HERE, "vocab_plan_shim.cpp"), "-o", lib],
                   check=True)
    F = C.CDLL(lib)
    for lib in (L, F):
        for f in (lib.dx_cost, lib.dw_cost):
            f.argtypes, f.restype = [C.c_int] * 4 + [C.c_longlong], C.c_float
    rng = random.Random(6)
    for _ in range(4000):
        n, d, V, room = round(2 ** rng.uniform(0, 13.5)), 64 * round(2 ** rng.uniform(0, 7)), round(2 ** rng.uniform(0, 17)), rng.choice((0, 1 << 22, 1 << 26))
        for tile in range(9):
            assert L.dx_cost(tile, n, d, V, room) == F.dx_cost(tile, n, d, V, room), (tile, n, d, V, room)
            assert L.dw_cost(tile, n, d, V, room) == F.dw_cost(tile, n, d, V, room), (tile, n, d, V, room)
