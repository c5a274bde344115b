"""Pages, windows and splits of the attention over a paged cache (csrc/attention_plan.h and .cpp: plain C++, the same functions that the kernels call)
without a GPU, built with -fsanitize=address,undefined."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_12357_amd", "csrc")
SETUP, MOST = 4, 2 ** 31 - 1 - 2 * 4096                       # the longest bound that a call takes


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    cxx = shutil.which(os.environ.get("CXX", "g++"))
    if cxx is None:
        pytest.skip("no host C++ compiler")
    out = str(tmp_path_factory.mktemp("plan") / "attention_plan_check")
    subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                    "-static-libasan", "-static-libubsan", "-Wall", "-Wextra", "-Werror", "-I", CSRC,
                    os.path.join(ROOT, "tests", "host", "attention_plan_check.cpp"), os.path.join(CSRC, "attention_plan.cpp"), "-o", out], check=True)
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0")
    env.pop("LD_PRELOAD", None)

    def run(lines):
        r = subprocess.run([out], input="".join(f"{line}\n" for line in lines), capture_output=True, text=True, check=True, env=env)
        got = [tuple(map(int, line.split())) for line in r.stdout.splitlines()]
        assert len(got) == len(lines)
        return got
    return run


def test_page_sizes(ask):
    sizes = [0, -4, 1, 2, 3, 4, 6, 8, 12, 16, 48, 64, 256, 1 << 20, (1 << 20) + 4]
    assert [n for n, in ask([f"shift {n}" for n in sizes])] == [-1, -1, -1, -1, -1, 2, -1, 3, -1, 4, -1, 6, 8, 20, -1]


def test_pages_of_positions(ask):
    """Numbers outside the cache, positions in front of the sequence and behind the table's row have no page; nothing outside the row is read."""
    row = [7, 0, -1, 9, 10, 11, -2147483648, 2147483647]
    for shift in (2, 4, 10):
        size = 1 << shift
        got = ask([f"page {shift} 10 {pos} " + " ".join(map(str, row)) for pos in (0, size - 1, size, 2 * size, 3 * size, 4 * size, 5 * size, 6 * size, 7 * size,
                                                                                     8 * size - 1, 8 * size, 2 ** 31 - 1, -1, -2 ** 31)])
        assert [p for p, in got] == [7, 7, 0, -1, 9, -1, -1, -1, -1, -1, -1, -1, -1, -1]
    assert ask(["page 4 10 0"]) == [(-1,)]                   # a row without entries


def test_what_a_token_sees(ask):
    """Lengths from nothing to the longest, windows and tables that end before, at and behind them."""
    lines, want = [], []
    for length in (-2 ** 31, -1, 0, 1, 2, 63, 64, 65, 1000, MOST - 1, MOST, MOST + 1, 2 ** 31 - 1):
        for max_len in (0, 1, 64, 1000, MOST):
            for window in (0, 1, 63, 64, 65, 2 ** 31 - 1):
                for shift, entries in ((2, 1), (4, 4), (4, 63), (20, 2048), (20, 2 ** 31 - 1)):
                    lines.append(f"seen {length} {max_len} {window} {entries} {shift}")
                    bad = length < 0 or length > max_len or length > entries << shift
                    first = max(0, length - window) if window else 0
                    want.append((0, 0, 1, 0) if bad else (0, 0, 0, 0) if length == 0 else (first, length, 0, -(-(length - first // 64 * 64) // 64)))
    assert ask(lines) == want


def _line(ask, workgroups, align, least, units, blocks):
    (got,) = ask([f"line {workgroups} {align} {least} {units} " + " ".join(map(str, blocks))])
    assert got[-1] == -1 and len(got) % 7 == 1
    return [got[i:i + 7] for i in range(0, len(got) - 1, 7)]


def test_every_block_belongs_to_one_workgroup(ask):
    """Shares are equal, in the order of the line; a workgroup has at most two units in part, its first and its last; parts of a unit know each other.
    Where units are rounded up, a workgroup has one of them."""
    rng = random.Random(1)
    for turn in range(120):
        align = rng.choice([0, 0, 4, 8])
        workgroups, least, units = rng.choice([1, 2, 7, 64, 512, 768, 1024]), rng.choice([1, 4, 8]), rng.choice([1, 2, 8, 5, 40])
        kind = rng.randrange(4)
        blocks = [rng.choice([0, 1, 2, rng.randint(0, 130)]) if kind else rng.randint(100, 3000) for _ in range(rng.choice([1, 2, 3, 30, 300]))]
        if kind == 3:
            blocks[rng.randrange(len(blocks))] = 2048
        places = lambda n: -(-n // align) * align if align else n + SETUP  # noqa: E731
        total = sum(places(n) for n in blocks if n) * units
        if align:
            workgroups = max(1, total // align)
        got = _line(ask, workgroups, align, least, units, blocks)
        each = align or max(least, -(-total // workgroups))
        # the line, unit by unit: SETUP places or none, the blocks, places up to a whole share or none
        place, line = {}, 0
        for b, n in enumerate(blocks):
            for unit in range(units if n else 0):
                place[b, unit] = line + (0 if align else SETUP)
                line += places(n)
        at, parts = -1, {}
        for w, b, unit, block, n, first, count in got:
            begin = place[b, unit]
            assert n >= 1 and block >= 0 and block + n <= blocks[b] and begin + block > at
            assert w * each <= begin + block and begin + block + n <= (w + 1) * each
            at = begin + block + n - 1
            parts.setdefault((b, unit), []).append((w, block, n))
            assert first == begin // each and count == (begin + blocks[b] - 1) // each - first + 1
        assert set(parts) == set(place)
        if align:
            assert len({w for w, *_ in got}) == len(got)
        slots = {}
        for (b, unit), p in parts.items():
            assert [w for w, _, _ in p] == list(range(p[0][0], p[0][0] + len(p)))
            assert [block for _, block, _ in p] == [sum(n for _, _, n in p[:i]) for i in range(len(p))] and sum(n for _, _, n in p) == blocks[b]
            for w, block, _ in p if len(p) > 1 else []:
                key = (w, block == 0)                        # where its sums go
                assert key not in slots
                slots[key] = (b, unit)


def test_plans(ask):
    """Grids hold the longest line that a call can have; where there is little work a workgroup has one unit."""
    cases = [(1, 8, 4, 131072, 0), (64, 8, 4, 8192, 0), (1, 16, 1, 200, 0), (33, 1, 71, 5000, 1000), (1, 1, 1, 0, 0), (1, 1, 1, 1, 1), (0, 8, 4, 100, 0),
             (4096, 16, 24, MOST, 0), (256, 8, 8, 131072, 0), (1, 1, 16, MOST, 0), (5000, 8, 4, 500, 0), (1 << 20, 8, 4, 64, 0), (8, 8, 4, 4096, 0)]
    plans = ask([f"plan {b} {h} {g} {m} {w} 512 256" for b, h, g, m, w in cases])
    for (b, h, g, m, w), (fits, *plan) in zip(cases, plans):
        span = min(m, w + 63) if 0 < w < m else m
        units, blocks = b * h * -(-g // 16), max(1, -(-span // 64))
        assert fits == (units * (blocks + 8) < 2 ** 30) or units * (blocks + 4) >= 2 ** 29
        if fits:
            workgroups, align, split, few, waves = plan
            assert waves == (1 if blocks <= 8 and units > 512 else 4)
            assert workgroups * 256 < 2 ** 32 and (workgroups <= 4096 or not split)
            if align:
                assert workgroups == max(1, units * -(-blocks // align)) and split == (blocks > align)
            else:
                assert workgroups == 2048 // waves and split
    got = [p[2] if p[0] else None for p in plans]
    assert got == [0, 0, 4, 8, 4, 4, 4, None, 0, 0, 0, 0, 8] and plans[3][4] == 1 and plans[0][4] == 0


def test_units_of_their_own_waves(ask):
    """Units of up to eight blocks have a wave each where there are more of them than workgroups, up to two rounds of waves, or one for units of one
    block; beyond, waves share the line."""
    cases = [(128, 300, 0), (512, 512, 0), (513, 512, 0), (65, 65, 0), (65, 64, 0), (257, 64, 0), (64, 64, 0), (64, 300, 0), (128, 513, 0), (100, 5000, 400), (100, 5000, 500)]
    got = ask([f"plan {b} 8 4 {m} {w} 512 256" for b, m, w in cases])
    assert [p[5] for p in got] == [1, 1, 1, 1, 1, 1, 4, 4, 4, 1, 4]
    assert [p[2] for p in got] == [8, 8, 0, 8, 8, 0, 8, 8, 0, 8, 0]
    assert [p[1] for p in got] == [1024, 4096, 2048, 520, 520, 2048, 512, 512, 512, 800, 512]
