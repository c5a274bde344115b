"""Pages, windows and splits of the attention over a paged cache (csrc/attention_plan.h and .cpp: plain C++, the same functions that the kernels call)
without a GPU, built with -fsanitize=address,undefined."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_12357_amd", "csrc")
CUS, MOST = 256, 2 ** 31 - 1 - 2 * 4096                       # the longest bound that a call takes


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
                    lines.append(f"seen {length} {max_len} {window} {entries} {shift} 64 0")
                    bad = length < 0 or length > max_len or length > entries << shift
                    first = max(0, length - window) if window else 0
                    want.append((0, 0, 1) if bad else (0, 0, 0) if length == 0 else (first, length, 0))
    assert [g[:3] for g in ask(lines)] == want


def test_parts_cover_what_is_seen_once(ask):
    rng = random.Random(1)
    cases = []
    for _ in range(400):
        max_len = rng.choice([1, 2, 64, 65, rng.randint(1, 10000), rng.randint(1, 2 ** 22), MOST])
        window = rng.choice([0, 0, 1, 63, 64, 65, rng.randint(1, 5000), rng.randint(1, max_len)])
        cases.append((rng.choice([1, 2, rng.randint(1, 500)]), rng.choice([1, 2, 8, 16]), rng.choice([1, 4, 16, 17, 71]), max_len, window))
    plans = ask([f"plan {b} {h} {g} {m} {w} {CUS}" for b, h, g, m, w in cases])
    lines, which = [], []
    for (b, h, g, max_len, window), (split, parts) in zip(cases, plans):
        assert split % 64 == 0 and 64 <= split <= 4096 and parts >= 1
        for length in {0, 1, max_len, max_len // 2, max(0, max_len - 63), min(max_len, window), min(max_len, window + 1), rng.randint(0, max_len)}:
            some = range(parts) if parts < 40 else sorted({0, 1, parts - 1} | {rng.randrange(parts) for _ in range(10)})
            for s in some:
                lines.append(f"seen {length} {max_len} {window} {2 ** 29} 4 {split} {s}")
                which.append((length, split, parts, s))
    ends = {}
    for (length, split, parts, s), (first, end, bad, begin, stop) in zip(which, ask(lines)):
        assert not bad and begin <= stop <= end and stop - begin <= split
        if begin < stop:
            assert begin % 64 == 0 and begin == first // 64 * 64 + s * split
            assert stop == end or stop == begin + split
            # its pages' numbers fit, and so does the sum of positions
            assert ((begin + split - 1) >> 2) - (begin >> 2) + 1 <= 1024 and begin + split + 4096 < 2 ** 31
        if s == 0 and length:
            assert begin <= first < stop
        if s == parts - 1:
            assert first // 64 * 64 + (s + 1) * split >= end     # nothing is left behind the last part
        ends[(length, split, s)] = (begin, stop)


def test_few_long_sequences_are_split_and_full_batches_less(ask):
    (one,), (many,), (short,) = (ask([f"plan {b} 8 4 {m} 0 {CUS}"]) for b, m in ((1, 131072), (256, 131072), (1, 200)))
    assert one[1] * 8 >= CUS and many[0] >= one[0] and short[1] == 1
