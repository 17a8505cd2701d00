"""-m "not gpu": what the operators of include/dba_beam.h work out about places in memory, compiled for the host with sanitizers."""
import itertools
import os
import random
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
MOST = 2**31 - 1


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path_factory.mktemp("bounds") / "beam_bounds_driver")
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-fsanitize=address,undefined", "-fno-sanitize-recover",
                    os.path.join(HERE, "beam_bounds_driver.cpp"), "-o", exe], check=True, timeout=300)

    def ask(queries):
        text = "".join(" ".join(map(str, q)) + "\n" for q in queries)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [[int(x) for x in line.split()] for line in out.splitlines()]
    return ask


def test_span_of_a_chain(driver):
    cases = list(itertools.product([-3, 0, 1, 7, 100, 1000, MOST], [-MOST, 0, 1, 5, 40, 100, MOST - 500, MOST - 64, MOST - 10, MOST],
                                   [(1, 0), (6, 0), (6, 5), (70, 30), (1 << 22, 0), (1 << 22, (1 << 22) - 1)], [1, 100, MOST - 1023]))
    got = driver([("chain", prefix, tree, n, last, limit) for prefix, tree, (n, last), limit in cases])
    assert len(got) == len(cases)
    for (prefix, tree, (n, last), limit), g in zip(cases, got):
        p = min(max(prefix, 0), limit)
        want = min(max(prefix, 0) + max(tree, 0), p + max(0, max(tree, 0) - n + last + 1), limit)
        assert g == [p, want], (prefix, tree, n, last, limit)


def bytes_of(at, length, axes):
    starts = {at}
    for count, stride in axes:
        starts = {s + i * stride for s in starts for i in range(count)}
    return {s + i for s in starts for i in range(length)}


def query(a, b, steps=1 << 16):
    return ("meet", steps) + tuple(x for at, length, axes in (a, b) for x in (at, length, *(y for ax in axes for y in ax)))


def test_places_that_meet(driver):
    """Random tensors, among them views of one tensor, against the sets of their bytes."""
    rng = random.Random(3)
    cases = []
    for i in range(6000):
        base = [(rng.randint(1, 4), s) for s in rng.sample([0, 1, 2, 3, 4, 6, 8, 12, 16, 24, 31, 60], 3)]
        pair = []
        for _ in range(2):
            axes = [(rng.randint(1, 4), s) if rng.random() < 0.3 else (c, s) for c, s in base] if i % 2 else [
                (rng.randint(1, 4), rng.choice([0, 1, 2, 3, 5, 8, 13, 16, 40, 64])) for _ in range(3)]
            rng.shuffle(axes)
            pair.append((1000 + rng.randint(0, 60), rng.randint(1, 5), axes))
        cases.append(pair)
    got = driver([query(a, b) for a, b in cases])
    found = 0
    for (a, b), (meets, nested) in zip(cases, got):
        x = bytes_of(*a)
        want = bool(x & bytes_of(*b))
        found += want
        assert meets == want, (a, b)
        if nested:
            pieces = a[1]
            for count, _ in a[2]:
                pieces *= count
            assert len(x) == pieces, a
    assert 1000 < found < 5500


def test_places_of_views(driver):
    """Rows of a packed record, keys beside values, a slice beside the rest; far addresses; pieces without bytes."""
    MB = 1 << 20
    k, v = ((AT, 64, [(64, 40 * MB), (20, 2 * MB), (8, 128)]) for AT in (MB, MB + 64))
    assert driver([query(k, v), query(k, k), query(k, (MB + 63, *v[1:]))]) == [[0, 1], [1, 1], [1, 1]]
    one, rest = (MB, 512, [(64, 40 * MB), (20, 2 * MB), (1, 0)]), (MB + 512, 96, [(64, 40 * MB), (20, 2 * MB), (5, 100)])
    assert driver([query(one, rest), query(rest, one), query((MB, 513, one[2]), rest)]) == [[0, 1], [0, 1], [1, 1]]
    every2, every3 = (MB, 1, [(1000, 6), (1, 0), (1, 0)]), (MB + 1, 1, [(500, 9), (1, 0), (1, 0)])
    assert driver([query(every2, every3), query(every2, every3, 40)]) == [[0, 1], [1, 1]]       # too few steps to tell
    far = (1 << 46, 1 << 31, [(65535, 1 << 32), (64, 1 << 49), (1, 0)])
    assert driver([query(far, ((1 << 46) + (1 << 31), *far[1:])), query(far, far), query((MB, 0, k[2]), k)]) == [[0, 1], [1, 1], [0, 1]]
