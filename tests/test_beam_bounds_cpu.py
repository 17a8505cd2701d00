"""-m "not gpu": what the operators of include/dba_beam.h work out about places in memory, compiled for the host with sanitizers."""
import itertools
import os
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
