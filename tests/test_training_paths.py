"""CPU: which way the tests' sizes take through the training attention's launches, by
the library's own rules, through a small host program linked with it."""
import os
import subprocess

import pytest

from paper_2608_12780_amd import binding as B
from paper_2608_12780_amd import build

import training_paths as P

PROBE = r"""
#include <cstdio>
#include <cstdlib>
#include "kernels.h"
int main(int, char **argv) {
  const int heads = atoi(argv[1]), n = atoi(argv[2]), d = atoi(argv[3]), bf16 = atoi(argv[4]), c_q = atoi(argv[5]);
  printf("%d %d %d %d %d", scope::train_lists_slots(heads, n, c_q), scope::attention_ordered(heads, n, d, c_q),
         scope::train_query_parts(heads, n, d, bf16, c_q), scope::train_key_parts(heads, n, bf16, c_q),
         scope::train_orders_keys(n, c_q));
}
"""


@pytest.fixture(scope="module")
def ways(tmp_path_factory):
    B.lib()
    d = tmp_path_factory.mktemp("probe")
    src, exe = d / "probe.cpp", d / "probe"
    src.write_text(PROBE)
    rocm = os.path.dirname(os.path.dirname(build.HIPCC))
    cmd = ["g++", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", "-I", f"{rocm}/include",
           "-I", build.CSRC, str(src), "-o", str(exe), B.LIB_PATH,
           f"-Wl,-rpath,{os.path.dirname(os.path.abspath(B.LIB_PATH))}", f"-Wl,-rpath,{rocm}/lib",
           f"-L{rocm}/lib", "-lamdhip64", "-Wl,--allow-shlib-undefined"]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(heads, n, d, dtype, c_q):
        """(way of the bf16 kernels by queries, their parts, parts of dK and dV, whether
        keys run by signature)"""
        out = subprocess.run([str(exe), *map(str, (heads, n, d, int(dtype == "bf16"), c_q))],
                             capture_output=True, text=True, check=True)
        listed, ordered, queries, keys, by_signature = map(int, out.stdout.split())
        way = "listed" if listed else "ordered" if ordered and queries == 1 else "by cost"
        return way, queries, keys, bool(by_signature)
    return run


@pytest.mark.parametrize("case", P.ORDERED)
def test_block_order(ways, case):
    assert ways(*case[:5])[:2] == ("ordered", 1)


@pytest.mark.parametrize("case", P.BY_COST)
def test_slots_by_cost(ways, case):
    assert ways(*case[:5])[:2] == ("by cost", 1)


@pytest.mark.parametrize("case", P.BY_COST_PARTS)
def test_slots_by_cost_in_parts(ways, case):
    way, queries, keys, _ = ways(*case[:5])
    assert way == "by cost" and queries > 1 and keys > 1


@pytest.mark.parametrize("case", P.LISTED_PARTS)
def test_listed_in_parts(ways, case):
    way, queries, keys, _ = ways(*case[:5])
    assert way == "listed" and queries > 1 and keys > 1


def test_long_sequences(ways):
    sparse, f32, dense, many = (ways(*case[:5]) for case in P.LONG)
    assert sparse == ("ordered", 1, 1, True)
    assert f32[1] > 1 and f32[2] > 1 and f32[3]
    assert dense == ("by cost", 1, 1, False)
    assert many[0] == "by cost" and many[1] > 1 and many[2] > 1 and many[3]
