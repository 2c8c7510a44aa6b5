"""The order in which blocks take the pieces of a divided row of work (csrc/block_order.h), compiled for the host: every piece once, the XCDs evenly."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_26246_amd", "csrc")
PROGRAM = """
#include <cstdio>
#include "block_order.h"
int main() {
  for (int n = 1; n <= 1024; ++n) {
    std::printf("%d", n);
    for (int b = 0; b < n; ++b) std::printf(" %d", slimattn::piece_of_block(b, n));
    std::printf("\\n");
  }
}
"""


@pytest.fixture(scope="module")
def orders(tmp_path_factory):
    at = tmp_path_factory.mktemp("order")
    (at / "p.cpp").write_text(PROGRAM)
    subprocess.run([shutil.which("g++") or "/opt/rocm/llvm/bin/clang++", "-std=c++17", "-I", CSRC, str(at / "p.cpp"), "-o", str(at / "p")], check=True)
    lines = subprocess.run([str(at / "p")], check=True, capture_output=True, text=True).stdout.splitlines()
    return {int(x.split()[0]): [int(y) for y in x.split()[1:]] for x in lines}


def test_every_piece_once(orders):
    assert len(orders) == 1024
    for n, order in orders.items():
        assert sorted(order) == list(range(n))


def test_every_xcd_has_its_share_as_one_run(orders):
    # block b runs on XCD b % 8, however many blocks without work were launched behind the n
    for n, order in orders.items():
        shares = [order[x::8] for x in range(8)]
        assert max(map(len, shares)) - min(map(len, shares)) <= 1
        for s in shares:
            assert s == list(range(s[0], s[0] + len(s))) if s else n < 8
