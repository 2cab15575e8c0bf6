"""Dropout's generator (csrc/philox.h) with the host's compiler: the published values of Philox 4x32-10 (the known answers of Random123, the authors'
library: counters and keys of zeros, of ones, and of the digits of pi), and the tests' own form of it."""
import subprocess

import numpy as np

from block_reference import philox
from paper_2006_09791_amd import build

KNOWN = [((0, 0, 0, 0), 0, (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
         ((0xffffffff,) * 4, 0xffffffffffffffff, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
         ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), 0x299f31d0a4093822, (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]

PROGRAM = r"""
#include <cstdio>
#include "philox.h"

int main() {
    unsigned c[4];
    unsigned long long key;
    while (std::scanf("%u %u %u %u %llu", c, c + 1, c + 2, c + 3, &key) == 5) {
        const gspc::Philox p = gspc::philox(c[0], c[1], c[2], c[3], key);
        std::printf("%u %u %u %u\n", p.word[0], p.word[1], p.word[2], p.word[3]);
    }
}
"""


def test_known_answers_and_the_tests_own_form(tmp_path):
    (tmp_path / "philox.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "philox")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wno-unknown-pragmas", "-I", build.CSRC, str(tmp_path / "philox.cpp"), "-o", exe], check=True)
    rng = np.random.default_rng(0)
    asked = [(c, k) for c, k, _ in KNOWN] + [(tuple(int(w) for w in rng.integers(1 << 32, size=4)), int(rng.integers(1 << 63)) * 2 + 1) for _ in range(500)]
    text = "\n".join(" ".join(map(str, (*c, k))) for c, k in asked)
    out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
    got = [tuple(map(int, line.split())) for line in out]
    assert got[:3] == [w for *_, w in KNOWN]
    assert got == [tuple(int(w) for w in philox(c, k)) for c, k in asked]
