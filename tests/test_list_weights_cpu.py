"""How attn_paged_tc.cuh counts the steps of a list and what they weigh, on the host: against counts made one by one, and up to 2^31 - 1
common keys (a block table may name a page many times, so so many slots need no such cache)."""
import os
import random
import subprocess

import pytest

from paper_2506_12355_b200 import build

PROGRAM = r"""
#include <cstdio>
#include <cstring>
#include "attn_paged_tc.cuh"
int main() {
    char what;
    int n, len, base, group, twin;
    while (std::scanf(" %c %d %d %d %d %d", &what, &n, &len, &base, &group, &twin) == 6) {
        attn_paged_tc::Params p;
        std::memset(&p, 0, sizeof(p));
        p.tile_tokens = 128 / group;
        p.twin_weight = twin;
        const int t2 = 2 * p.tile_tokens;
        if (what == 'p') {
            attn_paged_tc::Unit<true> u{0, n, 0, len, (n + t2 - 1) / t2};
            const attn_paged::Sharing s{p.tile_tokens, 0, 0, 0};
            std::printf("%d %lld %lld\n", u.steps_of(n), static_cast<long long>(u.head_weight(p)),
                        static_cast<long long>(attn_paged::list_cost(n, len, s, 1, 0)));
        } else {
            attn_paged_tc::Unit<false> u{0, n, base, len, (n + t2 - 1) / t2};
            std::printf("%d %lld 0\n", u.steps_of(n), static_cast<long long>(u.head_weight(p)));
        }
    }
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    at = tmp_path_factory.mktemp("weights")
    (at / "weights.cu").write_text(PROGRAM)
    flags = [f for f in build.NVCC_FLAGS if f not in ("-shared", "-Xcompiler", "-fPIC", "-O3")]
    subprocess.check_call([os.environ.get("NVCC", "nvcc")] + flags + ["-O1", "-I", build.CSRC, "-o", str(at / "weights"), str(at / "weights.cu")])

    def run(rows):
        text = "".join("%s %d %d %d %d %d\n" % row for row in rows)
        out = subprocess.run([str(at / "weights")], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


LIST_COST = 4


def expected(what, n, length, base, group, twin):
    tile = 128 // group
    pairs = -(-n // (2 * tile))
    weight = last = tiles = 0
    for i in range(pairs):
        two = n - i * 2 * tile > tile
        seen = length if what == "p" else max(base, 0) + min(n, (i + 1) * 2 * tile)      # keys that the pair's last token sees
        last = -(-seen // 128)
        weight += LIST_COST + last * (2 if two or i < pairs - 1 else twin)
        tiles += 2 if two else 1
    return last, weight, last * tiles if what == "p" else 0


def test_steps_and_weights(program):
    rng = random.Random(5)
    rows = []
    for _ in range(3000):
        what, n, group = rng.choice("pf"), rng.choice([1, 2, rng.randint(1, 300), rng.randint(1, 3000)]), rng.choice([1, 2, 3, 4, 7, 8, 20, 128])
        length = rng.choice([1, 127, 128, 129, rng.randint(1, 5000), rng.randint(1, 200000)])
        rows.append((what, n, length, length - n, group, rng.choice([1, 2])))
    for row, got in zip(rows, program(rows)):
        assert got == expected(*row), row


@pytest.mark.parametrize("length", [2 ** 31 - 1, 2 ** 31 - 127, 2 ** 31 - 128, 2 ** 31 - 129])
def test_lengths_up_to_the_last(program, length):
    rows = [(what, n, length, length - n, group, 2) for what in "pf" for n in (1, 40, 300) for group in (1, 4)]
    for row, got in zip(rows, program(rows)):
        assert got == expected(*row), row
