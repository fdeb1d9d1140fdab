"""The plan of the loss over a vocabulary (csrc/vocab_loss_plan.h), built on the host: which tiles the GPU tests' sizes take, and how large the workspace gets."""
import os
import subprocess

import pytest

from paper_2502_08141_amd import build, lowra
from tests.vocab_loss_sizes import TILES, UNITS

_MAIN = """
#include "vocab_loss_plan.h"
#include <cstdio>
int main() {
    int M, V, K, grad;
    while (std::scanf("%d %d %d %d", &M, &V, &K, &grad) == 4) {
        const lowra::LossPlan l = lowra::loss_plan(M, V, K, grad != 0, UNITS);
        std::printf("%d %d %d %d %d %d %d %zu\\n", 1 << l.shift, l.tokens, l.grad_tokens, l.splits, l.words, l.tiles, l.rows, l.bytes);
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "main.cpp").write_text(_MAIN.replace("UNITS", str(UNITS)))
    subprocess.run(["g++", "-O1", "-std=c++17", "-I" + build.CSRC, str(d / "main.cpp"), "-o", str(d / "plan")], check=True)

    def of(sizes):
        text = subprocess.run([str(d / "plan")], input="\n".join(" ".join(str(int(v)) for v in s) for s in sizes), capture_output=True, text=True, check=True).stdout
        return [dict(zip(("words", "tokens", "grad_tokens", "splits", "split_words", "tiles", "rows", "bytes"), map(int, line.split()))) for line in text.splitlines()]
    return of


def test_tiles_of_the_gpu_tests_sizes(plan):
    for (M, V, K, words, tokens, grad_tokens), l in zip(TILES, plan([(*t[:3], 1) for t in TILES])):
        assert (l["words"], l["tokens"], l["grad_tokens"]) == (words, tokens, grad_tokens), (M, V, K, l)
    # every first product with every second one that goes with it, one tile and several splits
    assert {t[3:5] for t in TILES} == {(128, 64), (128, 128), (256, 64), (256, 128), (256, 192), (256, 256)}
    assert {t[5] for t in TILES} == {64, 128, 192, 256}


def test_plans_hold_together(plan):
    """Splits cover the words in whole tiles and none is empty; a piece's tokens are the batch's, or a multiple of 256."""
    sizes = [(M, V, K, g) for M in (1, 63, 65, 129, 257, 1000, 4096, 100000, 1 << 30) for V in (1, 129, 1003, 32000, 50265, 130000, 1 << 21) for K in (8, 64, 1032, 4096, 16384, 1 << 20) for g in (0, 1)]
    for (M, V, K, g), l in zip(sizes, plan(sizes)):
        assert l["tiles"] == -(-V // l["words"]) and l["split_words"] % l["words"] == 0
        assert 0 < l["splits"] <= 64 and (l["splits"] - 1) * l["split_words"] < l["tiles"] * l["words"] <= l["splits"] * l["split_words"]
        assert l["rows"] == M or (l["rows"] < M and (not g or l["rows"] % 256 == 0) and l["rows"] >= 256)
        # one piece: exponentials of 256 MiB or of 256 tokens, partial sums of 64 MiB beyond one of each, which are 128 MiB or 256 tokens', and of a
        # token 12 bytes a tile, a flag of four for 32 tokens a tile, and 12 bytes
        if g:
            rows = max(256, l["rows"])
            assert l["bytes"] <= max(256 << 20, 512 * (V + 255)) + (64 << 20) + max(128 << 20, 1024 * K) + rows * l["tiles"] * 13 + rows * 24 + (1 << 12), (M, V, K, l)
        else:
            assert l["bytes"] <= 192 << 20, (M, V, K, l)


def test_library_agrees(plan):
    """The library reports the plan's workspace (without a device it assumes as many units)."""
    sizes = [(4096, 32000, 4096, 1), (333, 32000, 4096, 0), (777, 50265, 1024, 1)]
    for (M, V, K, g), l in zip(sizes, plan(sizes)):
        assert lowra.lowra_vocab_loss_workspace_bytes(M, V, K, bool(g)) == l["bytes"]
