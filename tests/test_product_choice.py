"""Which kernels octo_op_product runs, without a GPU: every token has one, launches fit, and rows are held only where the registers have room for them."""
import random
import subprocess

import pytest

import dispatch

SOURCE = r'''
#include "csrc/product_choice.h"
#include <cstdio>
using namespace octo;
int main() {
  int n, k_bytes, cols, gated, to8, bits, words, exact8;
  while (scanf("%d %d %d %d %d %d %d %d", &n, &k_bytes, &cols, &gated, &to8, &bits, &words, &exact8) == 8) {
    for (int from = 0; from < n;) {
      const ProductChoice c = product_choice(n - from, k_bytes, cols, gated, to8, bits, words, exact8);
      printf("%d %lld %d ", c.variant, c.blocks, c.tokens);
      if (c.tokens < 1) return 1;
      from += c.tokens;
    }
    printf("\n");
  }
}
'''


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("product")
    (d / "choice.cpp").write_text(SOURCE)
    dispatch.compile_host(["-o", str(d / "choice"), str(d / "choice.cpp")])

    def run(calls):
        text = "".join("%d %d %d %d %d %d %d %d\n" % c for c in calls)
        out = subprocess.run([str(d / "choice")], input=text, capture_output=True, text=True, check=True).stdout.splitlines()
        assert len(out) == len(calls)
        result = []
        for line in out:
            v = [int(w) for w in line.split()]
            result.append([tuple(v[i:i + 3]) for i in range(0, len(v), 3)])
        return result
    return run


TILES = {1: (256, 256), 2: (128, 128), 3: (128, 64), 4: (128, 128)}
# what is built, by the bits of x and w; exact: rows of 8 bits that go through bf16
BUILT = {32: {2, 3, 4, 10, 20, 40, 11, 21, 41, 22, 42, 44}, 16: {1, 2, 3, 4, 10, 20, 40, 11, 21, 41, 22, 24}, 8: {1, 2, 3, 4, 10, 20, 40, 11, 21, 41}}


def test_every_token_has_a_kernel(ask):
    rng = random.Random(0)
    calls = []
    for _ in range(20000):
        bits = rng.choice([32, 16, 8])
        n = rng.choice([rng.randint(1, 70), rng.randint(1, 600), rng.randint(1, 20000)])
        k = 16 * rng.choice([rng.randint(1, 64), rng.randint(1, 1100)])
        to8 = rng.random() < 0.3
        cols = rng.choice([rng.randint(1, 600), rng.randint(1, 9000), rng.randint(1, 140000)])
        if to8:
            cols = (cols + 31) // 32 * 32
        words = bits != 8 or rng.random() < 0.7
        calls.append((n, k, cols, rng.random() < 0.4, to8, bits, words, bits == 8 and (not words or rng.random() < 0.3)))
    for call, kernels in zip(calls, ask(calls)):
        n, k, cols, gated, to8, bits, words, exact8 = call
        rows = cols * (2 if gated else 1)
        assert sum(t for _, _, t in kernels) == n and len(kernels) <= 2, call
        for variant, blocks, tokens in kernels:
            assert variant in BUILT[bits] and not (exact8 and variant == 1), call
            if variant < 10:
                r, t = TILES[variant]
                assert blocks == -(-rows // r) * -(-tokens // t), call
            else:
                r, t = variant // 10, variant % 10
                outs = r * (8 if gated else 16)
                assert blocks == -(-cols // outs) * -(-tokens // (16 * max(t, 1))), call
                assert not gated or r > 1, call                        # gates and what they are a gate of are tiles of one block
                assert not to8 or outs % 32 == 0, call                 # a group of 32 outputs is one block's
                if not t:                                              # held
                    assert tokens <= 16 and words and k <= 1024 * ({1: 8, 2: 8, 4: 4} if bits == 8 else {1: 16, 2: 16, 4: 8})[r], call
        if len(kernels) == 2:                                          # whole rounds, then tokens that smaller tiles do in one
            (first, _, tokens), (second, _, _) = kernels
            assert first == 1 and tokens % 256 == 0 and second != 1, call


def test_choices_that_were_measured(ask):
    assert [k[0][0] for k in ask([(1, 8192, 4096, 0, 0, 16, 1, 0), (16, 4096, 12288, 1, 0, 8, 1, 0), (16, 4096, 12288, 1, 1, 8, 1, 0), (64, 8192, 4096, 0, 0, 16, 1, 0),
                                 (128, 8192, 4096, 0, 0, 16, 1, 0), (1024, 8192, 4096, 0, 0, 16, 1, 0), (2048, 8192, 4096, 0, 0, 16, 1, 0), (8192, 8192, 8192, 0, 0, 16, 1, 0)])] == \
        [10, 20, 40, 22, 3, 4, 2, 1]
    assert [k[:2] for k in ask([(12800, 8192, 4096, 0, 0, 16, 1, 0)])[0]] == [(1, 768), (3, 256)]
