"""How octo_op_attend cuts keys into parts, without a GPU: every piece of a call has a block, every part its place in the workspace."""
import random
import subprocess

import pytest

import dispatch

SOURCE = r'''
#include "csrc/attend_choice.h"
#include <cstdio>
#include <vector>
using namespace octo;
int main() {
  octo_attend_op op{};
  int cus;
  while (scanf("%d %d %d %d %d %d %d %d %d %d", &op.dtype, &op.kv_format, &op.dim, &op.q_heads, &op.kv_heads, &op.n_seq, &op.n_q, &op.max_q, &op.max_kv, &cus) == 10) {
    std::vector<int> q(op.n_seq), kv(op.n_seq);
    for (int i = 0; i < op.n_seq; ++i) if (scanf("%d %d", &q[i], &kv[i]) != 2) return 1;
    const Plan p = plan_of(&op, cus);
    const int group = op.q_heads / op.kv_heads;
    // what attend_tile_kernel finds from the lengths
    CutSums s{0, 0, 0};
    std::vector<long long> blocks(op.n_seq), tiles(op.n_seq);
    for (int i = 0; i < op.n_seq; ++i) {
      blocks[i] = ((long long)q[i] * group + 127) / 128; tiles[i] = q[i] ? ((long long)kv[i] + 63) / 64 : 0;
      s.work += (float)blocks[i] * tiles[i] * op.kv_heads; s.whole += (float)blocks[i] * op.kv_heads; s.longest = std::max(s.longest, (int)tiles[i]);
    }
    const long long there = launch_blocks(&op, p);
    const int least = cut_least(s, p.n_split);
    int most[3];
    float pieces[3];
    for (int c = 0; c < 3; ++c) {
      most[c] = cut_most(s, p.slots, least, c);
      pieces[c] = 0;
      for (int i = 0; i < op.n_seq; ++i) pieces[c] += (float)(blocks[i] * op.kv_heads * ((tiles[i] + most[c] - 1) / most[c] > 1 ? (tiles[i] + most[c] - 1) / most[c] : 1));
    }
    const int part = cut_tiles(s, most, pieces, p.slots, least, p.even_tiles, (float)op.n_seq * p.row_blocks * op.kv_heads, (float)there);
    long long needs = 0;
    int parts = 1;
    for (int i = 0; i < op.n_seq; ++i) {
      const int n = parts_of(kv[i], p.cut ? even_part(kv[i], part) : p.part_keys);
      parts = std::max(parts, n);
      needs += blocks[i] * op.kv_heads * n;
    }
    if (p.n_split > 1 && join_blocks(&op) > MOST_BLOCKS) return 1;
    printf("%d %d %lld %lld %d %d\n", p.kernel == TILES, p.cut, needs, there, parts, p.n_split);
  }
}
'''
TYPES = {"f32": 0, "f16": 1, "bf16": 2}


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    d = tmp_path_factory.mktemp("attend")
    (d / "choice.cpp").write_text(SOURCE)
    dispatch.compile_host(["-o", str(d / "choice"), str(d / "choice.cpp"), "-L", dispatch.ROCM + "/lib", "-lamdhip64", "-Wl,-rpath," + dispatch.ROCM + "/lib"])

    def run(calls):
        """(type, 4 bits, dim, query heads, key heads, [lengths of queries], [of keys], what the host states as the longest of each, compute units): per call
        (on attend_tile_kernel, cut on the device, pieces of 128 rows, blocks there, most parts of a sequence, parts in the workspace)."""
        text = []
        for dtype, four, dim, hq, hk, q, kv, (max_q, max_kv), cus in calls:
            text.append(" ".join(map(str, [TYPES[dtype], int(four), dim, hq, hk, len(q), max(sum(q), max_q), max_q, max_kv, cus] + [x for pair in zip(q, kv) for x in pair])))
        out = subprocess.run([str(d / "choice")], input="\n".join(text) + "\n", capture_output=True, text=True, check=True).stdout.split("\n")
        return [tuple(map(int, o.split())) for o in out[:len(calls)]]
    return run


def _spread(rng, lo, hi):
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def _calls(seed, count, lengths):
    """Drawn calls; lengths(rng, n, most) -> the lengths of n sequences of up to `most`."""
    rng = random.Random(seed)
    for _ in range(count):
        n, hk, four = _spread(rng, 1, 256), rng.choice([1, 2, 4, 8]), rng.random() < 0.5
        q, kv = lengths(rng, n, _spread(rng, 1, 4096)), lengths(rng, n, _spread(rng, 300, 131072))
        stated = (max(q), max(kv)) if rng.random() < 0.7 else (max(q) + rng.randint(0, 200), max(kv) + rng.randint(0, 5000))
        yield (rng.choice(["bf16", "f16"]), four, rng.choice([32, 64, 96, 128] if four else [8, 64, 72, 80, 128]), hk * rng.choice([1, 2, 4, 5, 8, 17]), hk,
               q, kv, stated, rng.choice([256, 256, 256, 304, 64]))


def _alike(rng, n, most):
    return [most] * n


def _nearly_alike(rng, n, most):
    return [most - rng.randint(0, most // 16) for _ in range(n)]


def _any(rng, n, most):
    return [rng.choice([most, rng.randint(0, most)]) for _ in range(n - 1)] + [most]


@pytest.mark.parametrize("lengths", [_alike, _nearly_alike, _any])
def test_every_piece_has_a_block_and_every_part_a_place(ask, lengths):
    calls = list(_calls(1, 4000, lengths))
    cut = 0
    for call, (tiles, is_cut, pieces, blocks, parts, room) in zip(calls, ask(calls)):
        assert parts <= max(room, 1), (call[:5], call[7:])
        if is_cut:
            cut += 1
            assert room > 1 and pieces <= blocks, (call[:5], len(call[5]), max(call[5]), max(call[6]), pieces, blocks)
    assert cut > 400


def test_calls_of_more_than_three_rounds_of_pieces(ask):
    """Equal sequences whose best number of parts makes more pieces than three rounds of blocks."""
    calls = [(dtype, four, dim, hq, hk, [q] * n, [kv] * n, (q, kv), 256) for dtype, four, dim, hq, hk, n, q, kv in [
        ("bf16", False, 128, 32, 8, 2, 2049, 12800), ("bf16", False, 128, 32, 8, 4, 600, 12800), ("f16", True, 128, 32, 8, 4, 600, 12800), ("bf16", False, 128, 32, 8, 1, 2200, 12800),
        ("f16", True, 128, 32, 8, 17, 96, 20440), ("f16", True, 128, 32, 8, 5, 197, 49903), ("f16", False, 80, 16, 8, 6, 642, 21877), ("bf16", True, 128, 17, 1, 171, 1, 51200)]]
    for call, (tiles, cut, pieces, blocks, parts, room) in zip(calls, ask(calls)):
        assert tiles and cut and parts > 1 and pieces <= blocks and parts <= room, (call[:5], pieces, blocks, parts, room)


@pytest.mark.parametrize("long", [False, True], ids=["stated", "there"])
def test_as_many_keys_as_are_taken(ask, long):
    """The largest number of keys that a call may state, with short sequences and with such a one."""
    most = 0x7FFFFF00
    calls = [(dtype, four, dim, 4 * hk, hk, [q] * n, [most if long else 700] * n, (q, most), 256) for dtype, four, dim in (("bf16", False, 128), ("f32", False, 64), ("f16", True, 96))
             for hk in (1, 8) for n in (1, 3, 30, 200, 300) for q in (1, 9, 40, 700)]
    for call, (tiles, cut, pieces, blocks, parts, room) in zip(calls, ask(calls)):
        assert 1 <= parts <= room <= 128 and (not cut or pieces <= blocks) and (parts == 1) == (not long or room == 1), (call[:5], len(call[5]), call[5][0], parts, room, pieces, blocks)


@pytest.mark.parametrize("keys", [2 ** 30 + 64, 2 ** 30 + 3 * 64 + 1, 2 ** 31 - 5 * 64, 2 ** 31 - 2 ** 24])
def test_sequences_longer_than_fp32_counts(ask, keys):
    """More than 2^24 tiles: no sequence may have more parts than the workspace."""
    calls = [("bf16", False, 64, 17 * hk, hk, q, [keys] * len(q), (max(q), keys), 256) for hk in (1, 2) for q in ([1], [5], [300], [5, 1], [300, 2], [40, 1, 0])]
    for call, (tiles, cut, pieces, blocks, parts, room) in zip(calls, ask(calls)):
        assert tiles and cut and 1 <= parts <= room and pieces <= blocks, (call[3:6], parts, room, pieces, blocks)


@pytest.mark.parametrize("n_q,q_heads,kv_heads", [(2 ** 28, 8, 8), (2 ** 28, 8, 1), (2 ** 29 - 1, 5, 5), (2 ** 31 - 1, 1, 1), (2 ** 31 - 1, 4, 2), (2 ** 19, 4096, 4096)])
def test_rows_that_32_bits_do_not_number(n_q, q_heads, kv_heads):
    """Refused before any launch: a sequence's queries times heads are row numbers in the kernels."""
    import ctypes as C

    from paper_2502_01277_amd import binding
    from test_tokens_host import _attend_op
    op = _attend_op()
    op.dim, op.n_seq, op.n_q, op.max_q, op.q_heads, op.kv_heads = 8, 1, n_q, n_q, q_heads, kv_heads
    assert binding.lib().octo_op_attend(C.byref(op), None, None) == binding.EINVAL and binding.lib().octo_op_attend_workspace_bytes(C.byref(op)) == 0


@pytest.mark.parametrize("n_seq,q_heads,kv_heads,max_q,max_kv", [(2 ** 21, 8, 8, 1, 600), (2 ** 24, 1, 1, 3, 9000), (2 ** 27, 1, 1, 3, 49), (2 ** 20, 64, 16, 1, 4096), (2 ** 22, 32, 4, 100, 64), (5, 4096, 1, 200000, 700)])
def test_more_blocks_than_a_launch_takes(n_seq, q_heads, kv_heads, max_q, max_kv):
    """Refused before any launch."""
    import ctypes as C

    from paper_2502_01277_amd import binding
    from test_tokens_host import _attend_op
    L, op = binding.lib(), _attend_op()
    op.dim, op.n_seq, op.n_q, op.max_q, op.max_kv, op.q_heads, op.kv_heads = 8, n_seq, 2 ** 31 - 1, max_q, max_kv, q_heads, kv_heads
    assert L.octo_op_attend(C.byref(op), None, None) == binding.EINVAL and L.octo_op_attend_workspace_bytes(C.byref(op)) == 0
