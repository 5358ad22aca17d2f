// Which kernel octo_op_product runs.  Host arithmetic only: no HIP header is needed to compile this file.
#pragma once

namespace octo {

struct ProductChoice { int variant; long long blocks; };

// Up to 16 tokens stay in the registers of 8 wavefronts while one group of weights after the other passes: the steps of 128 bytes of k that a wavefront has room for, with
// r x 16 rows of w a group.  Rows of 8 bits carry exponents and are widened, which takes registers too.
constexpr int product_held_steps(int r, bool rows8) { return r == 4 ? (rows8 ? 4 : 8) : rows8 ? 8 : 16; }

// variant: 1, 2, 3: tiles in LDS of 256 x 256, 128 x 128 and 128 x 64 (rows of w x tokens); 10 R + T: operands straight from memory, R x 16 rows of w and T x 16 tokens a block;
// 10 R: the same with up to 16 tokens, held.
// held_bytes: bytes of k of rows that can be held (0: exponents that are not aligned words); rows8: x and w in 8 bits.
// to8: results in 8 bits, whose groups of 32 outputs one block holds.  exact8: rows of 8 bits that go through bf16, which has no tiles of 256 x 256.
inline ProductChoice product_choice(int n, int held_bytes, int cols, bool gated, bool to8, bool rows8, bool exact8) {
  const long long rows = gated ? 2ll * cols : cols;
  auto blocks = [&](int bn, int bm) { return (rows + bn - 1) / bn * ((n + bm - 1) / bm); };
  auto few = [&](int r, int t) { const int outs = gated ? 8 * r : 16 * r; return ProductChoice{10 * r + t, (cols + outs - 1ll) / outs * ((n + 16ll * t - 1) / (16 * t))}; };
  if (n <= 16 && held_bytes) {
    // Two sets of 16 rows a group where x leaves room and there are groups enough for every CU (16 tokens, 8 bits 4096 -> 24576: 22.5 us, one set 25.2; bf16 4096 -> 131072
    // 212.6, one set 183.5, with less on its way for each)
    const int r = gated && to8 ? 4 : gated || to8 || (held_bytes <= 4096 && rows >= 32 * 256) ? 2 : 1;
    if (held_bytes <= 1024 * product_held_steps(r, rows8)) return {10 * r, few(r, 1).blocks};
  }
  if (n <= 64 || blocks(128, 64) < 128) {
    const int t = n <= 16 ? 1 : n <= 32 || (gated && to8) ? 2 : 4;
    if (gated && to8) return few(4, t);
    return few(gated || to8 || t > 1 || rows > 16 * 512 ? 2 : 1, t);
  }
  if (!exact8 && blocks(256, 256) >= 256) return {1, blocks(256, 256)};
  if (blocks(128, 128) >= 256) return {2, blocks(128, 128)};
  return {3, blocks(128, 64)};
}

}  // namespace octo
