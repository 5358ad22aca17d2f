// Which kernels octo_op_product runs.  Host arithmetic only: no HIP header is needed to compile this file.
#pragma once

namespace octo {

struct ProductChoice { int variant; long long blocks; int tokens; };   // tokens: how many of the n the kernel takes; the others are chosen for anew

// Up to 16 tokens stay in the registers of 8 wavefronts while one group of weights after the other passes: the steps of 128 bytes of k that a wavefront has room for, with
// r x 16 rows of w a group.  Rows of 8 bits carry exponents and are widened, which takes registers too.
constexpr int product_held_steps(int r, bool rows8) { return r == 4 ? (rows8 ? 4 : 8) : rows8 ? 8 : 16; }

// variant: 1, 2: tiles in LDS of 256 x 256 and 128 x 128 (rows of w x tokens) with two stages; 3, 4: of 128 x 64 and 128 x 128 with four; 10 R + T: operands straight from memory,
// R x 16 rows of w and T x 16 tokens a block; 10 R: the same with up to 16 tokens, held.
// bits: of a value of x and w.  words: exponents of 8 bits come in aligned words.  to8: results in 8 bits, whose groups of 32 outputs one block holds.  bytes8: rows of 8 bits whose exponents
// come byte by byte, for which there are no tiles of 256 x 256.  direct: results leave tiles straight from registers (ProductArgs).
inline ProductChoice product_choice(int n, int k_bytes, int cols, bool gated, bool to8, int bits, bool words, bool bytes8, bool direct = true) {
  const long long rows = gated ? 2ll * cols : cols;
  auto blocks = [&](int bn, int bm) { return (rows + bn - 1) / bn * ((n + bm - 1ll) / bm); };
  auto few = [&](int r, int t) { const int outs = gated ? 8 * r : 16 * r; return ProductChoice{10 * r + t, (cols + outs - 1ll) / outs * ((n + 16ll * t - 1) / (16 * t)), n}; };
  if (n <= 16) {
    if (words) {
      // Two sets of 16 rows a group where x leaves room and there are groups enough for every CU (16 tokens, 8 bits 4096 -> 24576: 22.5 us, one set 25.2; bf16 4096 -> 131072
      // 212.6, one set 183.5, with less on its way for each)
      const int r = gated && to8 ? 4 : gated || to8 || (k_bytes <= 4096 && rows >= 32 * 256) ? 2 : 1;
      if (k_bytes <= 1024 * product_held_steps(r, bits == 8)) return {10 * r, few(r, 1).blocks, n};
    }
    return few(gated && to8 ? 4 : gated || to8 || rows > 16 * 512 ? 2 : 1, 1);
  }
  if (bits == 32) {
    // fp32's products are the bound, and blocks as small as it takes spread them (4096 -> 4096: 64 tokens 34 us, 64 x 64 a block 81, tiles 132; 512 tokens 2048 -> 2048: 60, 43 and 70)
    const ProductChoice square = few(4, 4);
    if (square.blocks <= 128) return few(gated && to8 ? 4 : 2, 2);
    if (square.blocks <= 256) return square;
  } else if (bits == 16 && !(gated && to8)) {
    // A block a CU (64 tokens, 4096 -> 4096: 17.1 us, tiles 18.9; 1024 -> 4096 6.6 and 7.6; with two blocks a CU, 128 tokens, 31.2 and 18.9).  Larger ones for short rows whose results leave tiles
    // through LDS, which takes as long as some ten steps: bf16 without activation, in 17 sizes of up to 256 blocks and 2560 bytes 0.65 to 1.09 of the tiles' time (308 tokens, 1160 -> 1100: 7.3 and
    // 9.3; 1000 tokens, 904 -> 470: 7.1 and 11.0), GELU 0.44 to 0.81; rows of 2816 to 4096 bytes 1.12 to 1.16, beyond 256 blocks 1.17 to 1.56.  Straight from registers tiles are as fast (0.86 to 1.14).
    if (few(2, 2).blocks <= 256) return few(2, 2);
    if (!direct && k_bytes <= 2560 && few(2, 4).blocks <= 256) return few(2, 4);
  } else if (bits == 8) {
    // The same (64 tokens, 4096 -> 1024: 9.5 us, two sets of rows a block 13.0, tiles 15.7; 32 tokens, 4096 -> 4096: 13.0, tiles 25.7).  Tiles that take exponents byte by byte are slow beyond a
    // block a CU too (64 tokens, 4000 -> 4096: 14.3, tiles 34.8; 300 tokens, 4000 -> 2000: 34.8, tiles 39.4; 1000 tokens, 4000 -> 1000: 45.8, tiles 40.7).
    if (!gated && !to8 && few(1, 1).blocks <= 256) return few(1, 1);
    if (!(gated && to8) && few(2, 1).blocks <= 256) return few(2, 1);
    if (!words && few(4, 1).blocks <= 768) return few(4, 1);
  }
  if (!bytes8 && bits != 32 && blocks(256, 256) >= 256) {              // fp32, 4096 cubed: 1158 us, tiles of 128 x 128 953
    // Whole rounds of 256 CUs; few tiles that are left over would take a round of their own, in which smaller ones are done in a third of the time.
    const long long across = (rows + 255) / 256, all = blocks(256, 256), m = all / 256 * 256 / across * 256;
    const long long rest = n - m;
    if (rest > 0 && m > 0 && (rows + 127) / 128 * ((rest + 127) / 128) <= 256) return {1, across * (m / 256), (int)m};
    return {1, all, n};
  }
  // Four stages where a CU has one block, two where it has two (bf16, 4096 -> 4096: 512 tokens 21.9 us, with two stages 37.3; 1024 tokens 33.4, two stages 44.3; 2048 tokens 65.3
  // and 59.3).
  if (n <= 64 || blocks(128, 64) <= 256) return {3, blocks(128, 64), n};
  return {blocks(128, 128) <= 256 ? 4 : 2, blocks(128, 128), n};
}

}  // namespace octo
