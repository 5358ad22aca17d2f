// Which kernel octo_op_attend starts, and how the keys are cut into parts: on the host by sizes, and in attend_tile_kernel by the lengths on the
// device, in arithmetic that both sides have here.
#pragma once
#include <algorithm>
#include <cmath>

#include "octo_internal.h"

namespace octo {

constexpr int MAX_PARTS = 128;
enum { DIRECT_OWN = 0, DIRECT_SHARE = 1, DIRECT_SHARE2 = 2 };      // 16 rows a wavefront, 16 or 32 a block whose wavefronts share the keys
enum { SHARED_KEYS = 1, OWN_ROWS = 2, TILES = 3 };          // as in the kernel id; 4 there: SHARED_KEYS with 32 rows, 5: TILES with parts cut on the device

struct Plan { int kernel, how, row_blocks, n_split, part_keys, cut, slots, even_tiles; };

__host__ __device__ inline int parts_of(int n_kv, int part_keys) { return n_kv > part_keys ? (n_kv - 1) / part_keys + 1 : 1; }
// A sequence's part where parts are cut to `most` tiles of 64 keys: as many parts as that takes, of equal length.
__host__ __device__ inline int even_part(int n_kv, int most) {
  const int tiles = (n_kv + 63) / 64, n = tiles > most ? (tiles + most - 1) / most : 1;
  return 64 * (tiles ? (tiles + n - 1) / n : 1);
}

// Parts cut on the device.  What the lengths there sum up to: blocks x tiles and blocks over all sequences and key heads, and the tiles of the longest sequence.
struct CutSums { float work, whole; int longest; };
constexpr float CUT_ROUNDS[3] = {0.85f, 1.85f, 2.85f};       // what of the last round may be lost to sequences shorter than a part
// No sequence may have more parts than the workspace holds.
__host__ __device__ inline int cut_least(const CutSums& s, int n_split) {
  const int n = (s.longest + n_split - 1) / n_split;
  return n > 4 ? n : 4;
}
__host__ __device__ inline int cut_most(const CutSums& s, float slots, int least, int c) {
  const int n = (int)ceilf(s.work / (slots * CUT_ROUNDS[c]));
  return n > least ? n : least;
}
// The longest part in tiles, of most[c], which take pieces[c] blocks, or without parts: the least estimated end.  In tiles: a block's start and end are as long as
// three, the join as four; without parts the longest sequence may come last.  Where the sequences are as long as each other and as the host stated (`stated` blocks), even_tiles,
// if the `blocks` there are enough for its pieces.
__host__ __device__ inline int cut_tiles(const CutSums& s, const int* most, const float* pieces, float slots, int least, int even_tiles, float stated, float blocks) {
  int part = s.longest > 1 ? s.longest : 1;
  const float longest = (float)s.longest;
  float best = s.whole <= slots ? longest + 3.f : s.work / slots + longest + 3.f;
#pragma unroll
  for (int c = 0; c < 3; ++c) {
    const float end = ceilf(pieces[c] / slots) * (most[c] + 3.f) + 4.f;
    if (end < best) { best = end; part = most[c]; }
  }
  if (even_tiles > 0 && s.work >= s.whole * longest * (15.f / 16.f) && s.whole >= stated * (15.f / 16.f)) {
    const int even = least > even_tiles ? least : even_tiles;
    if (s.whole * (float)((s.longest + even - 1) / even) <= blocks) part = even;
  }
  return part;
}
// Blocks to start.  A sequence's pieces are at most those of its work in parts of that length and one more for each block of rows: of most[c], together CUT_ROUNDS rounds and
// `whole`; of even_tiles, `whole` times the parts of the longest sequence.
inline long long cut_blocks(const Plan& p, long long whole, int max_kv) {
  const int tiles = (max_kv + 63) / 64, even = p.even_tiles > 0 ? (tiles + p.even_tiles - 1) / p.even_tiles : 1;
  return std::max(3 * p.slots + whole, whole * even);
}

// The number of parts with the least estimated end for blocks of equal length on TILES, `at_once` of them on a compute unit: the unit with the most blocks takes them in
// rounds, alone a block has 1 / 1.6 of what the unit does with two or three, and its start and end are as long as six tiles;
// the join as twelve, and for every part 0.6 and 0.4 for a million values written and read.
// 79 calls of equal lengths, timed in turn: 3.3 % less in the mean than with three blocks a unit (5 x 197 queries over 49903 keys of 4 bits, 32 / 8 heads of 128, 1424 -> 903 us;
// 6 x 642 over 21877, 16 / 8 heads of 80, 844 -> 630), single ones more (59 x 33 over 36264 of 4 bits, 2 heads of 64, 164 -> 230).
inline long long even_parts(long long blocks, double outputs, int max_kv, int cus, int at_once) {
  const int tiles = std::max(1, (max_kv + 63) / 64);
  if (blocks > 65536) return 1;                             // over a hundred rounds: the last one is nothing
  double best = 1e30;
  long long n = 1;
  for (int k = 1; k <= std::max(1, std::min(MAX_PARTS, max_kv / 256)); ++k) {
    const int part = (tiles + k - 1) / k;
    const long long parts = (tiles + part - 1) / part, most = (blocks * parts + cus - 1) / cus, last = most % at_once;
    const double end = (most / at_once * at_once / 1.6 + (last > 1 ? last / 1.6 : last)) * (part + 6) + (parts > 1 ? 12 + parts * (0.6 + 4e-7 * outputs) : 0);
    if (end < best) { best = end; n = parts; }
  }
  return n;
}

// Which kernel, by the rows of the longest sequence, their tiles of 16 over all sequences and heads, and the keys ("512 x 49": 512 sequences of 2 heads and 49
// keys; us, bf16, dim 128, where nothing else is said).
//   OWN_ROWS where there are tiles for all wavefronts and few keys to share: 512 x 49, 8 / 16 / 32 / 48 rows 9.7 / 11.4 / 15.0 / 19.5 against 12.1 / 13.3 / 20.2 /
//     27.3 (SHARED_KEYS) and 14.1 / 14.5 / 15.6 / 17.0 (TILES); from 4 bits also 400 keys, 20 and 48 rows: 22.8, 30.3 : 26.5, 36.1 : 32.2, 36.7; fp32,
//     512 x 400, dim 64, 20 and 128 rows: 52.8, 153 : 66.0, 187.
//   SHARED_KEYS for up to 16 rows, for all else in fp32, and where the whole call is short, as its wavefronts are quickly done: 4 x 400, 128 rows 8.2 against 13.7
//     (TILES); 64 x 400, 32, 64 and 96 rows: 10.9, 12.7, 17.5 : 14.1, 14.6, 15.5; further for few long sequences (4 x 24000, 64 and 128 rows: 32, 44 : 40, 46; but
//     64 x 3000, 64 rows 59.9 : 59.6) and from 4 bits, which TILES converts first and then puts in LDS (64 x 3000, 64 and 128 rows: 33, 42 : 47, 60).
//   TILES for the rest: 64 x 3000, 128 rows 70 against 76; 512 x 400: 66 against 112; many short ones: 137 sequences of 4084 rows and 37 keys 89 against 205.
// SHARED_KEYS with 32 rows a block instead of 16 where there are many tiles: the keys are read and put in order half as often (64 x 3000, 64 and 128 rows: 75, 131 ->
//   60, 76; from 4 bits 33, 54 -> 33, 42; fp32, dim 64: 88, 161 -> 79, 114), but a short call is longer (4 x 400: 8.2 -> 10.0; fp32, 77 rows in 5 tiles 29 -> 37).
// Parts of the keys: as many as give every compute unit two blocks (TILES and fp32, which take longer for a key: three; OWN_ROWS: four), of at least 256 keys, and, where sequences may
//   differ in length, up to sixteen blocks of 2048 keys, for an even end: 16 single tokens over up to 51200 keys of 4 bits 131 -> 117 us, 17 questions
//   of up to 96 tokens over up to 20440 keys 486 -> 453.  With TILES the rows
//   tell: as many as n_seq x max_q, then sequences are alike, and even_parts has it: 64 x 3000, 128 rows 71 -> 59 us, 4 x 1600, 900 rows 55 -> 40,
//   13 questions of 475 rows (20 / 4 heads of 96) over 42138 keys of 4 bits 718 -> 498.
// A long call of up to 256 sequences on TILES cuts its parts on the device, where the lengths are (cut_piece; n_split is then the most a sequence can have): 24 tiles for every place a
//   block can have at least, as looking at all lengths takes a block 5 us.  Where it finds them alike it takes even_parts's length
//   (0.7 % of the 3.3 there; 3.2 % over 16 calls of equal queries and ragged keys).
inline Plan plan_of(const octo_attend_op* op, int cus) {
  Plan p{};
  const long long rows = (long long)op->max_q * (op->q_heads / op->kv_heads), pairs = (long long)op->n_seq * op->kv_heads, blocks16 = pairs * ((rows + 15) / 16);
  const bool f32 = op->dtype == OCTO_F32, four_bits = op->kv_format == OCTO_KV_CACHE4;
  const double work = (double)blocks16 * op->max_kv / cus;          // keys a compute unit reads if every tile reads its own
  const bool many = blocks16 >= 4ll * cus, long_enough = !many || op->max_kv >= 384;
  if (many && (f32 ? op->max_kv <= 512 : four_bits ? op->max_kv <= 512 && rows <= 48 : op->max_kv <= 128 && rows <= 32)) p.kernel = OWN_ROWS;
  else if (f32 || rows <= 16) p.kernel = SHARED_KEYS;
  else if (four_bits) p.kernel = (long_enough && work <= 5500) || (rows <= 128 && op->max_kv >= 2048 && work <= 13000) ? SHARED_KEYS : TILES;
  else p.kernel = long_enough && work <= (rows <= 32 ? 3000 : rows <= 128 && op->max_kv >= 8192 ? 6000 : 1000) ? SHARED_KEYS : TILES;
  const bool tiles = p.kernel == TILES;
  const long long tiles16 = (rows + 15) / 16;
  const bool pairs_of_tiles = f32 ? work >= 1500 && (tiles16 % 2 == 0 || tiles16 > 6) : four_bits ? rows > 64 && work >= 4000 : work >= (rows <= 32 ? 2000 : 400);
  p.how = p.kernel == OWN_ROWS ? DIRECT_OWN : p.kernel == SHARED_KEYS && rows > 16 && pairs_of_tiles ? DIRECT_SHARE2 : DIRECT_SHARE;
  const int block_rows = tiles ? 128 : p.how == DIRECT_SHARE2 ? 32 : 16;
  p.row_blocks = (int)((rows + block_rows - 1) / block_rows);
  const long long blocks = p.kernel == OWN_ROWS ? (blocks16 + 3) / 4 : pairs * p.row_blocks;
  const bool alike = tiles && op->n_q >= (long long)op->n_seq * op->max_q * 15 / 16;
  auto parts = [&](int target, int least) { return blocks > 0 ? std::min<long long>((long long)target * cus / blocks, op->max_kv / least) : 1; };
  long long n = parts(p.kernel == OWN_ROWS ? 4 : f32 || tiles ? 3 : 2, 256);
  if (!alike) n = std::max(n, parts(16, 2048));
  const int at_once = op->dim <= 64 ? 3 : 2;
  const long long even = alike ? even_parts(blocks, (double)op->n_q * op->q_heads * op->dim, op->max_kv, cus, at_once) : 1;
  auto split = [&](long long n) {
    n = std::max(1ll, std::min<long long>(n, MAX_PARTS));
    p.part_keys = (int)((op->max_kv + n * 64 - 1) / (n * 64)) * 64;
    p.n_split = parts_of(op->max_kv, p.part_keys);
  };
  split(std::max(n, even));
  p.slots = cus * at_once;                                 // blocks of attend_tile_kernel at a time
  p.cut = tiles && p.n_split > 1 && op->n_seq <= 256 && (double)blocks * ((op->max_kv + 63) / 64) >= 24.0 * p.slots;
  p.even_tiles = alike ? (int)(((op->max_kv + 63) / 64 + even - 1) / even) : 0;
  if (alike && !p.cut) split(even);
  return p;
}

// Blocks that read the same keys run on one die, where the sets of keys share out evenly over the eight.
inline bool by_die(const Plan& p, long long sets) { return p.row_blocks > 1 && (sets % 8 == 0 || sets >= 64); }
// Blocks of the first launch.  HIP counts the threads of a launch, 256 a block, in 32 bits.
constexpr long long MOST_BLOCKS = 0xFFFFFF;
inline long long launch_blocks(const octo_attend_op* op, const Plan& p) {
  const long long whole = (long long)op->n_seq * op->kv_heads * p.row_blocks, sets = (long long)op->n_seq * op->kv_heads * p.n_split;
  if (p.cut) return cut_blocks(p, whole, op->max_kv);
  if (p.kernel == OWN_ROWS) return (whole * p.n_split + 3) / 4;
  return (by_die(p, sets) ? (sets + 7) / 8 * 8 : sets) * p.row_blocks;
}

// Blocks of attend_join_kernel, 8 rows of a sequence each; calls with parts are of so few blocks that these are far from MOST_BLOCKS.
inline long long join_blocks(const octo_attend_op* op) { return op->n_seq * (((long long)op->max_q * op->q_heads + 7) / 8); }

}  // namespace octo
