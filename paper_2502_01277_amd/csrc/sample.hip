// octo_op_sample: one token of each row of logits.
//
// With the tokens of a row in the order of their logits (equal ones by index) and w = exp((x - max) / temperature), top-k, top-p and min-p each keep a beginning of that order; what
// they keep in common is one too, and is known by its last token.  The token is drawn in the order of indices: the first at which the sum of the kept weights passes u times all.
//
// A workgroup takes a row; few long ones of fp32 and fp16 are shared (sample_parts).  Sums of weights decide which token a border falls on, so they are made of integers: the exponent is taken in
// fp64, w from a table of 1024 steps an octave and a remainder that fp32 holds to 2^-35, and rounded to multiples of 2^-shift of the largest, whose sums in 64 bits are the same in any order.
// The bound is arithmetic, an exponential of twenty instructions for each logit (an instruction for each of 131072 logits takes a compute unit 0.85 us), so it is computed where it has to be:
//   - top_k of up to LISTED: the k-th largest of the threads' own largest logits is no larger than the k-th largest of all; what is not below it, little more than k logits, is put in order in LDS.
//   - bf16: a row has few different logits.  Codes of the 16 octaves below the largest magnitude are counted, 4096 of them, and all sums are those of counts times weights.
//   - else borders are found by a histogram of counts and weights over 64 octaves of w, 64 bins each; the tokens of the bin that holds the border are listed, one more histogram of the
//     list's own range leaves few of them (a sort of the whole list: 16 us more), which are put in order.  Where they are too many to list (equal logits, say), bits of the logits
//     themselves make further histograms.  The same where the others do not fit (more equal logits than are listed, borders in codes that are not counted).
// Measured (MI355X), top-p 0.9: 1 x 8192 bf16 21 us, 1 x 32768 27, fp32 40; 1 x 131072 bf16 49, fp32 76 (alone 113: of the 76, two looks at a row by one workgroup take 15 each, at the 35 GB/s that a compute unit draws from beyond its L2); 512 x 100003 bf16 100, fp32 214; the first 50 of 1 x 32768 15 (with votes on 20 bits of a key one after the other 17).
#include <cmath>
#include <type_traits>

#include "mfma_common.h"
#include "octo_internal.h"

namespace octo {
namespace {

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = 16, BINS = 4096, SORTED = 2048, LISTED = 512, MOST_PARTS = 8;
typedef unsigned long long u64;

struct SampleArgs {
  const void* logits; long long row;
  const float *u, *temperature, *top_p, *min_p; const int* top_k;
  float all_temperature, all_top_p, all_min_p; int all_top_k;
  int* token; float* logprob; int* kept;
  const int* n_dyn;
  int vocab, shift;
  int parts;                // workgroups of a row where there are few rows, or 0
  float* part_best; u64* part_weight; unsigned* part_count;           // [n][parts], and histograms [n][parts][BINS]
};

// Floats as integers of the same order, both zeros alike.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned b = __float_as_uint(v + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ float unordered(unsigned k) { return __uint_as_float(k & 0x80000000u ? k & 0x7FFFFFFFu : ~k); }

constexpr int STEPS = 1024;    // of an octave
// 2^(j / STEPS) by the exponential's series, rounded a few times
struct Octave { double v[STEPS]; };
constexpr Octave make_octave() {
  Octave o{};
  for (int j = 0; j < STEPS; ++j) {
    const double x = j * (0.69314718055994530942 / STEPS);
    double sum = 1.0;
    for (int n = 24; n > 0; --n) sum = 1.0 + sum * x / n;
    o.v[j] = sum;
  }
  return o;
}
__device__ const Octave octave = make_octave();
// w of a logit in units of 2^-shift.  The exponent t is in steps of an octave, in fp64: its nearest integer picks w from the table, what is left, at most half a step, a factor 1 + eps that
// fp32 holds to 2^-35 of w.
struct Weigher {
  const double* table;      // 2^(j / STEPS), in LDS
  double best, factor;      // t = (v - best) factor
  int shift;
  double least;             // min-p as an exponent in steps: weights have no bits where it may lie
  __device__ __forceinline__ bool dropped(float v) const { return ((double)v - best) * factor < least; }
  static constexpr u64 ZERO = 0x4330000000000000ull;                 // 2^52: integers added to it lie in its low bits
  __device__ __forceinline__ double steps(float v) const {
    return fmax(((double)v - best) * factor, -73728.0);           // 72 octaves down nothing is left; also for what is no number (-infinity, NaN, at an infinite temperature too)
  }
  __device__ __forceinline__ double scaled(double t, int* k) const {
    const double m = t + 6755399441055744.0;                         // 1.5 * 2^52: the nearest integer is in the low bits
    *k = (int)__double_as_longlong(m);
    const float f = (float)(t - (m - 6755399441055744.0));
    const float eps = f * fmaf(f, fmaf(f, 5.1696e-11f, 2.29097850e-7f), 6.76901543e-4f);         // 2^(f / STEPS) - 1, coefficients (ln 2 / STEPS)^n / n!
    const double w = __longlong_as_double(__double_as_longlong(table[*k & (STEPS - 1)]) + ((long long)((*k >> 10) + shift) << 52));
    return fma(w, (double)eps, w);
  }
  __device__ __forceinline__ double scaled(float v) const { int k; return scaled(steps(v), &k); }
  static __device__ __forceinline__ u64 bits(double w) { return (u64)__double_as_longlong(w + 4503599627370496.0); }      // ZERO + the nearest integer
  static __device__ __forceinline__ u64 whole(double w) { return bits(w) - ZERO; }
  __device__ __forceinline__ u64 operator()(float v) const { return whole(scaled(v)); }
  static __device__ __forceinline__ int bin_of(int k) { return min(-k >> 4, BINS - 1); }
  __device__ __forceinline__ int bin(float v) const { return bin_of((int)__double_as_longlong(steps(v) + 6755399441055744.0)); }
};

template <typename V> __device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
  return v;
}
template <typename V> __device__ __forceinline__ V wave_scan(V v, int lane) {      // inclusive
#pragma unroll
  for (int d = 1; d < 64; d *= 2) { const V o = __shfl_up(v, d); if (lane >= d) v += o; }
  return v;
}

// RANGE_WORDS: counts of codes, two of 16 bits a word, for each of CODE_RANGES parts of the row (bf16 alone)
constexpr int CODE_RANGES = 8;
template <int RANGE_WORDS> struct SampleShared {
  unsigned codes[CODE_RANGES][RANGE_WORDS];
  double table[STEPS];
  u64 weight[BINS];
  unsigned count[BINS];
  u64 list[SORTED];
  u64 wave_w[SAMPLE_WAVES];
  unsigned wave_c[SAMPLE_WAVES];
  float wave_max[SAMPLE_WAVES], wave_big[SAMPLE_WAVES];
  unsigned key_min, key_max;
  int listed, bin, token, cut;
  unsigned bin_count, key, at, before_c;
  u64 before_w, tiny_w;
};

// The last token that is kept: all whose ordered logit is above `key`, and of those equal to it the ones up to index `at`.
struct Last { unsigned key; int at; };

// Positions are indices plus the distance of the row's start from the last 16-byte border before it, so that vectors are aligned.
template <typename T> struct SampleRow {
  static constexpr int VEC = 16 / sizeof(T), DEPTH = 4;
  const T* x; int skew, end;
  bool odd;                 // a row with infinite logits is one of zeros and ones: those weigh 1, the others that may be drawn nothing
  __device__ __forceinline__ SampleRow(const SampleArgs& a, int row) : x((const T*)a.logits + row * a.row), odd(false) {
    skew = (int)(((uintptr_t)x & 15) / sizeof(T)); end = a.vocab + skew;
  }
  __device__ __forceinline__ u32x4 load(int p) const {
    u32x4 v;
    if (p >= skew && p + VEC <= end) {
      v = *(const u32x4*)(x + (p - skew));
    } else {
#pragma unroll
      for (int e = 0; e < VEC; ++e) ((T*)&v)[e] = p + e >= skew && p + e < end ? x[p + e - skew] : (T)-INFINITY;
    }
    if (odd) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) { const float f = (float)((T*)&v)[e]; ((T*)&v)[e] = (T)(f == INFINITY ? 0.f : f > -INFINITY ? -1.f : -INFINITY); }
    }
    return v;
  }
  // f(position, vector) of the positions from, from + stride ...
  template <typename F> __device__ __forceinline__ void vectors(int from, int count, int stride, F&& f) const {
    for (int i0 = 0; i0 < count; i0 += DEPTH) {
      u32x4 v[DEPTH];
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) if (i0 + d < count) v[d] = load(from + (i0 + d) * stride);
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) if (i0 + d < count) f(from + (i0 + d) * stride, v[d]);
    }
  }
  static __device__ __forceinline__ float value(const u32x4& v, int e) { return (float)((const T*)&v)[e]; }
  // f(index, logit) of every token there that may be drawn
  template <typename F> __device__ __forceinline__ void each(int from, int count, int stride, F&& f) const {
    vectors(from, count, stride, [&](int p, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float f32 = value(v, e);
        if (f32 > -INFINITY) f(p + e - skew, f32);                   // neither -infinity nor NaN
      }
    });
  }
  // vectors of a lane where `ways` workgroups share the row; a part is whole vectors of all threads of one
  __device__ __forceinline__ int tiles(int ways) const { return (end + ways * SAMPLE_THREADS * VEC - 1) / (ways * SAMPLE_THREADS * VEC); }
};

// What a row is drawn by.
struct SampleChoice {
  float temperature, top_p, min_p; int top_k;
  __device__ __forceinline__ SampleChoice(const SampleArgs& a, int row)
      : temperature(a.temperature ? a.temperature[row] : a.all_temperature), top_p(a.top_p ? a.top_p[row] : a.all_top_p), min_p(a.min_p ? a.min_p[row] : a.all_min_p),
        top_k(a.top_k ? a.top_k[row] : a.all_top_k) {}
  __device__ __forceinline__ bool first_alone() const { return !(temperature > 0) || top_k == 1 || top_p <= 0 || min_p > 1; }
  __device__ __forceinline__ bool short_list() const { return top_k > 0 && top_k <= LISTED; }
  __device__ __forceinline__ double factor() const { return (double)STEPS * 1.4426950408889634 / (double)temperature; }
};

// ---- few rows: the largest logit and the histogram of weights by `parts` workgroups a row ----------------------------------
template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_best_kernel(SampleArgs a) {
  __shared__ float wave_max[SAMPLE_WAVES];
  const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts, tid = threadIdx.x;
  if (a.n_dyn && row >= *a.n_dyn) return;
  const SampleRow<T> x(a, row);
  const int tiles = x.tiles(a.parts), stride = SAMPLE_THREADS * x.VEC;
  float best = -INFINITY;
  x.vectors(part * tiles * stride + tid * x.VEC, tiles, stride, [&](int, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < x.VEC; ++e) best = fmaxf(best, x.value(v, e));          // the other one where one is NaN
  });
#pragma unroll
  for (int d = 1; d < 64; d *= 2) best = fmaxf(best, __shfl_xor(best, d));
  if (!(tid & 63)) wave_max[tid >> 6] = best;
  __syncthreads();
  if (tid) return;
  for (int w = 0; w < SAMPLE_WAVES; ++w) best = fmaxf(best, wave_max[w]);
  a.part_best[blockIdx.x] = best;
}

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_part_kernel(SampleArgs a) {
  __shared__ double table[STEPS];
  __shared__ u64 weight[BINS];
  __shared__ unsigned count[BINS];
  const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts, tid = threadIdx.x;
  if (a.n_dyn && row >= *a.n_dyn) return;
  const SampleChoice by(a, row);
  float best = -INFINITY;
  for (int p = 0; p < a.parts; ++p) best = fmaxf(best, a.part_best[row * a.parts + p]);
  if (!(best > -INFINITY) || best == INFINITY || by.first_alone() || by.short_list()) return;       // rows that the last kernel does alone
  const SampleRow<T> x(a, row);
  const Weigher weigh{table, (double)best, by.factor(), a.shift, -INFINITY};
  table[tid] = octave.v[tid];
  for (int b = tid; b < BINS; b += SAMPLE_THREADS) { weight[b] = 0; count[b] = 0; }
  __syncthreads();
  const int tiles = x.tiles(a.parts), stride = SAMPLE_THREADS * x.VEC;
  unsigned below = 0;                                                // of the last bin, which words that are ruled out by a number share: they weigh nothing
  x.each(part * tiles * stride + tid * x.VEC, tiles, stride, [&](int, float v) __attribute__((always_inline)) {
    int k;
    const u64 q = Weigher::whole(weigh.scaled(weigh.steps(v), &k));
    const int bin = Weigher::bin_of(k);
    if (bin == BINS - 1) { ++below; return; }
    if (q) atomicAdd(&weight[bin], q);
    atomicAdd(&count[bin], 1u);
  });
  below = wave_sum(below);
  if (!(tid & 63) && below) atomicAdd(&count[BINS - 1], below);
  __syncthreads();
  u64* const to_w = a.part_weight + (long long)blockIdx.x * BINS;
  unsigned* const to_c = a.part_count + (long long)blockIdx.x * BINS;
  for (int b = tid; b < BINS; b += SAMPLE_THREADS) { to_w[b] = weight[b]; to_c[b] = count[b]; }
}

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a) {
  constexpr int VEC = SampleRow<T>::VEC;
  constexpr bool CODES = std::is_same<T, __bf16>::value;
  __shared__ SampleShared<CODES ? BINS / 2 : 1> s;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (a.n_dyn && row >= *a.n_dyn) return;
  const SampleChoice by(a, row);
  const float temperature = by.temperature, top_p = by.top_p, min_p = by.min_p;
  const int top_k = by.top_k;
  const float u = fminf(fmaxf(a.u[row], 0.f), 0.99999994f);

  // a wavefront has a range of positions, lanes have neighbouring vectors
  SampleRow<T> x(a, row);
  const int skew = x.skew, tiles = x.tiles(1);                       // vectors of a lane
  const int range_len = tiles * 64 * VEC;                            // positions of a wavefront
  auto vectors = [&](int from, int count, int stride, auto&& f) __attribute__((always_inline)) { x.vectors(from, count, stride, f); };
  auto each = [&](int from, int count, int stride, auto&& f) __attribute__((always_inline)) { x.each(from, count, stride, f); };
  auto value = [&](const u32x4& v, int e) __attribute__((always_inline)) { return x.value(v, e); };
  const int mine = wave * range_len + lane * VEC;
  auto all = [&](auto&& f) __attribute__((always_inline)) { each(mine, tiles, 64 * VEC, f); };
  auto answer = [&](int token, int kept, double logprob) {
    a.token[row] = token;
    if (a.kept) a.kept[row] = kept;
    if (a.logprob) a.logprob[row] = (float)logprob;
  };

  s.table[tid] = octave.v[tid];
  if (by.short_list())
    for (int b = tid; b < BINS; b += SAMPLE_THREADS) { s.count[b] = 0; ((unsigned*)s.weight)[b] = 0; }
  // the largest logit, of this thread and of all, and the largest magnitude
  float own = -INFINITY, big = 0.f;
  const bool in_parts = !std::is_same<T, __bf16>::value && a.parts && !by.short_list();
  if (in_parts) { if (tid < a.parts) own = a.part_best[row * a.parts + tid]; }
  else vectors(mine, tiles, 64 * VEC, [&](int, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const float f = value(v, e);
      own = fmaxf(own, f);                                           // the other one where one is NaN
      if (sizeof(T) == 2) big = fmaxf(big, f > -INFINITY ? fabsf(f) : 0.f);
    }
  });
  float best = own;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) { best = fmaxf(best, __shfl_xor(best, d)); big = fmaxf(big, __shfl_xor(big, d)); }
  if (!lane) { s.wave_max[wave] = best; s.wave_big[wave] = big; }
  if (tid == 0) { s.listed = 0; s.at = 0x7FFFFFFF; s.token = -1; s.cut = 0x7FFFFFFF; s.tiny_w = 0; }
  __syncthreads();
  for (int w = 0; w < SAMPLE_WAVES; ++w) { best = fmaxf(best, s.wave_max[w]); big = fmaxf(big, s.wave_big[w]); }
  if (!(best > -INFINITY)) {
    if (!tid) answer(-1, 0, -INFINITY);
    return;
  }
  if (by.first_alone()) {
    // the first in order alone
    all([&](int i, float v) { if (v == best) atomicMin(&s.at, (unsigned)i); });
    __syncthreads();
    if (!tid) answer((int)s.at, 1, 0.0);
    return;
  }
  const bool odd = x.odd = best == INFINITY, split = in_parts && !odd;
  if (odd) { best = 0.f; own = own == INFINITY ? 0.f : own > -INFINITY ? -1.f : -INFINITY; }
  const double factor = odd ? 1e6 : by.factor();
  const Weigher weigh{s.table, (double)best, factor, a.shift, min_p > 0 ? log2((double)min_p) * STEPS : -INFINITY};
  const bool by_p = top_p < 1.0f;
  const bool by_min = min_p > 0;                                     // NaN: none

  // sums over the threads before this one and over all; ends with all threads past its use of LDS
  auto block_scan = [&](u64 w, unsigned c, u64* before_w, unsigned* before_c, u64* all_w, unsigned* all_c) __attribute__((always_inline)) {
    const u64 sw = wave_scan(w, lane); const unsigned sc = wave_scan(c, lane);
    if (lane == 63) { s.wave_w[wave] = sw; s.wave_c[wave] = sc; }
    __syncthreads();
    u64 bw = 0, aw = 0; unsigned bc = 0, ac = 0;
    for (int v = 0; v < SAMPLE_WAVES; ++v) {
      if (v == wave) { bw = aw; bc = ac; }
      aw += s.wave_w[v]; ac += s.wave_c[v];
    }
    *before_w = bw + sw - w; *before_c = bc + sc - c; *all_w = aw; *all_c = ac;
    __syncthreads();
  };
  auto sort_list = [&](int log2_padded) {                             // ascending
    for (int lk = 1; lk <= log2_padded; ++lk)
      for (int lj = lk - 1; lj >= 0; --lj) {
        for (int p = tid; p < 1 << (log2_padded - 1); p += SAMPLE_THREADS) {
          const int lo = p >> lj << (lj + 1) | (p & ((1 << lj) - 1)), hi = lo + (1 << lj);
          const u64 x0 = s.list[lo], x1 = s.list[hi];
          if ((x0 > x1) == ((lo >> lk & 1) == 0)) { s.list[lo] = x1; s.list[hi] = x0; }
        }
        __syncthreads();
      }
  };
  auto logprob_of = [&](float v, u64 kept_w) { return weigh.steps(v) * (0.69314718055994530942 / STEPS) - log(ldexp((double)kept_w, -a.shift)); };

  // ---- a short list -----------------------------------------------------------------------------------------------------
  if (by.short_list()) {
    // The largest key of 24 bits that top_k threads reach with their own largest logit, by two counts of 12 bits, larger ones first (0 where fewer have any).
    const unsigned own_key = own > -INFINITY ? ordered(own) : 0;
    unsigned* const low = (unsigned*)s.weight;
    auto pick = [&](const unsigned* counts, unsigned need) {          // the bin that brings the count to `need`
      const u32x4 c = *(const u32x4*)(counts + 4 * tid);
      const unsigned c4 = c[0] + c[1] + c[2] + c[3], sc = wave_scan(c4, lane);
      if (lane == 63) s.wave_c[wave] = sc;
      if (!tid) s.bin = -1;
      __syncthreads();
      unsigned bc = sc - c4;
      for (int v = 0; v < wave; ++v) bc += s.wave_c[v];
      if (bc < need && bc + c4 >= need) {
        int b = 0;
        while (bc + c[b] < need) bc += c[b++];
        s.bin = 4 * tid + b; s.before_c = bc;
      }
      __syncthreads();
      return s.bin;
    };
    if (own_key) atomicAdd(&s.count[4095 - (own_key >> 20)], 1u);
    __syncthreads();
    unsigned floor_key = 0;
    const int upper = pick(s.count, (unsigned)top_k);
    if (upper >= 0) {
      const unsigned digit = 4095 - upper, need = (unsigned)top_k - s.before_c;
      if (own_key >> 20 == digit) atomicAdd(&low[4095 - (own_key >> 8 & 4095)], 1u);
      __syncthreads();
      floor_key = digit << 20 | (unsigned)(4095 - pick(low, need)) << 8;
    }
    if (own_key >= floor_key) {                                       // others have none
      all([&](int i, float v) {
        if (ordered(v) < floor_key) return;
        if (*(volatile int*)&s.listed > SORTED) return;              // too many already
        const int at = atomicAdd(&s.listed, 1);
        if (at < SORTED) s.list[at] = (u64)~ordered(v) << 32 | (unsigned)i;      // ascending: larger logits first, equal ones by index
      });
    }
    __syncthreads();
    const int listed = s.listed;
    if (listed <= SORTED) {
      const double limit = by_p ? (double)top_p : 2.0;
      if (listed <= 256) {
        // Few: places in the order and sums before an entry are counted, four threads an entry.
        const int i = tid & 255, part = tid >> 8;
        const u64 entry = i < listed ? s.list[i] : ~0ull;
        const float v = unordered(~(unsigned)(entry >> 32));
        const double w = i < listed ? weigh.scaled(v) : 0.0;
        const u64 q = i < listed ? Weigher::whole(w) : 0;
        if (tid < 256) { s.weight[i] = q; s.weight[256 + i] = 0; s.count[i] = 0; }
        __syncthreads();
        unsigned place = 0; u64 before = 0;
        for (int j = part; j < listed; j += 4) if (s.list[j] < entry) { ++place; before += s.weight[j]; }
        if (place) { atomicAdd(&s.count[i], place); atomicAdd(&s.weight[256 + i], before); }
        __syncthreads();
        place = s.count[i]; before = s.weight[256 + i];
        const bool chosen = tid < listed && place < (unsigned)top_k;
        u64 sum = wave_sum(chosen ? q : 0);
        if (!lane) s.wave_w[wave] = sum;
        __syncthreads();
        sum = s.wave_w[0] + s.wave_w[1] + s.wave_w[2] + s.wave_w[3];
        const bool keep = chosen && (!place || ((double)before < limit * (double)sum && !weigh.dropped(v)));
        if (tid < 256) { s.weight[i] = keep ? q : 0; s.weight[256 + i] = 0; }
        const int kept = __syncthreads_count(keep);
        before = 0;
        for (int j = part; j < listed; j += 4) if ((unsigned)s.list[j] < (unsigned)entry) before += s.weight[j];
        if (before) atomicAdd(&s.weight[256 + i], before);
        sum = wave_sum(keep ? q : 0);
        if (!lane) s.wave_w[wave] = sum;
        __syncthreads();
        sum = s.wave_w[0] + s.wave_w[1] + s.wave_w[2] + s.wave_w[3];
        before = s.weight[256 + i];
        const double target = (double)u * (double)sum;
        if (keep && !((double)before > target) && (double)(before + q) > target) answer((int)(unsigned)entry, kept, logprob_of(v, sum));
        return;
      }
      int padded = 1;
      while (1 << padded < listed) ++padded;
      for (int i = listed + tid; i < 1 << padded; i += SAMPLE_THREADS) s.list[i] = ~0ull;
      __syncthreads();
      sort_list(padded);
      // an entry a thread
      const int k = min(top_k, listed);
      u64 entry = ~0ull, q = 0, bw, aw; unsigned bc, ac;
      double w = 0.0;
      if (tid < k) { entry = s.list[tid]; w = weigh.scaled(unordered(~(unsigned)(entry >> 32))); q = Weigher::whole(w); }
      block_scan(q, 0, &bw, &bc, &aw, &ac);
      const bool keep = tid < k && (!tid || ((double)bw < limit * (double)aw && !weigh.dropped(unordered(~(unsigned)(entry >> 32)))));
      // what is kept is a beginning; in the order of the indices
      const int kept = __syncthreads_count(keep);
      padded = 1;
      while (1 << padded < kept) ++padded;
      if (tid < kept) { s.list[tid] = entry << 32 | (unsigned)tid; s.weight[tid] = q; }
      else if (tid < 1 << padded) s.list[tid] = ~0ull;
      const unsigned key = ~(unsigned)(entry >> 32);
      s.count[tid] = key;
      __syncthreads();
      sort_list(padded);
      const u64 by_index = tid < kept ? s.list[tid] : 0;
      const u64 qi = tid < kept ? s.weight[(unsigned)by_index] : 0;
      block_scan(qi, 0, &bw, &bc, &aw, &ac);
      const double target = (double)u * (double)aw;
      if (qi && !((double)bw > target) && (double)(bw + qi) > target)
        answer((int)(by_index >> 32), kept, logprob_of(unordered(s.count[(unsigned)by_index]), aw));
      return;
    }
    __syncthreads();
    if (!tid) s.listed = 0;
    __syncthreads();
  }

  Last last{0, 0x7FFFFFFF};
  u64 kept_w = 0; unsigned kept = 0;
  bool counted = false;                                              // by the codes of bf16

  // ---- codes of bf16 ------------------------------------------------------------------------------------------------------
  // Entry j of the order: codes of positive logits from the largest down, 0 .. 2047, then of negative ones.  Codes of smaller magnitude than the 16 octaves ("tiny") lie between them; they are listed.
  const int base = max((int)(__float_as_uint(big) >> 23) - 15, 0) << 7;         // the least code of the octaves
  auto entry_of = [&](unsigned code) __attribute__((always_inline)) -> int {    // -1: tiny
    const int off = (int)(code & 0x7FFF) - base;
    return off < 0 ? -1 : code > 0x8000 ? 2048 + off : 2047 - off;              // both zeros are alike
  };
  auto code_of_entry = [&](int j) -> float { return __uint_as_float((unsigned)(j < 2048 ? base + 2047 - j : 0x8000 | (base + j - 2048)) << 16); };
  unsigned ties = 0;                                                 // how many of the last code are kept
  int last_entry = BINS;
  u64 last_q = 0;
  bool tiny_kept = true;
  // Parts of long rows are counted apart, and the draw needs no look at all tokens for their sums (512 x 100003 top-p 122 -> 101 us; 1 x 8192 20 -> 23).
  const bool apart = tiles >= 4;
  const int code_ranges = apart ? CODE_RANGES : 1, code_range = apart ? wave / (SAMPLE_WAVES / CODE_RANGES) : 0, code_len = range_len * (SAMPLE_WAVES / CODE_RANGES);
  if constexpr (CODES) {
    if (!odd && big < INFINITY && (by_p || top_k > 0) && code_len < 65536) {
      for (int b = tid; b < code_ranges * BINS / 2; b += SAMPLE_THREADS) s.codes[0][b] = 0;
      __syncthreads();
      vectors(mine, tiles, 64 * VEC, [&](int, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const unsigned code = (e & 1 ? v[e / 2] >> 16 : v[e / 2] & 0xFFFF);
          if ((code & 0x7FFF) > 0x7F80 || code == 0xFF80) continue;             // NaN, -infinity
          const int j = entry_of(code);
          if (j >= 0) { atomicAdd(&s.codes[code_range][j >> 1], (j & 1) ? 0x10000u : 1u); continue; }
          // more than are listed do not fit and are not counted on (words ruled out by -1e9 make all others tiny: 1 x 131072, one in a hundred ruled out, top-p, 612 us with all of them added up, so 159)
          if (*(volatile int*)&s.listed > SORTED) continue;
          const float t = __uint_as_float(code << 16);
          const int at = atomicAdd(&s.listed, 1);
          atomicAdd(&s.tiny_w, weigh(t));
          if (at < SORTED) s.list[at] = (u64)code_range << 32 | ordered(t);
        }
      });
      __syncthreads();
      const unsigned tiny_c = (unsigned)s.listed;
      const u64 tiny_w = s.tiny_w;
      // four entries a thread, and the tiny ones before those of thread 512
      const int first = tid == 512 ? -1 : 0;
      u64 q[4], w4 = tid == 512 ? tiny_w : 0; unsigned c[4], c4 = tid == 512 ? tiny_c : 0;
      int cut = 0x7FFFFFFF;                                          // the first entry that min-p drops
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = 0;
      for (int d = 0; d < code_ranges; ++d) {
        const unsigned lo = s.codes[d][2 * tid], hi = s.codes[d][2 * tid + 1];
        c[0] += lo & 0xFFFF; c[1] += lo >> 16; c[2] += hi & 0xFFFF; c[3] += hi >> 16;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s.count[4 * tid + e] = c[e];
        const double w = c[e] ? weigh.scaled(code_of_entry(4 * tid + e)) : 0.0;
        q[e] = Weigher::whole(w);
        s.weight[4 * tid + e] = q[e];
        w4 += q[e] * c[e]; c4 += c[e];
        if (c[e] && weigh.dropped(code_of_entry(4 * tid + e))) cut = min(cut, 4 * tid + e);
      }
      if (by_min) atomicMin(&s.cut, cut);
      u64 bw, aw; unsigned bc, ac;
      block_scan(w4, c4, &bw, &bc, &aw, &ac);
      kept_w = aw; kept = ac;
      bool fits = tiny_c <= SORTED;
      // an entry at which the count or the weight reaches its limit becomes the last one, with as many of its tokens as that takes
      auto border = [&](bool by_count, unsigned limit_c, double limit_w) {
        if (!tid) s.bin = -2;
        __syncthreads();
        u64 w = bw; unsigned n = bc;
        for (int e = first; e < 4; ++e) {
          const unsigned ce = e < 0 ? tiny_c : c[e < 0 ? 0 : e];
          const u64 all_e = e < 0 ? tiny_w : q[e < 0 ? 0 : e] * ce;
          const bool before = by_count ? n < limit_c : !n || (double)w < limit_w, after = by_count ? n + ce >= limit_c : (double)(w + all_e) >= limit_w;
          if (ce && before && after) { s.bin = e < 0 ? -1 : 4 * tid + e; s.before_c = n; s.before_w = w; }
          n += ce; w += all_e;
        }
        __syncthreads();
        const int j = s.bin;
        const unsigned n0 = s.before_c; const u64 w0 = s.before_w;
        __syncthreads();
        if (j == -2) return;                                         // not reached: all are kept
        if (j == -1) { fits = false; return; }
        const unsigned ce = s.count[j]; const u64 qe = s.weight[j];
        unsigned m = ce;
        if (by_count) m = limit_c - n0;
        else if (qe) {
          const double need = ceil((limit_w - (double)w0) / (double)qe);
          m = need < 1 ? 1 : need > ce ? ce : (unsigned)need;
          while (m > 1 && (double)(w0 + (m - 1) * qe) >= limit_w) --m;
          while (m < ce && (double)(w0 + m * qe) < limit_w) ++m;
        }
        if (j > last_entry || (j == last_entry && m >= ties)) return;
        last_entry = j; ties = m; last_q = qe; kept_w = w0 + m * qe; kept = n0 + m;
      };
      if (top_k > 0) border(true, (unsigned)top_k, 0.0);
      if (by_p) border(false, 0, (double)top_p * (double)kept_w);
      if (by_min) {
        // tiny ones lie on both sides of the least weight, or all on one
        int tiny_in = 0, tiny_out = 0;
        for (int i = tid; i < (int)min(tiny_c, (unsigned)SORTED); i += SAMPLE_THREADS) { const float t = unordered((unsigned)s.list[i]); if (weigh.dropped(t)) tiny_out = 1; else tiny_in = 1; }
        tiny_in = __syncthreads_or(tiny_in); tiny_out = __syncthreads_or(tiny_out);
        const int j = min(s.cut, BINS);                              // the first counted entry that is dropped
        if (tiny_out && tiny_in && last_entry >= 2048) fits = false;
        const int stop = tiny_out && j > 2048 ? 2048 : j;
        if (stop < BINS && stop <= last_entry) {
          // everything before entry `stop` is kept
          if (tid == stop / 4) {
            u64 w = bw; unsigned n = bc;
            if (tid == 512 && !tiny_out) { w += tiny_w; n += tiny_c; }
            for (int e = 0; e < stop % 4; ++e) { w += q[e] * c[e]; n += c[e]; }
            s.before_w = w; s.before_c = n;
          }
          __syncthreads();
          kept_w = s.before_w; kept = s.before_c; last_entry = stop; ties = 0; last_q = 0;
          __syncthreads();
        }
        if (tiny_out) tiny_kept = false;
      }
      if (last_entry < 2048) tiny_kept = false;
      if (fits) {
        // weights of what is not kept, and of the last code, whose tokens are counted, become none
        for (int j = tid; j < BINS; j += SAMPLE_THREADS) if (j >= last_entry) s.weight[j] = 0;
        counted = true;
      }
      __syncthreads();
      if (!fits) { kept_w = 0; kept = 0; if (!tid) s.listed = 0; __syncthreads(); }
    }
  }

  // the logit that lies `bins` bins below the largest, rounded down or up: what is beyond it needs no exponent to be told from those of a bin two further in
  auto above = [&](int bins, bool up) __attribute__((always_inline)) {
    const double v = (double)best - (double)bins * 16.0 / factor;
    return up ? __double2float_ru(v) : __double2float_rd(v);
  };
  // bin b of all parts, on its way from memory at once (0 of parts that are not there)
  auto of_parts = [&](int b, u64 (&w)[MOST_PARTS], unsigned (&c)[MOST_PARTS]) __attribute__((always_inline)) {
    const long long at = (long long)row * a.parts * BINS + b;
#pragma unroll
    for (int p = 0; p < MOST_PARTS; ++p) {
      w[p] = 0; c[p] = 0;
      if (p < a.parts) { w[p] = a.part_weight[at + p * BINS]; c[p] = a.part_count[at + p * BINS]; }
    }
  };
  // f(index, logit) of the tokens between two logits, which are few: one branch a vector
  auto between = [&](float low, float high, auto&& f) __attribute__((always_inline)) {
    vectors(mine, tiles, 64 * VEC, [&](int p, const u32x4& vec) __attribute__((always_inline)) {
      bool any = false;
#pragma unroll
      for (int e = 0; e < VEC; ++e) any |= (value(vec, e) >= low) & (value(vec, e) <= high);
      if (!any) return;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float v = value(vec, e);
        if (v >= low && v <= high && v > -INFINITY) f(p + e - skew, v);
      }
    });
  };

  if (!counted) {
    // ---- histograms of weights ------------------------------------------------------------------------------------------------
    if (top_k > 0 || by_p) {
      // One border: the first token in order at which the count reaches `limit_c` (by_count), or the weight `limit_w`.  Its bin is looked for among the bins of w, then among bits of the
      // logits, until few enough share it; those are sorted.  Returns the weight up to and with the token; all of it, and `last` as it was, where the limit is not reached.
      auto clear = [&]() { for (int b = tid; b < BINS; b += SAMPLE_THREADS) { s.weight[b] = 0; s.count[b] = 0; } __syncthreads(); };
      auto find_bin = [&](bool by_count, unsigned limit_c, double limit_w, unsigned base_c, u64 base_w) {
        // four bins a thread
        u64 w = 0; unsigned c = 0;
        for (int b = 0; b < 4; ++b) { w += s.weight[4 * tid + b]; c += s.count[4 * tid + b]; }
        u64 bw, aw; unsigned bc, ac;
        block_scan(w, c, &bw, &bc, &aw, &ac);
        bw += base_w; bc += base_c;
        if (!tid) { s.bin = -1; s.before_w = aw; }
        __syncthreads();
        const bool before = by_count ? bc < limit_c : !bc || (double)bw < limit_w, after = by_count ? bc + c >= limit_c : bc + c && (double)(bw + w) >= limit_w;
        if (c && before && after) {
          for (int b = 0; b < 4; ++b) {
            const unsigned cb = s.count[4 * tid + b]; const u64 wb = s.weight[4 * tid + b];
            if (cb && (by_count ? bc + cb >= limit_c : (double)(bw + wb) >= limit_w)) { s.bin = 4 * tid + b; s.bin_count = cb; s.before_c = bc; s.before_w = bw; break; }
            bc += cb; bw += wb;
          }
        }
        __syncthreads();
      };
      auto border = [&](bool by_count, unsigned limit_c, double limit_w) -> u64 {
        // s.weight and s.count are over the bins of w here
        find_bin(by_count, limit_c, limit_w, 0, 0);
        const int w_bin = s.bin;
        unsigned size = s.bin_count, base_c = s.before_c, mask = 0, bits = 0;
        u64 base_w = s.before_w;
        __syncthreads();
        if (w_bin < 0) return base_w;
        // the last bin holds whatever lies 64 octaves down or more: words ruled out by large numbers, most words at a low temperature
        const float low = w_bin == BINS - 1 ? -INFINITY : above(w_bin + 2, false), high = above(w_bin - 2, true);
        auto none_reached = [&]() { const u64 w = base_w + s.before_w; __syncthreads(); return w; };
        auto in_group = [&](float v) __attribute__((always_inline)) { return (ordered(v) & mask) == bits && weigh.bin(v) == w_bin; };
        for (int level = 0; size > SORTED && level < 3; ++level) {
          const int down = level == 0 ? 20 : level == 1 ? 8 : 0, digits = level < 2 ? 4096 : 256;
          clear();
          between(low, high, [&](int, float v) {
            if (!in_group(v)) return;
            const int d = digits - 1 - (int)(ordered(v) >> down & (digits - 1));
            const u64 q = weigh(v);
            if (q) atomicAdd(&s.weight[d], q);
            // lanes with the digit of the first of them, equal logits most often, are counted together (1 x 131072 fp32, 99 % ruled out by -1e9, top_k 3500 and top-p: 754 us one by one,
            // with the last bin's one by one as well, so 238)
            const int first = __builtin_amdgcn_readfirstlane(d);
            const u64 alike = __ballot(d == first);
            if (d != first) atomicAdd(&s.count[d], 1u);
            else if (lane == __ffsll(alike) - 1) atomicAdd(&s.count[d], (unsigned)__popcll(alike));
          });
          __syncthreads();
          find_bin(by_count, limit_c, limit_w, base_c, base_w);
          if (s.bin < 0) return none_reached();
          bits |= (unsigned)(digits - 1 - s.bin) << down; mask |= (unsigned)(digits - 1) << down;
          size = s.bin_count; base_c = s.before_c; base_w = s.before_w;
          __syncthreads();
        }
        if (size > SORTED) {
          // more equal logits than can be sorted: they are in the order of their indices, and all weigh the same
          const u64 q = weigh(unordered(bits));
          unsigned m = 1;
          if (by_count) m = limit_c - base_c;
          else if (q) {
            const double need = ceil((limit_w - (double)base_w) / (double)q);
            m = need < 1 ? 1 : need > size ? size : (unsigned)need;
            while (m > 1 && (double)(base_w + (m - 1) * q) >= limit_w) --m;
            while (m < size && (double)(base_w + m * q) < limit_w) ++m;
          }
          unsigned c = 0;
          all([&](int, float v) { c += ordered(v) == bits; });
          c = wave_sum(c);
          u64 bw, aw; unsigned bc, ac;
          block_scan(0, lane ? 0 : c, &bw, &bc, &aw, &ac);
          bc = __shfl(bc, 0);
          if (bc < m && bc + c >= m) {
            // in this wavefront's range: vector by vector, in the order of the indices
            for (int i = 0; i < tiles; ++i) {
              unsigned here = 0;
              each(mine + i * 64 * VEC, 1, 0, [&](int, float v) { here += ordered(v) == bits; });
              const unsigned up = wave_scan(here, lane), sum = __shfl(up, 63);
              if (bc + sum >= m) {
                unsigned at = bc + up - here;
                each(mine + i * 64 * VEC, 1, 0, [&](int index, float v) { if (ordered(v) == bits && ++at == m) s.at = (unsigned)index; });
                break;
              }
              bc += sum;
            }
          }
          __syncthreads();
          last = Last{bits, (int)s.at};
          __syncthreads();
          return base_w + m * q;
        }
        if (!tid) { s.listed = 0; s.key_min = 0xFFFFFFFFu; s.key_max = 0; s.key = 0; s.at = 0x7FFFFFFF; s.before_w = base_w; }
        __syncthreads();
        between(low, high, [&](int i, float v) {
          if (!in_group(v)) return;
          const int at = atomicAdd(&s.listed, 1);
          if (at < SORTED) s.list[at] = (u64)~ordered(v) << 32 | (unsigned)i;      // larger logits first, equal ones by index
        });
        __syncthreads();
        size = min((unsigned)s.listed, (unsigned)SORTED);
        // two entries a thread
        u64 entry[2];
        for (int e = 0; e < 2; ++e) entry[e] = tid + e * SAMPLE_THREADS < (int)size ? s.list[tid + e * SAMPLE_THREADS] : ~0ull;
        auto key_of = [](u64 x) { return (unsigned)(x >> 32); };
        auto logit_of = [&](u64 x) { return unordered(~key_of(x)); };
        if (size > 64) {
          // one more histogram, of the list's own range of logits
          unsigned lo = min(key_of(entry[0]), key_of(entry[1])), hi = max(entry[0] == ~0ull ? 0u : key_of(entry[0]), entry[1] == ~0ull ? 0u : key_of(entry[1]));
#pragma unroll
          for (int d = 1; d < 64; d *= 2) { lo = min(lo, (unsigned)__shfl_xor((int)lo, d)); hi = max(hi, (unsigned)__shfl_xor((int)hi, d)); }
          if (!lane) { atomicMin(&s.key_min, lo); atomicMax(&s.key_max, hi); }
          clear();
          lo = s.key_min; hi = s.key_max;
          const int down = max(20 - __clz(hi - lo | 1), 0);
          for (int e = 0; e < 2; ++e)
            if (entry[e] != ~0ull) { const int d = (int)((key_of(entry[e]) - lo) >> down); atomicAdd(&s.weight[d], weigh(logit_of(entry[e]))); atomicAdd(&s.count[d], 1u); }
          __syncthreads();
          find_bin(by_count, limit_c, limit_w, base_c, base_w);
          if (s.bin < 0) return none_reached();
          const unsigned digit = (unsigned)s.bin;
          size = s.bin_count; base_c = s.before_c; base_w = s.before_w;
          for (int e = 0; e < 2; ++e) if (entry[e] != ~0ull && (key_of(entry[e]) - lo) >> down != digit) entry[e] = ~0ull;
          if (!tid) s.listed = 0;
          __syncthreads();
          for (int e = 0; e < 2; ++e) if (entry[e] != ~0ull) s.list[atomicAdd(&s.listed, 1)] = entry[e];
          __syncthreads();
        }
        auto decide = [&](u64 x, bool before, bool after, u64 w) { if (before && after) { s.key = ~key_of(x); s.at = (unsigned)x; s.before_w = w; } };
        if (size <= 64) {
          // what lies before an entry is added up by its own thread
          const u64 x = tid < (int)size ? s.list[tid] : ~0ull, q = tid < (int)size ? weigh(logit_of(x)) : 0;
          if (tid < 64) s.weight[tid] = q;
          __syncthreads();
          unsigned c = base_c; u64 w = base_w;
          if (tid < (int)size) {
            for (int j = 0; j < (int)size; ++j) if (s.list[j] < x) { ++c; w += s.weight[j]; }
            decide(x, by_count ? c < limit_c : !c || (double)w < limit_w, by_count ? c + 1 >= limit_c : (double)(w + q) >= limit_w, w + q);
          }
        } else {
          int padded = 1;
          while (1 << padded < (int)size) ++padded;
          for (int i = (int)size + tid; i < 1 << padded; i += SAMPLE_THREADS) s.list[i] = ~0ull;
          __syncthreads();
          sort_list(padded);
          u64 q[2] = {0, 0}; unsigned c = 0;
          for (int e = 0; e < 2; ++e) if (2 * tid + e < (int)size) { q[e] = weigh(logit_of(s.list[2 * tid + e])); ++c; }
          u64 bw, aw; unsigned bc, ac;
          block_scan(q[0] + q[1], c, &bw, &bc, &aw, &ac);
          bw += base_w; bc += base_c;
          for (int e = 0; e < (int)c; ++e) {
            const bool before = by_count ? bc < limit_c : !bc || (double)bw < limit_w;
            ++bc; bw += q[e];
            decide(s.list[2 * tid + e], before, by_count ? bc >= limit_c : (double)bw >= limit_w, bw);
          }
        }
        __syncthreads();
        last = Last{s.key, (int)s.at};
        const u64 sum = s.before_w;
        __syncthreads();
        return sum;
      };
      auto histogram = [&]() {
        if (split) {
          for (int b = tid; b < BINS; b += SAMPLE_THREADS) {
            u64 w = 0, w8[MOST_PARTS]; unsigned c = 0, c8[MOST_PARTS];
            of_parts(b, w8, c8);
#pragma unroll
            for (int p = 0; p < MOST_PARTS; ++p) { w += w8[p]; c += c8[p]; }
            s.weight[b] = w; s.count[b] = c;
          }
          __syncthreads();
          return;
        }
        clear();
        unsigned below = 0;                                          // of the last bin, as in sample_part_kernel
        all([&](int, float v) {
          int k;
          const u64 q = Weigher::whole(weigh.scaled(weigh.steps(v), &k));
          const int bin = Weigher::bin_of(k);
          if (bin == BINS - 1) { ++below; return; }
          if (q) atomicAdd(&s.weight[bin], q);
          atomicAdd(&s.count[bin], 1u);
        });
        below = wave_sum(below);
        if (!lane && below) atomicAdd(&s.count[BINS - 1], below);
        __syncthreads();
      };
      histogram();
      u64 total = 0;                                                 // the weight that top-p takes a share of
      if (top_k > 0) {
        total = border(true, (unsigned)top_k, 0.0);
      } else {
        u64 w = 0, bw; unsigned bc, ac;
        for (int b = 0; b < 4; ++b) w += s.weight[4 * tid + b];
        block_scan(w, 0, &bw, &bc, &total, &ac);
      }
      if (by_p) {
        const Last k_last = last;
        if (top_k > 0) histogram();                                  // the border's own histograms may have taken their place
        border(false, 0u, (double)top_p * (double)total);
        // of two beginnings the shorter one
        if (top_k > 0 && (k_last.key > last.key || (k_last.key == last.key && k_last.at < last.at))) last = k_last;
      }
    }
  }

  // ---- the draw -------------------------------------------------------------------------------------------------------------
  // Weights of what is kept by ranges of positions; f(index, logit, weight, kept) in a lane's own order.  Where codes were counted, tokens of the last code come with ~0 for their weight: the
  // first `ties` of them by index are kept.
  auto weights = [&](int from, int count, int stride, auto&& f) __attribute__((always_inline)) {
    if constexpr (std::is_same<T, __bf16>::value) {
      if (counted) {
        vectors(from, count, stride, [&](int p, const u32x4& v) __attribute__((always_inline)) {
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const unsigned code = (e & 1 ? v[e / 2] >> 16 : v[e / 2] & 0xFFFF);
            if ((code & 0x7FFF) > 0x7F80 || code == 0xFF80) continue;
            const int j = entry_of(code);
            const float value16 = __uint_as_float(code << 16);
            if (j >= 0) f(p + e - skew, value16, j == last_entry ? ~0ull : s.weight[j], true);
            else if (tiny_kept) f(p + e - skew, value16, weigh(value16), true);
          }
        });
        return;
      }
    }
    vectors(from, count, stride, [&](int p, const u32x4& vec) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const float v = value(vec, e);
        bool keep = v > -INFINITY;
        if (last.key) {                                              // the same for all
          const unsigned key = ordered(v);
          keep = keep && (key > last.key || (key == last.key && p + e - skew <= last.at));
        }
        const double w = weigh.scaled(keep ? v : -INFINITY);
        keep = keep && !weigh.dropped(v);
        f(p + e - skew, v, keep ? Weigher::whole(w) : 0ull, keep);
      }
    });
  };
  const bool by_counts = CODES && counted && apart;
  const int ranges = split ? a.parts : by_counts ? CODE_RANGES : SAMPLE_WAVES;
  const int draw_len = split ? x.tiles(a.parts) * SAMPLE_THREADS * VEC : by_counts ? code_len : range_len;
  if (by_counts) {
    // sums of counts times weights; `count`: of the last code
    if constexpr (CODES) {
      if (tid < CODE_RANGES) { s.wave_w[tid] = 0; s.wave_c[tid] = last_entry < BINS ? s.codes[tid][last_entry >> 1] >> (last_entry & 1) * 16 & 0xFFFF : 0; }
      __syncthreads();
      u64 q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] = s.weight[4 * tid + e];
#pragma unroll
      for (int d = 0; d < CODE_RANGES; ++d) {
        const unsigned lo = s.codes[d][2 * tid], hi = s.codes[d][2 * tid + 1];
        const u64 w = wave_sum(q[0] * (lo & 0xFFFF) + q[1] * (lo >> 16) + q[2] * (hi & 0xFFFF) + q[3] * (hi >> 16));
        if (!lane && w) atomicAdd(&s.wave_w[d], w);
      }
      if (tiny_kept) for (int i = tid; i < s.listed; i += SAMPLE_THREADS) atomicAdd(&s.wave_w[s.list[i] >> 32], weigh(unordered((unsigned)s.list[i])));
    }
  } else if (split) {
    // Bins before the last one are kept as a whole, their sums are there for each part; tokens of the others are looked at one by one.
    int whole = last.key ? weigh.bin(unordered(last.key)) : BINS;
    float low = last.key ? unordered(last.key) : -INFINITY;
    if (by_min) {
      const int bins = (int)fmin(-log2((double)min_p) * (STEPS / 16), (double)BINS);
      whole = min(whole, max(bins - 1, 0));
      if (bins < BINS) low = fmaxf(low, above(bins + 3, false));
    }
    if (tid < SAMPLE_WAVES) { s.wave_w[tid] = 0; s.wave_c[tid] = 0; }
    __syncthreads();
    u64 sums[MOST_PARTS] = {}; unsigned counts[MOST_PARTS] = {};
    for (int b = tid; b < whole; b += SAMPLE_THREADS) {
      u64 w[MOST_PARTS]; unsigned c[MOST_PARTS];
      of_parts(b, w, c);
#pragma unroll
      for (int p = 0; p < MOST_PARTS; ++p) { sums[p] += w[p]; counts[p] += c[p]; }
    }
#pragma unroll
    for (int p = 0; p < MOST_PARTS; ++p) {
      const u64 w = wave_sum(sums[p]); const unsigned c = wave_sum(counts[p]);
      if (!lane && c) { atomicAdd(&s.wave_w[p], w); atomicAdd(&s.wave_c[p], c); }
    }
    if (whole < BINS) {
      const float high = above(whole - 2, true);
      between(low, high, [&](int i, float v) {
        if (weigh.bin(v) < whole) return;
        const unsigned key = ordered(v);
        if (last.key && !(key > last.key || (key == last.key && i <= last.at))) return;
        if (weigh.dropped(v)) return;
        const int p = (i + skew) / draw_len;
        atomicAdd(&s.wave_w[p], weigh(v)); atomicAdd(&s.wave_c[p], 1u);
      });
    }
  } else {
    u64 sum = 0; unsigned count = 0;                                 // count: of what is kept, or of the last code
    weights(mine, tiles, 64 * VEC, [&](int, float, u64 q, bool keep) __attribute__((always_inline)) {
      if (counted) { if (q == ~0ull) ++count; else sum += q; }
      else { sum += q; count += keep; }
    });
    sum = wave_sum(sum); count = wave_sum(count);
    if (!lane) { s.wave_w[wave] = sum; s.wave_c[wave] = count; }
  }
  __syncthreads();
  if (!counted) for (int w = 0; w < ranges; ++w) { kept_w += s.wave_w[w]; kept += s.wave_c[w]; }
  const double target = (double)u * (double)kept_w;
  // weight up to a point: w of other tokens and n of the last code
  auto weight_of = [&](u64 w, unsigned n) { return counted ? w + (u64)min(n, ties) * last_q : w; };
  u64 before = 0; unsigned before_n = 0; int range = 0;
  for (; range < ranges - 1; ++range) {
    const u64 w = before + s.wave_w[range]; const unsigned n = before_n + s.wave_c[range];
    if ((double)weight_of(w, n) > target) break;
    before = w; before_n = n;
  }
  __syncthreads();
  // the range that the target is in, in pieces of neighbouring vectors of all threads
  for (int p0 = range * draw_len; p0 < (range + 1) * draw_len; p0 += SAMPLE_THREADS * VEC) {
    const bool in = p0 + tid * VEC < (range + 1) * draw_len;
    u64 here = 0; unsigned here_n = 0;
    if (in) weights(p0 + tid * VEC, 1, 0, [&](int, float, u64 q, bool) { if (counted && q == ~0ull) ++here_n; else here += q; });
    u64 bw, aw; unsigned bn, an;
    block_scan(here, here_n, &bw, &bn, &aw, &an);
    bw += before; bn += before_n;
    if (in && !((double)weight_of(bw, bn) > target) && (double)weight_of(bw + here, bn + here_n) > target) {
      bool found = false;
      weights(p0 + tid * VEC, 1, 0, [&](int i, float v, u64 q, bool) {
        if (found) return;
        if (counted && q == ~0ull) ++bn; else bw += q;
        if ((double)weight_of(bw, bn) > target) {
          found = true;
          s.token = i;
          answer(i, (int)kept, logprob_of(v, kept_w));
        }
      });
    }
    __syncthreads();
    if (s.token >= 0) return;
    before += aw; before_n += an;
  }
}

}  // namespace
}  // namespace octo

using namespace octo;

namespace {
// Workgroups of a row where rows are few and long, or 0.  fp32, top-p: 1 x 131072 113 us alone, so 76; 48 x 131072 115 and 94; 1 x 262144 200 and 115; but 128 x 131072 126 and 133,
// 1 x 32768 37 and 41.  Counting the codes of bf16 takes less (1 x 131072 49, shared by weights 91), a short list needs no weights of all tokens.
int sample_parts(const octo_sample_op* op) {
  const bool short_list = !op->d_top_k && op->top_k > 0 && op->top_k <= LISTED;
  if (op->dtype == OCTO_BF16 || op->n < 1 || op->n > 64 || op->vocab < 65536 || short_list) return 0;
  return 256 / op->n < MOST_PARTS ? 256 / op->n : MOST_PARTS;
}
constexpr size_t PART_BYTES = (size_t)BINS * (sizeof(u64) + sizeof(unsigned)) + sizeof(float);
bool sample_sizes(const octo_sample_op* op) { return op && op->dtype >= OCTO_F32 && op->dtype <= OCTO_BF16 && op->n >= 0 && op->n <= 0x3FFFFF && op->vocab >= 1 && op->vocab <= OCTO_MAX_VOCAB; }
}  // namespace

extern "C" size_t octo_op_sample_workspace_bytes(const octo_sample_op* op) { return sample_sizes(op) ? (size_t)op->n * sample_parts(op) * PART_BYTES : 0; }

extern "C" octo_status octo_op_sample(const octo_sample_op* op, void* hip_stream) {
  if (!sample_sizes(op)) return OCTO_EINVAL;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  if (!op->d_logits || (uintptr_t)op->d_logits % es || op->row < 0 || !op->d_u || !op->d_token) return OCTO_EINVAL;
  if (((uintptr_t)op->d_u | (uintptr_t)op->d_token | (uintptr_t)op->d_temperature | (uintptr_t)op->d_top_k | (uintptr_t)op->d_top_p | (uintptr_t)op->d_min_p | (uintptr_t)op->d_logprob |
       (uintptr_t)op->d_kept | (uintptr_t)op->d_n) & 3) return OCTO_EINVAL;
  if (!op->n) return OCTO_OK;
  SampleArgs a{};
  a.logits = op->d_logits; a.row = op->row; a.u = op->d_u;
  a.temperature = op->d_temperature; a.top_k = op->d_top_k; a.top_p = op->d_top_p; a.min_p = op->d_min_p;
  a.all_temperature = op->temperature; a.all_top_k = op->top_k; a.all_top_p = op->top_p; a.all_min_p = op->min_p;
  a.token = op->d_token; a.logprob = op->d_logprob; a.kept = op->d_kept; a.n_dyn = op->d_n; a.vocab = op->vocab;
  int bits = 0;
  while ((1 << bits) < op->vocab) ++bits;
  a.shift = 62 - bits < 50 ? 62 - bits : 50;                         // a sum of `vocab` weights of up to one stays within 63 bits
  const size_t need = octo_op_sample_workspace_bytes(op);
  if (op->d_workspace && need) {
    if (op->workspace_bytes < need || (uintptr_t)op->d_workspace & 15) return OCTO_EINVAL;
    a.parts = sample_parts(op);
    const size_t all = (size_t)op->n * a.parts;
    a.part_weight = (u64*)op->d_workspace; a.part_count = (unsigned*)(a.part_weight + all * BINS); a.part_best = (float*)(a.part_count + all * BINS);
  }
  hipStream_t s = (hipStream_t)hip_stream;
  const dim3 grid((unsigned)op->n), block(SAMPLE_THREADS);
  if (a.parts) {
    const dim3 wide((unsigned)(op->n * a.parts));
    if (op->dtype == OCTO_F32) { hipLaunchKernelGGL(sample_best_kernel<float>, wide, block, 0, s, a); hipLaunchKernelGGL(sample_part_kernel<float>, wide, block, 0, s, a); }
    else { hipLaunchKernelGGL(sample_best_kernel<_Float16>, wide, block, 0, s, a); hipLaunchKernelGGL(sample_part_kernel<_Float16>, wide, block, 0, s, a); }
  }
  if (op->dtype == OCTO_F32) hipLaunchKernelGGL(sample_kernel<float>, grid, block, 0, s, a);
  else if (op->dtype == OCTO_F16) hipLaunchKernelGGL(sample_kernel<_Float16>, grid, block, 0, s, a);
  else hipLaunchKernelGGL(sample_kernel<__bf16>, grid, block, 0, s, a);
  return hipGetLastError() == hipSuccess ? OCTO_OK : OCTO_EHIP;
}
