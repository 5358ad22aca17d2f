// octo_op_sample: one token of each row of logits.
//
// With the tokens of a row in the order of their logits (equal ones by index) and w = exp((x - max) / temperature), top-k, top-p and min-p each keep a beginning of that order; what
// they keep in common is one too, and is known by its last token.  The token is drawn in the order of indices: the first at which the sum of the kept weights passes u times all.
//
// A workgroup takes a row.  Sums of weights decide which token a border falls on, so they are made of integers: w is computed in fp64 (64 steps an octave from a table, the rest by a
// polynomial, 1e-15 off) and rounded to multiples of 2^-shift of the largest, whose sums in 64 bits are the same in any order.  Borders are found by a histogram of
// counts and weights over 64 octaves of w, 64 bins each; the tokens of the bin that holds the border are sorted.  Where they are too many (equal logits, say), bits of the
// logits themselves make further histograms.
#include <cmath>

#include "mfma_common.h"
#include "octo_internal.h"

namespace octo {
namespace {

constexpr int SAMPLE_THREADS = 1024, SAMPLE_WAVES = 16, BINS = 4096, SORTED = 2048;
typedef unsigned long long u64;

struct SampleArgs {
  const void* logits; long long row;
  const float *u, *temperature, *top_p, *min_p; const int* top_k;
  float all_temperature, all_top_p, all_min_p; int all_top_k;
  int* token; float* logprob; int* kept;
  const int* n_dyn;
  int vocab, shift;
};

// 2^(j / 64), j = 0 .. 63
struct ExpTable { double v[64]; };
ExpTable exp_table() {
  ExpTable t;
  for (int j = 0; j < 64; ++j) t.v[j] = std::exp2(j / 64.0);
  return t;
}

// Floats as integers of the same order.
__device__ __forceinline__ unsigned ordered(float v) {
  const unsigned b = __float_as_uint(v);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

struct Weigher {
  const double* table;      // in LDS
  double inverse;           // 1 / temperature
  float max;
  int shift;
  // w of a logit in units of 2^-shift, its bin, and w itself
  __device__ __forceinline__ u64 operator()(float v, int* bin, double* w) const {
    double x = v == max ? 0.0 : ((double)v - (double)max) * inverse;
    x = fmax(x, -50.0);                                              // e^-50 < 2^-72; also where it is no number (an infinite maximum, an infinite temperature)
    const double kd = rint(x * 92.33248261689366);               // 64 / ln 2
    const double r = fma(kd, -0.010830424696249145, x), r2 = fma(kd, -3.623510646634843e-19, r);
    const int k = (int)kd;
    double p = fma(r2, 1.0 / 120, 1.0 / 24);
    p = fma(p, r2, 1.0 / 6); p = fma(p, r2, 0.5); p = fma(p, r2, 1.0); p = fma(p, r2, 1.0);
    *w = ldexp(p * table[k & 63], k >> 6);
    *bin = min(-k, BINS - 1);
    // adding 2^52 leaves the nearest integer in the low bits
    return (u64)__double_as_longlong(ldexp(*w, shift) + 4503599627370496.0) - 0x4330000000000000ull;
  }
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

struct SampleShared {
  double table[64];
  u64 weight[BINS];
  unsigned count[BINS];
  u64 list[SORTED];
  u64 wave_w[SAMPLE_WAVES];
  unsigned wave_c[SAMPLE_WAVES];
  float wave_max[SAMPLE_WAVES];
  int wave_at[SAMPLE_WAVES];
  int listed, bin, token;
  unsigned bin_count, key, at, before_c;
  u64 before_w;
};

template <typename T>
__global__ __launch_bounds__(SAMPLE_THREADS) void sample_kernel(SampleArgs a, ExpTable table) {
  constexpr int VEC = 16 / sizeof(T), DEPTH = 4;
  __shared__ SampleShared s;
  const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (a.n_dyn && row >= *a.n_dyn) return;
  const T* const x = (const T*)a.logits + row * a.row;
  if (tid < 64) s.table[tid] = table.v[tid];

  // Positions are indices plus the distance of the row's start from the last 16-byte border before it, so that vectors are aligned; a wavefront has a range of them, lanes have
  // neighbouring vectors.
  const int skew = (int)(((uintptr_t)x & 15) / sizeof(T)), end = a.vocab + skew;
  const int tiles = (end + SAMPLE_WAVES * 64 * VEC - 1) / (SAMPLE_WAVES * 64 * VEC);                 // vectors of a lane
  auto load = [&](int p) __attribute__((always_inline)) -> u32x4 {
    u32x4 v;
    if (p >= skew && p + VEC <= end) return *(const u32x4*)(x + (p - skew));
#pragma unroll
    for (int e = 0; e < VEC; ++e) ((T*)&v)[e] = p + e >= skew && p + e < end ? x[p + e - skew] : (T)-INFINITY;
    return v;
  };
  // f(index, logit) of every token of the positions from, from + stride ... that may be drawn
  auto each = [&](int from, int count, int stride, auto&& f) __attribute__((always_inline)) {
    for (int i0 = 0; i0 < count; i0 += DEPTH) {
      u32x4 v[DEPTH];
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) if (i0 + d < count) v[d] = load(from + (i0 + d) * stride);
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        if (i0 + d >= count) break;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float f32 = (float)((const T*)&v[d])[e];
          if (f32 > -INFINITY) f(from + (i0 + d) * stride + e - skew, f32);          // neither -infinity nor NaN
        }
      }
    }
  };
  const int mine = wave * tiles * 64 * VEC + lane * VEC;
  auto all = [&](auto&& f) __attribute__((always_inline)) { each(mine, tiles, 64 * VEC, f); };

  // the best token, and how many there are
  float best = -INFINITY; int best_at = 0x7FFFFFFF; unsigned there = 0;
  all([&](int i, float v) { ++there; if (v > best || (v == best && i < best_at)) { best = v; best_at = i; } });
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const float v = __shfl_xor(best, d); const int i = __shfl_xor(best_at, d);
    if (v > best || (v == best && i < best_at)) { best = v; best_at = i; }
  }
  there = wave_sum(there);
  if (!lane) { s.wave_max[wave] = best; s.wave_at[wave] = best_at; s.wave_c[wave] = there; }
  __syncthreads();
  there = 0;
  for (int w = 0; w < SAMPLE_WAVES; ++w) {
    const float v = s.wave_max[w]; const int i = s.wave_at[w];
    if (v > best || (v == best && i < best_at)) { best = v; best_at = i; }
    there += s.wave_c[w];
  }
  __syncthreads();

  const float temperature = a.temperature ? a.temperature[row] : a.all_temperature;
  if (!there || !(temperature > 0)) {
    if (!tid) {
      a.token[row] = there ? best_at : -1;
      if (a.kept) a.kept[row] = there ? 1 : 0;
      if (a.logprob) a.logprob[row] = there ? 0.f : -INFINITY;
    }
    return;
  }
  const int top_k = a.top_k ? a.top_k[row] : a.all_top_k;
  const float top_p = a.top_p ? a.top_p[row] : a.all_top_p, min_p = a.min_p ? a.min_p[row] : a.all_min_p;
  const Weigher weigh{s.table, 1.0 / (double)temperature, best, a.shift};

  // the last token that top-k and top-p keep: all whose ordered logit is above `last_key`, and of those equal to it the ones up to index `last_at`
  unsigned last_key = 0; int last_at = 0x7FFFFFFF;
  const bool by_k = top_k > 0 && (unsigned)top_k < there, by_p = top_p < 1.0f;

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

  u64 total = 0;                                                     // the weight that top-p takes a share of
  if (by_k || by_p) {
    // One border: the first token in order at which the count reaches `limit_c` (by_count), or the weight `limit_w`.  Its bin is looked for among the bins of w, then among bits of the logits, until
    // few enough share it; those are sorted.  Returns the weight up to and with the token.
    auto clear = [&]() { for (int b = tid; b < BINS; b += SAMPLE_THREADS) { s.weight[b] = 0; s.count[b] = 0; } __syncthreads(); };
    auto find_bin = [&](bool by_count, unsigned limit_c, double limit_w, unsigned base_c, u64 base_w) {
      // four bins a thread
      u64 w = 0; unsigned c = 0;
      for (int b = 0; b < 4; ++b) { w += s.weight[4 * tid + b]; c += s.count[4 * tid + b]; }
      u64 bw, aw; unsigned bc, ac;
      block_scan(w, c, &bw, &bc, &aw, &ac);
      bw += base_w; bc += base_c;
      if (!tid) s.bin = -1;
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
      auto in_group = [&](float v, int* bin, double* w, u64* q) __attribute__((always_inline)) {
        *q = weigh(v, bin, w);
        return *bin == w_bin && (ordered(v) & mask) == bits;
      };
      for (int level = 0; size > SORTED && level < 3; ++level) {
        const int down = level == 0 ? 20 : level == 1 ? 8 : 0, digits = level < 2 ? 4096 : 256;
        clear();
        all([&](int, float v) {
          int bin; double w; u64 q;
          if (in_group(v, &bin, &w, &q)) { const int d = digits - 1 - (int)(ordered(v) >> down & (digits - 1)); atomicAdd(&s.weight[d], q); atomicAdd(&s.count[d], 1u); }
        });
        __syncthreads();
        find_bin(by_count, limit_c, limit_w, base_c, base_w);
        bits |= (unsigned)(digits - 1 - s.bin) << down; mask |= (unsigned)(digits - 1) << down;
        size = s.bin_count; base_c = s.before_c; base_w = s.before_w;
        __syncthreads();
      }
      if (size > SORTED) {
        // more equal logits than can be sorted: they are in the order of their indices, and all weigh the same
        int bin; double wd;
        const unsigned sign = bits & 0x80000000u ? bits & 0x7FFFFFFFu : ~bits;
        const u64 q = weigh(__uint_as_float(sign), &bin, &wd);
        unsigned m = 1;
        if (by_count) m = limit_c - base_c;
        else if (q) {
          const double need = ceil((limit_w - (double)base_w) / (double)q);
          m = need < 1 ? 1 : need > size ? size : (unsigned)need;
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
            const unsigned up = wave_scan(here, lane), last = __shfl(up, 63);
            if (bc + last >= m) {
              unsigned at = bc + up - here;
              each(mine + i * 64 * VEC, 1, 0, [&](int index, float v) { if (ordered(v) == bits && ++at == m) s.at = (unsigned)index; });
              break;
            }
            bc += last;
          }
        }
        __syncthreads();
        last_key = bits; last_at = (int)s.at;
        __syncthreads();
        return base_w + m * q;
      }
      if (!tid) s.listed = 0;
      int padded = 2;
      while (padded < (int)size) padded *= 2;
      __syncthreads();
      for (int i = tid; i < padded; i += SAMPLE_THREADS) s.list[i] = ~0ull;
      __syncthreads();
      all([&](int i, float v) {
        int bin; double w; u64 q;
        if (in_group(v, &bin, &w, &q)) s.list[atomicAdd(&s.listed, 1)] = (u64)~ordered(v) << 32 | (unsigned)i;      // ascending: larger logits first, equal ones by index
      });
      __syncthreads();
      for (int k = 2; k <= padded; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
          for (int p = tid; p < padded / 2; p += SAMPLE_THREADS) {
            const int lo = 2 * j * (p / j) + p % j, hi = lo + j;
            const u64 x0 = s.list[lo], x1 = s.list[hi];
            if ((x0 > x1) == ((lo & k) == 0)) { s.list[lo] = x1; s.list[hi] = x0; }
          }
          __syncthreads();
        }
      // two entries a thread
      u64 q[2] = {0, 0}; unsigned c = 0;
      for (int e = 0; e < 2; ++e) {
        if (2 * tid + e >= (int)size) continue;
        const unsigned key = ~(unsigned)(s.list[2 * tid + e] >> 32);
        int bin; double w;
        q[e] = weigh(__uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key), &bin, &w);
        ++c;
      }
      u64 bw, aw; unsigned bc, ac;
      block_scan(q[0] + q[1], c, &bw, &bc, &aw, &ac);
      bw += base_w; bc += base_c;
      for (int e = 0; e < (int)c; ++e) {
        const bool before = by_count ? bc < limit_c : !bc || (double)bw < limit_w;
        ++bc; bw += q[e];
        const bool after = by_count ? bc >= limit_c : (double)bw >= limit_w;
        if (before && after) { s.key = ~(unsigned)(s.list[2 * tid + e] >> 32); s.at = (unsigned)s.list[2 * tid + e]; s.before_w = bw; }
      }
      __syncthreads();
      last_key = s.key; last_at = (int)s.at;
      const u64 sum = s.before_w;
      __syncthreads();
      return sum;
    };
    auto histogram = [&]() {
      clear();
      all([&](int, float v) {
        int bin; double w;
        const u64 q = weigh(v, &bin, &w);
        atomicAdd(&s.weight[bin], q);
        atomicAdd(&s.count[bin], 1u);
      });
      __syncthreads();
    };
    histogram();
    {
      u64 w = 0, bw; unsigned bc, ac;
      for (int b = 0; b < 4; ++b) w += s.weight[4 * tid + b];
      block_scan(w, 0, &bw, &bc, &total, &ac);
    }
    if (by_k) total = border(true, (unsigned)top_k, 0.0);
    if (by_p) {
      const unsigned k_key = last_key; const int k_at = last_at;
      if (by_k) histogram();                                         // the border's own histograms may have taken their place
      border(false, 0u, (double)top_p * (double)total);
      // of two beginnings the shorter one
      if (by_k && (k_key > last_key || (k_key == last_key && k_at < last_at))) { last_key = k_key; last_at = k_at; }
    }
  }

  // kept weights by ranges of positions
  auto keeps = [&](int i, float v, double w) __attribute__((always_inline)) {
    const unsigned key = ordered(v);
    return (key > last_key || (key == last_key && i <= last_at)) && (!(w < (double)min_p) || i == best_at);
  };
  u64 sum = 0; unsigned count = 0;
  all([&](int i, float v) {
    int bin; double w;
    const u64 q = weigh(v, &bin, &w);
    if (keeps(i, v, w)) { sum += q; ++count; }
  });
  sum = wave_sum(sum); count = wave_sum(count);
  if (!lane) { s.wave_w[wave] = sum; s.wave_c[wave] = count; }
  __syncthreads();
  u64 kept_w = 0; unsigned kept = 0;
  for (int w = 0; w < SAMPLE_WAVES; ++w) { kept_w += s.wave_w[w]; kept += s.wave_c[w]; }
  const float u = fminf(fmaxf(a.u[row], 0.f), 0.99999994f);
  const double target = (double)u * (double)kept_w;
  u64 before = 0; int range = 0;
  for (; range < SAMPLE_WAVES - 1; ++range) {
    if ((double)(before + s.wave_w[range]) > target) break;
    before += s.wave_w[range];
  }
  if (!tid) s.token = -1;
  __syncthreads();
  // the range that the target is in, in pieces of neighbouring vectors of all threads
  for (int p0 = range * tiles * 64 * VEC; p0 < (range + 1) * tiles * 64 * VEC; p0 += SAMPLE_THREADS * VEC) {
    const bool in = p0 + tid * VEC < (range + 1) * tiles * 64 * VEC;
    u64 here = 0;
    if (in) each(p0 + tid * VEC, 1, 0, [&](int i, float v) { int bin; double w; const u64 q = weigh(v, &bin, &w); if (keeps(i, v, w)) here += q; });
    u64 bw, aw; unsigned bc, ac;
    block_scan(here, 0, &bw, &bc, &aw, &ac);
    bw += before;
    if (in && here && !((double)bw > target) && (double)(bw + here) > target) {
      bool found = false;
      each(p0 + tid * VEC, 1, 0, [&](int i, float v) {
        int bin; double w;
        const u64 q = weigh(v, &bin, &w);
        if (!keeps(i, v, w) || found) return;
        bw += q;
        if ((double)bw > target) {
          found = true;
          s.token = i;
          a.token[row] = i;
          if (a.kept) a.kept[row] = (int)kept;
          if (a.logprob) a.logprob[row] = (float)((v == best ? 0.0 : ((double)v - (double)best) * weigh.inverse) - log(ldexp((double)kept_w, -a.shift)));
        }
      });
    }
    __syncthreads();
    if (s.token >= 0) return;
    before += aw;
  }
}

}  // namespace
}  // namespace octo

using namespace octo;

extern "C" octo_status octo_op_sample(const octo_sample_op* op, void* hip_stream) {
  if (!op || (op->dtype != OCTO_F32 && op->dtype != OCTO_F16 && op->dtype != OCTO_BF16)) return OCTO_EINVAL;
  const int es = op->dtype == OCTO_F32 ? 4 : 2;
  if (op->n < 0 || op->n > 0x3FFFFF || op->vocab < 1 || op->vocab > OCTO_MAX_VOCAB || !op->d_logits || (uintptr_t)op->d_logits % es || op->row < 0 || !op->d_u || !op->d_token) return OCTO_EINVAL;
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
  static const ExpTable table = exp_table();
  hipStream_t s = (hipStream_t)hip_stream;
  const dim3 grid((unsigned)op->n), block(SAMPLE_THREADS);
  if (op->dtype == OCTO_F32) hipLaunchKernelGGL(sample_kernel<float>, grid, block, 0, s, a, table);
  else if (op->dtype == OCTO_F16) hipLaunchKernelGGL(sample_kernel<_Float16>, grid, block, 0, s, a, table);
  else hipLaunchKernelGGL(sample_kernel<__bf16>, grid, block, 0, s, a, table);
  return hipGetLastError() == hipSuccess ? OCTO_OK : OCTO_EHIP;
}
