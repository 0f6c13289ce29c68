// The next token of each row of logits, from a given uniform number.
//
// With weights w_i = exp((l_i - max l) / T), the kept tokens are a prefix of the
// order by (logit descending, index ascending): of top_k tokens, then the
// shortest one whose weights reach top_p of theirs, then those of weight min_p
// and more (the first token always stays).  The token drawn is the first index
// whose running sum of kept weights exceeds u times their total.
//
// The weights are binary64, and their sums binary64 or 64-bit integers of a finer unit
// than the draws can tell: a running sum of 262144 binary32 weights moves by about 1e-8
// with the order of its terms, and as much of the draws would change.
//
// Two launches.  The first reads every logit once: per chunk of 16384 it counts
// the logits in 2047 bins from the chunk's largest one down, and adds up weights.
// Bins are the values' upper 16 bits in order, but for 64 equal ones between
// -1/8 and 1/8, where those bits are finer than a logit's meaning: 2047 bins reach
// from any usual largest logit over 0 to far below it.  A bf16 bin outside that
// band is one value, and its weight its count times the value's; the other bins'
// weights are added as 64-bit integers in units of 2^-48 of the chunk's largest
// weight, and where the row's bins are summed in units of 2^-(62 - log2 n) of the row's
// (2^-44 of 262144 logits), so that no order of the additions matters.
//
// The second launch, one workgroup a row, finds the kept prefix and the chunk of
// the drawn token from counts and sums, and reads that chunk again.  Where the
// prefix ends inside a bin of several values it sorts that bin's logits.  A row
// whose prefix ends below the bins among logits that have a weight, or in a bin of
// several values with more than 2048 logits, goes through passes over the row by that
// one workgroup instead: 64 rows of 262144 take 1.1 to 1.4 ms then.
//
// 64 bf16 rows of 262144: 26 us for the scan (33 MB, 1.3 TB/s), which issues 39 vector and
// 27 scalar instructions for 64 logits: the vector units are busy half of its cycles, the
// scalar ones a third, LDS an eighth.  37 for the draw, a chain of steps on one workgroup a
// row: the row's bins (12 us), the prefix, the chunks' sums (4) and the chunk (4 to 15); 24
// more where a prefix ends among the values around 0.  One row: 11 and 21 us (with bins from
// the largest logit to 0 only, 26 for both, but passes over the row where a prefix ends
// below 0).  131 f32 rows of 100003: 31 and 46 us.
#include <cmath>
#include <cstdint>

#include "device.h"
#include "kernels.h"

namespace w8a8 {

namespace {

constexpr int kThreads = 1024;
constexpr int kVec = 8;                        // consecutive logits of a thread
constexpr int kBlock = kThreads * kVec;        // logits a workgroup takes at a time
constexpr int kMaxBlocks = kSampleMaxVocab / kBlock;
constexpr uint32_t kMinusInf = 0x007fffffu;    // key of -inf

// order-preserving bits of a logit; -0 is 0, NaN is below -inf
__device__ __forceinline__ uint32_t key_of(float l) {
  if (l != l) return 0;
  const uint32_t b = __float_as_uint(l + 0.0f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  if (key == 0) return -INFINITY;
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// 16 bytes of a row, which need not lie at a multiple of 16 (f32 rows of odd length do not):
// the loads take any address.  Logit by logit 131 such rows of 100003 took 44 us to scan,
// not 28, and 87 to draw from, not 44.
typedef uint32_t Four __attribute__((ext_vector_type(4)));
typedef Four Four32 __attribute__((aligned(4)));
typedef Four Four16 __attribute__((aligned(2)));

struct Row {
  const void* base;
  int64_t n;
  bool bf;
  uint32_t top;   // key of the largest logit
  double best, inv_t;
};

__device__ __forceinline__ uint32_t key_at(const Row& r, int64_t i) {
  if (i >= r.n) return 0;
  return key_of(r.bf ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(r.base)[i])
                     : reinterpret_cast<const float*>(r.base)[i]);
}

// the keys of eight logits from index i on (a multiple of 8); 0 behind the row
__device__ __forceinline__ void keys8(const Row& r, int64_t i, uint32_t (&k)[kVec]) {
  if (i + kVec <= r.n) {
    if (r.bf) {
      const Four w = *reinterpret_cast<const Four16*>(reinterpret_cast<const uint16_t*>(r.base) + i);
#pragma unroll
      for (int e = 0; e < kVec; ++e) k[e] = key_of(bf16_bits_to_float((w[e >> 1] >> (16 * (e & 1))) & 0xffffu));
    } else {
      const Four32* p = reinterpret_cast<const Four32*>(reinterpret_cast<const float*>(r.base) + i);
      const Four a = p[0], b = p[1];
#pragma unroll
      for (int e = 0; e < kVec; ++e) k[e] = key_of(__uint_as_float(e < 4 ? a[e] : b[e - 4]));
    }
  } else {
#pragma unroll
    for (int e = 0; e < kVec; ++e) k[e] = key_at(r, i + e);
  }
}

// e^x for x <= 0, within 2^-51 of it (0 below -708): x = (32 m + j) ln2 / 32 + y with
// |y| <= ln2 / 64, e^y by its series to y^6 (the next term is below 2^-57), 2^(j/32)
// from a table.  Half the instructions of a general exp, which bounded the scan.
__device__ const double kExp2Table[32] = {  // 2^(j / 32)
    0x1.0000000000000p+0, 0x1.059b0d3158574p+0, 0x1.0b5586cf9890fp+0, 0x1.11301d0125b51p+0,
    0x1.172b83c7d517bp+0, 0x1.1d4873168b9aap+0, 0x1.2387a6e756238p+0, 0x1.29e9df51fdee1p+0,
    0x1.306fe0a31b715p+0, 0x1.371a7373aa9cbp+0, 0x1.3dea64c123422p+0, 0x1.44e086061892dp+0,
    0x1.4bfdad5362a27p+0, 0x1.5342b569d4f82p+0, 0x1.5ab07dd485429p+0, 0x1.6247eb03a5585p+0,
    0x1.6a09e667f3bcdp+0, 0x1.71f75e8ec5f74p+0, 0x1.7a11473eb0187p+0, 0x1.82589994cce13p+0,
    0x1.8ace5422aa0dbp+0, 0x1.93737b0cdc5e5p+0, 0x1.9c49182a3f090p+0, 0x1.a5503b23e255dp+0,
    0x1.ae89f995ad3adp+0, 0x1.b7f76f2fb5e47p+0, 0x1.c199bdd85529cp+0, 0x1.cb720dcef9069p+0,
    0x1.d5818dcfba487p+0, 0x1.dfc97337b9b5fp+0, 0x1.ea4afa2a490dap+0, 0x1.f50765b6e4540p+0,
};
__device__ __forceinline__ double exp_of(double x) {
  if (!(x > -708.0)) return 0.0;
  const double k = rint(x * 46.16624130844683);  // 32 / ln2
  double y = __builtin_fma(k, -0.021660849392446835, x);  // ln2 / 32: 36 bits, so that the product is exact
  y = __builtin_fma(k, -5.145609244655338e-14, y);  // ... and the rest
  const int i = (int)k;
  double e = __builtin_fma(y, 1.0 / 720.0, 1.0 / 120.0);
  e = __builtin_fma(y, e, 1.0 / 24.0);
  e = __builtin_fma(y, e, 1.0 / 6.0);
  e = __builtin_fma(y, e, 0.5);
  e = __builtin_fma(y, e, 1.0);
  const double root = kExp2Table[i & 31];
  return ldexp(__builtin_fma(root * y, e, root), i >> 5);
}

__device__ __forceinline__ double weight(const Row& r, uint32_t key) {
  if (key == r.top) return 1.0;
  if (key <= kMinusInf || r.best == INFINITY) return 0.0;
  return exp_of(((double)value_of(key) - r.best) * r.inv_t);
}

// The same as a call: code that runs once a row waits for its instructions to be
// fetched, and each inlined exponential is 200 bytes of them.
__device__ __attribute__((noinline)) double exp_call(double x) { return exp_of(x); }
__device__ __forceinline__ double weight_call(const Row& r, uint32_t key) {
  if (key == r.top) return 1.0;
  if (key <= kMinusInf || r.best == INFINITY) return 0.0;
  return exp_call(((double)value_of(key) - r.best) * r.inv_t);
}

__device__ __forceinline__ double last_lane(double v) {
  const uint64_t b = __builtin_bit_cast(uint64_t, v);
  const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)b, 63), hi = (uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), 63);
  return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ double wave_sum64(double v) { return last_lane(wave_scan(v)); }

// sum over the workgroup, in a fixed order; every thread gets it
__device__ double group_sum(double v, double* red) {
  v = wave_sum64(v);
  __syncthreads();
  if (lane_id() == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int i = 0; i < kThreads / kWave; ++i) s += red[i];
  return s;
}

// The first index whose running sum of f(key, index) exceeds `target`; if the
// rounding of the sums leaves none, the last index with f > 0; -1 if there is none.
// total: set to the sum over all.
template <class F>
__device__ int64_t walk(const Row& r, double u, bool share, F f, double* sums, double* red, int64_t* found, double* total) {
  const int n_blocks = (int)((r.n + kBlock - 1) / kBlock);
  uint32_t k[kVec];
  for (int b = 0; b < n_blocks; ++b) {
    const int64_t i = (int64_t)b * kBlock + threadIdx.x * kVec;
    keys8(r, i, k);
    double s = 0.0;
    for (int e = 0; e < kVec; ++e) s += i + e < r.n ? f(k[e], i + e) : 0.0;
    s = group_sum(s, red);
    if (threadIdx.x == 0) sums[b] = s;
  }
  __syncthreads();
  double all = 0.0;
  for (int b = 0; b < n_blocks; ++b) all += sums[b];
  *total = all;
  const double target = share ? u * all : u;
  int at = -1;
  double before = 0.0, run = 0.0;
  for (int b = 0; b < n_blocks; ++b) {
    if (sums[b] > 0.0) {
      at = b;
      before = run;
    }
    run += sums[b];
    if (run > target && sums[b] > 0.0) break;
  }
  if (at < 0) return -1;
  // within the block: each thread's sum, the sums of the threads before it
  const int64_t i = (int64_t)at * kBlock + threadIdx.x * kVec;
  keys8(r, i, k);
  double own = 0.0;
  for (int e = 0; e < kVec; ++e) own += i + e < r.n ? f(k[e], i + e) : 0.0;
  const double scan = wave_scan(own);
  __syncthreads();
  if (lane_id() == kWave - 1) red[threadIdx.x >> 6] = scan;
  if (threadIdx.x == 0) found[0] = INT64_MAX, found[1] = -1;
  __syncthreads();
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += red[w];
  double c = before + (scan - own);
  for (int e = 0; e < kVec; ++e) {
    const double v = i + e < r.n ? f(k[e], i + e) : 0.0;
    c += v;
    if (v > 0.0) {
      if (c > target) {
        atomicMin((unsigned long long*)&found[0], (unsigned long long)(i + e));
        break;
      }
      atomicMax((long long*)&found[1], (long long)(i + e));
    }
  }
  __syncthreads();
  return found[0] != INT64_MAX ? found[0] : found[1];
}

// Sums of weights that do not depend on the order: hi + lo / unit in units of 1 / unit, a
// power of two with which all n weights of a row stay below 2^63, so that a weight counts
// down to 1 / unit^2 (2^-76 of 2^24 logits, 2^-88 of 262144).
struct Sum2 {
  unsigned long long hi, lo;  // lo < unit
};
__device__ __forceinline__ void add2(Sum2& a, unsigned long long hi, unsigned long long lo, int bits) {
  lo += a.lo;
  a.hi += hi + (lo >> bits);
  a.lo = lo & ((1ull << bits) - 1);
}
// x >= 0 as such a sum, its last part rounded by `round`
template <class R>
__device__ __forceinline__ void split2(double x, double unit, R round, unsigned long long* hi, unsigned long long* lo) {
  const double h = floor(x * unit);
  *hi = (unsigned long long)h;
  *lo = (unsigned long long)round((x * unit - h) * unit);
}

// Digit by digit, the key of the logit at which the running sum of f(key) over the
// descending order reaches `goal`; *above: the sum of the larger keys.  unit: 2^bits.
template <class F>
__device__ uint32_t select(const Row& r, double goal, F f, unsigned long long (*hist)[2], uint32_t* pick, int bits, double* above) {
  uint32_t prefix = 0;
  const double unit = ldexp(1.0, bits);
  Sum2 over = {0, 0}, want = {0, 0};
  unsigned long long hi, lo;
  split2(goal, unit, [](double x) { return ceil(x); }, &hi, &lo);
  add2(want, hi, lo, bits);
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (threadIdx.x < 256) hist[threadIdx.x][0] = hist[threadIdx.x][1] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x * kVec; i < r.n; i += kBlock) {
      uint32_t ks[kVec];
      keys8(r, i, ks);
      for (int e = 0; e < kVec; ++e) {
        const uint32_t k = ks[e];
        if (i + e < r.n && (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8)))) {
          split2(f(k), unit, [](double x) { return rint(x); }, &hi, &lo);
          if (hi) atomicAdd(&hist[(k >> shift) & 255][0], hi);
          if (lo) atomicAdd(&hist[(k >> shift) & 255][1], lo);
        }
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      Sum2 run = over, at = over;
      int last = -1;
      for (int b = 255; b >= 0; --b) {
        if (!(hist[b][0] | hist[b][1])) continue;
        last = b;
        at = run;
        add2(run, hist[b][0], hist[b][1], bits);
        if (run.hi > want.hi || (run.hi == want.hi && run.lo >= want.lo)) break;
      }
      pick[0] = (uint32_t)max(last, 0);
      hist[256][0] = at.hi;
      hist[256][1] = at.lo;
    }
    __syncthreads();
    prefix |= pick[0] << shift;
    over = {hist[256][0], hist[256][1]};
  }
  *above = ((double)over.hi + (double)over.lo / unit) / unit;
  return prefix;
}

// LDS of the passes over a row
struct PassLds {
  double sums[kMaxBlocks];
  double red[kThreads / kWave];
  unsigned long long hist[257][2];
  int64_t found[2];
  uint32_t pick[1], tops[kThreads / kWave];
};

struct RowArgs {
  float t, top_p, min_p, u;
  int top_k;
  bool greedy, k_on, p_on;  // which limits apply
  double least;             // smallest weight kept
};
__device__ __forceinline__ RowArgs row_args(const SampleParams& p, int64_t row) {
  RowArgs a;
  a.t = p.temperature ? p.temperature[row] : p.temperature_all;
  a.top_k = p.top_k ? p.top_k[row] : p.top_k_all;
  a.top_p = p.top_p ? p.top_p[row] : p.top_p_all;
  a.min_p = p.min_p ? p.min_p[row] : p.min_p_all;
  a.u = p.u[row] > 0.0f ? p.u[row] : 0.0f;  // NaN: 0
  a.greedy = !(a.t > 0.0f);
  a.k_on = !a.greedy && a.top_k > 0 && a.top_k < p.n;
  a.p_on = !a.greedy && a.top_p < 1.0f;
  a.least = !a.greedy && a.min_p > 0.0f ? fmin((double)a.min_p, 1.0) : 0.0;
  return a;
}
__device__ __forceinline__ Row row_of(const SampleParams& p, int64_t row, bool bf) {
  Row r;
  r.bf = bf;
  r.n = p.n;
  r.base = bf ? (const void*)(reinterpret_cast<const uint16_t*>(p.logits) + row * p.ld)
              : (const void*)(reinterpret_cast<const float*>(p.logits) + row * p.ld);
  return r;
}

// A row in passes over it, by a workgroup of kThreads.
__device__ void draw_in_passes(const SampleParams& p, int64_t row, Row r, const RowArgs& a, int bits, PassLds& s) {
  uint32_t top = 0;
  for (int64_t i = threadIdx.x * kVec; i < r.n; i += kBlock) {
    uint32_t k[kVec];
    keys8(r, i, k);
    for (int e = 0; e < kVec; ++e) top = max(top, k[e]);
  }
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  __syncthreads();
  if (lane_id() == 0) s.tops[threadIdx.x >> 6] = top;
  __syncthreads();
  for (int i = 0; i < kThreads / kWave; ++i) top = max(top, s.tops[i]);
  r.top = top;
  r.best = (double)value_of(top);
  r.inv_t = 1.0 / (double)a.t;
  if (top <= kMinusInf) {  // nothing to draw from
    if (threadIdx.x == 0) {
      p.token[row] = -1;
      if (p.prob) p.prob[row] = 0.0f;
    }
    return;
  }
  // the kept prefix: keys above thr, and thr itself up to index cut
  uint32_t thr = a.greedy ? top : 0;
  int64_t cut = INT64_MAX;
  double ties = a.greedy ? 1.0 : 0.0, total;
  if (a.k_on) {
    double above;
    thr = select(r, (double)a.top_k, [](uint32_t) { return 1.0; }, s.hist, s.pick, 0, &above);
    ties = (double)a.top_k - above;
  }
  if (a.p_on) {
    const uint32_t floor_key = thr;
    const double floor_ties = ties;
    double z = 0.0;
    for (int64_t i = threadIdx.x * kVec; i < r.n; i += kBlock) {
      uint32_t k[kVec];
      keys8(r, i, k);
      for (int e = 0; e < kVec; ++e)
        if (i + e < r.n && (floor_ties == 0.0 || k[e] > floor_key)) z += weight_call(r, k[e]);
    }
    z = group_sum(z, s.red);
    if (floor_ties > 0.0) z += floor_ties * weight_call(r, floor_key);
    const double goal = (double)fmaxf(a.top_p, 0.0f) * z;
    double above;
    thr = select(r, goal, [&](uint32_t k) { return k >= floor_key ? weight_call(r, k) : 0.0; }, s.hist, s.pick, bits, &above);
    const double w = weight_call(r, thr);
    ties = w > 0.0 ? fmax(1.0, ceil((goal - above) / w)) : (double)r.n;
    if (floor_ties > 0.0 && thr == floor_key) ties = fmin(ties, floor_ties);
  }
  if (ties > 0.0)
    cut = walk(r, ties - 0.5, false, [&](uint32_t k, int64_t) { return k == thr ? 1.0 : 0.0; }, s.sums, s.red, s.found, &total);
  const int64_t token = walk(r, (double)a.u, true, [&](uint32_t k, int64_t i) {
    if (k < thr || (k == thr && i > cut)) return 0.0;
    if (a.greedy) return 1.0;
    const double w = weight_call(r, k);
    return w < a.least ? 0.0 : w; }, s.sums, s.red, s.found, &total);
  if (threadIdx.x == 0) {
    p.token[row] = token;
    if (p.prob) p.prob[row] = (float)((a.greedy ? 1.0 : weight_call(r, key_at(r, token))) / total);
  }
}

// ------------------------------------------------------------------ bins

constexpr int kChunk = 16384;
constexpr int kBins = 2048;      // from the largest logit down; the last one: all others
constexpr int kBand = 32;        // bins on either side of 0, kBand / 256 = 1/8 wide
constexpr uint32_t kBandBits = 0x3e00;  // upper 16 bits of 1/8
constexpr int kMaxChunks = kSampleMaxVocab / kChunk;
constexpr int kScanThreads = 512;
constexpr int kList = 2048;      // logits of one bin that are sorted

// value of a key's upper 16 bits
__device__ __forceinline__ float value16(uint32_t k16) {
  return bf16_bits_to_float(k16 & 0x8000u ? k16 & 0x7fffu : ~k16 & 0xffffu);
}
// A key's place in the order of bins: 0 .. 31 and -1 .. -32 in the band, one for
// each value of the upper 16 bits above and below it.
__device__ __forceinline__ int place_of(uint32_t key) {
  const uint32_t k16 = key >> 16;
  const bool neg = !(k16 & 0x8000u);
  const uint32_t mag = neg ? 0x7fffu - k16 : k16 - 0x8000u;
  const int x = mag >= kBandBits ? (int)(mag - kBandBits) + kBand : (int)(bf16_bits_to_float(mag) * 256.0f);
  return neg ? -1 - x : x;
}
__device__ __forceinline__ bool in_band(int place) { return place < kBand && place >= -kBand; }
// upper 16 bits of a place outside the band; 0 where there is no such value
__device__ __forceinline__ uint32_t key16_at(int place) {
  const int x = place < 0 ? -1 - place : place;
  const uint32_t mag = (uint32_t)(x - kBand) + kBandBits;
  return mag > 0x7f80u ? 0u : place < 0 ? 0x7fffu - mag : 0x8000u + mag;
}
// the smallest key of a place
__device__ __forceinline__ uint32_t first_key(int place) {
  if (!in_band(place)) return key16_at(place) << 16;
  return key_of((float)place * (1.0f / 256.0f));  // -(x + 1) / 256 for place -1 - x
}

// Per row and chunk in the workspace.
struct ChunkWs {
  unsigned long long* fix;  // [rows][chunks][fixed] weights in 2^-48 of the chunk's largest:
                            // of the band's bins (bf16) or of all (f32)
  double* tail;             // [rows][chunks] weights of the last bin, relative to the chunk's largest
  uint16_t* count;          // [rows][chunks][kBins]
  uint32_t* top;            // [rows][chunks] the largest logit's key
  int chunks, fixed;
};
ChunkWs chunk_ws(void* ws, int64_t rows, int64_t n, bool bf) {
  ChunkWs w;
  w.chunks = (int)((n + kChunk - 1) / kChunk);
  w.fixed = bf ? 2 * kBand : kBins;
  const int64_t all = rows * w.chunks;
  w.fix = reinterpret_cast<unsigned long long*>(ws);
  w.tail = reinterpret_cast<double*>(w.fix + all * w.fixed);
  w.count = reinterpret_cast<uint16_t*>(w.tail + all);
  w.top = reinterpret_cast<uint32_t*>(w.count + all * kBins);
  return w;
}
constexpr double kFix = 281474976710656.0;  // 2^48: 2^14 weights up to 1 stay below 2^62

__device__ __forceinline__ uint32_t wave_top(uint32_t top) {
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  return top;
}
// what the weights below the bins matter for
__device__ __forceinline__ bool needs_tail(const RowArgs& a) {
  return !a.greedy && !a.k_on && (a.p_on || a.least == 0.0);
}

// Bits of a logit: 0 .. 0x7fff upper bits of its magnitude, and its sign (not of 0).
// The bin's place as place_of gives it.
__device__ __forceinline__ int place_of_bits(uint32_t b16) {
  const uint32_t mag = b16 & 0x7fffu;
  const int x = mag >= kBandBits ? (int)mag - (int)(kBandBits - kBand) : (int)(bf16_bits_to_float(mag) * 256.0f);
  return b16 > 0x8000u ? ~x : x;
}

// Logits of a thread: V vectors of eight, kept as they come.
template <bool BF>
struct Vec;
template <>
struct Vec<true> {
  Four a;
  __device__ __forceinline__ uint32_t bits(int e) const {  // of the binary32 value
    return e & 1 ? a[e >> 1] & 0xffff0000u : a[e >> 1] << 16;
  }
  __device__ __forceinline__ void load(const Row& r, int64_t i) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(r.base) + i;
    if (i + 8 <= r.n) {
      a = *reinterpret_cast<const Four16*>(p);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)  // NaN behind the row
        a[e] = (i + 2 * e < r.n ? p[2 * e] : 0x7fffu) | ((i + 2 * e + 1 < r.n ? p[2 * e + 1] : 0x7fffu) << 16);
    }
  }
};
template <>
struct Vec<false> {
  Four a, b;
  __device__ __forceinline__ uint32_t bits(int e) const { return e < 4 ? a[e] : b[e - 4]; }
  __device__ __forceinline__ void load(const Row& r, int64_t i) {
    const float* p = reinterpret_cast<const float*>(r.base) + i;
    if (i + 8 <= r.n) {
      a = reinterpret_cast<const Four32*>(p)[0];
      b = reinterpret_cast<const Four32*>(p)[1];
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) (e < 4 ? a : b)[e & 3] = __float_as_uint(i + e < r.n ? p[e] : NAN);
    }
  }
};

// registers: four workgroups a CU for f32 (all of 131 x 100003 logits at once); bf16 spills with
// as few, and 64 x 262144 logits took 28 us where they took 25 with more
template <bool BF>
__global__ __launch_bounds__(kScanThreads, BF ? 4 : 8) void sample_scan_kernel(SampleParams p, ChunkWs ws) {
  constexpr int V = kChunk / kScanThreads / kVec, kFixed = BF ? 2 * kBand : kBins;
  static_assert(V * kVec == 32, "a bit of a word for each logit of a thread");
  __shared__ uint32_t hist[kBins];
  __shared__ unsigned long long fix[kFixed];
  __shared__ float tops[kScanThreads / kWave];
  __shared__ double red[kScanThreads / kWave];
  const int64_t row = blockIdx.y, at = row * ws.chunks + blockIdx.x;
  Row r = row_of(p, row, BF);
  const int64_t i0 = (int64_t)blockIdx.x * kChunk + threadIdx.x * kVec;
  Vec<BF> x[V];
#pragma unroll
  for (int v = 0; v < V; ++v) x[v].load(r, i0 + v * kScanThreads * kVec);
  const RowArgs a = row_args(p, row);
  for (int i = threadIdx.x; i < kBins; i += kScanThreads) hist[i] = 0;
  for (int i = threadIdx.x; i < kFixed; i += kScanThreads) fix[i] = 0;
  float top = NAN;  // of numbers; NaN where there is none
  bool nan = false;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < kVec; e += 2) {
      const float f0 = __uint_as_float(x[v].bits(e)), f1 = __uint_as_float(x[v].bits(e + 1));
      nan |= __builtin_isunordered(f0, f1);
      top = fmaxf(fmaxf(top, f0), f1);
    }
  if (__any(nan)) {  // the maximum of a number and a signalling NaN is NaN: numbers alone
    top = NAN;
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        const float f = __uint_as_float(x[v].bits(e));
        top = f == f ? fmaxf(top, f) : top;
      }
  }
  for (int m = 32; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
  if (lane_id() == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kScanThreads / kWave; ++i) top = fmaxf(top, tops[i]);
  r.top = key_of(top);
  const bool live = !a.greedy && r.top > kMinusInf, tail = live && needs_tail(a);
  r.best = (double)top;
  r.inv_t = 1.0 / (double)a.t;
  const int first = place_of(r.top);
  // Weights that can matter: of logits in bins of several values, and below the
  // bins; a logit below min_p of the chunk's largest is below it of the row's, and
  // no sum needs it where there is no top_p.
  float least = -INFINITY;
  if (a.least > 0.0 && !a.p_on) {
    least = (float)((double)top + (double)a.t * log(a.least));
    least -= fabsf(least) * 1e-6f + fabsf(top) * 1e-6f;  // above any rounding of the two
    if (!(fabsf(least) < INFINITY)) least = -INFINITY;
  }
  const bool all = !BF && live && least == -INFINITY;  // every f32 weight, where it stands
  double rest = 0.0;
  auto add = [&](uint32_t key, int place) {
    const int d = first - place;
    const double w = weight(r, key);
    if (d < kBins - 1)
      atomicAdd(&fix[BF ? place + kBand : d], (unsigned long long)rint(w * kFix));
    else
      rest += w;
  };
  uint32_t todo = 0;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const uint32_t b = x[v].bits(e), b16 = BF || b != 0x80000000u ? b >> 16 : 0u;
      const float f = __uint_as_float(b);
      // f32: -0 is 0, and another value with upper bits 0x8000 lies below it
      const int place = BF || b <= 0x80000000u || b16 != 0x8000u ? place_of_bits(b16) : -1, d = first - place;
      const bool number = f == f, in = number && d < kBins - 1;
      if (in) atomicAdd(&hist[d], 1u);
      if (in ? (!BF || in_band(place)) && f >= least : number && tail) {
        if (all)
          add(key_of(f), place);
        else
          todo |= 1u << (8 * v + e);
      }
    }
  if (!live) todo = 0;
  // a few of a thread's bf16 logits: those that any lane has, one at a time (in
  // the loop above each would cost the whole wave its exponential)
  while (todo) {
    const int bit = __builtin_ctz(todo);
    todo &= todo - 1;
    const uint32_t key = key_at(r, i0 + (bit >> 3) * (kScanThreads * kVec) + (bit & 7));
    add(key, place_of(key));
  }
  rest = wave_sum64(rest);
  if (lane_id() == 0) red[threadIdx.x >> 6] = rest;
  __syncthreads();
  uint32_t* out = reinterpret_cast<uint32_t*>(ws.count + at * kBins);
  for (int i = threadIdx.x; i < kBins / 2; i += kScanThreads) out[i] = hist[2 * i] | (hist[2 * i + 1] << 16);
  for (int i = threadIdx.x; i < kFixed; i += kScanThreads) ws.fix[at * kFixed + i] = fix[i];
  if (threadIdx.x == 0) {
    ws.top[at] = r.top;
    double s = 0.0;
    for (int i = 0; i < kScanThreads / kWave; ++i) s += red[i];
    ws.tail[at] = s;
  }
}

// inclusive scan over the workgroup, thread order; red: one entry a wave
template <class T>
__device__ T group_scan(T v, T* red) {
  v = wave_scan(v);
  __syncthreads();
  if (lane_id() == kWave - 1) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T before = 0;
#pragma unroll
  for (int w = 0; w < kThreads / kWave - 1; ++w) before += w < (int)(threadIdx.x >> 6) ? red[w] : T(0);  // all reads at once
  return before + v;
}

struct DrawLds {
  union {
    double w[kBins];            // weight of a logit of each bin that is one value
    uint32_t n_bin[kBins];      // before it: the row's counts
  };
  double sum[kMaxChunks];       // kept weight of each chunk
  double scale[kMaxChunks];     // weight of its largest logit
  int off[kMaxChunks];          // bins from the row's largest logit to the chunk's
  int ties[kMaxChunks];         // kept logits of the prefix's last bin
  union {
    unsigned long long list[kList];  // a bin's logits, ~key and index: ascending is the order of the prefix
    unsigned long long f_bin[kBins]; // before it: the row's weights, in 1 / unit of its largest
  };
  double redd[kThreads / kWave], at, goal, target, total;
  uint32_t redu[kThreads / kWave];
  int bin, n, found, last, chunk;
};
union DrawUnion {
  DrawLds d;
  PassLds p;
};

// The m logits of bin b of a row into s.list, in order.  A call, like exp_call:
// five places need it, none of them in every row.  One workgroup reads the row, and
// what it does for each logit bounds that (48 us of 262144 when it formed the bin of
// each), so a logit's bits are compared with the range that the bin is of them.
template <bool BF>
__device__ __attribute__((noinline)) void gather_bin(const Row& r, DrawLds& s, const uint16_t* count, int C, int first, int b, uint32_t m) {
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6;
  constexpr int kWaves = kThreads / kWave, kParts = 8;  // parts of a chunk, so that few chunks occupy all waves
  constexpr int kLoads = kChunk / kParts / (kWave * kVec);
  // the bin's magnitudes, upper 16 bits: [m0, m1); of the infinities no NaN
  const int place = first - b, x = place < 0 ? ~place : place;
  const uint32_t m0 = x < kBand ? __float_as_uint((float)x * (1.0f / 256.0f)) >> 16 : (uint32_t)(x - kBand) + kBandBits;
  const uint32_t m1 = x < kBand ? __float_as_uint((float)(x + 1) * (1.0f / 256.0f)) >> 16 : m0 + 1;
  const uint32_t sign = place < 0 ? 0x80000000u : 0u;
  const uint32_t lo = sign | (m0 << 16) | (place == -1 ? 1u : 0u);  // -0 is 0, of place 0
  const uint32_t span = m0 == 0x7f80u ? 1u : (sign | (m1 << 16)) - lo;
  const bool zero = place == 0;
  __syncthreads();
  if (tid == 0) s.n = 0;
  for (int i = tid; i < kList; i += kThreads) s.list[i] = ~0ull;
  __syncthreads();
  for (int cp = wave; cp < C * kParts; cp += kWaves) {
    const int c = cp / kParts, d = b - s.off[c];
    if (d < 0 || !count[(int64_t)c * kBins + d]) continue;
    const int64_t at0 = (int64_t)c * kChunk + (cp % kParts) * (kChunk / kParts) + lane * kVec;
    Vec<BF> y[kLoads];
#pragma unroll
    for (int v = 0; v < kLoads; ++v) y[v].load(r, at0 + v * kWave * kVec);  // NaN behind the row
#pragma unroll
    for (int v = 0; v < kLoads; ++v) {
      uint32_t hits = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) hits |= y[v].bits(e) - lo < span ? 1u << e : 0u;
      if (zero) {
#pragma unroll
        for (int e = 0; e < kVec; ++e) hits |= y[v].bits(e) == 0x80000000u ? 1u << e : 0u;
      }
      if (hits) {
        int at = atomicAdd(&s.n, __popc(hits));
        do {
          const int e = __builtin_ctz(hits);
          hits &= hits - 1;
          uint32_t bits = y[v].bits(0);
#pragma unroll
          for (int f = 1; f < kVec; ++f) bits = e == f ? y[v].bits(f) : bits;
          if (at < kList)
            s.list[at] = ((unsigned long long)~key_of(__uint_as_float(bits)) << 32) | (unsigned long long)(at0 + v * kWave * kVec + e);
          ++at;
        } while (hits);
      }
    }
  }
  __syncthreads();
  int size = 2;
  while (size < (int)m) size *= 2;
  for (int len = 2; len <= size; len *= 2)
    for (int step = len / 2; step >= 1; step /= 2) {
      if (tid < size / 2) {
        const int i = 2 * tid - (tid & (step - 1)), j = i + step;
        const unsigned long long x = s.list[i], y = s.list[j];
        if ((x > y) == ((i & len) == 0)) {
          s.list[i] = y;
          s.list[j] = x;
        }
      }
      // the 64 pairs of a wave are of 128 neighbours where step <= 64, and a wave's LDS accesses
      // are in order: 10 of 66 steps of 2048 logits need the workgroup's barrier
      if (max(step, step > 1 ? step / 2 : len) > kWave) {
        __syncthreads();
      } else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
      }
    }
  __syncthreads();
}

template <bool BF>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleParams p, ChunkWs ws, int bits) {
  constexpr int kFixed = BF ? 2 * kBand : kBins;
  static_assert(kBins == 2 * kThreads && kList == 2 * kThreads && kChunk == 16 * kThreads, "a thread has two bins");
  __shared__ DrawUnion lds;
  DrawLds& s = lds.d;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, lane = lane_id(), wave = tid >> 6, C = ws.chunks;
  const double unit = ldexp(1.0, bits);
  constexpr int kWaves = kThreads / kWave;
  const uint32_t* tops = ws.top + row * C;
  const uint16_t* count = ws.count + row * C * kBins;
  const unsigned long long* fix = ws.fix + row * C * kFixed;
  // counts of chunk c, those of bins below `end`: a lane has pairs 64 apart
  constexpr int kPairs = kBins / (2 * kWave);
  auto load_counts = [&](int c, int end, uint32_t(&v)[kPairs]) {
    const uint32_t* src = reinterpret_cast<const uint32_t*>(count + (int64_t)c * kBins) + lane;
#pragma unroll
    for (int i = 0; i < kPairs; ++i) v[i] = 2 * kWave * i < end ? src[kWave * i] : 0u;
  };
  // f32: the weights of kAhead pairs of them, all loads before the first use (3 of
  // 90 us of 131 rows of 100003)
  constexpr int kAhead = 8;
  auto load_fixed = [&](int c, int i0, int end, ulonglong2(&v)[kAhead]) {
    const ulonglong2* src = reinterpret_cast<const ulonglong2*>(fix + (int64_t)c * kFixed) + lane;
#pragma unroll
    for (int i = 0; i < kAhead; ++i) v[i] = 2 * kWave * (i0 + i) < end ? src[kWave * (i0 + i)] : ulonglong2{0, 0};
  };
  uint32_t q[kPairs];
  if (wave < C) load_counts(wave, kBins, q);
  const RowArgs a = row_args(p, row);
  Row r = row_of(p, row, BF);
  uint32_t top = 0;
  for (int c = tid; c < C; c += kThreads) top = max(top, tops[c]);
  top = wave_top(top);
  if (lane == 0) s.redu[wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kWaves; ++i) top = max(top, s.redu[i]);
  if (top <= kMinusInf) {
    if (tid == 0) {
      p.token[row] = -1;
      if (p.prob) p.prob[row] = 0.0f;
    }
    return;
  }
  r.top = top;
  r.best = (double)value_of(top);
  r.inv_t = 1.0 / (double)a.t;
  const int first = place_of(top);
  for (int c = tid; c < C; c += kThreads) {
    s.off[c] = first - place_of(tops[c]);
    s.scale[c] = a.greedy ? 0.0 : weight_call(r, tops[c]) / kFix;
  }
  __syncthreads();
  // a logit's weight in bin b where the bin is one value; the bin's sum in chunk c otherwise
  auto one_value = [&](int b) { return BF && !in_band(first - b); };
  auto value_weight = [&](int b) {
    const uint32_t k16 = key16_at(first - b);
    return a.greedy || !k16 ? 0.0 : weight_call(r, k16 & 0x8000u ? k16 << 16 : (k16 << 16) | 0xffffu);
  };
  auto fixed_sum = [&](int c, int b) {
    return (double)fix[(int64_t)c * kFixed + (BF ? first - b + kBand : b - s.off[c])] * s.scale[c];
  };
  // ---- the row's bins: a wave a chunk, its counts two at a time (lanes two apart in LDS)
  for (int b = tid; b < kBins; b += kThreads) s.n_bin[b] = 0;
  for (int b = tid; b < kFixed; b += kThreads) s.f_bin[b] = 0;
  __syncthreads();
  for (int c = wave; c < C; c += kWaves) {
    const int off = s.off[c];
    const double scale = s.scale[c] * unit;
    if (c != wave) load_counts(c, kBins, q);
    if constexpr (BF) {
      const unsigned long long f = fix[(int64_t)c * kFixed + lane];
      if (f) atomicAdd(&s.f_bin[lane], (unsigned long long)rint((double)f * scale));
    }
#pragma unroll
    for (int i0 = 0; i0 < kPairs; i0 += kAhead) {
      ulonglong2 f[kAhead];
      if constexpr (!BF) load_fixed(c, i0, kBins, f);
#pragma unroll
      for (int i = i0; i < i0 + kAhead; ++i) {
        const int b = 2 * (kWave * i + lane) + off;
        const uint32_t m0 = q[i] & 0xffffu, m1 = q[i] >> 16;
        if (m0 && b < kBins - 1) atomicAdd(&s.n_bin[b], m0);
        if (m1 && b + 1 < kBins - 1) atomicAdd(&s.n_bin[b + 1], m1);
        if constexpr (!BF) {
          if (f[i - i0].x && b < kBins - 1) atomicAdd(&s.f_bin[b], (unsigned long long)rint((double)f[i - i0].x * scale));
          if (f[i - i0].y && b + 1 < kBins - 1) atomicAdd(&s.f_bin[b + 1], (unsigned long long)rint((double)f[i - i0].y * scale));
        }
      }
    }
  }
  __syncthreads();
  // ---- bins 2 tid, 2 tid + 1: counts, weights, running sums before them
  const int b0 = 2 * tid;
  uint32_t n[2];
  double w[2], sum[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int b = b0 + j;
    n[j] = s.n_bin[b];
    w[j] = n[j] && one_value(b) ? value_weight(b) : 0.0;
    sum[j] = !n[j] ? 0.0 : one_value(b) ? (double)n[j] * w[j] : (double)s.f_bin[BF ? first - b + kBand : b] / unit;
  }
  __syncthreads();  // s.w is where the counts are
  s.w[b0] = w[0];
  s.w[b0 + 1] = w[1];
  uint32_t n_before[2];
  double s_before[2];
  n_before[0] = group_scan(n[0] + n[1], s.redu) - (n[0] + n[1]);
  n_before[1] = n_before[0] + n[0];
  s_before[0] = group_scan(sum[0] + sum[1], s.redd) - (sum[0] + sum[1]);
  s_before[1] = s_before[0] + sum[0];
  // ---- weights below the bins, by chunk (a wave a chunk)
  double below = 0.0;
  if (needs_tail(a)) {
    for (int c = wave; c < C; c += kWaves) {
      const int off = s.off[c];
      double x = 0.0;
      for (int d = max(0, kBins - 1 - off) + lane; d < kBins - 1; d += kWave) {
        const uint32_t m = count[(int64_t)c * kBins + d];
        if (m) x += one_value(off + d) ? (double)m * value_weight(off + d) : fixed_sum(c, off + d);
      }
      x = wave_sum64(x);
      if (lane == 0) s.sum[c] = x + ws.tail[row * C + c] * (s.scale[c] * kFix);
    }
    __syncthreads();
    for (int c = 0; c < C; ++c) below += s.sum[c];
  }

  // ---- the kept prefix: all bins before `bin`, and the first `kept` logits of it
  int bin = kBins;        // kBins: everything, kBins - 1: everything in the bins
  uint32_t kept = 0, many = 0;  // many: all logits of the bin
  int listed = -1;        // the bin whose logits are in the list, in order
  bool lost = false;
  bool all_binned = false;  // known: nothing below the bins has any weight
  // the logits of bin b (m of them) into the list, in order
  auto gather = [&](int b, uint32_t m) {
    if (listed != b) gather_bin<BF>(r, s, count, C, first, b, m);
    listed = b;
  };
  auto list_weight = [&](int i) { return weight_call(r, ~(uint32_t)(s.list[i] >> 32)); };
  // the one bin `here` is true for becomes the prefix's last
  auto take = [&](bool here0, bool here1, uint32_t k0, uint32_t k1) {
    __syncthreads();
    if (tid == 0) s.bin = kBins;
    __syncthreads();
    if (here0 || here1) {
      const int j = here1 ? 1 : 0;
      s.bin = b0 + j;
      s.n = (int)(j ? k1 : k0);
      s.last = (int)n[j];
      s.at = s_before[j];
      s.goal = w[j];
    }
    __syncthreads();
    bin = s.bin;
    if (bin < kBins) {
      kept = (uint32_t)s.n;
      many = (uint32_t)s.last;
    }
  };
  if (a.greedy) {
    take(tid == 0, false, 1, 0);
    lost = !one_value(0) && many > kList;
    if (!lost && !one_value(0)) gather(0, many);
  }
  double at = 0.0, value = 0.0;  // weights before the bin; its value's
  if (a.k_on) {
    const uint32_t k = (uint32_t)a.top_k;
    take(n_before[0] < k && k <= n_before[0] + n[0], n_before[1] < k && k <= n_before[1] + n[1], k - n_before[0], k - n_before[1]);
    at = s.at;
    value = s.goal;
    if (bin == kBins) {
      // Fewer logits than top_k in the bins.  Where all others weigh nothing (a row of which a
      // grammar allows few tokens, the rest at -inf or at the type's lowest value), what is in the
      // bins is all that can be drawn, and the row needs no passes: 64 such rows of 262144 took
      // 1.1 ms with them, and take 0.11 with this look for the largest logit below the bins.
      const uint32_t edge = first_key(first - (kBins - 2));
      uint32_t next = 0;
      for (int64_t i = tid * kVec; i < r.n; i += kBlock) {
        uint32_t k8[kVec];
        keys8(r, i, k8);
#pragma unroll
        for (int e = 0; e < kVec; ++e) next = max(next, k8[e] < edge ? k8[e] : 0u);
      }
      next = wave_top(next);
      __syncthreads();
      if (lane == 0) s.redu[wave] = next;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWaves; ++i) next = max(next, s.redu[i]);
      lost = weight_call(r, next) > 0.0;
      all_binned = !lost;
    } else {
      lost = !one_value(bin) && kept < many && many > kList;
    }
  }
  if (a.p_on && !lost) {
    // what the tokens so far weigh
    const int last = bin;
    const uint32_t most = kept;
    double z;
    if (last == kBins) {
      __syncthreads();
      if (tid == kThreads - 1) s.total = s_before[1] + sum[1];
      __syncthreads();
      z = s.total + below;
    } else if (one_value(last)) {
      z = at + (double)kept * value;
    } else if (kept == many) {
      __syncthreads();
      if (tid == last / 2) s.total = s_before[last & 1] + sum[last & 1];
      __syncthreads();
      z = s.total;
    } else {
      gather(last, many);
      double x = 0.0;
      for (uint32_t i = tid; i < kept; i += kThreads) x += list_weight((int)i);
      z = at + group_sum(x, s.redd);
    }
    const double goal = (double)fmaxf(a.top_p, 0.0f) * z;
    // the last bin with a token before which the goal is not reached
    __syncthreads();
    if (tid == 0) s.bin = 0;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (n[j] && b0 + j <= last && s_before[j] < goal) atomicMax(&s.bin, b0 + j);
    __syncthreads();
    const int end = s.bin;
    if (last == kBins) lost = s.total < goal;  // not reached within the bins
    if (!lost) {
      take(b0 == end, b0 + 1 == end, n[0], n[1]);
      at = s.at;
      value = s.goal;
      const uint32_t limit = end == last ? most : many;
      if (one_value(end)) {
        kept = value > 0.0 ? (uint32_t)fmin(fmax(1.0, ceil((goal - at) / value)), (double)limit) : limit;
      } else if (many > kList) {
        lost = true;
      } else {
        gather(end, many);
        const double x0 = 2 * tid < (int)many ? list_weight(2 * tid) : 0.0, x1 = 2 * tid + 1 < (int)many ? list_weight(2 * tid + 1) : 0.0;
        const double upto = at + group_scan(x0 + x1, s.redd);
        uint32_t before = (2 * tid < (int)many && upto - x1 - x0 < goal) + (2 * tid + 1 < (int)many && upto - x1 < goal);
        before = group_scan(before, s.redu);
        __syncthreads();
        if (tid == kThreads - 1) s.n = (int)before;
        __syncthreads();
        kept = min(max((uint32_t)s.n, 1u), limit);
      }
    }
  }
  if (a.least > 0.0 && !lost) {
    // the first bin with a token below min_p
    __syncthreads();
    if (tid == 0) s.bin = kBins;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 2; ++j)
      if (n[j] && b0 + j <= bin && (one_value(b0 + j) ? w[j] : weight_call(r, first_key(first - b0 - j))) < a.least) atomicMin(&s.bin, b0 + j);
    __syncthreads();
    const int end = s.bin;
    if (end < kBins) {
      const uint32_t most = end == bin ? kept : ~0u;
      take(b0 == end, b0 + 1 == end, 0, 0);
      if (!one_value(end)) {
        lost = many > kList;
        if (!lost) {
          gather(end, many);
          uint32_t x = 0;
          for (uint32_t i = tid; i < many; i += kThreads) x += list_weight((int)i) >= a.least ? 1u : 0u;
          x = group_scan(x, s.redu);
          __syncthreads();
          if (tid == kThreads - 1) s.n = (int)x;
          __syncthreads();
          kept = min((uint32_t)s.n, most);
        }
      }
    } else if (bin == kBins) {  // logits below the bins may still be kept
      lost = !all_binned && weight_call(r, first_key(first - (kBins - 2))) >= a.least;
      bin = kBins - 1;
      kept = many = 0;
    }
  }
  if (all_binned && bin == kBins) bin = kBins - 1;
  if (!lost && bin < kBins - 1 && !one_value(bin) && kept > 0 && kept < many) {
    lost = many > kList;
    if (!lost) gather(bin, many);
  }
  if (lost) {
    __syncthreads();
    draw_in_passes(p, row, r, a, bits, lds.p);
    return;
  }

  // ---- kept weight of each chunk
  const bool single = bin < kBins - 1 && one_value(bin), whole = kept == many;
  const double tie_weight = a.greedy ? 1.0 : bin < kBins - 1 ? s.w[bin] : 0.0;
  __syncthreads();
  if (single && wave == 0) {  // of equal logits the lowest indexes
    uint32_t left = kept;
    for (int c0 = 0; c0 < C; c0 += kWave) {
      const int c = c0 + lane;
      const int d = c < C ? bin - s.off[c] : -1;
      const uint32_t m = d >= 0 ? count[(int64_t)c * kBins + d] : 0u;
      const uint32_t upto = wave_scan(m);
      const uint32_t before = upto - m;
      if (c < C) s.ties[c] = (int)min(m, left > before ? left - before : 0u);
      const uint32_t all = __shfl(upto, kWave - 1);
      left -= min(left, all);
    }
  }
  __syncthreads();
  for (int c = wave; c < C; c += kWaves) {
    const int off = s.off[c];
    double x = 0.0;
    const int end = a.greedy ? 0 : min(bin, kBins - 1) - off;
    if constexpr (BF) {
      load_counts(c, end, q);
      const int d = first - (lane - kBand) - off;  // the lane's bin of the band
      if (d >= 0 && d < end) x = fixed_sum(c, d + off);
#pragma unroll
      for (int i = 0; i < kPairs; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t m = e ? q[i] >> 16 : q[i] & 0xffffu;
          const int d = 2 * (kWave * i + lane) + e;
          if (m && d < end && one_value(d + off)) x += (double)m * s.w[d + off];
        }
    } else {
#pragma unroll
      for (int i0 = 0; i0 < kPairs; i0 += kAhead) {
        ulonglong2 f[kAhead];
        load_fixed(c, i0, end, f);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int d = 2 * (kWave * (i0 + i) + lane);
          if (d < end) x += (double)f[i].x * s.scale[c];
          if (d + 1 < end) x += (double)f[i].y * s.scale[c];
        }
      }
    }
    if (bin < kBins - 1 && kept > 0) {
      if (single) {
        if (lane == 0) x += (double)s.ties[c] * tie_weight;
      } else if (whole && !a.greedy) {
        if (lane == 0 && bin >= off) x += fixed_sum(c, bin);
      } else {
        for (uint32_t i = lane; i < kept; i += kWave)
          if ((int)((uint32_t)s.list[i] / kChunk) == c) x += a.greedy ? 1.0 : list_weight((int)i);
      }
    }
    x = wave_sum64(x);
    if (lane == 0) s.sum[c] = bin == kBins ? x + s.sum[c] : x;
  }
  __syncthreads();
  if (wave == 0) {  // its chunk, by running sums of 64 at a time
    double all = 0.0;
    for (int c0 = 0; c0 < C; c0 += kWave) {
      all += wave_sum64(c0 + lane < C ? s.sum[c0 + lane] : 0.0);
    }
    const double target = (double)a.u * all;
    double run = 0.0, before = 0.0;
    int at_c = 0;
    for (int c0 = 0; c0 < C; c0 += kWave) {
      const double own = c0 + lane < C ? s.sum[c0 + lane] : 0.0;
      const double v = wave_scan(own);
      const uint64_t some = __ballot(own > 0.0), past = __ballot(own > 0.0 && run + v > target);
      if (some) {  // the first one past the target, else the last one with any
        const int i = past ? __builtin_ctzll(past) : 63 - __builtin_clzll(some);
        at_c = c0 + i;
        before = run + (__shfl(v, i) - __shfl(own, i));
      }
      if (past) break;
      run += last_lane(v);
    }
    if (lane == 0) {
      s.total = all;
      s.chunk = at_c;
      s.target = target - before;
      s.found = kChunk;
      s.last = -1;
    }
  }
  __syncthreads();
  // ---- the token within its chunk: eight logits a thread, twice
  const int c = s.chunk;
  const unsigned long long cut = !single && kept > 0 && bin < kBins - 1 && !(whole && !a.greedy) ? s.list[kept - 1] : ~0ull;
  const uint32_t most = single ? (uint32_t)s.ties[c] : 0u;
  const double target = s.target, total = s.total;
  double before = 0.0, mine_x = 0.0;
  uint32_t ranked = 0;
  int64_t mine_i = 0;
#pragma unroll 1
  for (int h = 0; h < kChunk / kBlock; ++h) {
    const int64_t i0 = (int64_t)c * kChunk + h * kBlock + tid * kVec;
    uint32_t k[kVec], rank = ranked;
    keys8(r, i0, k);
    if (single) {
      uint32_t mine = 0;
#pragma unroll
      for (int e = 0; e < kVec; ++e) mine += k[e] && first - place_of(k[e]) == bin ? 1u : 0u;
      const uint32_t upto = group_scan(mine, s.redu);
      rank += upto - mine;
      if (tid == kThreads - 1) s.n = (int)(ranked + upto);
    }
    double x[kVec], own = 0.0;
    uint32_t todo = 0;  // logits that need an exponential: few of a bf16 row's, so one a lane at a time
#pragma unroll
    for (int e = 0; e < kVec; ++e) {
      const int b = min(first - place_of(k[e]), kBins - 1);  // the last one: all below the bins
      x[e] = 0.0;
      if (k[e] && b <= bin && (b < kBins - 1 || bin == kBins)) {
        if (b == bin && single) {
          x[e] = rank < most ? tie_weight : 0.0;
          ++rank;
        } else if (b < kBins - 1 && one_value(b)) {
          x[e] = a.greedy ? 0.0 : s.w[b];
        } else {
          const unsigned long long id = ((unsigned long long)~k[e] << 32) | (unsigned long long)(i0 + e);
          if (b < bin || (kept > 0 && id <= cut)) todo |= 1u << e;
        }
      }
    }
    while (todo) {
      const int bit = __builtin_ctz(todo);
      todo &= todo - 1;
      uint32_t key = k[0];
#pragma unroll
      for (int e = 1; e < kVec; ++e) key = bit == e ? k[e] : key;
      const double w1 = a.greedy ? 1.0 : weight_call(r, key);
#pragma unroll
      for (int e = 0; e < kVec; ++e) x[e] = bit == e ? w1 : x[e];
    }
#pragma unroll
    for (int e = 0; e < kVec; ++e) own += x[e];
    // The first thread whose running sum passes the target; where rounding leaves
    // none, the last one with a kept logit.
    const double upto = before + group_scan(own, s.redd);
    if (own > 0.0) {
      const uint64_t past = __ballot(upto > target), some = __ballot(true);  // one lane a wave has a say
      if (past ? lane == __builtin_ctzll(past) : lane == 63 - __builtin_clzll(some)) {
        if (past) atomicMin(&s.found, h * kThreads + tid);
        else atomicMax(&s.last, h * kThreads + tid);
        double run = upto - own;
        int hit = -1;
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          if (x[e] > 0.0 && (hit < 0 || !(run > target))) {
            hit = e;
            mine_x = x[e];
          }
          run += x[e];
        }
        mine_i = i0 + hit;
      }
    }
    if (tid == kThreads - 1) s.at = upto;
    __syncthreads();
    if (s.found < kChunk) break;
    before = s.at;
    ranked = single ? (uint32_t)s.n : 0u;
    __syncthreads();
  }
  const int who = s.found < kChunk ? s.found : s.last;
  if (who >= 0 && tid == who % kThreads) {
    p.token[row] = mine_i;
    if (p.prob) p.prob[row] = (float)(mine_x / total);
  }
}

template <bool BF>
hipError_t sample_launch(const SampleParams& p, void* ws, hipStream_t st) {
  int log2n = 0;
  while (((int64_t)1 << log2n) < p.n) ++log2n;
  const int bits = 62 - log2n;  // n weights up to 1 in units of 2^-bits stay below 2^63
  const ChunkWs w = chunk_ws(ws, p.rows, p.n, BF);
  sample_scan_kernel<BF><<<dim3((unsigned)w.chunks, (unsigned)p.rows), kScanThreads, 0, st>>>(p, w);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  sample_draw_kernel<BF><<<dim3((unsigned)p.rows), kThreads, 0, st>>>(p, w, bits);
  return hipGetLastError();
}

}  // namespace

size_t sample_ws_bytes(int64_t rows, int64_t n, bool bf16) {
  const int64_t all = rows * ((n + kChunk - 1) / kChunk);
  return (size_t)all * ((bf16 ? 2 * kBand : kBins) * sizeof(unsigned long long) + kBins * sizeof(uint16_t) +
                        sizeof(double) + sizeof(uint32_t));
}

hipError_t launch_sample(const SampleParams& p, bool bf16, void* ws, hipStream_t st) {
  return bf16 ? sample_launch<true>(p, ws, st) : sample_launch<false>(p, ws, st);
}

}  // namespace w8a8
