// The next token of each row of logits, from a given uniform number.
//
// With weights w_i = exp((l_i - max l) / T), the kept tokens are a prefix of the
// order by (logit descending, index ascending): of top_k tokens, then the
// shortest one whose weights reach top_p of theirs, then those of weight min_p
// and more (the first token always stays).  The token drawn is the first index
// whose running sum of kept weights exceeds u times their total.
//
// The weights and their sums are binary64: a running sum of 262144 binary32
// weights moves by about 1e-8 with the order of its terms, and as much of the
// draws would change.  A prefix is given by the key of its last logit (the
// logit's bits in an order-preserving form) and the index of its last tie.
//
// A row of bf16 logits has few distinct values near its largest one, so two
// launches suffice, the first of which reads every logit once: per chunk of 8192
// it counts the logits on each of the 1023 values up to the chunk's largest and
// adds up the weights of the rest.  The second launch, one workgroup a row,
// finds the kept prefix and the chunk that holds the drawn token from the counts
// alone (a value's weight times its count), and reads that chunk again.  Rows
// whose prefix ends below those values (and f32 rows) go through passes over
// the row instead.
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

struct Row {
  const void* base;
  int64_t n;
  bool bf, wide;  // wide: 16-byte loads
  uint32_t top;   // key of the largest logit
  double best, t;
};

__device__ __forceinline__ uint32_t key_at(const Row& r, int64_t i) {
  if (i >= r.n) return 0;
  return key_of(r.bf ? bf16_bits_to_float(reinterpret_cast<const uint16_t*>(r.base)[i])
                     : reinterpret_cast<const float*>(r.base)[i]);
}

__device__ __forceinline__ void keys8(const Row& r, int64_t i, uint32_t (&k)[kVec]) {
#pragma unroll
  for (int e = 0; e < kVec; ++e) k[e] = key_at(r, i + e);
}

__device__ __forceinline__ double weight(const Row& r, uint32_t key) {
  if (key == r.top) return 1.0;
  if (key <= kMinusInf || r.best == INFINITY) return 0.0;
  return exp(((double)value_of(key) - r.best) / r.t);
}

__device__ __forceinline__ double wave_sum64(double v) {
  for (int m = 32; m >= 1; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

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
  double scan = own;
  for (int m = 1; m < kWave; m <<= 1) {
    const double o = __shfl_up(scan, m);
    if (lane_id() >= m) scan += o;
  }
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

// Digit by digit, the key of the logit at which the running measure over the
// descending order reaches `goal`; *above: the measure of the larger keys.
template <class F>
__device__ uint32_t select(const Row& r, double goal, F f, unsigned long long* hist, uint32_t* pick, double unit, double* above) {
  uint32_t prefix = 0;
  unsigned long long over = 0;
  const unsigned long long want = (unsigned long long)ceil(goal * unit);
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (threadIdx.x < 256) hist[threadIdx.x] = 0;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < r.n; i += kThreads) {
      const uint32_t k = key_at(r, i);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) {
        const unsigned long long v = f(k);
        if (v) atomicAdd(&hist[(k >> shift) & 255], v);
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      unsigned long long run = over;
      int last = -1;
      unsigned long long at = over;
      for (int b = 255; b >= 0; --b) {
        if (!hist[b]) continue;
        last = b;
        at = run;
        run += hist[b];
        if (run >= want) break;
      }
      pick[0] = (uint32_t)max(last, 0);
      hist[256] = at;
    }
    __syncthreads();
    prefix |= pick[0] << shift;
    over = hist[256];
  }
  *above = (double)over;
  return prefix;
}

// LDS of the passes over a row
struct PassLds {
  double sums[kMaxBlocks];
  double red[kThreads / kWave];
  unsigned long long hist[257];
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
__device__ void draw_in_passes(const SampleParams& p, int64_t row, Row r, const RowArgs& a, double unit, PassLds& s) {
  uint32_t top = 0;
  for (int64_t i = threadIdx.x; i < r.n; i += kThreads) top = max(top, key_at(r, i));
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  __syncthreads();
  if (lane_id() == 0) s.tops[threadIdx.x >> 6] = top;
  __syncthreads();
  for (int i = 0; i < kThreads / kWave; ++i) top = max(top, s.tops[i]);
  r.top = top;
  r.best = (double)value_of(top);
  r.t = (double)a.t;
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
    thr = select(r, (double)a.top_k, [](uint32_t) { return 1ull; }, s.hist, s.pick, 1.0, &above);
    ties = (double)a.top_k - above;
  }
  if (a.p_on) {
    const uint32_t floor_key = thr;
    const double floor_ties = ties;
    double z = 0.0;
    for (int64_t i = threadIdx.x; i < r.n; i += kThreads) {
      const uint32_t k = key_at(r, i);
      if (floor_ties == 0.0 || k > floor_key) z += weight(r, k);
    }
    z = group_sum(z, s.red);
    if (floor_ties > 0.0) z += floor_ties * weight(r, floor_key);
    const double goal = (double)fmaxf(a.top_p, 0.0f) * z;
    double above;
    thr = select(r, goal, [&](uint32_t k) {
      return k >= floor_key ? (unsigned long long)rint(weight(r, k) * unit) : 0ull; }, s.hist, s.pick, unit, &above);
    const double w = weight(r, thr);
    ties = w > 0.0 ? fmax(1.0, ceil((goal - above / unit) / w)) : (double)r.n;
    if (floor_ties > 0.0 && thr == floor_key) ties = fmin(ties, floor_ties);
  }
  if (ties > 0.0)
    cut = walk(r, ties - 0.5, false, [&](uint32_t k, int64_t) { return k == thr ? 1.0 : 0.0; }, s.sums, s.red, s.found, &total);
  const int64_t token = walk(r, (double)a.u, true, [&](uint32_t k, int64_t i) {
    if (k < thr || (k == thr && i > cut)) return 0.0;
    if (a.greedy) return 1.0;
    const double w = weight(r, k);
    return w < a.least ? 0.0 : w; }, s.sums, s.red, s.found, &total);
  if (threadIdx.x == 0) {
    p.token[row] = token;
    if (p.prob) p.prob[row] = (float)((a.greedy ? 1.0 : weight(r, key_at(r, token))) / total);
  }
}

// ------------------------------------------------------------------ f32 rows

__global__ __launch_bounds__(kThreads) void sample_passes_kernel(SampleParams p, double unit) {
  __shared__ PassLds s;
  const int64_t row = blockIdx.x;
  draw_in_passes(p, row, row_of(p, row, false), row_args(p, row), unit, s);
}

// ------------------------------------------------------------------ bf16 rows

constexpr int kChunk = 8192;
constexpr int kBins = 1024;      // values below the largest; the last bin: all others
constexpr int kMaxChunks = kSampleMaxVocab / kChunk;
constexpr int kScanThreads = 256;

// Per row and chunk in the workspace.
struct ChunkWs {
  uint16_t* count;   // [rows][chunks][kBins]
  double* tail;      // [rows][chunks] weights of the last bin's logits, relative to the chunk's largest
  uint32_t* top;     // [rows][chunks] the largest logit's 16-bit key
  int chunks;
};
__host__ __device__ inline ChunkWs chunk_ws(void* ws, int64_t rows, int64_t n) {
  ChunkWs w;
  w.chunks = (int)((n + kChunk - 1) / kChunk);
  const int64_t all = rows * w.chunks;
  w.count = reinterpret_cast<uint16_t*>(ws);
  w.tail = reinterpret_cast<double*>(w.count + all * kBins);
  w.top = reinterpret_cast<uint32_t*>(w.tail + all);
  return w;
}

// the weight of value `key16` next to a largest logit `top16`
__device__ __forceinline__ double weight16(uint32_t key16, uint32_t top16, double best, double t) {
  if (key16 == top16) return 1.0;
  if (key16 <= (kMinusInf >> 16) || best == INFINITY) return 0.0;
  const uint32_t b = key16 & 0x8000u ? key16 & 0x7fffu : ~key16 & 0xffffu;
  return exp(((double)bf16_bits_to_float(b) - best) / t);
}
__device__ __forceinline__ float value16(uint32_t key16) {
  return bf16_bits_to_float(key16 & 0x8000u ? key16 & 0x7fffu : ~key16 & 0xffffu);
}
__device__ __forceinline__ uint32_t key16_of(uint32_t b) {
  if ((b & 0x7fffu) > 0x7f80u) return 0;       // NaN
  if (b == 0x8000u) b = 0;                     // -0
  return b & 0x8000u ? ~b & 0xffffu : b | 0x8000u;
}

// eight logits from index i on, as keys; 0 behind the row
__device__ __forceinline__ void keys16x8(const uint16_t* row, int64_t i, int64_t n, bool wide, uint32_t (&k)[8]) {
  if (wide && i + 8 <= n) {
    const uint4 r = *reinterpret_cast<const uint4*>(row + i);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = key16_of((w[e >> 1] >> (16 * (e & 1))) & 0xffffu);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = i + e < n ? key16_of(row[i + e]) : 0u;
  }
}

__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(SampleParams p, ChunkWs ws) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t tops[kScanThreads / kWave];
  __shared__ double red[kScanThreads / kWave];
  constexpr int V = kChunk / kScanThreads / 8;
  const int64_t row = blockIdx.y, at = row * ws.chunks + blockIdx.x;
  const uint16_t* base = reinterpret_cast<const uint16_t*>(p.logits) + row * p.ld;
  const bool wide = (reinterpret_cast<uintptr_t>(base) & 15u) == 0;
  const int64_t i0 = (int64_t)blockIdx.x * kChunk + threadIdx.x * 8;
  uint32_t k[V][8], top = 0;
#pragma unroll
  for (int v = 0; v < V; ++v) keys16x8(base, i0 + v * kScanThreads * 8, p.n, wide, k[v]);
  for (int i = threadIdx.x; i < kBins; i += kScanThreads) hist[i] = 0;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, k[v][e]);
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if (lane_id() == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kScanThreads / kWave; ++i) top = max(top, tops[i]);
  const RowArgs a = row_args(p, row);
  // the weights below the counted values matter where no count limits the prefix
  const bool tail = !a.greedy && !a.k_on && (a.p_on || a.least == 0.0) && top > (kMinusInf >> 16);
  const double best = (double)value16(top);
  double rest = 0.0;
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t d = top - k[v][e];
      if (d < kBins - 1) {
        if (k[v][e]) atomicAdd(&hist[d], 1u);
      } else if (tail) {
        rest += weight16(k[v][e], top, best, (double)a.t);
      }
    }
  rest = wave_sum64(rest);
  if (lane_id() == 0) red[threadIdx.x >> 6] = rest;
  __syncthreads();
  uint32_t* out = reinterpret_cast<uint32_t*>(ws.count + at * kBins);
  for (int i = threadIdx.x; i < kBins / 2; i += kScanThreads) out[i] = hist[2 * i] | (hist[2 * i + 1] << 16);
  if (threadIdx.x == 0) {
    ws.top[at] = top;
    double s = 0.0;
    for (int i = 0; i < kScanThreads / kWave; ++i) s += red[i];
    ws.tail[at] = s;
  }
}

// inclusive scan over the workgroup, thread order; red: one entry a wave
template <class T>
__device__ T group_scan(T v, T* red) {
  for (int m = 1; m < kWave; m <<= 1) {
    const T o = __shfl_up(v, m);
    if (lane_id() >= m) v += o;
  }
  __syncthreads();
  if (lane_id() == kWave - 1) red[threadIdx.x >> 6] = v;
  __syncthreads();
  T before = 0;
  for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) before += red[w];
  return before + v;
}

struct DrawLds {
  double w[kBins];            // weight of each value of the row, 0 where not kept
  double sum[kMaxChunks];     // kept weight of each chunk
  int off[kMaxChunks];        // the chunk's largest value, counted from the row's
  int ties[kMaxChunks];       // kept logits of the prefix's last value
  double redd[kThreads / kWave];
  uint32_t redu[kThreads / kWave];
  int bin, found, last;
  double at_bin, target, total;
  int chunk;
};
union DrawUnion {
  DrawLds d;
  PassLds p;
};

__global__ __launch_bounds__(kThreads) void sample_draw_kernel(SampleParams p, ChunkWs ws, double unit) {
  static_assert(kThreads == kBins && kChunk == 8 * kThreads, "a thread has one value and eight logits of a chunk");
  __shared__ DrawUnion lds;
  DrawLds& s = lds.d;
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x, C = ws.chunks;
  const uint32_t* tops = ws.top + row * C;
  const uint16_t* count = ws.count + row * C * kBins;
  const RowArgs a = row_args(p, row);
  const double t = (double)a.t;
  uint32_t top = 0;
  for (int c = tid; c < C; c += kThreads) top = max(top, tops[c]);
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if (lane_id() == 0) s.redu[tid >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / kWave; ++i) top = max(top, s.redu[i]);
  if (top <= (kMinusInf >> 16)) {
    if (tid == 0) {
      p.token[row] = -1;
      if (p.prob) p.prob[row] = 0.0f;
    }
    return;
  }
  const double best = (double)value16(top);
  for (int c = tid; c < C; c += kThreads) s.off[c] = (int)(top - tops[c]);
  if (tid == 0) s.bin = kBins;
  __syncthreads();
  // ---- value tid of the row: count, weight, running sums
  uint32_t n = 0;
  if (tid < kBins - 1)
    for (int c = 0; c < C; ++c) {
      const int d = tid - s.off[c];
      n += d >= 0 ? count[(int64_t)c * kBins + d] : 0u;
    }
  const double w = a.greedy ? (tid == 0 ? 1.0 : 0.0) : tid < kBins - 1 && (uint32_t)tid <= top ? weight16(top - tid, top, best, t) : 0.0;
  const uint32_t upto_n = group_scan(n, s.redu);
  const double upto_w = group_scan((double)n * w, s.redd);
  // weights below the counted values, each chunk's (a wave a chunk)
  double below = 0.0;
  const bool tail = !a.greedy && !a.k_on && (a.p_on || a.least == 0.0);
  if (tail) {
    for (int c = tid >> 6; c < C; c += kThreads / kWave) {
      const int off = s.off[c];
      double x = 0.0;
      for (int d = max(0, kBins - 1 - off) + lane_id(); d < kBins - 1; d += kWave) {
        const uint32_t m = count[(int64_t)c * kBins + d];
        if (m) x += (double)m * weight16((uint32_t)max((int)top - off - d, 0), top, best, t);
      }
      x = wave_sum64(x) + ws.tail[row * C + c] * weight16(tops[c], top, best, t);
      if (lane_id() == 0) s.sum[c] = x;
    }
    __syncthreads();
    for (int c = 0; c < C; ++c) below += s.sum[c];
  }
  // ---- the kept prefix: values before `bin`, and `ties` logits of it
  int bin = kBins;  // none: all are kept
  double ties = 0.0, z = 0.0;
  bool lost = false;  // ends below the counted values
  auto take = [&](bool here, double x) {  // the one thread whose value it is tells the others
    __syncthreads();
    if (tid == 0) s.bin = kBins;
    __syncthreads();
    if (here) {
      s.bin = tid;
      s.at_bin = x;
    }
    __syncthreads();
    bin = s.bin;
    ties = s.at_bin;
  };
  if (a.greedy) {
    bin = 0;
    ties = 1.0;
  }
  if (a.k_on) {
    const uint32_t k = (uint32_t)a.top_k;
    take(upto_n >= k && upto_n - n < k, (double)(k - (upto_n - n)));
    lost = bin == kBins;
  }
  if (a.p_on && !lost) {
    const int last = bin;
    const double most = ties;
    // what the top_k tokens weigh, or all
    __syncthreads();
    if (tid == (last == kBins ? kBins - 1 : last))
      s.total = last == kBins ? upto_w + below : upto_w - (double)n * w + most * w;
    __syncthreads();
    z = s.total;
    const double goal = (double)fmaxf(a.top_p, 0.0f) * z, before = upto_w - (double)n * w;
    // the last value with a token before which the goal is not reached
    __syncthreads();
    if (tid == 0) s.bin = 0;
    __syncthreads();
    if (n > 0 && tid <= last && before < goal) atomicMax(&s.bin, tid);
    __syncthreads();
    const int end = s.bin;
    // beyond the counted values: their sum does not reach the goal
    if (last == kBins) {
      __syncthreads();
      if (tid == kBins - 1) s.total = upto_w;
      __syncthreads();
      lost = s.total < goal;
    }
    if (!lost) {
      take(tid == end, w > 0.0 ? fmin(fmax(1.0, ceil((goal - before) / w)), tid == last ? most : (double)n) : (double)n);
    }
  }
  if (!a.greedy && !a.k_on && !a.p_on && a.least > 0.0) {
    __syncthreads();
    if (tid == kBins - 2) s.total = w;
    __syncthreads();
    lost = s.total >= a.least;
    bin = kBins - 1;  // what the counted values hold
  }
  if (lost) {
    __syncthreads();
    draw_in_passes(p, row, row_of(p, row, true), a, unit, lds.p);
    return;
  }
  // ---- kept weight of each chunk
  __syncthreads();
  s.w[tid] = w < a.least || tid > bin ? 0.0 : w;
  __syncthreads();
  if (tid == 0) {  // ties go to the lowest indexes
    double left = ties;
    if (bin < kBins - 1)
      for (int c = 0; c < C; ++c) {
        const int d = bin - s.off[c];
        const double m = d >= 0 ? fmin((double)count[(int64_t)c * kBins + d], left) : 0.0;
        s.ties[c] = (int)m;
        left -= m;
      }
  }
  __syncthreads();
  for (int c = tid >> 6; c < C; c += kThreads / kWave) {
    const int off = s.off[c];
    double x = 0.0;
    for (int d = lane_id(); d < min(bin, kBins - 1) - off; d += kWave)
      x += (double)count[(int64_t)c * kBins + d] * s.w[d + off];
    x = wave_sum64(x);
    if (bin < kBins - 1) x += (double)s.ties[c] * s.w[bin];
    if (bin == kBins) x += s.sum[c];
    if (lane_id() == 0) s.sum[c] = x;
  }
  __syncthreads();
  if (tid == 0) {
    double all = 0.0;
    for (int c = 0; c < C; ++c) all += s.sum[c];
    const double target = (double)a.u * all;
    double run = 0.0, before = 0.0;
    int at = 0;
    for (int c = 0; c < C; ++c) {
      if (s.sum[c] > 0.0) {
        at = c;
        before = run;
      }
      run += s.sum[c];
      if (run > target && s.sum[c] > 0.0) break;
    }
    s.total = all;
    s.chunk = at;
    s.target = target - before;
    s.found = kChunk;
    s.last = -1;
  }
  __syncthreads();
  // ---- the token within its chunk
  const int c = s.chunk;
  const uint16_t* base = reinterpret_cast<const uint16_t*>(p.logits) + row * p.ld;
  uint32_t k[8];
  keys16x8(base, (int64_t)c * kChunk + tid * 8, p.n, (reinterpret_cast<uintptr_t>(base) & 15u) == 0, k);
  uint32_t mine = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) mine += top - k[e] == (uint32_t)bin ? 1 : 0;
  uint32_t rank = bin < kBins - 1 ? group_scan(mine, s.redu) - mine : 0;
  double x[8], own = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const uint32_t d = top - k[e];
    x[e] = 0.0;
    if (d < kBins - 1) {
      x[e] = s.w[d];
      if (d == (uint32_t)bin) {
        if (rank >= (uint32_t)s.ties[c]) x[e] = 0.0;
        ++rank;
      }
    } else if (bin == kBins && k[e]) {
      x[e] = weight16(k[e], top, best, t);
    }
    own += x[e];
  }
  const double upto = group_scan(own, s.redd);
  double run = upto - own;
  const double target = s.target;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    run += x[e];
    if (x[e] > 0.0) {
      if (run > target) atomicMin(&s.found, tid * 8 + e);
      else atomicMax(&s.last, tid * 8 + e);
    }
  }
  __syncthreads();
  const int hit = s.found < kChunk ? s.found : s.last;
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (tid * 8 + e == hit) {
      p.token[row] = (int64_t)c * kChunk + hit;
      if (p.prob) p.prob[row] = (float)(x[e] / s.total);
    }
}

}  // namespace

size_t sample_ws_bytes(int64_t rows, int64_t n, bool bf16) {
  if (!bf16) return 0;
  const int64_t all = rows * ((n + kChunk - 1) / kChunk);
  return (size_t)all * (kBins * sizeof(uint16_t) + sizeof(double) + sizeof(uint32_t));
}

hipError_t launch_sample(const SampleParams& p, bool bf16, void* ws, hipStream_t st) {
  int log2n = 0;
  while (((int64_t)1 << log2n) < p.n) ++log2n;
  const double unit = ldexp(1.0, 62 - log2n);
  if (!bf16) {
    sample_passes_kernel<<<dim3((unsigned)p.rows), kThreads, 0, st>>>(p, unit);
    return hipGetLastError();
  }
  const ChunkWs w = chunk_ws(ws, p.rows, p.n);
  sample_scan_kernel<<<dim3((unsigned)w.chunks, (unsigned)p.rows), kScanThreads, 0, st>>>(p, w);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  sample_draw_kernel<<<dim3((unsigned)p.rows), kThreads, 0, st>>>(p, w, unit);
  return hipGetLastError();
}

}  // namespace w8a8
