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
  if (key <= kMinusInf) return 0.0;
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

}  // namespace

// One workgroup a row, some passes over the row each.
__global__ __launch_bounds__(kThreads) void sample_kernel(SampleParams p, bool bf, double unit) {
  __shared__ double sums[kMaxBlocks];
  __shared__ double red[kThreads / kWave];
  __shared__ unsigned long long hist[257];
  __shared__ int64_t found[2];
  __shared__ uint32_t pick[1], tops[kThreads / kWave];
  const int64_t row = blockIdx.x;
  Row r;
  r.bf = bf;
  r.n = p.n;
  r.base = bf ? (const void*)(reinterpret_cast<const uint16_t*>(p.logits) + row * p.ld)
              : (const void*)(reinterpret_cast<const float*>(p.logits) + row * p.ld);
  const float t = p.temperature ? p.temperature[row] : p.temperature_all;
  const int top_k = p.top_k ? p.top_k[row] : p.top_k_all;
  const float top_p = p.top_p ? p.top_p[row] : p.top_p_all;
  const float min_p = p.min_p ? p.min_p[row] : p.min_p_all;
  uint32_t top = 0;
  for (int64_t i = threadIdx.x; i < r.n; i += kThreads) top = max(top, key_at(r, i));
  for (int m = 32; m >= 1; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m));
  if (lane_id() == 0) tops[threadIdx.x >> 6] = top;
  __syncthreads();
  for (int i = 0; i < kThreads / kWave; ++i) top = max(top, tops[i]);
  r.top = top;
  r.best = (double)value_of(top);
  r.t = (double)t;
  if (value_of(top) == -INFINITY) {  // nothing to draw from
    if (threadIdx.x == 0) {
      p.token[row] = -1;
      if (p.prob) p.prob[row] = 0.0f;
    }
    return;
  }
  const bool greedy = !(t > 0.0f);
  // the kept prefix: keys above thr, and thr itself up to index cut
  uint32_t thr = 0;
  int64_t cut = INT64_MAX;
  double ties = 0.0, total;
  if (greedy) {
    thr = top;
    ties = 1.0;
  } else {
    if (top_k > 0 && top_k < r.n) {
      double above;
      thr = select(r, (double)top_k, [](uint32_t) { return 1ull; }, hist, pick, 1.0, &above);
      ties = (double)top_k - above;
    }
    if (top_p < 1.0f) {
      const uint32_t floor_key = thr;
      const double floor_ties = ties;
      double z = 0.0;
      for (int64_t i = threadIdx.x; i < r.n; i += kThreads) {
        const uint32_t k = key_at(r, i);
        if (floor_ties == 0.0 || k > floor_key) z += weight(r, k);
      }
      z = group_sum(z, red);
      if (floor_ties > 0.0) z += floor_ties * weight(r, floor_key);
      const double goal = (double)fmaxf(top_p, 0.0f) * z;
      double above;
      thr = select(r, goal, [&](uint32_t k) {
        return k >= floor_key ? (unsigned long long)rint(weight(r, k) * unit) : 0ull; }, hist, pick, unit, &above);
      const double w = weight(r, thr);
      ties = w > 0.0 ? fmax(1.0, ceil((goal - above / unit) / w)) : (double)r.n;
      if (floor_ties > 0.0 && thr == floor_key) ties = fmin(ties, floor_ties);
    }
  }
  if (ties > 0.0)
    cut = walk(r, ties - 0.5, false, [&](uint32_t k, int64_t) { return k == thr ? 1.0 : 0.0; }, sums, red, found, &total);
  const double least = min_p > 0.0f ? fmin((double)min_p, 1.0) : 0.0;
  const float u = p.u[row] > 0.0f ? p.u[row] : 0.0f;  // NaN: 0
  const int64_t token = walk(r, (double)u, true, [&](uint32_t k, int64_t i) {
    if (k < thr || (k == thr && i > cut)) return 0.0;
    if (greedy) return 1.0;
    const double w = weight(r, k);
    return w < least ? 0.0 : w; }, sums, red, found, &total);
  if (threadIdx.x == 0) {
    p.token[row] = token;
    if (p.prob) p.prob[row] = (float)((greedy ? 1.0 : weight(r, key_at(r, token))) / total);
  }
}

hipError_t launch_sample(const SampleParams& p, bool bf16, hipStream_t st) {
  int log2n = 0;
  while (((int64_t)1 << log2n) < p.n) ++log2n;
  sample_kernel<<<dim3((unsigned)p.rows), kThreads, 0, st>>>(p, bf16, ldexp(1.0, 62 - log2n));
  return hipGetLastError();
}

}  // namespace w8a8
