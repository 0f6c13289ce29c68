// Rotary positions, and the rows of a fused QKV projection rotated and stored
// in a paged key/value cache.
//
// A head of d elements carries rot / 2 pairs; pair j of the token at position p
// is turned by the angle p * freq[j]:
//   (a, b) -> scale * (a cos - b sin, b cos + a sin),
// pairs (j, j + rot/2) in the half layout, (2j, 2j + 1) in the interleaved one.
// The angle is formed in binary64 (at position 10^6 a binary32 product is off
// by up to 0.06 rad), as a number of turns, of which only the fraction counts.
//
// One wave takes one row (token).  Heads are cut into units of 16 elements,
// eight pairs or sixteen elements that pass; lane l takes units l, l + 64, ...
// Memory bounds all three kernels: 4095 rows of 18 f32 heads of 128 (75 MB) take 17 us, 4.4 TB/s,
// and 2039-token prompts appended and read back (144 MB) 30 us, 4.8 TB/s, where a copy of
// 2 GiB reaches 4.96; the angles, formed once a row and unit, are hidden behind it.
#include "device.h"
#include "kernels.h"

namespace w8a8 {

namespace {

// 16 elements of a unit, in binary32
template <bool BF>
__device__ __forceinline__ void load8(const void* base, int64_t at, float* v) {
  if constexpr (BF) {
    const uint4 r = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(base) + at);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = bf16_bits_to_float(w[i] & 0xffffu);
      v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(base) + at);
    const float4 a = p[0], b = p[1];
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
  }
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  return (uint32_t)float_to_bf16_bits(lo) | ((uint32_t)float_to_bf16_bits(hi) << 16);
}

template <bool BF>
__device__ __forceinline__ void store8(void* base, int64_t at, const float* v) {
  if constexpr (BF) {
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(base) + at) =
        make_uint4(pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7]));
  } else {
    float4* p = reinterpret_cast<float4*>(reinterpret_cast<float*>(base) + at);
    p[0] = make_float4(v[0], v[1], v[2], v[3]);
    p[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// cos and sin of pair j0 .. j0 + 7 at position pos, times scale
__device__ __forceinline__ void turns8(const double* freq, int j0, double pos, float scale, float* c, float* s) {
  constexpr double kInvTwoPi = 0.15915494309189533577;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const double t = pos * (freq[j0 + i] * kInvTwoPi);
    const float f = (float)(2.0 * (t - rint(t)));  // half turns in [-1, 1]
    float sn, cs;
    sincospif(f, &sn, &cs);
    c[i] = cs * scale;
    s[i] = sn * scale;
  }
}

// offsets of the two runs of 8 elements that unit u of a head holds
__device__ __forceinline__ void unit_at(int u, int rot, bool inter, int* a, int* b) {
  const bool split = !inter && 16 * u < rot;
  *a = split ? 8 * u : 16 * u;
  *b = split ? rot / 2 + 8 * u : 16 * u + 8;
}

// a unit's pairs turned: x[0..7], x[8..15] are the runs of unit_at
__device__ __forceinline__ void turn(float* x, bool inter, const float* c, const float* s) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float& a = inter ? x[2 * i] : x[i];
    float& b = inter ? x[2 * i + 1] : x[i + 8];
    const float p = a * c[i] - b * s[i], q = b * c[i] + a * s[i];
    a = p;
    b = q;
  }
}

}  // namespace

template <bool BF, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(RopeParams p) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;
  const int units = p.d / 16, all = p.heads * units;
  const double pos = (double)p.pos[row];
  float c[8], s[8];
  int have = -1;
  for (int i = lane_id(); i < all; i += kWave) {
    const int h = i / units, u = i - h * units;
    int a, b;
    unit_at(u, p.rot, INTER, &a, &b);
    float x[16];
    const int64_t in = row * p.ldx + (int64_t)h * p.d, out = row * p.ldy + (int64_t)h * p.d;
    load8<BF>(p.x, in + a, x);
    load8<BF>(p.x, in + b, x + 8);
    if (16 * u < p.rot) {
      if (have != u) turns8(p.freq, 8 * u, pos, p.scale, c, s);
      have = u;
      turn(x, INTER, c, s);
    }
    store8<BF>(p.y, out + a, x);
    store8<BF>(p.y, out + b, x + 8);
  }
}

// The cached row (page, slot) of a sequence's position, or -1: outside the
// table, or in a page that it does not hold.
__device__ __forceinline__ int64_t cached_row(const PagedKv& kv, const PagedBatch& b, int seq, int pos) {
  if (pos < 0 || (pos >> kv.page_log2) >= b.max_pages) return -1;
  const int page = b.table[(int64_t)seq * b.max_pages + (pos >> kv.page_log2)];
  if (page < 0 || page >= kv.n_pages) return -1;
  return (((int64_t)page * kv.n_kv) << kv.page_log2) + (pos & ((1 << kv.page_log2) - 1));
}

// the sequence of a row and its position there; false behind the last sequence
__device__ __forceinline__ bool row_position(const PagedBatch& b, int64_t row, int* seq, int* pos) {
  int count = 0;
  for (int base = 0; base < b.n_seqs; base += kWave) {
    const int s = base + lane_id();
    const uint64_t m = __ballot(s < b.n_seqs && b.q_start[s] <= row);
    count += __popcll(m);
    if (m != ~0ull) break;
  }
  if (count == 0) return false;
  *seq = count - 1;
  const int end = b.q_start[count];
  if (row >= end) return false;
  *pos = max(b.ctx_len[count - 1], 0) - (int)(end - row);
  return true;
}

// Row of the projection -> rotated queries (bf16), rotated key and value rows of
// the cache.  A key or value row is quantised from its binary32 values (s = max
// |x| / 127, codes rne(x / s)), with no rounding to bf16 between the rotation and
// the codes; the maximum runs over the D / 16 lanes that hold the head.
template <int D, bool I8, bool INTER>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams p) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;  // whole wave
  int seq, pos;
  if (!row_position(p.batch, row, &seq, &pos)) return;
  constexpr int U = D / 16;
  const int u = lane_id() % U, hk = p.n_heads + p.kv.n_kv, all = hk + p.kv.n_kv;
  const int64_t at = cached_row(p.kv, p.batch, seq, pos);
  const bool rotates = 16 * u < p.rot;
  float c[8], s[8];
  if (rotates) turns8(p.freq, 8 * u, (double)pos, p.scale, c, s);
  for (int h = lane_id() / U; h < all; h += kWave / U) {  // the lanes of a head stay together
    int a = 16 * u, b = 16 * u + 8;
    if (h < hk) unit_at(u, p.rot, INTER, &a, &b);
    float x[16];
    const uint16_t* src = p.qkv + row * p.ld + (int64_t)h * D;
    load8<true>(src, a, x);
    load8<true>(src, b, x + 8);
    if (h < hk && rotates) turn(x, INTER, c, s);
    if (h < p.n_heads) {
      uint16_t* dst = p.q + row * p.ldq + (int64_t)h * D;
      store8<true>(dst, a, x);
      store8<true>(dst, b, x + 8);
      continue;
    }
    const bool key = h < hk;
    const int j = h - (key ? p.n_heads : hk);
    const int64_t r = at + ((int64_t)j << p.kv.page_log2);
    if constexpr (I8) {
      float m = fabsf(x[0]);  // of numbers; NaN where a row has none, so that it stays NaN
#pragma unroll
      for (int i = 1; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
      m = fmaxf(m, lane_xor<1>(m));
      m = fmaxf(m, lane_xor<2>(m));
      m = fmaxf(m, lane_xor<4>(m));
      if constexpr (U == 16) m = fmaxf(m, lane_xor<8>(m));
      const float sc = m / 127.0f;
      const float inv = 1.0f / sc;
      uint32_t w[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w[i] = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[i] |= sc != 0.0f ? (uint32_t)(uint8_t)code_of(x[4 * i + e], sc, inv, true) << (8 * e) : 0u;
      }
      if (at >= 0) {
        int8_t* dst = reinterpret_cast<int8_t*>(key ? p.kv.k : p.kv.v) + r * D;
        *reinterpret_cast<uint2*>(dst + a) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2*>(dst + b) = make_uint2(w[2], w[3]);
        if (u == 0) (key ? p.kv.sk : p.kv.sv)[r] = sc;
      }
    } else if (at >= 0) {
      void* dst = key ? p.kv.k : p.kv.v;
      store8<true>(dst, r * D + a, x);
      store8<true>(dst, r * D + b, x + 8);
    }
  }
}

// The cached rows of the batch's new tokens as bf16; zeros where the page table
// holds no page.  One wave per row, lanes over the heads' units.
template <int D, bool I8>
__global__ __launch_bounds__(256) void kv_read_kernel(KvReadParams p) {
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= p.rows) return;  // whole wave
  int seq, pos;
  if (!row_position(p.batch, row, &seq, &pos)) return;
  constexpr int U = D / 16;
  const int u = lane_id() % U, all = 2 * p.kv.n_kv;
  const int64_t at = cached_row(p.kv, p.batch, seq, pos);
  for (int h = lane_id() / U; h < all; h += kWave / U) {
    const bool key = h < p.kv.n_kv;
    const int j = key ? h : h - p.kv.n_kv;
    const int64_t r = at + ((int64_t)j << p.kv.page_log2);
    float x[16] = {};
    if (at >= 0) {
      if constexpr (I8) {
        const uint4 raw = *reinterpret_cast<const uint4*>(reinterpret_cast<const int8_t*>(key ? p.kv.k : p.kv.v) + r * D + 16 * u);
        const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
        const float sc = (key ? p.kv.sk : p.kv.sv)[r];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = (float)(int8_t)(uint8_t)(w[i >> 2] >> (8 * (i & 3))) * sc;
      } else {
        load8<true>(key ? p.kv.k : p.kv.v, r * D + 16 * u, x);
        load8<true>(key ? p.kv.k : p.kv.v, r * D + 16 * u + 8, x + 8);
      }
    }
    uint16_t* dst = (key ? p.k_out : p.v_out) + (row * p.kv.n_kv + j) * D + 16 * u;
    store8<true>(dst, 0, x);
    store8<true>(dst, 8, x + 8);
  }
}

static dim3 row_grid(int64_t rows) { return dim3((unsigned)((rows + 3) / 4)); }

hipError_t launch_rope(const RopeParams& p, bool bf16, bool inter, hipStream_t st) {
  const dim3 g = row_grid(p.rows);
  if (bf16)
    inter ? rope_kernel<true, true><<<g, 256, 0, st>>>(p) : rope_kernel<true, false><<<g, 256, 0, st>>>(p);
  else
    inter ? rope_kernel<false, true><<<g, 256, 0, st>>>(p) : rope_kernel<false, false><<<g, 256, 0, st>>>(p);
  return hipGetLastError();
}

template <int D>
static hipError_t append_launch(const AppendParams& p, bool inter, hipStream_t st) {
  const dim3 g = row_grid(p.rows);
  if (p.kv.sk)
    inter ? kv_append_kernel<D, true, true><<<g, 256, 0, st>>>(p) : kv_append_kernel<D, true, false><<<g, 256, 0, st>>>(p);
  else
    inter ? kv_append_kernel<D, false, true><<<g, 256, 0, st>>>(p) : kv_append_kernel<D, false, false><<<g, 256, 0, st>>>(p);
  return hipGetLastError();
}

hipError_t launch_kv_append(const AppendParams& p, int head_dim, bool inter, hipStream_t st) {
  return head_dim == 256 ? append_launch<256>(p, inter, st) : append_launch<128>(p, inter, st);
}

hipError_t launch_kv_read(const KvReadParams& p, int head_dim, hipStream_t st) {
  const dim3 g = row_grid(p.rows);
  if (head_dim == 256)
    p.kv.sk ? kv_read_kernel<256, true><<<g, 256, 0, st>>>(p) : kv_read_kernel<256, false><<<g, 256, 0, st>>>(p);
  else
    p.kv.sk ? kv_read_kernel<128, true><<<g, 256, 0, st>>>(p) : kv_read_kernel<128, false><<<g, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace w8a8
