// Attention of new tokens over a paged key/value cache.
//
// The cache holds INT8 codes with per-row scales or bf16 rows, in pages of a
// power of two of positions.  A sequence's new tokens are its last positions
// (their rows are in the cache already); the token at position pos attends the
// positions j <= pos, j > pos - window whose page the table holds, and a token
// without any gets zeros.
//
// The query heads of one key/value head and the new tokens of a sequence are
// the rows of one product: row r is head r % group of token r / group.  Scores
// are formed transposed, keys x rows, so that a lane holds one row's scores and
// the softmax needs two exchanges between lanes; in that layout they are the
// second operand of the transposed value product, values x weights, as they
// stand.  Maximum, sum and outputs run in binary32 along the keys.
#include <algorithm>

#include "device.h"
#include "kernels.h"

namespace w8a8 {

namespace {

constexpr int kStep = 32;          // keys a wave takes at a time
constexpr int kPass = 4 * kStep;   // ... and a workgroup

// INT8 code e of a word (exact in bf16)
__device__ __forceinline__ float byte_f(uint32_t w, int e) {
  return (float)(int8_t)(uint8_t)(w >> (8 * e));
}
// the bf16 pair of two binary32 values whose low 16 bits are dropped
__device__ __forceinline__ int pair_hi(float lo, float hi) {
  return (int)__builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// A tile of BM rows of one sequence.  Sequence s has slots floor(q_start[s] *
// group / BM) + s and up, one for each of its tiles at least: a workgroup finds
// its sequence without a prefix sum, and slots between the sequences are empty.
struct Tile {
  int seq, q0, q_len, row0;
  int first;  // position of the first new token
};
template <int BM>
__device__ __forceinline__ bool find_tile(const PagedAttnParams& p, int64_t slot, Tile* t) {
  int count = 0;
  for (int base = 0; base < p.batch.n_seqs; base += kWave) {
    const int s = base + lane_id();
    const uint64_t m = __ballot(s < p.batch.n_seqs && (int64_t)p.batch.q_start[min(s, p.batch.n_seqs)] * p.group / BM + s <= slot);
    count += __popcll(m);
    if (m != ~0ull) break;
  }
  if (count == 0) return false;
  const int s = count - 1, q0 = p.batch.q_start[s], q1 = p.batch.q_start[s + 1];
  if (q0 < 0 || q1 > p.rows || q1 <= q0) return false;
  const int64_t row0 = (slot - (int64_t)q0 * p.group / BM - s) * BM;
  if (row0 < 0 || row0 >= (int64_t)(q1 - q0) * p.group) return false;
  t->seq = s;
  t->q0 = q0;
  t->q_len = q1 - q0;
  t->first = max(p.batch.ctx_len[s], 0) - t->q_len;
  t->row0 = (int)row0;
  return true;
}

}  // namespace

// Sixteen rows a workgroup.  Each of its four waves walks every fourth group of
// 32 keys, straight from memory: a lane's pieces of a key row are what lies
// together in memory (any assignment of the dimensions to the product's K
// positions serves), and its 16 bytes of a value row are one output dimension
// of sixteen products.  The weights go in as two bf16 values (16 significant
// bits).
template <int D, bool I8>
__global__ __launch_bounds__(256) void attn_paged_kernel(PagedAttnParams p) {
  constexpr int KI = I8 ? D / 64 : D / 32;  // 16-byte pieces of a lane's quarter of a key row
  constexpr int E = D / 16;                 // dimensions of a lane's part of a value row
  constexpr int VW = I8 ? E / 4 : E / 2;    // ... in words
  constexpr int ROWB = I8 ? D : 2 * D;
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float ored[2][16][LD];
  __shared__ float om[4][16], ol[4][16];

  Tile tl;
  if (!find_tile<16>(p, blockIdx.x, &tl)) return;  // whole workgroup
  const int j = blockIdx.y;
  const int tid = threadIdx.x, w = tid >> 6, l = lane_id(), n = l & 15, g = l >> 4;
  const int first = tl.first, rows = tl.q_len * p.group, row = tl.row0 + n;
  const int pos = row < rows ? first + row / p.group : -1;
  const int from = pos < 0 ? 0 : max(0, pos + 1 - p.window);
  const int hi = min(first + min(rows - 1, tl.row0 + 15) / p.group + 1, p.batch.max_pages << p.kv.page_log2);  // exclusive
  // in [0, hi], so that no position below leaves 32 bits: a first position down to
  // -2^25 and a window up to 2^30 (the launcher's bound) are within them, too
  const int lo = min(max(0, first + tl.row0 / p.group + 1 - p.window), max(hi, 0));
  const int32_t* table = p.batch.table + (int64_t)tl.seq * p.batch.max_pages;

  v4i q[D / 32];
  {
    const int r = min(row, rows - 1);
    const uint16_t* src = p.q + (int64_t)(tl.q0 + r / p.group) * p.ldq + (int64_t)(j * p.group + r % p.group) * D;
#pragma unroll
    for (int c = 0; c < D / 32; ++c) {
      const int d0 = I8 ? 64 * (c >> 1) + 16 * g + 8 * (c & 1) : 32 * c + 8 * g;
      q[c] = *reinterpret_cast<const v4i*>(src + d0);
    }
  }

  float run_m = -INFINITY, run_l = 0.0f;
  v4f acc[E];  // dimensions E (4 g + r) + e of row n
#pragma unroll
  for (int e = 0; e < E; ++e) acc[e] = v4f{0.f, 0.f, 0.f, 0.f};

  for (int r0 = (lo & ~(kStep - 1)) + kStep * w; r0 < hi; r0 += kPass) {
    float sc[8], vs[8];
    uint32_t vc[8][VW];
    // ---- scores of two 16-key tiles
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int k0 = r0 + 16 * t;
      const int page = k0 < hi ? table[k0 >> p.kv.page_log2] : -1;
      const bool held = page >= 0 && page < p.kv.n_pages;
      const int64_t at = held ? ((((int64_t)page * p.kv.n_kv + j) << p.kv.page_log2) + (k0 & ((1 << p.kv.page_log2) - 1))) : 0;
      const int8_t* kp = reinterpret_cast<const int8_t*>(p.kv.k) + (at + n) * ROWB + 16 * g;
      uint4 kc[KI];
      const bool in = held && k0 + n >= lo && k0 + n < hi;  // other rows are not read
#pragma unroll
      for (int i = 0; i < KI; ++i)
        kc[i] = in ? *reinterpret_cast<const uint4*>(kp + 64 * i) : make_uint4(0, 0, 0, 0);
      v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        v4i kf;
        if constexpr (I8) {
          const uint4 u = kc[c >> 1];
          const uint32_t a = c & 1 ? u.z : u.x, b = c & 1 ? u.w : u.y;
          kf = v4i{pair_hi(byte_f(a, 0), byte_f(a, 1)), pair_hi(byte_f(a, 2), byte_f(a, 3)),
                   pair_hi(byte_f(b, 0), byte_f(b, 1)), pair_hi(byte_f(b, 2), byte_f(b, 3))};
        } else {
          kf = __builtin_bit_cast(v4i, kc[c]);
        }
        s = mma_bf16(kf, q[c], s);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = k0 + 4 * g + i;
        const bool live = held && key >= lo && key < hi;
        float x = s[i] * p.scale_log2;
        vs[4 * t + i] = 1.0f;
        if constexpr (I8) {
          x *= live ? p.kv.sk[at + 4 * g + i] : 0.0f;
          vs[4 * t + i] = live ? p.kv.sv[at + 4 * g + i] : 0.0f;
        }
        sc[4 * t + i] = held && key >= from && key <= pos ? x : -INFINITY;
        const uint32_t* vp = reinterpret_cast<const uint32_t*>(reinterpret_cast<const int8_t*>(p.kv.v) + (at + 4 * g + i) * ROWB) + VW * n;
#pragma unroll
        for (int c = 0; c < VW; ++c) vc[4 * t + i][c] = live ? vp[c] : 0u;
      }
    }
    // ---- running softmax
    float mx = run_m;
#pragma unroll
    for (int i = 0; i < 8; ++i) mx = fmaxf(mx, sc[i]);
    mx = fmaxf(mx, lane_xor<16>(mx));
    mx = fmaxf(mx, lane_xor<32>(mx));
    const float ref = mx == -INFINITY ? 0.0f : mx;  // nothing seen yet: weights of 0
    const float corr = __builtin_amdgcn_exp2f(run_m - ref);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sc[i] = __builtin_amdgcn_exp2f(sc[i] - ref);
      sum += sc[i];
    }
    sum += lane_xor<16>(sum);
    sum += lane_xor<32>(sum);
    run_l = run_l * corr + sum;
    run_m = mx;
    // ---- the weights as two bf16 values
    v4i hi2, lo2;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float a[2], b[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float wt = I8 ? (sc[i + k] == 0.0f ? 0.0f : sc[i + k] * vs[i + k]) : sc[i + k];
        a[k] = bf16_bits_to_float(float_to_bf16_bits(wt));
        b[k] = bf16_bits_to_float(float_to_bf16_bits(wt - a[k]));
      }
      hi2[i >> 1] = pair_hi(a[0], a[1]);
      lo2[i >> 1] = pair_hi(b[0], b[1]);
    }
#pragma unroll
    for (int e = 0; e < E; ++e) {
      v4i vf;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        if constexpr (I8)
          vf[i >> 1] = pair_hi(byte_f(vc[i][e >> 2], e & 3), byte_f(vc[i + 1][e >> 2], e & 3));
        else
          vf[i >> 1] = (int)__builtin_amdgcn_perm(vc[i + 1][e >> 1], vc[i][e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
      }
      acc[e] = mma_bf16(vf, lo2, mma_bf16(vf, hi2, acc[e] * corr));
    }
  }

  // ---- the four waves
  if (g == 0) {
    om[w][n] = run_m;
    ol[w][n] = run_l;
  }
  __syncthreads();
  const float m = fmaxf(fmaxf(om[0][n], om[1][n]), fmaxf(om[2][n], om[3][n]));
  const float ref = m == -INFINITY ? 0.0f : m;
  const float f = __builtin_amdgcn_exp2f(run_m - ref);
  auto slot = [&](int r, int e) -> float4& {
    return *reinterpret_cast<float4*>(&ored[w & 1][n][E * (4 * g + r) + e]);
  };
  if (w >= 2) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < E; e += 4)
        slot(r, e) = make_float4(acc[e][r] * f, acc[e + 1][r] * f, acc[e + 2][r] * f, acc[e + 3][r] * f);
  }
  __syncthreads();
  if (w < 2) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float4 o = slot(r, e);
        o.x += acc[e][r] * f;
        o.y += acc[e + 1][r] * f;
        o.z += acc[e + 2][r] * f;
        o.w += acc[e + 3][r] * f;
        slot(r, e) = o;
      }
  }
  __syncthreads();
  // ---- 16 rows of D: thread tid has eight dimensions of a row
  for (int i = tid; i < 16 * D / 8; i += 256) {
    const int rr = i / (D / 8), d0 = 8 * (i % (D / 8)), r = tl.row0 + rr;
    if (r >= rows) break;
    const float mr = fmaxf(fmaxf(om[0][rr], om[1][rr]), fmaxf(om[2][rr], om[3][rr]));
    const float rref = mr == -INFINITY ? 0.0f : mr;
    float den = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) den += ol[k][rr] * __builtin_amdgcn_exp2f(om[k][rr] - rref);
    uint32_t o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float x = ored[0][rr][d0 + 2 * k] + ored[1][rr][d0 + 2 * k];
      const float y = ored[0][rr][d0 + 2 * k + 1] + ored[1][rr][d0 + 2 * k + 1];
      o[k] = (uint32_t)float_to_bf16_bits(den == 0.0f ? 0.0f : x / den) |
             ((uint32_t)float_to_bf16_bits(den == 0.0f ? 0.0f : y / den) << 16);
    }
    uint16_t* dst = p.out + (int64_t)(tl.q0 + r / p.group) * p.ldo + (int64_t)(j * p.group + r % p.group) * D + d0;
    *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

hipError_t launch_attn_paged(const PagedAttnParams& p, int head_dim, hipStream_t st) {
  const dim3 g((unsigned)(p.rows * p.group / 16 + p.batch.n_seqs), (unsigned)p.kv.n_kv);
  if (head_dim == 256)
    p.kv.sk ? attn_paged_kernel<256, true><<<g, 256, 0, st>>>(p) : attn_paged_kernel<256, false><<<g, 256, 0, st>>>(p);
  else
    p.kv.sk ? attn_paged_kernel<128, true><<<g, 256, 0, st>>>(p) : attn_paged_kernel<128, false><<<g, 256, 0, st>>>(p);
  return hipGetLastError();
}

}  // namespace w8a8
