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
#include <type_traits>

#include "device.h"
#include "kernels.h"

namespace w8a8 {

namespace {

constexpr int kStep = 32;          // keys a wave takes at a time
constexpr int kPass = 4 * kStep;   // ... and a workgroup
constexpr int kRows = 16;          // rows of the row-tile kernel
constexpr int kSplitSeqs = 512;    // sequences that the row kernel's workgroups share out among them

// INT8 code e of a word (exact in bf16)
__device__ __forceinline__ float byte_f(uint32_t w, int e) {
  return (float)(int8_t)(uint8_t)(w >> (8 * e));
}
// the bf16 pair of two binary32 values whose low 16 bits are dropped
__device__ __forceinline__ int pair_hi(float lo, float hi) {
  return (int)__builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}

// Arrays that no kernel writes, read through the scalar cache where the index is the
// same for a wave.
typedef const __attribute__((address_space(4))) int32_t* ConstInts;

// The new tokens of sequence s, false where it has none (or its arrays are not
// what they should be: rows outside the call, more tokens than the workspace is
// for; those rows are not touched).
struct Seq {
  int q0, q_len;
  int first;  // position of the first new token
};
__device__ __forceinline__ bool seq_at(const PagedAttnParams& p, int q0, int q1, int ctx, Seq* t) {
  if (q0 < 0 || q1 > p.rows || q1 <= q0 || q1 - q0 > p.max_q) return false;
  t->q0 = q0;
  t->q_len = q1 - q0;
  t->first = max(ctx, 0) - t->q_len;
  return true;
}
__device__ __forceinline__ bool seq_of(const PagedAttnParams& p, int s, Seq* t) {  // s: the same for a wave
  const ConstInts start = (ConstInts)p.batch.q_start;
  return seq_at(p, start[s], start[s + 1], ((ConstInts)p.batch.ctx_len)[s], t);
}
// sum over a wave
__device__ __forceinline__ uint32_t total(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(v), kWave - 1); }

// Keys [lo, hi) that rows row0 .. row1 of a sequence attend, lo in [0, hi]: no
// position below leaves 32 bits (first positions from -2^25, windows and tables up
// to 2^30).  Pieces of `piece` keys from lo rounded down to a step; one at least.
struct Keys {
  int lo, hi, begin, pieces;
};
__device__ __forceinline__ Keys keys_of(const PagedAttnParams& p, const Seq& t, int row0, int row1, int piece) {
  Keys k;
  k.hi = min(t.first + row1 / p.group + 1, p.batch.max_pages << p.kv.page_log2);
  k.lo = min(max(0, t.first + row0 / p.group + 1 - p.window), max(k.hi, 0));
  k.begin = k.lo & ~(kStep - 1);
  k.pieces = max((k.hi - k.begin + piece - 1) / piece, 1);
  return k;
}
// Where the piece of `piece` keys from `begin` on ends, of keys up to hi.  (The sum of
// begin and piece can pass 32 bits: a context beyond a table of 2^30 positions.)
__host__ __device__ constexpr int piece_end(int begin, int hi, int piece) {
  return hi - begin < piece ? hi : begin + piece;
}
static_assert(piece_end((1 << 30) - 32, 1 << 30, 1 << 30) == 1 << 30, "the last keys of the largest table");
static_assert(piece_end(0, -(1 << 30), 512) == -(1 << 30) && piece_end(512, 2000, 512) == 1024, "no keys; a piece in the middle");

// The sum of all passes over the slots, rounded up: the fewest passes of a piece.  The sum
// is one modulo 2^32: of 512 sequences of 2^30 positions, 2^32 passes, it is 0, which
// means nothing else (without any pass no answer is used).
__host__ __device__ constexpr uint32_t fewest_passes(uint32_t sum, uint32_t slots) { return (sum - 1) / slots + 1; }
static_assert(fewest_passes(0, kSplitSeqs) == 1u << 23, "512 sequences of 2^30 positions");
static_assert(fewest_passes(1, 512) == 1 && fewest_passes(512, 512) == 1 && fewest_passes(513, 512) == 2, "rounded up");

// Work of the row kernel: a sequence of at most 16 rows, or a piece of its keys.
//
// Contexts differ by much and only the GPU knows them, so the pieces are counted here:
// L passes of 128 keys are the fewest for which all pieces of all sequences, ceil(passes
// / L) of each, are at most p.row_pieces, what the CUs hold at once; a sequence is then
// cut evenly.  64 contexts of 600 to 16384 keys (240 MB) took 62 us in pieces of a fixed
// length, whose workgroups did not all fit and were not evenly spread over the XCDs.
struct RowWork {
  Seq t;
  Keys ks;
  int seq, piece, slot0;  // keys of a piece, slot of the sequence's first one
};
// of a slot, or (slot < 0) of sequence `seq`; false: none
__device__ __forceinline__ bool row_work(const PagedAttnParams& p, int slot, int seq, RowWork* w) {
  uint32_t k[kSplitSeqs / kWave], len = 1;
  int slot0 = seq = slot >= 0 ? slot : seq;
  uint32_t pieces = 1;
  if (p.row_pieces) {
    uint32_t sum = 0;
#pragma unroll
    for (int c = 0; c < kSplitSeqs / kWave; ++c) {
      const int s = c * kWave + lane_id();
      k[c] = 0;
      if (s < p.batch.n_seqs) {
        Seq t;
        if (seq_at(p, p.batch.q_start[s], p.batch.q_start[s + 1], p.batch.ctx_len[s], &t) && t.q_len * p.group <= p.max_rows)
          k[c] = (uint32_t)keys_of(p, t, 0, t.q_len * p.group - 1, kPass).pieces;
      }
      sum += k[c];
    }
    const uint32_t slots = (uint32_t)p.row_pieces;
    len = max(fewest_passes(total(sum), slots), 1u);
    for (;;) {  // to the longest at the latest: a piece a sequence, of which there are no more than slots
      uint32_t n = 0;
#pragma unroll
      for (int c = 0; c < kSplitSeqs / kWave; ++c)
        if (c * kWave < p.batch.n_seqs) n += (k[c] + len - 1) / len;
      if (total(n) <= slots) break;
      len += max(len / 16, 1u);
    }
    uint32_t before = 0;
    bool found = false;
#pragma unroll
    for (int c = 0; c < kSplitSeqs / kWave; ++c)
      if (c * kWave < p.batch.n_seqs) {
        const uint32_t mine = (k[c] + len - 1) / len, upto = before + wave_scan(mine), from = upto - mine;
        const uint64_t hit = slot >= 0 ? __ballot(from <= (uint32_t)slot && (uint32_t)slot < upto) : seq / kWave == c ? 1ull << (seq % kWave) : 0ull;
        if (hit && !found) {
          const int at = __builtin_ctzll(hit);
          found = true;
          seq = c * kWave + at;
          slot0 = __builtin_amdgcn_readlane((int)from, at);
          pieces = (uint32_t)__builtin_amdgcn_readlane((int)mine, at);
          len = (uint32_t)__builtin_amdgcn_readlane((int)((k[c] + max(mine, 1u) - 1) / max(mine, 1u)), at);
          break;
        }
        before = (uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1);
      }
    if (!found || pieces == 0) return false;
  }
  seq = __builtin_amdgcn_readfirstlane(seq);
  if (!seq_of(p, seq, &w->t)) return false;
  const int rows = w->t.q_len * p.group;
  if (rows > p.max_rows) return false;
  w->seq = seq;
  w->slot0 = __builtin_amdgcn_readfirstlane(slot0);
  w->piece = p.row_pieces ? __builtin_amdgcn_readfirstlane((int)len) * kPass : 1 << 30;
  w->ks = keys_of(p, w->t, 0, rows - 1, w->piece);
  return true;
}

}  // namespace

// Sequences of at most 16 rows, one a workgroup, and for long contexts a piece of
// its keys (row_work).  Each of the four waves walks every fourth group of 32 keys, straight
// from memory: a lane's pieces of a key row are what lies together in memory (any
// assignment of the dimensions to the product's K positions serves), and its 16
// bytes of a value row are one output dimension of sixteen products.  The weights
// go in as two bf16 values (16 significant bits).  The next group's keys and
// values are loaded as soon as the registers of this one's are free.  Rows of a
// held page are read whatever they hold; what no row attends is masked out of the
// scores, and zeroed in bf16 values (a weight of 0 times NaN).
//
// Memory bounds it: 64 contexts of 2048 to 16384 positions (240 MB of INT8) take 52 us,
// 4.6 TB/s with the 6 us before the first loads return and the last workgroups' ends
// (without the conversions or half the products 3 to 8 us less); 40 windows of 1024
// (131 MB of bf16) 32 us.  Registers for two workgroups a CU: with one, the windows took
// 5 us more.
template <int D, bool I8>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(PagedAttnParams p) {
  constexpr int KI = I8 ? D / 64 : D / 32;  // 16-byte pieces of a lane's quarter of a key row
  constexpr int E = D / 16;                 // dimensions of a lane's part of a value row
  constexpr int VW = I8 ? E / 4 : E / 2;    // ... in words
  constexpr int ROWB = I8 ? D : 2 * D;
  constexpr int LD = D + 4;
  __shared__ __attribute__((aligned(16))) float ored[2][kRows][LD];
  __shared__ float om[4][kRows], ol[4][kRows];

  RowWork work;
  const int slot = blockIdx.x, j = blockIdx.y;
  if (!row_work(p, slot, 0, &work)) return;  // whole workgroup
  const Seq tl = work.t;
  const Keys ks = work.ks;
  const int seq = work.seq, rows = tl.q_len * p.group, split = slot - work.slot0;
  if (split >= ks.pieces) return;
  const int begin = ks.begin + split * work.piece, lo = ks.lo, hi = piece_end(begin, ks.hi, work.piece);
  const int tid = threadIdx.x, w = __builtin_amdgcn_readfirstlane(tid >> 6), l = lane_id(), n = l & 15, g = l >> 4;
  const int pos = n < rows ? tl.first + n / p.group : -1;
  const int from = pos < 0 ? 0 : max(0, pos + 1 - p.window);
  const ConstInts table = (ConstInts)(p.batch.table + (int64_t)seq * p.batch.max_pages);
  const int page_mask = (1 << p.kv.page_log2) - 1;

  uint4 kc[2][KI];       // key row 16 t + n, bytes 64 i + 16 g .. + 15
  uint32_t vc[8][VW];    // value row 16 t + 4 g + i (at 4 t + i), dimensions E n .. + E - 1
  float4 sk[2], sv[2];   // INT8: scales of rows 16 t + 4 g .. + 3
  bool held[2];
  int64_t at[2];
  // the pages of two 16-key tiles (wave-uniform: scalar loads)
  auto locate = [&](int r0) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int k0 = r0 + 16 * t;
      const int page = k0 < hi ? table[k0 >> p.kv.page_log2] : -1;
      held[t] = page >= 0 && page < p.kv.n_pages;
      at[t] = held[t] ? ((((int64_t)page * p.kv.n_kv + j) << p.kv.page_log2) + (k0 & page_mask)) : 0;
    }
  };
  auto load_k = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int8_t* kp = reinterpret_cast<const int8_t*>(p.kv.k) + (at[t] + n) * ROWB + 16 * g;
#pragma unroll
      for (int i = 0; i < KI; ++i) kc[t][i] = *reinterpret_cast<const uint4*>(kp + 64 * i);
      if constexpr (I8) sk[t] = *reinterpret_cast<const float4*>(p.kv.sk + at[t] + 4 * g);
    }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int8_t* vp = reinterpret_cast<const int8_t*>(p.kv.v) + (at[t] + 4 * g) * ROWB + 4 * VW * n;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if constexpr (VW >= 4) {
#pragma unroll
          for (int c = 0; c < VW; c += 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(vp + i * ROWB + 4 * c);
            vc[4 * t + i][c] = x.x;
            vc[4 * t + i][c + 1] = x.y;
            vc[4 * t + i][c + 2] = x.z;
            vc[4 * t + i][c + 3] = x.w;
          }
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(vp + i * ROWB);
          vc[4 * t + i][0] = x.x;
          vc[4 * t + i][1] = x.y;
        }
      }
      if constexpr (I8) sv[t] = *reinterpret_cast<const float4*>(p.kv.sv + at[t] + 4 * g);
    }
  };

  int r0 = begin + kStep * w;
  if (r0 < hi) {
    locate(r0);
    load_k();
    load_v();
  }
  v4i q[D / 32];
  {
    const int r = min(n, rows - 1);
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

  for (; r0 < hi; r0 += kPass) {
    const bool more = r0 + kPass < hi;
    // ---- scores of two 16-key tiles
    float sc[8], vs[8];
    const bool h0 = held[0], h1 = held[1];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        v4i kf;
        if constexpr (I8) {
          const uint4 u = kc[t][c >> 1];
          const uint32_t a = c & 1 ? u.z : u.x, b = c & 1 ? u.w : u.y;
          kf = v4i{pair_hi(byte_f(a, 0), byte_f(a, 1)), pair_hi(byte_f(a, 2), byte_f(a, 3)),
                   pair_hi(byte_f(b, 0), byte_f(b, 1)), pair_hi(byte_f(b, 2), byte_f(b, 3))};
        } else {
          kf = __builtin_bit_cast(v4i, kc[t][c]);
        }
        s = mma_bf16(kf, q[c], s);
      }
      const float ks4[4] = {I8 ? sk[t].x : 1.f, I8 ? sk[t].y : 1.f, I8 ? sk[t].z : 1.f, I8 ? sk[t].w : 1.f};
      const float vs4[4] = {I8 ? sv[t].x : 1.f, I8 ? sv[t].y : 1.f, I8 ? sv[t].z : 1.f, I8 ? sv[t].w : 1.f};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = r0 + 16 * t + 4 * g + i;
        const float x = s[i] * (I8 ? ks4[i] * p.scale_log2 : p.scale_log2);
        sc[4 * t + i] = (t ? h1 : h0) && key >= from && key <= pos && key < hi ? x : -INFINITY;
        vs[4 * t + i] = vs4[i];
      }
    }
    if constexpr (!I8) {
      if (!(h0 && h1 && r0 >= lo && r0 + kStep <= hi)) {  // wave-uniform
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int key = r0 + 16 * (i >> 2) + 4 * g + (i & 3);
          const bool live = (i < 4 ? h0 : h1) && key >= lo && key < hi;
#pragma unroll
          for (int c = 0; c < VW; ++c) vc[i][c] = live ? vc[i][c] : 0u;
        }
      }
    }
    if (more) {
      locate(r0 + kPass);
      load_k();
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
      const float x = sc[i];
      sc[i] = __builtin_amdgcn_exp2f(x - ref);
      sum += sc[i];
      if constexpr (I8) sc[i] = x == -INFINITY ? 0.0f : sc[i] * vs[i];  // a scale no row attends may be NaN
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
        a[k] = bf16_bits_to_float(float_to_bf16_bits(sc[i + k]));
        b[k] = bf16_bits_to_float(float_to_bf16_bits(sc[i + k] - a[k]));
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
    if (more) load_v();
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
  auto sums = [&](int r, int e) -> float4& {
    return *reinterpret_cast<float4*>(&ored[w & 1][n][E * (4 * g + r) + e]);
  };
  if (w >= 2) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < E; e += 4)
        sums(r, e) = make_float4(acc[e][r] * f, acc[e + 1][r] * f, acc[e + 2][r] * f, acc[e + 3][r] * f);
  }
  __syncthreads();
  if (w < 2) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        float4 o = sums(r, e);
        o.x += acc[e][r] * f;
        o.y += acc[e + 1][r] * f;
        o.z += acc[e + 2][r] * f;
        o.w += acc[e + 3][r] * f;
        sums(r, e) = o;
      }
  }
  __syncthreads();
  // ---- rows of D: thread tid has eight dimensions of a row
  for (int i = tid; i < rows * D / 8; i += 256) {
    const int r = i / (D / 8), d0 = 8 * (i % (D / 8));
    const float mr = fmaxf(fmaxf(om[0][r], om[1][r]), fmaxf(om[2][r], om[3][r]));
    const float rref = mr == -INFINITY ? 0.0f : mr;
    float den = 0.0f, x[8];
#pragma unroll
    for (int k = 0; k < 4; ++k) den += ol[k][r] * __builtin_amdgcn_exp2f(om[k][r] - rref);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = ored[0][r][d0 + k] + ored[1][r][d0 + k];
    if (ks.pieces > 1) {
      const int64_t piece = ((int64_t)j * p.row_pieces + slot) * p.max_rows + r;
      float4* dst = reinterpret_cast<float4*>(p.part + piece * D + d0);
      dst[0] = make_float4(x[0], x[1], x[2], x[3]);
      dst[1] = make_float4(x[4], x[5], x[6], x[7]);
      if (d0 == 0) p.part_ml[piece] = make_float2(mr, den);
    } else {
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        o[k] = (uint32_t)float_to_bf16_bits(den == 0.0f ? 0.0f : x[2 * k] / den) |
               ((uint32_t)float_to_bf16_bits(den == 0.0f ? 0.0f : x[2 * k + 1] / den) << 16);
      uint16_t* dst = p.out + (int64_t)(tl.q0 + r / p.group) * p.ldo + (int64_t)(j * p.group + r % p.group) * D + d0;
      *reinterpret_cast<uint4*>(dst) = make_uint4(o[0], o[1], o[2], o[3]);
    }
  }
}

// The pieces of a sequence's rows, one workgroup for all of them: D / 4 threads have four
// dimensions of a row each, and where there are few rows several such groups add
// every G-th piece; the groups' sums are added in order.  6 to 7 us, of which the launch
// and finding the pieces are 5; a workgroup for each row took 15 of 40 x 4 sequences' heads.
template <int D>
__device__ __forceinline__ void join_rows(const PagedAttnParams& p, int seq, int j) {
  constexpr int T = D / 4, S = 1024 / T;
  __shared__ float4 red[S][T];
  RowWork work;
  if (!row_work(p, -1, seq, &work)) return;  // whole workgroup
  const int rows = work.t.q_len * p.group, pieces = work.ks.pieces;
  if (pieces == 1) return;  // written already
  int G = S;
  while (G * rows > S) G >>= 1;
  const int s = threadIdx.x / T, t = threadIdx.x % T, r = s / G, g = s % G;
  const int64_t base = ((int64_t)j * p.row_pieces + work.slot0) * p.max_rows + min(r, rows - 1);
  float m = -INFINITY, den = 0.0f;
  for (int i = t; i < pieces; i += T) m = fmaxf(m, p.part_ml[base + (int64_t)i * p.max_rows].x);
#pragma unroll
  for (int k = T / 2; k >= 1; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
  const float ref = m == -INFINITY ? 0.0f : m;
  for (int i = t; i < pieces; i += T) {
    const float2 ml = p.part_ml[base + (int64_t)i * p.max_rows];
    den += ml.y * __builtin_amdgcn_exp2f(ml.x - ref);
  }
#pragma unroll
  for (int k = T / 2; k >= 1; k >>= 1) den += __shfl_xor(den, k);
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = g; i < pieces; i += G) {
    const int64_t at = base + (int64_t)i * p.max_rows;
    const float f = __builtin_amdgcn_exp2f(p.part_ml[at].x - ref);
    const float4 x = reinterpret_cast<const float4*>(p.part + at * D)[t];
    o.x += x.x * f;
    o.y += x.y * f;
    o.z += x.z * f;
    o.w += x.w * f;
  }
  red[s][t] = o;
  __syncthreads();
  if (g != 0 || r >= rows) return;
  for (int i = 1; i < G; ++i) {
    const float4 x = red[s + i][t];
    o.x += x.x;
    o.y += x.y;
    o.z += x.z;
    o.w += x.w;
  }
  auto bits = [&](float x) { return (uint32_t)float_to_bf16_bits(den == 0.0f ? 0.0f : x / den); };
  uint16_t* dst = p.out + (int64_t)(work.t.q0 + r / p.group) * p.ldo + (int64_t)(j * p.group + r % p.group) * D + 4 * t;
  *reinterpret_cast<uint2*>(dst) = make_uint2(bits(o.x) | (bits(o.y) << 16), bits(o.z) | (bits(o.w) << 16));
}

// ------------------------------------------------------------------ more than 16 rows

constexpr int kTile = 128;     // rows of a workgroup
typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

__device__ v4i kZeros = {0, 0, 0, 0};  // what stands for a row that is not read
typedef const __attribute__((address_space(1))) v4i* GlobalVec;

// Tiles of sequence s, of the sequences of more than 16 rows.
__device__ __forceinline__ uint32_t tiles_of(const PagedAttnParams& p, int s) {
  Seq t;
  if (s >= p.batch.n_seqs || !seq_at(p, p.batch.q_start[s], p.batch.q_start[s + 1], 0, &t)) return 0;
  const int rows = t.q_len * p.group;
  return rows > kRows ? (uint32_t)((rows + kTile - 1) / kTile) : 0u;
}
// all tiles of the batch
__device__ __forceinline__ int count_tiles(const PagedAttnParams& p) {
  uint32_t n = 0;
  for (int base = 0; base < p.batch.n_seqs; base += kWave) n += tiles_of(p, base + lane_id());
  return (int)min(total(n), (uint32_t)p.tile_slots);  // fewer than counted only where sequences overlap
}
// tile number `tile`, sequence by sequence; false: none
__device__ __forceinline__ bool tile_of(const PagedAttnParams& p, int tile, Seq* t, int* seq, int* row0) {
  uint32_t before = 0;
  for (int base = 0; base < p.batch.n_seqs; base += kWave) {
    const uint32_t mine = tiles_of(p, base + lane_id()), upto = before + wave_scan(mine);
    const uint64_t hit = __ballot(upto - mine <= (uint32_t)tile && (uint32_t)tile < upto);
    if (hit) {
      const int at = __builtin_ctzll(hit);
      *seq = base + at;
      *row0 = (tile - __builtin_amdgcn_readlane((int)(upto - mine), at)) * kTile;
      return seq_of(p, base + at, t);
    }
    before = (uint32_t)__builtin_amdgcn_readlane((int)upto, kWave - 1);
  }
  return false;
}

__device__ __forceinline__ v16f mma32_bf16(v4i a, v4i b, v16f c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
// v of this lane and of the one 32 away
__device__ __forceinline__ float max32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// v, as something that the compiler cannot form ahead of the loop: what a single
// instruction makes of it would be held in a register each.
__device__ __forceinline__ int here(int v) {
  asm volatile("" : "+v"(v));
  return v;
}
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {  // one v_cvt_pk_bf16_f32
  return __builtin_bit_cast(uint32_t, v2bf{(__bf16)lo, (__bf16)hi});
}
// 16 bytes a lane from memory into LDS at `lds` (wave-uniform) + 16 * lane, without a
// register.  In assembly because the compiler, which cannot tell the two buffers
// apart, waits for the builtin's loads before the transposing reads of the present
// tile; the wait is at the barrier that ends the buffer's filling.
__device__ __forceinline__ void load_lds16(GlobalVec src, uint32_t lds) {
  lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(src), "s"(lds) : "m0", "memory");
}
// N such loads 1024 bytes apart, both in LDS and from `from` (wave-uniform); load i at
// lane offset off ^ (s1 if i is odd) ^ (s2 if i >= 2).
template <int N>
__device__ __forceinline__ void load_lds16_rows(const char* from, uint32_t off, uint32_t s1, uint32_t s2, uint32_t lds) {
  const uint64_t f = (uint64_t)(uintptr_t)from;
  const uint64_t base = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(f >> 32)) << 32) |
                        (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)f);
  lds = (uint32_t)__builtin_amdgcn_readfirstlane((int)lds);
  if constexpr (N == 4)
    asm volatile("s_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %4\n\tglobal_load_lds_dwordx4 %1, %4 offset:1024\n\t"
                 "global_load_lds_dwordx4 %2, %4 offset:2048\n\tglobal_load_lds_dwordx4 %3, %4 offset:3072"
                 : : "v"(off), "v"(off ^ s1), "v"(off ^ s2), "v"(off ^ s1 ^ s2), "s"(base), "s"(lds) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2\n\tglobal_load_lds_dwordx4 %1, %2 offset:1024"
                 : : "v"(off), "v"(off ^ s1), "s"(base), "s"(lds) : "m0", "memory");
}
// 128 rows of a sequence.  Eight waves, four row groups of 32 rows times two key
// groups: key group k takes the 32-key tiles k, k + 2, ... of the piece, from its
// own half of LDS, where the tile after the present one is being put meanwhile.
// With 32 x 32 products a wave's scores (keys x rows) leave each lane 16 keys of one
// row; as bf16 they are the second operand of the value product (dimensions x
// keys) times (keys x rows), whose first operand the transposing LDS read takes
// from value rows as they lie.  Rows of a tile are D bf16 values, the 16-byte chunks of
// a key row at index ^ (row % 16), of a value row at index ^ (4 (row % 4)), so that
// what is read in one cycle (the same chunk of 16 key rows; 64 bytes of four value
// rows) covers the 64 banks once.  INT8 codes become
// bf16 (exactly) on the way into LDS, once for the four row groups; a key's scale
// multiplies its scores, a value's its weight.  The weights are rounded to bf16, each
// by half a step (2^-8 of it) at most and independently of the others, which moves
// results about as much as their own rounding to bf16 does (the two together: 0.0023 of the
// results' size, the latter alone 0.0016, over 8192 positions).
// The reference of the exponentials follows the running maximum only when that
// has grown by 2^8, so that the outputs are seldom rescaled (binary32 sums have the
// room, and the rounding of the weights is relative).
//
// 8192 tokens of one prompt, 4 heads of 256, bf16: 160 us, 0.86 PFLOP/s of the pairs
// that are attended, where a large library product reaches 1.27.  A step of 64 keys takes
// 5100 cycles of a SIMD: 2 x 1024 of matrix instructions (40 %), and between them the reads
// of LDS, 100 vector instructions and 16 exponentials of 4 cycles and more a wave (all
// vector instructions: 30 %), and two barriers; the waves wait for those and for loads 27 %
// of their time, and as long for their turn to issue.  509 tokens over 8192 positions, 16
// heads of 128, INT8: 73 us, of whose cycles vector instructions (codes to bf16, two scales,
// weights) take 40 % and matrix instructions 19 %; the waves wait 44 % of their time, and
// a fifth of LDS' busy cycles are bank conflicts.  INT8 heads of 256 do not fit their
// registers (19 of 256 spilled, 76 bytes a lane): the prompt of 8192 tokens takes 252 us a
// call, where bf16 takes 169.
template <int D, bool I8>
__global__ __launch_bounds__(512) void attn_tile_kernel(PagedAttnParams p) {
  constexpr int NC = D / 16, NB = D / 32;  // 16-dimension steps of a score, 32-dimension blocks of a result
  constexpr int ROWL = 2 * D, TILEB = kStep * ROWL;          // bytes of a row and of a tile in LDS
  constexpr int ROWG = I8 ? D : 2 * D;                       // ... of a cached row
  constexpr int LOADS = 8 * ROWG / 1024;                     // 16-byte loads of a lane for its wave's 8 rows
  extern __shared__ __attribute__((aligned(16))) char smem[];
  // [key group][buffer][key | value] tiles, then [key group][tile % 4][keys' 32 | values' 32] scales
  float* scales = reinterpret_cast<float*>(smem + 8 * TILEB);

  Seq tl;
  int seq, row0;
  // The workgroups with work come first, without gaps: what is one round of the CUs is
  // spread evenly over them.  With empty ones between, some of 256 equal pieces waited for
  // another's end (64 tiles over 8192 keys: 126 us instead of 76).
  const int n_tiles = count_tiles(p);
  const uint32_t id = blockIdx.x + gridDim.x * (blockIdx.y + gridDim.y * blockIdx.z);
  if (n_tiles == 0 || id >= (uint32_t)n_tiles * gridDim.y * gridDim.z) return;
  const int slot = n_tiles - 1 - (int)(id % n_tiles);  // the longest ranges of keys first
  const int j = (int)(id / n_tiles % gridDim.y), split = (int)(id / n_tiles / gridDim.y);
  if (!tile_of(p, slot, &tl, &seq, &row0)) return;  // whole workgroup
  const int rows = tl.q_len * p.group;
  const Keys ks = keys_of(p, tl, row0, min(row0 + kTile, rows) - 1, p.tile_piece);
  if (split >= ks.pieces) return;
  const int begin = ks.begin + split * p.tile_piece, lo = ks.lo, hi = piece_end(begin, ks.hi, p.tile_piece);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = lane_id(), n = l & 31, g = l >> 5;
  const int rg = w & 3, kg = w >> 2;
  const int wrow = row0 + 32 * rg, row = wrow + n;       // the wave's first row, the lane's row
  const int pos = row < rows ? tl.first + row / p.group : -1;
  const int from = pos < 0 ? 0 : max(0, pos + 1 - p.window);
  const bool any = wrow < rows;                           // wave-uniform, as the next two
  const int pos0 = tl.first + wrow / p.group, pos1 = tl.first + min(wrow + 31, rows - 1) / p.group;
  const ConstInts table = (ConstInts)(p.batch.table + (int64_t)seq * p.batch.max_pages);
  const int page_mask = (1 << p.kv.page_log2) - 1;

  // maxima are taken of unscaled scores: a negative scale's sign goes into the queries
  const float scale = fabsf(p.scale_log2);
  const int flip = p.scale_log2 < 0.0f ? (int)0x80008000u : 0;
  v4i q[NC];
  {
    const int r = min(row, rows - 1);
    const uint16_t* src = p.q + (int64_t)(tl.q0 + r / p.group) * p.ldq + (int64_t)(j * p.group + r % p.group) * D + 8 * g;
#pragma unroll
    for (int c = 0; c < NC; ++c) q[c] = *reinterpret_cast<const v4i*>(src + 16 * c) ^ flip;
  }

  char* const mine = smem + kg * 4 * TILEB;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)mine + 8 * rg * ROWL;
  // where chunk 0 of row r of a tile lies in it: v = 0 keys, 1 values (the rest by xor)
  auto swizzle = [](int r, int v) { return v ? 4 * (r & 3) : r & 15; };
  constexpr int kChunks = ROWL / 16, kRowsLoad = 64 / kChunks;  // bf16: rows of a load
  v4i raw[I8 ? 2 * LOADS : 1];  // INT8: codes on their way, keys then values
  float raw_s = 0.0f;           // and scales: lane n of the keys, lane 32 + n of the values
  // pages of the two halves of a tile; -1 past the end or not held
  struct Pages {
    int a, b;
  };
  auto page_at = [&](int k0) {
    const int id = k0 < hi ? table[k0 >> p.kv.page_log2] : -1;
    return id < p.kv.n_pages ? max(id, -1) : -1;
  };
  auto pages = [&](int k0) { return Pages{page_at(k0), page_at(k0 + 16)}; };
  // The wave's 8 rows of the tile at k0 (they lie in one page) on their way: keys
  // (v = 0), values (v = 1), bf16 straight to buffer b.
  auto stage = [&](int k0, Pages pg, int b, int v) {
    const int id = rg >= 2 ? pg.b : pg.a, key = k0 + 8 * rg;
    const int64_t at = (((int64_t)max(id, 0) * p.kv.n_kv + j) << p.kv.page_log2) + (key & page_mask);
    const char* base = reinterpret_cast<const char*>(v ? p.kv.v : p.kv.k) + at * ROWG;
    if constexpr (I8) {  // whatever the rows hold: codes are finite, and what none attends has weight 0
#pragma unroll
      for (int i = 0; i < LOADS; ++i) raw[v * LOADS + i] = *(GlobalVec)(base + (uint32_t)(16 * l) + 1024 * i);
    } else if (id >= 0 && key >= lo && key + 8 <= hi) {  // all of them; wave-uniform
      const int ln = here(l), r = ln / kChunks;
      load_lds16_rows<LOADS>(base, r * ROWG + 16 * ((ln % kChunks) ^ swizzle(8 * rg + r, v)), 16 * swizzle(kRowsLoad, v),
                             16 * swizzle(2 * kRowsLoad, v), lds0 + (2 * b + v) * TILEB);
    } else {
#pragma unroll 1
      for (int i = 0; i < LOADS; ++i) {
        const int idx = 64 * i + here(l), r = idx / kChunks, c = idx % kChunks;
        uint64_t src = (uint64_t)(uintptr_t)(base + r * ROWG + 16 * (c ^ swizzle(8 * rg + r, v)));
        src = id >= 0 && key + r >= lo && key + r < hi ? src : (uint64_t)(uintptr_t)&kZeros;
        load_lds16((GlobalVec)(uintptr_t)src, lds0 + (2 * b + v) * TILEB + 1024 * i);
      }
    }
  };
  // INT8: scales of the keys at k0 and of the values at v0
  auto stage_scales = [&](int k0, Pages pk, int v0, Pages pv) {
    if constexpr (I8) {
      if (rg == 0) {
        const int key = (g ? v0 : k0) + n, id = g ? (n < 16 ? pv.a : pv.b) : (n < 16 ? pk.a : pk.b);
        const bool live = id >= 0 && key >= lo && key < hi;
        const int64_t a = ((int64_t)id * p.kv.n_kv + j) * (page_mask + 1) + (key & page_mask);
        raw_s = live ? (g ? p.kv.sv : p.kv.sk)[a] : 0.0f;
      }
    }
  };
  // INT8: the staged codes into buffer b as bf16, the scales into set t % 4 (keys) or
  // (t - 1) % 4 (values, one tile behind)
  auto put = [&](int b, int v) {
    if constexpr (I8) {
#pragma unroll
      for (int i = 0; i < LOADS; ++i) {
        const int idx = 64 * i + here(l), r = idx / (ROWG / 16), c = idx % (ROWG / 16);
        const v4i u = raw[v * LOADS + i];
        const uint32_t x[4] = {(uint32_t)u.x, (uint32_t)u.y, (uint32_t)u.z, (uint32_t)u.w};
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[2 * e] = (uint32_t)pair_hi(byte_f(x[e], 0), byte_f(x[e], 1));
          o[2 * e + 1] = (uint32_t)pair_hi(byte_f(x[e], 2), byte_f(x[e], 3));
        }
        char* dst = mine + (2 * b + v) * TILEB + (8 * rg + r) * ROWL;
        const int z = swizzle(8 * rg + r, v);
        *reinterpret_cast<uint4*>(dst + 16 * ((2 * c) ^ z)) = make_uint4(o[0], o[1], o[2], o[3]);
        *reinterpret_cast<uint4*>(dst + 16 * ((2 * c + 1) ^ z)) = make_uint4(o[4], o[5], o[6], o[7]);
      }
    }
  };
  auto put_scales = [&](int tk, int tv) {
    if constexpr (I8) {
      if (rg == 0) scales[(kg * 4 + ((g ? tv : tk) & 3)) * 64 + l] = raw_s;
    }
  };

  float ref = -INFINITY, sum = 0.0f;
  v16f acc[NB];  // dimensions 32 b + 8 (r / 4) + 4 g + r % 4 of row n
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[b][r] = 0.0f;

  // LDS addresses: chunk 2 c + g of key row n, at (2 c + g) ^ (n % 16); chunk 4 i + low of
  // the value rows vr = 4 g + (l % 16) / 4 (+ 8, + 16 h), at (4 i + low) ^ (4 (vr % 4)), whose
  // four dimensions are 32 i + 16 ((l / 16) % 2) + 4 (l % 4) and up
  const int vr = 4 * g + ((l >> 2) & 3);
  const int koff = n * ROWL + 16 * (g ^ (n & 15));
  const int voff = TILEB + vr * ROWL + 8 * (l & 1) + 16 * (2 * ((l >> 4) & 1) + ((l >> 1) & 1)) + 64 * (vr & 3);

  // h0, h1: the two pages held; whole: every row attends every key
  v16f s;     // a tile's scores
  v4i pw[2];  // a tile's weights
  auto key_frag = [&](const char* buf, int ko, int c) {
    return *reinterpret_cast<const v4i*>(buf + (ko ^ (32 * (c & 7))) + 256 * (c >> 3));
  };
  auto value_frag = [&](const char* buf, int vo, int u) {
    const int h = u / NB, i = u % NB;
    const char* a = buf + (vo ^ (64 * (i & 3))) + 16 * h * ROWL + 256 * (i >> 2);
    typedef __attribute__((address_space(3))) v4s* lds4;
    const v4s lo4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)a), hi4 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(a + 8 * ROWL));
    const int2 x = __builtin_bit_cast(int2, lo4), y = __builtin_bit_cast(int2, hi4);
    return v4i{x.x, x.y, y.x, y.y};
  };
  // Matrix products: scores of the tile in key buffer kb and, do_v, the value product
  // of the weights with value buffer vb, in turn (the scores are one chain, whose
  // latency the others fill); the reads of LDS some products ahead.  One form for all
  // tiles of the loop, seen or not (weights of 0): with a branch around the
  // products the compiler moves the 128 output registers about.
  auto products = [&](auto do_s, auto do_v, int kb, int vb) {
    constexpr bool DS = decltype(do_s)::value, DV = decltype(do_v)::value;
    constexpr int AH = DS && DV ? 2 : 3;
    static_assert(NC == 2 * NB, "as many products either way");
    const char* kbuf = mine + 2 * kb * TILEB;
    const char* vbuf = mine + 2 * vb * TILEB;
    const int ko = here(koff), vo = here(voff);
    v4i kf[AH], vf[AH];
    if constexpr (DS) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = 0.0f;
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < NC + AH; ++t) {
      const int u = t - AH;
      if (u >= 0) {
        if constexpr (DS) s = mma32_bf16(kf[u % AH], q[u], s);
        if constexpr (DV) acc[u % NB] = mma32_bf16(vf[u % AH], pw[u / NB], acc[u % NB]);
      }
      if (t < NC) {
        if constexpr (DS) kf[t % AH] = key_frag(kbuf, ko, t);
        if constexpr (DV) vf[t % AH] = value_frag(vbuf, vo, t);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Scores to weights.  h0, h1: the two pages held; whole: every row attends every key.
  auto weights = [&](int k0, int t, bool h0, bool h1, bool whole) {
    const float* sc = scales + (kg * 4 + (t & 3)) * 64 + 4 * g;
    float x[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) x[r] = s[r];
    if constexpr (I8) {
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float4 f = *reinterpret_cast<const float4*>(sc + 2 * r);
        x[r] *= f.x; x[r + 1] *= f.y; x[r + 2] *= f.z; x[r + 3] *= f.w;
      }
    }
    if (!whole) {  // keys from .. min(pos, hi - 1): one unsigned comparison each
      const int span = min(pos, hi - 1) - from;
      const uint32_t limit = (uint32_t)(span + 1), u = (uint32_t)(k0 + 4 * g - from);
#pragma unroll
      for (int r = 0; r < 16; ++r)
        x[r] = u + 8 * (r >> 2) + (r & 3) < (span >= 0 && (r < 8 ? h0 : h1) ? limit : 0u) ? x[r] : -INFINITY;
    }
    float mx = x[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, x[r]);
    mx = max32(mx) * scale;
    if (__any(mx > ref + 8.0f)) {
      const float next = fmaxf(ref, mx), corr = next == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - next);
      ref = next;
      sum *= corr;
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][r] *= corr;
    }
    const float m = ref == -INFINITY ? 0.0f : ref;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], scale, -m));
      sum += x[r];
    }
    if constexpr (I8) {
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const float4 f = *reinterpret_cast<const float4*>(sc + 32 + 2 * r);
        x[r] *= f.x; x[r + 1] *= f.y; x[r + 2] *= f.z; x[r + 3] *= f.w;
      }
      if (!whole) {  // a scale that this row does not attend may be NaN
        const int last = min(pos, hi - 1) - k0 - 4 * g, first = from - k0 - 4 * g;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int key = 8 * (r >> 2) + (r & 3);
          x[r] = key >= first && key <= last ? x[r] : 0.0f;
        }
      }
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
      pw[h] = v4i{(int)pack2(x[8 * h], x[8 * h + 1]), (int)pack2(x[8 * h + 2], x[8 * h + 3]),
                  (int)pack2(x[8 * h + 4], x[8 * h + 5]), (int)pack2(x[8 * h + 6], x[8 * h + 7])};
  };
  auto sync = []() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
    __builtin_amdgcn_sched_barrier(0);
  };

  // The two key groups' waves of a row group share a SIMD, half a tile apart: while
  // one is in its matrix products (values of a tile with scores of the next), the
  // other forms weights and sends for the tiles to come, so that matrix and vector
  // units work at the same time.  Tile t's keys and values are in the buffers t % 2; the
  // keys of t + 2 and the values of t + 1 are sent for as soon as those of t and t - 1
  // have been used.
  const int n_it = (hi - begin + 2 * kStep - 1) / (2 * kStep);
  const int key0 = begin + kStep * kg;
  auto sees = [&](int k0, Pages pg) {
    return any && k0 <= pos1 && k0 < hi && k0 + kStep > pos0 + 1 - p.window && max(pg.a, pg.b) >= 0;
  };
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  Pages pg0 = pages(key0), pg1 = pages(key0 + 2 * kStep), pg2 = pages(key0 + 4 * kStep);
  stage(key0, pg0, 0, 0);
  stage(key0, pg0, 0, 1);
  stage_scales(key0, pg0, key0, pg0);
  put(0, 0);
  put(0, 1);
  put_scales(0, 0);
  stage(key0 + 2 * kStep, pg1, 1, 0);
  stage_scales(key0 + 2 * kStep, pg1, key0, pg0);
  put(1, 0);
  put_scales(1, 0);
  __builtin_amdgcn_s_waitcnt((15 << 8) | (7 << 4));
  sync();
  if (kg == 1) sync();
  products(yes, no, 0, 0);
  if constexpr (I8) {  // the codes go through registers, half a step earlier
    stage(key0 + 4 * kStep, pg2, 0, 0);
    stage(key0 + 2 * kStep, pg1, 1, 1);
    stage_scales(key0 + 4 * kStep, pg2, key0 + 2 * kStep, pg1);
  }
  for (int t = 0; t < n_it; ++t) {
    const int k0 = key0 + 2 * kStep * t;
    sync();
    // weights of tile t
    const Pages pg3 = pages(k0 + 6 * kStep);  // here, so that the wait at the step's end finds it done
    if constexpr (!I8) {  // past the end: zeros, so that there are as many loads
      stage(k0 + 4 * kStep, pg2, t & 1, 0);
      stage(k0 + 2 * kStep, pg1, (t + 1) & 1, 1);
    }
    if (sees(k0, pg0))
      weights(k0, t, pg0.a >= 0, pg0.b >= 0, min(pg0.a, pg0.b) >= 0 && k0 + kStep - 1 <= pos0 && k0 > pos1 - p.window && k0 + kStep <= hi);
    else
      pw[0] = pw[1] = v4i{0, 0, 0, 0};
    put(t & 1, 0);
    put((t + 1) & 1, 1);
    put_scales(t + 2, t + 1);
    // the loads before this step's
    if constexpr (!I8) __builtin_amdgcn_s_waitcnt(((2 * LOADS) & 15) | (7 << 4) | (15 << 8));
    sync();
    // values of tile t, scores of tile t + 1 (behind the last: scores that nobody uses)
    __builtin_amdgcn_s_setprio(1);
    products(yes, yes, (t + 1) & 1, t & 1);
    __builtin_amdgcn_s_setprio(0);
    if constexpr (I8) {  // into registers while the last products are on, for the next step to put
      stage(k0 + 6 * kStep, pg3, (t + 1) & 1, 0);
      stage(k0 + 4 * kStep, pg2, t & 1, 1);
      stage_scales(k0 + 6 * kStep, pg3, k0 + 4 * kStep, pg2);
    }
    pg0 = pg1;
    pg1 = pg2;
    pg2 = pg3;
  }
  if (kg == 0) sync();

  // ---- the two key groups
  sum = sum32(sum);
  __builtin_amdgcn_s_waitcnt((15 << 8) | (7 << 4));  // the last loads into LDS, which takes the outputs now
  __syncthreads();
  int lane = threadIdx.x;  // from here on: what the loop need not hold registers for
  asm volatile("" : "+v"(lane));
  lane &= 63;
  const int ln = lane & 31, lg = lane >> 5, lrow = wrow + ln;
  float4* ex = reinterpret_cast<float4*>(smem) + rg * (64 * NB * 4);
  float2* exm = reinterpret_cast<float2*>(smem + 8 * TILEB) ;  // where the scales were: 4 x 32 pairs
  if (kg == 1) {
#pragma unroll
    for (int i = 0; i < NB; ++i)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        ex[(i * 4 + r / 4) * 64 + lane] = make_float4(acc[i][r], acc[i][r + 1], acc[i][r + 2], acc[i][r + 3]);
    if (lg == 0) exm[32 * rg + ln] = make_float2(ref, sum);
  }
  __syncthreads();
  if (kg == 1 || !any) return;
  const float2 o = exm[32 * rg + ln];
  const float top = fmaxf(ref, o.x), m = top == -INFINITY ? 0.0f : top;
  const float f0 = __builtin_amdgcn_exp2f(ref - m), f1 = __builtin_amdgcn_exp2f(o.x - m);
  sum = sum * f0 + o.y * f1;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  const int64_t part = (((int64_t)slot * p.kv.n_kv + j) * p.max_tile_pieces + split);
  float4* dst = reinterpret_cast<float4*>(p.tile_part) + (part * 4 + rg) * (64 * NB * 4) + lane;
  uint16_t* out = p.out + (int64_t)(tl.q0 + lrow / p.group) * p.ldo + (int64_t)(j * p.group + lrow % p.group) * D + 4 * lg;
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const float4 e = ex[(i * 4 + r / 4) * 64 + lane];
      const float4 x = make_float4(acc[i][r] * f0 + e.x * f1, acc[i][r + 1] * f0 + e.y * f1, acc[i][r + 2] * f0 + e.z * f1, acc[i][r + 3] * f0 + e.w * f1);
      if (ks.pieces > 1)
        dst[(i * 4 + r / 4) * 64] = x;
      else if (lrow < rows)
        *reinterpret_cast<uint2*>(out + 32 * i + 2 * r) = make_uint2(pack2(x.x * inv, x.y * inv), pack2(x.z * inv, x.w * inv));
    }
  if (ks.pieces > 1 && lg == 0) p.tile_ml[part * kTile + 32 * rg + ln] = make_float2(top, sum);
}

// The pieces of a tile: four waves join 32 rows, each a quarter of their dimensions, in
// the layout the pieces are in (11 us for the 43 MB of the prompt of 8192 tokens,
// whose pieces the memory-side cache holds).
template <int D>
__device__ __forceinline__ void join_tile(const PagedAttnParams& p, int slot, int j) {
  constexpr int NB = D / 32, Q = NB;  // float4 of a lane (NB * 4 / 4 waves)
  Seq tl;
  int seq, row0;
  const int rg = threadIdx.x >> 8, w = (threadIdx.x >> 6) & 3, l = lane_id(), n = l & 31, g = l >> 5;
  if (!tile_of(p, slot, &tl, &seq, &row0)) return;
  const int rows = tl.q_len * p.group, row = row0 + 32 * rg + n;
  if (row0 + 32 * rg >= rows) return;
  const int pieces = keys_of(p, tl, row0, min(row0 + kTile, rows) - 1, p.tile_piece).pieces;
  if (pieces == 1) return;  // written already
  const int64_t part = ((int64_t)slot * p.kv.n_kv + j) * p.max_tile_pieces;
  const float2* ml = p.tile_ml + part * kTile + 32 * rg + n;
  const float4* src = reinterpret_cast<const float4*>(p.tile_part) + (part * 4 + rg) * (64 * NB * 4) + w * Q * 64 + l;
  float top = -INFINITY, sum = 0.0f;
  for (int i = 0; i < pieces; ++i) top = fmaxf(top, ml[(int64_t)i * kTile].x);
  const float m = top == -INFINITY ? 0.0f : top;
  float4 acc[Q];
#pragma unroll
  for (int k = 0; k < Q; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 2
  for (int i = 0; i < pieces; ++i) {
    const float2 x = ml[(int64_t)i * kTile];
    const float f = __builtin_amdgcn_exp2f(x.x - m);
    sum += x.y * f;
#pragma unroll
    for (int k = 0; k < Q; ++k) {
      const float4 v = src[(int64_t)i * 4 * (64 * NB * 4) + k * 64];
      acc[k].x += v.x * f;
      acc[k].y += v.y * f;
      acc[k].z += v.z * f;
      acc[k].w += v.w * f;
    }
  }
  if (row >= rows) return;
  const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
  uint16_t* out = p.out + (int64_t)(tl.q0 + row / p.group) * p.ldo + (int64_t)(j * p.group + row % p.group) * D + 4 * g;
#pragma unroll
  for (int k = 0; k < Q; ++k)  // float4 w * Q + k: dimensions 8 of it
    *reinterpret_cast<uint2*>(out + 8 * (w * Q + k)) = make_uint2(pack2(acc[k].x * inv, acc[k].y * inv), pack2(acc[k].z * inv, acc[k].w * inv));
}

// Both joins in one launch, as either is mostly its launch.
template <int D>
__global__ __launch_bounds__(1024) void attn_join_kernel(PagedAttnParams p) {
  const int seqs = p.row_pieces ? p.batch.n_seqs : 0;
  if ((int)blockIdx.x < seqs)
    join_rows<D>(p, blockIdx.x, blockIdx.y);
  else
    join_tile<D>(p, blockIdx.x - seqs, blockIdx.y);
}

// ------------------------------------------------------------------ launches

// Row kernel: workgroups that the CUs hold at once, two each (pieces for three: 64 long
// contexts 56 us instead of 50, and as long where registers would let three in).
static constexpr int64_t kRowSlots = 512;
// Tile kernel: pieces for one workgroup a CU, which is what one holds; for two where the
// new tokens may be most of the context, as the keys of a prompt's tiles then differ from
// few to all (one tile of a piece each: 200 us of the prompt of 8192 tokens instead of
// 160).  Of 512 keys and more: a piece writes its 128 rows in binary32 and they are read
// again to be joined.
//
// The pieces of tiles follow from what the tables can hold, as the host knows no lengths:
// the prompt above takes 172 us a call with a table of 8192 positions and 193 with one of
// 32768 or more, a chunk of 509 tokens over 8192 positions (16 heads on 8 of 128, INT8) 102
// and 248.  Tiles of few rows cost as much as full ones: 64 sequences of 8 tokens with 4
// heads of 256 over 2325 to 16384 positions take 255 us, where one token each takes 59.
static constexpr int kTileSlots = 256, kTilePieceMin = 512;

void attn_paged_plan(PagedAttnParams* p, int64_t max_q, int64_t ctx_max) {
  // keys of any row and its neighbours; no key lies behind the 2^30 positions of the largest table
  const int64_t span = std::min<int64_t>(std::min<int64_t>(ctx_max, (int64_t)p->window + max_q) + kStep, 1 << 30);
  p->max_q = (int)max_q;
  p->max_rows = (int)std::min<int64_t>(max_q * p->group, kRows);
  // Pieces for each key/value head: the slots, or of more sequences than slots two rounds
  // of them.  More than that are not cut, which serves contexts of like lengths: of 129
  // sequences of 8 heads, one of 32768 positions among ones of 200 to 500, the long one is one
  // workgroup a head and takes 422 us.  Nor is it cut where the sequences take all slots
  // (128 such: 854 us).
  const int64_t rounds = (p->batch.n_seqs * (int64_t)p->kv.n_kv + kRowSlots - 1) / kRowSlots;
  p->row_pieces = p->batch.n_seqs <= kSplitSeqs && rounds <= 2 && span > kPass ? (int)(kRowSlots * rounds / p->kv.n_kv) : 0;
  p->tile_slots = 0;
  p->tile_piece = p->max_tile_pieces = 1;
  if (max_q * p->group > kRows) {
    // a last tile for each sequence of more than kRows rows
    p->tile_slots = (int)(p->rows * p->group / kTile + std::min<int64_t>(p->batch.n_seqs, p->rows * p->group / (kRows + 1)));
    const int64_t tiles = (p->rows * p->group / kTile + 1) * p->kv.n_kv;
    const int64_t target = 2 * max_q > ctx_max ? 2 * kTileSlots : kTileSlots, most = (target + tiles - 1) / tiles;
    int64_t piece = std::max<int64_t>((span + most - 1) / most, kTilePieceMin);
    piece = (piece + 2 * kStep - 1) / (2 * kStep) * (2 * kStep);
    p->tile_piece = (int)piece;
    p->max_tile_pieces = (int)((span + piece - 1) / piece);
  }
}

// Workspace: outputs of the row kernel's pieces, of the tile kernel's, then their
// maxima and sums.
static size_t row_parts(const PagedAttnParams& p) {
  return (size_t)p.kv.n_kv * p.row_pieces * p.max_rows;
}
static size_t tile_parts(const PagedAttnParams& p) {
  return p.max_tile_pieces == 1 ? 0 : (size_t)p.tile_slots * p.kv.n_kv * p.max_tile_pieces * kTile;
}
size_t attn_paged_ws_bytes(const PagedAttnParams& p, int head_dim) {
  return (row_parts(p) + tile_parts(p)) * (head_dim * sizeof(float) + sizeof(float2));
}

template <int D, bool I8>
static hipError_t tile_launch(const PagedAttnParams& p, hipStream_t st) {
  constexpr int kLds = 8 * kStep * 2 * D + 2048;
  auto kern = attn_tile_kernel<D, I8>;
  if constexpr (kLds > 64 * 1024) {
    static bool attr_set[64] = {};  // by device; benign race: every caller sets the same value
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev >= 64 || !attr_set[dev]) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
      if (e != hipSuccess) return e;
      if (dev < 64) attr_set[dev] = true;
    }
  }
  kern<<<dim3((unsigned)p.tile_slots, (unsigned)p.kv.n_kv, (unsigned)p.max_tile_pieces), 512, kLds, st>>>(p);
  return hipGetLastError();
}

template <int D, bool I8>
static hipError_t paged_launch(PagedAttnParams p, void* ws, hipStream_t st) {
  p.part = reinterpret_cast<float*>(ws);
  p.tile_part = p.part + row_parts(p) * D;
  p.part_ml = reinterpret_cast<float2*>(p.tile_part + tile_parts(p) * D);
  p.tile_ml = p.part_ml + row_parts(p);
  if (p.tile_slots) {
    const hipError_t e = tile_launch<D, I8>(p, st);
    if (e != hipSuccess) return e;
  }
  attn_rows_kernel<D, I8><<<dim3((unsigned)(p.row_pieces ? p.row_pieces : p.batch.n_seqs), (unsigned)p.kv.n_kv), 256, 0, st>>>(p);
  const hipError_t e = hipGetLastError();
  const int64_t joins = (p.row_pieces ? p.batch.n_seqs : 0) + (p.max_tile_pieces > 1 ? p.tile_slots : 0);
  if (e != hipSuccess || joins == 0) return e;
  attn_join_kernel<D><<<dim3((unsigned)joins, (unsigned)p.kv.n_kv), 1024, 0, st>>>(p);
  return hipGetLastError();
}

hipError_t launch_attn_paged(const PagedAttnParams& p, int head_dim, void* ws, hipStream_t st) {
  if (head_dim == 256) return p.kv.sk ? paged_launch<256, true>(p, ws, st) : paged_launch<256, false>(p, ws, st);
  return p.kv.sk ? paged_launch<128, true>(p, ws, st) : paged_launch<128, false>(p, ws, st);
}

}  // namespace w8a8
