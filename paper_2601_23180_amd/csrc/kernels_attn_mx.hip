// Tree-masked grouped-query attention over a context held in 4 bits (layout: mx.hpp) and the draft nodes' own K and V.
//
// For query row r (query head, node) of a kv head: scores s_j = q_r . K_j / sqrt(d) over the context's slots and the row's
// ancestors, one pass over the keys with the running maximum m and l = sum exp(s_j - m), o = sum exp(s_j - m) V_j, result o / l.
// Workgroups take a range of keys each and leave (m, l, o); a second launch adds them up in ascending order.  Short contexts take one workgroup for
// everything, and no second launch.
//
// A wavefront takes 32 keys at a time, straight from the cache to registers: a key's codes are so few bytes that sharing a
// tile through LDS would cost more than converting it once per 16 to 64 query rows.  K Q^T and V^T P^T go through 16 x 16 x 32
// matrix instructions in the transposed form (a query row per lane, so the softmax state is per lane), and the order of the
// reduction is chosen so that nothing moves between lanes: score register e of lane (ln, g) is the key 8 g + e of the
// tile, which is what the second product's operand wants of that lane.  bf16 queries are exact operands and probabilities
// are rounded to bf16, half a step of the result's own type.  fp32 queries and probabilities go as three parts of 8 bits, 24 in all: with two, results were
// off by 3.7e-6 of their size where fp32 torch is off by 8e-7, with three by 6e-7.  In a verification pass they go in two, 16 bits, like the pass's other operands.
//
// What bounds it: for few rows the reading (eight sequences of up to 32768 keys, 8 kv heads of 128, one token: 214 MB, cold, in 44 to 46 us; 285 MB in 46 where part of it lies in
// the last-level cache), launch and first data
// below 4096 keys or so; for many rows no one part (four sequences of 60 nodes and 32 heads over 16384 keys: 82 to 95 us by card, 0.7 to 0.8 PFLOP/s): a run of 32 keys
// under 32 rows is 34 matrix instructions of 16 cycles, about 110 vector instructions of conversion and 60 of softmax, a third of them exponentials.  Timed without the draft
// nodes, 88 us; with the keys' conversion left out 88, the values' 87, both 77, the exponentials 84, the loads 79.  Tried for that and not better: three wavefronts a SIMD (12
// registers spilled: 101); 64 rows a wavefront, which halves the conversions a row and leaves one wavefront a SIMD (106); operands converted once
// for all rows in LDS (86 to 106); each operand converted in front of its product instead of
// all at once (2 to 8 % slower).  Joining the partials in the last workgroup of a row instead of by a second launch: 10.6 + 3.8 us became 19 to 22, since what other
// workgroups wrote has to be read past the L2 in a chain of stamp, maxima and sums.
#include <float.h>

#include "mx.hpp"
#include "plan.hpp"

namespace ts {

namespace {

// Maximum, in natural-log units, that a partial is stored with, as kernels_attn.hip has it: -inf marks a partial without keys, which the
// merge skips; one whose scores are all NaN or all -inf is added up, so that the NaN in its sums reaches the row.
__device__ __forceinline__ float stored_max(float m_log2) { return fmaxf(m_log2 * 0.693147180559945f, -FLT_MAX); }

// A number as NP bf16 parts, each the largest that fits of what is left.  bf16 inputs are one part; fp32 ones three, which is all 24 bits, or
// two (rounded: 16 bits) in a verification pass, whose activations go to every product that way.
template <int NP>
__device__ __forceinline__ void split_value(float x, bf16 (&o)[NP]) {
  if constexpr (NP == 1) {
    o[0] = (bf16)x;
  } else if constexpr (NP == 2) {
    o[0] = (bf16)x;
    o[1] = (bf16)(x - (float)o[0]);
  } else {   // cut off, not rounded: exact, and nothing finite becomes infinite
    const float a = __uint_as_float(__float_as_uint(x) & 0xffff0000u), y = x - a;
    const float b = __uint_as_float(__float_as_uint(y) & 0xffff0000u);
    o[0] = (bf16)a; o[1] = (bf16)b; o[2] = (bf16)(y - b);
  }
}
// Eight queries, keys or values as operands
template <int NP>
__device__ __forceinline__ void split8(const f32x4 &x, const f32x4 &y, bf16x8 (&o)[NP]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    bf16 parts[NP];
    split_value<NP>(e < 4 ? x[e & 3] : y[e & 3], parts);
#pragma unroll
    for (int p = 0; p < NP; ++p) o[p][e] = parts[p];
  }
}
template <int NP>
__device__ __forceinline__ void load_parts(const float *p, bf16x8 (&o)[NP]) { split8<NP>(*(const f32x4 *)p, *(const f32x4 *)(p + 4), o); }
template <int NP>
__device__ __forceinline__ void load_parts(const bf16 *p, bf16x8 (&o)[NP]) {
  static_assert(NP == 1, "bf16 operands are exact");
  o[0] = *(const bf16x8 *)p;
}
// Two probabilities, elements e and e + 1
template <int NP>
__device__ __forceinline__ void prob_parts(f32x2 p, bf16x8 (&o)[NP], int e) {
  f32x2 rest = p;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const bf16x2 h = __builtin_convertvector(rest, bf16x2);
    o[i][e] = h[0]; o[i][e + 1] = h[1];
    if (i + 1 < NP) rest = f32x2{rest[0] - (float)h[0], rest[1] - (float)h[1]};
  }
}

// A wavefront's 32 keys as they lie in the cache, from slot s of block row r.  Lane (ln, g): of key 8 (ln / 4) + 4 t + ln % 4, t = 0, 1,
// the features (D / 4) g .., inside one block; of the keys 8 g .. 8 g + 7 the values of features 64 i + 4 ln .. + 3.
template <int D>
struct KeyCodes {
  uint32_t w[2][D / 32];
  uint32_t scale[2];
  // uniform bases and 32-bit lane offsets: the address arithmetic stays off the vector ALU
  __device__ __forceinline__ void load(const MxMap &m, size_t r, int s, uint32_t ln, uint32_t g) {
    const uint32_t at = 8 * (ln >> 2) + (ln & 3);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t *codes = m.k_codes + MxOffsets<D>::k_codes(m, r, s + 4 * t), *scales = m.k_scales + MxOffsets<D>::k_scales(m, r, s + 4 * t);
      if constexpr (D == 128) {
        const u32x4 x = *(const u32x4 *)(codes + (at * (D / 2) + g * (D / 8)));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[t][i] = x[i];
      } else {
        const u32x2 x = *(const u32x2 *)(codes + (at * (D / 2) + g * (D / 8)));
        w[t][0] = x[0]; w[t][1] = x[1];
      }
      scale[t] = scales[at * (D / 32) + g * (D / 32) / 4];
    }
  }
  // operand of reduction step i for 16 keys: features (D / 4) g + 8 i ..
  __device__ __forceinline__ bf16x8 operand(int t, int i) const { return mx_values(w[t][i], mx_scale(scale[t], 0)); }
};
template <int D>
struct ValueCodes {
  u32x4 w[D / 64];
  u32x2 scale[D / 64];
  __device__ __forceinline__ void load(const MxMap &m, size_t r, int s, uint32_t ln, uint32_t g) {
    const uint8_t *codes = m.v_codes + MxOffsets<D>::v_codes(m, r, s), *scales = m.v_scales + MxOffsets<D>::v_scales(m, r, s);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      w[i] = *(const u32x4 *)(codes + 256 * i + (g * (8 * D / 2) + ln * 16));
      scale[i] = *(const u32x2 *)(scales + 16 * i + (g * (8 * D / 32) + (ln >> 3) * 8));
    }
  }
  // only the first `left` of the lane's eight keys are tokens: the others become element 0 of the smallest scale, whatever lies there
  __device__ __forceinline__ void keep(int left) {
    const uint64_t mask = left <= 0 ? 0 : (left >= 8 ? ~0ull : (1ull << (8 * left)) - 1);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      scale[i][0] &= (uint32_t)mask;
      scale[i][1] &= (uint32_t)(mask >> 32);
#pragma unroll
      for (int x = 0; x < 4; ++x) w[i][x] &= (2 * x < left ? 0xffffu : 0u) | (2 * x + 1 < left ? 0xffff0000u : 0u);
    }
  }
  // operands of the features 64 i + 4 ln + j, j = 0 .. 3: the eight keys of the lane
  __device__ __forceinline__ void operands(int i, bf16x8 (&o)[4]) const {
    uint32_t f[4][4];   // [feature][pair of keys]
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float s0 = mx_scale(scale[i][x >> 1], (2 * x) & 3), s1 = mx_scale(scale[i][x >> 1], (2 * x + 1) & 3);
      union { bf16x2 v; uint32_t u; } a0, a1, b0, b1;   // features 0, 1 and 2, 3 of both keys
      a0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][x], s0, 0); a1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][x], s1, 2);
      b0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][x], s0, 1); b1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i][x], s1, 3);
      f[0][x] = __builtin_amdgcn_perm(a1.u, a0.u, 0x05040100); f[1][x] = __builtin_amdgcn_perm(a1.u, a0.u, 0x07060302);
      f[2][x] = __builtin_amdgcn_perm(b1.u, b0.u, 0x05040100); f[3][x] = __builtin_amdgcn_perm(b1.u, b0.u, 0x07060302);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = __builtin_bit_cast(bf16x8, u32x4{f[j][0], f[j][1], f[j][2], f[j][3]});
  }
};

// RB blocks of 16 query rows of a wavefront: their queries as operands, and the running sums.
//
// Probabilities are powers of two relative to a reference r per row, which is set kHead above the largest score of the row when one
// outgrows it: they stay at 1 and below, nothing finite overflows, and the reference, and with it the sums, moves once or twice on a long
// context instead of with every new maximum (32 rows have one in 60 % of 64 runs of random keys).  Whether a score has outgrown r is seen
// from the probabilities.  The sum of a row's weights comes from the matrix cores as one more feature that is 1.
constexpr float kHead = 8.f;
template <int D, int RB, typename T, int NP>
struct QueryRows {
  static constexpr int ST = D / 32, NV = D / 64, NO = 4 * NV;
  bf16x8 q[RB][ST][NP];   // lane (ln, g): features (D / 4) g + 8 t .. of row ln of each block
  float r[RB];
  f32x4 o[RB][NO + 1];    // o[rb][4 i + j][e]: feature 64 i + 16 g + 4 e + j of row ln; o[rb][NO]: the sum of its weights, four times

  static __device__ __forceinline__ float unit() { return 1.44269504088896f / sqrtf((float)D); }   // scores in powers of two
  __device__ __forceinline__ void start(const MxAttnArgs &a, const T *q0, int first_row, int p_rows, int ln, int g) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int pc = min(first_row + rb * 16 + ln, p_rows - 1), al = pc / a.n_nodes, node = pc - al * a.n_nodes;
      const T *p = q0 + node * a.q.row + al * D + g * (D / 4);
#pragma unroll
      for (int t = 0; t < ST; ++t) load_parts<NP>(p + 8 * t, q[rb][t]);
      r[rb] = -INFINITY;
#pragma unroll
      for (int i = 0; i <= NO; ++i) o[rb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  }
  static __device__ __forceinline__ void clear(f32x4 (&s)[RB][2]) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb][0] = s[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  // scores += step i of the reduction; kf: 2 x 16 keys
  __device__ __forceinline__ void score(f32x4 (&s)[RB][2], const bf16x8 &kf0, const bf16x8 &kf1, int i) const {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        s[rb][0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf0, q[rb][i][p], s[rb][0], 0, 0, 0);
        s[rb][1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf1, q[rb][i][p], s[rb][1], 0, 0, 0);
      }
  }
  // leaves the lane's keys out whose bits are not set
  static __device__ __forceinline__ void mask(f32x4 (&s)[2], uint32_t bits) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!((bits >> e) & 1u)) s[e >> 2][e & 3] = -INFINITY;
  }
  // returns the largest
  static __device__ __forceinline__ float powers(const f32x4 (&s)[2], float ref, bf16x8 (&pf)[NP]) {
    float p[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e >> 2][e & 3], unit(), -ref));   // 0 for a key left out
#pragma unroll
    for (int e = 0; e < 8; e += 2) prob_parts<NP>(f32x2{p[e], p[e + 1]}, pf, e);
    return fmaxf(fmaxf(fmaxf(fmaxf(p[0], p[1]), p[2]), fmaxf(fmaxf(p[3], p[4]), p[5])), fmaxf(p[6], p[7]));
  }
  // scores to probabilities, as operands; the largest, or a number above 1 where a lane has none (keys left out before the first one, NaN scores)
  __device__ __forceinline__ float weigh(const f32x4 (&s)[RB][2], bf16x8 (&pf)[RB][NP]) const {
    float top = 0.f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float t = powers(s[rb], r[rb], pf[rb]);
      top = t <= 1.f ? fmaxf(top, t) : 2.f;
    }
    return top;
  }
  // behind weigh: where a score has outgrown its row's reference, the reference and the sums move and the probabilities are taken again
  __device__ __forceinline__ void settle(const f32x4 (&s)[RB][2], bf16x8 (&pf)[RB][NP], float top) {
    if (__builtin_amdgcn_ballot_w64(top > 1.f) == 0) return;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float t = fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3]));
      t = fmaxf(t, fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3])));
      t = fmaxf(t, __shfl_xor(t, 16, 64));
      t = fmaxf(t, __shfl_xor(t, 32, 64)) * unit();
      const float r_new = t > r[rb] ? t + kHead : r[rb], alpha = t > r[rb] ? __builtin_amdgcn_exp2f(r[rb] - r_new) : 1.f;   // 0 at first
      r[rb] = r_new;
#pragma unroll
      for (int i = 0; i <= NO; ++i) o[rb][i] *= alpha;
      powers(s[rb], r_new == -INFINITY ? 0.f : r_new, pf[rb]);
    }
  }
  // sums += values of 16 features (i < NO; NO: the ones) times probabilities
  __device__ __forceinline__ void add(const bf16x8 &vf, const bf16x8 (&pf)[RB][NP], int i) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) o[rb][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[rb][p], o[rb][i], 0, 0, 0);
  }
  // into LDS, rows from `row` on
  __device__ __forceinline__ void store(float *lds, int ld, float *s_m, float *s_l, int row) const {
    const int lane = threadIdx.x & 63, ln = lane & 15, g = lane >> 4;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int to = row + rb * 16 + ln;
      if (g == 0) { s_m[to] = r[rb]; s_l[to] = o[rb][NO][0]; }
      float *p = lds + (size_t)to * ld + 16 * g;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) *(f32x4 *)(p + 64 * i + 4 * q) = f32x4{o[rb][4 * i][q], o[rb][4 * i + 1][q], o[rb][4 * i + 2][q], o[rb][4 * i + 3][q]};
    }
  }
  static __device__ __forceinline__ bf16x8 ones() {
    const bf16 x = (bf16)1.f;
    return bf16x8{x, x, x, x, x, x, x, x};
  }
};

// The draft nodes of one (sequence, kv head)
template <typename T>
struct OwnRows {
  const T *k, *v;
  int64_t k_row, v_row;
  int M;
  __device__ __forceinline__ OwnRows(const MxAttnArgs &a, int kvh, int b, int d)
      : k((const T *)a.k.p + b * a.k.seq + kvh * d), v((const T *)a.v.p + b * a.v.seq + kvh * d), k_row(a.k.row), v_row(a.v.row), M(a.n_nodes) {}
};

// Root paths of sequence b.  A tree given by its parents is turned into them in LDS (lds: kPathBytes): every node takes over what lies above it,
// twice as far each time.  Every thread of the workgroup comes here.
constexpr int kPathBytes = kMaxNodes * 20;
struct RootPaths {
  const MxAttnArgs &a;
  const uint64_t *lo, *hi;
  int b;
  __device__ __forceinline__ RootPaths(const MxAttnArgs &args, unsigned char *lds, int seq) : a(args), lo((uint64_t *)lds), hi(lo + kMaxNodes), b(seq) {
    if (a.anc || a.chain) return;
    uint64_t *l = (uint64_t *)lds, *h = l + kMaxNodes;
    int32_t *up = (int32_t *)(h + kMaxNodes);
    const int i = threadIdx.x, M = a.n_nodes;
    if (i < M) {
      AncMask m = {0, 0};
      m.set(i);
      l[i] = m.lo; h[i] = m.hi;
      up[i] = a.parent[b * M + i];
    }
    __syncthreads();
    for (int far = 1; far < M; far *= 2) {
      uint64_t x = 0, y = 0;
      int32_t u = 0;
      if (i < M) { u = up[i]; x = l[i] | l[u]; y = h[i] | h[u]; u = up[u]; }
      __syncthreads();
      if (i < M) { l[i] = x; h[i] = y; up[i] = u; }
      __syncthreads();
    }
  }
  __device__ __forceinline__ AncMask of(int node) const {
    if (a.anc) return a.anc[b * a.n_nodes + node];
    if (a.chain) return AncMask{node < 63 ? (2ull << node) - 1 : ~0ull, node < 64 ? 0ull : (node < 127 ? (2ull << (node - 64)) - 1 : ~0ull)};
    return AncMask{lo[node], hi[node]};
  }
};

enum { kOutPanels, kOutF32, kOutBf16, kPartials };
// four features from kk on of result row r
template <int OUT>
__device__ __forceinline__ void store_result(const MxAttnArgs &a, int r, int kk, const f32x4 &o) {
  if constexpr (OUT == kOutF32) {
    *(f32x4 *)((float *)a.out + r * a.out_row + kk) = o;
    return;
  }
  bf16x4 h;
#pragma unroll
  for (int e = 0; e < 4; ++e) h[e] = (bf16)o[e];
  if constexpr (OUT == kOutBf16) {
    *(bf16x4 *)((bf16 *)a.out + r * a.out_row + kk) = h;
  } else {   // operand layout of the O projection, where they lie side by side
    bf16x4 rest;
#pragma unroll
    for (int e = 0; e < 4; ++e) rest[e] = (bf16)(o[e] - (float)h[e]);
    *(bf16x4 *)((bf16 *)a.out + ol_offset(r, kk, 0, (int)a.out_panel)) = h;
    *(bf16x4 *)((bf16 *)a.out + ol_offset(r, kk, 1, (int)a.out_panel)) = rest;
  }
}

// Softmax sums of 16 query rows over draft nodes n_begin .. n_end, by one wavefront with 16 x 16 x 4 fp32 instructions, 16 nodes at a time.
// Lane (ln, g): features D/4 g .. of node / query row ln for the scores, which come out as nodes 4 g + e of row ln; features D/16 ln .. of the
// nodes 4 g + e for the second product.
template <int D, typename T>
struct OwnSums {
  static constexpr int F = D / 16;   // features a lane takes
  float m, l;       // of row ln; m in powers of two
  f32x4 o[F];       // o[f][e]: feature (4 g + e) F + f
  __device__ __forceinline__ void store(float *row) const {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int f = 0; f < F; f += 4) *(f32x4 *)(row + (4 * g + e) * F + f) = f32x4{o[f][e], o[f + 1][e], o[f + 2][e], o[f + 3][e]};
  }
  __device__ __forceinline__ OwnSums(const OwnRows<T> &x, const T *q, const AncMask &path, int n_begin, int n_end) {
    const int lane = threadIdx.x & 63, ln = lane & 15, g = lane >> 4;
    const float scale = 1.44269504088896f / sqrtf((float)D);
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int n0 = n_begin; n0 < n_end; n0 += 16) {
      const uint32_t mine = (uint32_t)((n0 < 64 ? path.lo : path.hi) >> (n0 & 63)) & 0xffffu;
      if (__builtin_amdgcn_ballot_w64(mine != 0) == 0) continue;
      const T *kp = x.k + min(n0 + ln, x.M - 1) * x.k_row + g * (D / 4), *qp = q + g * (D / 4);
      f32x4 s0 = f32x4{0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int t = 0; t < D / 16; t += 4) {
        f32x4 kv[4], qv[4];
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (t + u < D / 16) { kv[u] = load4(kp + 4 * (t + u)); qv[u] = load4(qp + 4 * (t + u)); }
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (t + u < D / 16) {
            s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[u][0], qv[u][0], s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[u][1], qv[u][1], s1, 0, 0, 0);
            s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[u][2], qv[u][2], s0, 0, 0, 0);
            s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[u][3], qv[u][3], s1, 0, 0, 0);
          }
      }
      float p[4], top = m;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = (mine >> (4 * g + e)) & 1u ? (s0[e] + s1[e]) * scale : -INFINITY;
        top = fmaxf(top, p[e]);
      }
      top = fmaxf(top, __shfl_xor(top, 16, 64));
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float m_safe = top == -INFINITY ? 0.f : top, alpha = __builtin_amdgcn_exp2f(m - m_safe);
      m = top;
      l *= alpha;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        p[e] = __builtin_amdgcn_exp2f(p[e] - m_safe);   // 0 for other branches
        l += p[e];
      }
#pragma unroll
      for (int f0 = 0; f0 < F; f0 += 4) {   // a quarter of the features at a time: registers
        f32x4 v[4];
        bool odd = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = load4(x.v + min(n0 + 4 * g + e, x.M - 1) * x.v_row + ln * F + f0);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (!(__builtin_fabsf(v[e][j]) < INFINITY)) { odd = true; v[e][j] = 0.f; }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          o[f0 + j] *= alpha;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[f0 + j] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[e][j], p[e], o[f0 + j], 0, 0, 0);
        }
        if (__builtin_amdgcn_ballot_w64(odd) != 0) {   // infinities and NaNs: for each row those of its own ancestors only
#pragma unroll 1
          for (int k = 0; k < 16; ++k) {
            const float w = __shfl((k & 3) == 0 ? p[0] : (k & 3) == 1 ? p[1] : (k & 3) == 2 ? p[2] : p[3], ln + 16 * (k >> 2), 64);
            if (!((mine >> k) & 1u)) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const f32x4 y = load4(x.v + (n0 + k) * x.v_row + (4 * g + e) * F + f0);
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (!(__builtin_fabsf(y[j]) < INFINITY)) o[f0 + j][e] += w * y[j];
            }
          }
        }
      }
    }
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
  }
};

// OwnSums of the 16 rows from first_row on (p_rows and more: none) as a partial.  lds: kPathBytes; every thread of the workgroup comes here.
template <int D, typename T>
__device__ __forceinline__ void own_rows(const MxAttnArgs &a, unsigned char *lds, int kvh, int b, int first_row, int n_begin, int n_end, size_t part) {
  const RootPaths paths(a, lds, b);
  const T *q0 = (const T *)a.q.p + b * a.q.seq + kvh * a.group * D;
  const OwnRows<T> x(a, kvh, b, D);
  const int p_rows = a.group * x.M, row = first_row + (threadIdx.x & 15);
  if (first_row >= p_rows) return;   // wave-uniform
  const int pc = min(row, p_rows - 1), al = pc / x.M, node = pc - al * x.M;
  const AncMask path = paths.of(node);
  const OwnSums<D, T> sums(x, q0 + node * a.q.row + al * D, path, n_begin, n_end);
  if (row >= p_rows) return;
  if ((threadIdx.x & 63) < 16) {
    a.part_m[part + row] = sums.m == -INFINITY && (path.lo | path.hi) == 0 ? -INFINITY : stored_max(sums.m);
    a.part_l[part + row] = sums.l;
  }
  sums.store(a.part_o + (part + row) * D);
}

// the workgroup behind all others stores the nodes' rows, which nobody reads here
template <int D, int NW, typename T>
__device__ __forceinline__ void append_rows(const MxAttnArgs &a, int kvh, int b) {
  const int wave = threadIdx.x >> 6, ctx = a.ctx.v[b];
  const OwnRows<T> x(a, kvh, b, D);
  for (int i = (ctx / kMxGroup + wave) * kMxGroup; i < ctx + x.M; i += NW * kMxGroup) mx_store_group<D, T>(a.c, b, kvh, i, ctx, x.M, x.k, x.k_row, x.v, x.v_row);
}

// the low `left` bits of eight
__device__ __forceinline__ uint32_t low_bits(int left) { return left <= 0 ? 0u : (left >= 8 ? 255u : (1u << left) - 1); }

}  // namespace

// RB blocks of 16 query rows a wavefront; RW wavefronts side by side hold the rows of a workgroup, and KG groups of them take every KG-th run
// of 32 keys, straight from the cache to registers; the groups' sums meet in LDS at the end.
//
// OUT = kPartials: four wavefronts; grid (kv head, rows, part).  The first parts take the draft nodes, kMxOwnNodes each, so that the splits behind fill in as those end
// (four sequences of 60 nodes over 16384 keys: 82 us, 109 with them last); then the splits, a.keys keys each whatever sequence they belong to; then a
// workgroup for each sequence that stores its nodes' rows.  Row groups of the same keys land on one XCD where the kv heads are a multiple of 8.
// Else: short contexts.  One workgroup of eight wavefronts takes its rows over all keys and nodes and writes their results, which saves the partials' way
// through memory and the launch behind them; RB of the wavefronts take the draft nodes, 16 rows each.
template <int D, int RB, int RW, typename T, int NP, int OUT, bool PAGED>
__global__ __launch_bounds__(OUT == kPartials ? 256 : 512, OUT != kPartials || RB > 1 ? 2 : 3) void k_mx_attn(MxAttnArgs a) {
  constexpr bool kWhole = OUT != kPartials;
  constexpr int NW = kWhole ? 8 : 4, KG = kWhole ? 8 - RB : 4 / RW, R = 16 * RB * RW, ST = D / 32, NV = D / 64;
  constexpr int LD = D + 4, kSums = kWhole ? KG + 1 : KG;   // rows of sums in LDS: those of the groups, then those of the nodes
  __shared__ __attribute__((aligned(16))) float sums[kSums * R * LD];
  __shared__ float s_m[kSums * R], s_l[kSums * R];
  __shared__ __attribute__((aligned(16))) unsigned char path_lds[kWhole ? kPathBytes : 16];
  const int kvh = blockIdx.x, row0 = blockIdx.y * R, lane = threadIdx.x & 63, ln = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rw = kWhole ? 0 : wave % RW, kg = kWhole ? wave - RB : wave / RW;
  const int n_own = kWhole ? 0 : a.n_own, n_main = kWhole ? a.batch : a.split0[a.batch], p_rows = a.group * a.n_nodes, first_row = row0 + rw * RB * 16;
  int z = (int)blockIdx.z - n_own * a.batch;
  if (z >= n_main) {
    if (blockIdx.y == 0) append_rows<D, NW, T>(a, kvh, z - n_main);
    return;
  }
  if (z < 0) {   // first of all: the others fill in as these end
    const int b = (int)blockIdx.z / a.n_own, n = (int)blockIdx.z - b * a.n_own, n0 = n * kMxOwnNodes;
    static_assert(kWhole || sizeof(sums) >= kPathBytes, "the nodes' root paths lie there");
    return own_rows<D, T>(a, (unsigned char *)sums, kvh, b, wave * 16 < R ? row0 + wave * 16 : p_rows, n0, min(n0 + kMxOwnNodes, a.n_nodes),
                          a.part(a.split0[b + 1] + b * a.n_own + n, kvh));
  }
  int b = 0;
  if (kWhole) b = z;
  else
    while (z >= a.split0[b + 1]) ++b;
  const int ctx = a.ctx.v[b], k_begin = kWhole ? 0 : (z - a.split0[b]) * a.keys, k_end = kWhole ? ctx : min(ctx, k_begin + a.keys);
  const size_t part = a.part(z + b * n_own, kvh);
  const T *q0 = (const T *)a.q.p + b * a.q.seq + kvh * a.group * D;
  if constexpr (kWhole) {
    const RootPaths paths(a, path_lds, b);
    if (kg < 0) {
      const int row = row0 + wave * 16, at = KG * R + wave * 16 + ln;
      if (a.k.p && row < p_rows) {   // wave-uniform
        const OwnRows<T> nodes(a, kvh, b, D);
        const int pc = min(row + ln, p_rows - 1), al = pc / a.n_nodes, node = pc - al * a.n_nodes;
        const OwnSums<D, T> own(nodes, q0 + node * a.q.row + al * D, paths.of(node), 0, a.n_nodes);
        if (g == 0) { s_m[at] = own.m; s_l[at] = own.l; }
        own.store(sums + at * LD);
      } else if (g == 0) {
        s_m[at] = -INFINITY;
        s_l[at] = 0.f;
      }
    } else if (kg * 32 >= ctx) {   // no run
      for (int i = lane; i < R; i += 64) { s_m[kg * R + i] = -INFINITY; s_l[kg * R + i] = 0.f; }
    }
  }

  if (!kWhole || (kg >= 0 && kg * 32 < ctx)) {   // wave-uniform
    // the codes of a run are requested where those of the run before are used; past the end the last keys are read again and left out
    const int first = k_begin + kg * 32, last = (k_end - 1) & ~31;
    KeyCodes<D> kc;
    ValueCodes<D> vc;
    size_t r = a.c.block(b, kvh, min(first, last));
    auto at = [&](int k0) { return PAGED ? k0 % kKvPage : k0; };
    kc.load(a.c, r, at(min(first, last)), ln, g);
    vc.load(a.c, r, at(min(first, last)), ln, g);
    if (PAGED) r = a.c.block(b, kvh, min(first + 32 * KG, last));
    QueryRows<D, RB, T, NP> x;
    x.start(a, q0, first_row, p_rows, ln, g);
    if (first_row < p_rows)   // wave-uniform
      for (int k0 = first; k0 < k_end; k0 += 32 * KG) {
        const int next = at(min(k0 + 32 * KG, last));
        f32x4 s[RB][2];
        x.clear(s);
        bf16x8 kf[ST][2];
#pragma unroll
        for (int i = 0; i < ST; ++i)
#pragma unroll
          for (int t = 0; t < 2; ++t) kf[i][t] = kc.operand(t, i);
        kc.load(a.c, r, next, ln, g);
#pragma unroll
        for (int i = 0; i < ST; ++i) x.score(s, kf[i][0], kf[i][1], i);
        if (k0 + 32 > k_end) {   // wave-uniform: the keys end in here
          const int left = k_end - (k0 + 8 * g);
          vc.keep(left);
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) x.mask(s[rb], low_bits(left));
        }
        bf16x8 pf[RB][NP];
        x.settle(s, pf, x.weigh(s, pf));
        x.add(x.ones(), pf, 4 * NV);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
          bf16x8 vf[4];
          vc.operands(i, vf);
#pragma unroll
          for (int j = 0; j < 4; ++j) x.add(vf[j], pf, 4 * i + j);
        }
        vc.load(a.c, r, next, ln, g);
        if (PAGED) r = a.c.block(b, kvh, min(k0 + 64 * KG, last));
      }
    x.store(sums, LD, s_m, s_l, kg * R + rw * RB * 16);
  }
  __syncthreads();

  // whole rows, the groups in ascending order
  for (int i = threadIdx.x; i < min(R, p_rows - row0) * (D / 4); i += 64 * NW) {
    const int r = i / (D / 4), f = i % (D / 4) * 4;
    float m = s_m[r], l = 0.f;
#pragma unroll
    for (int k = 1; k < kSums; ++k) m = fmaxf(m, s_m[k * R + r]);
    f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
      const float mk = s_m[k * R + r], lk = s_l[k * R + r], w = __builtin_amdgcn_exp2f(mk - m);
      const f32x4 ok = *(const f32x4 *)(sums + (k * R + r) * LD + f);
      const bool some = mk != -INFINITY || lk != 0.f;   // else no key, or scores of -infinity alone; NaN scores leave no maximum but a NaN sum
      l += some ? lk * w : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += some ? ok[e] * w : 0.f;
    }
    if constexpr (kWhole) {
      const int al = (row0 + r) / a.n_nodes, node = row0 + r - al * a.n_nodes;
      const float den = ctx > 0 || a.k.p ? l : 1.f;   // no key at all: 0
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = o[e] / den;
      store_result<OUT>(a, b * a.n_nodes + node, (kvh * a.group + al) * D + f, o);
    } else {
      if (f == 0) {
        a.part_m[part + row0 + r] = stored_max(m);
        a.part_l[part + row0 + r] = l;
      }
      *(f32x4 *)(a.part_o + (part + row0 + r) * D + f) = o;
    }
  }
}

// Join the partials of a row and kv head.  A wavefront takes 64 features of a head, four a lane, and a quarter of the partials on every 16 lanes, all
// of them requested at once: the time is that of one read, not of one behind another.  The quarters are joined as the partials are, in a fixed order.  A row that saw
// no key at all (no context, no nodes of its own) is 0.
template <int D, int NB, int OUT>
__global__ __launch_bounds__(1024) void k_mx_merge(MxAttnArgs a) {
  const int r = blockIdx.x, kvh = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int M = a.n_nodes, b = r / M, node = r - b * M, n = a.split0[b + 1] - a.split0[b] + a.n_own;
  const int al = wave / (D / 64), f = (wave & (D / 64 - 1)) * 64 + (lane & 15) * 4, quarter = lane >> 4;
  const size_t first = a.part(a.split0[b] + b * a.n_own, kvh) + al * M + node, step = a.part(1, 0);
  float m = -INFINITY, l = 0.f;
  f32x4 o = f32x4{0.f, 0.f, 0.f, 0.f};
  if (n > 0) {
    float pm[NB], pl[NB];
    f32x4 po[NB];
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const size_t idx = first + min(quarter + 4 * i, n - 1) * step;
      pm[i] = a.part_m[idx];
      pl[i] = a.part_l[idx];
      po[i] = *(const f32x4 *)(a.part_o + idx * D + f);
    }
#pragma unroll
    for (int i = 0; i < NB; ++i) m = fmaxf(m, quarter + 4 * i < n ? pm[i] : -INFINITY);
    m = fmaxf(m, __shfl_xor(m, 16, 64));
    m = fmaxf(m, __shfl_xor(m, 32, 64));
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      if (quarter + 4 * i >= n || pm[i] == -INFINITY) continue;
      const float w = __builtin_amdgcn_exp2f((pm[i] - m) * 1.44269504088896f);
      o += po[i] * w;
      l += pl[i] * w;
    }
#pragma unroll
    for (int x = 16; x < 64; x *= 2) {
      l += __shfl_xor(l, x, 64);
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], x, 64);
    }
  }
  const float den = m == -INFINITY ? 1.f : l;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = o[e] / den;
  if (quarter == 0) store_result<OUT>(a, r, (kvh * a.group + al) * D + f, o);
}

namespace {
template <int D, int OUT>
void launch_merge(hipStream_t st, const MxAttnArgs &a) {
  const dim3 grid(a.batch * a.n_nodes, a.c.n_kv), block(a.group * D);   // <= 1024 (group <= 8, d <= 128)
  static_assert(4 * 16 >= kMaxAttnSplits, "every partial is read at once");
  int n = 0;
  for (int b = 0; b < a.batch; ++b) n = max(n, a.split0[b + 1] - a.split0[b] + a.n_own);
  if (n <= 4 * 2) hipLaunchKernelGGL((k_mx_merge<D, 2, OUT>), grid, block, 0, st, a);
  else if (n <= 4 * 4) hipLaunchKernelGGL((k_mx_merge<D, 4, OUT>), grid, block, 0, st, a);
  else if (n <= 4 * 8) hipLaunchKernelGGL((k_mx_merge<D, 8, OUT>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_mx_merge<D, 16, OUT>), grid, block, 0, st, a);
}

template <int D, typename T, int NP, int OUT>
void launch_rows(hipStream_t st, const MxAttnArgs &a) {
  const dim3 grid(a.c.n_kv, a.n_row_groups, (a.whole ? a.batch : a.split0[a.batch] + a.n_own * a.batch) + (a.append ? a.batch : 0));
#define TS_MX(THREADS, ...)                                                                                          \
  do {                                                                                                              \
    if (a.c.page_table) hipLaunchKernelGGL((k_mx_attn<D, __VA_ARGS__, true>), grid, dim3(THREADS), 0, st, a);          \
    else hipLaunchKernelGGL((k_mx_attn<D, __VA_ARGS__, false>), grid, dim3(THREADS), 0, st, a);                        \
  } while (0)
  if (a.whole) {
    if (a.form == kMxRows16) TS_MX(512, 1, 1, T, NP, OUT); else TS_MX(512, 2, 1, T, NP, OUT);
    return;
  }
  if (a.form == kMxRows16) TS_MX(256, 1, 1, T, NP, kPartials);
  else if (a.form == kMxRows32) TS_MX(256, 2, 1, T, NP, kPartials);
  else TS_MX(256, 2, 2, T, NP, kPartials);
#undef TS_MX
  launch_merge<D, OUT>(st, a);
}

template <int D>
void launch_d(hipStream_t st, const MxAttnArgs &a) {
  if (a.out_row == 0) launch_rows<D, float, 2, kOutPanels>(st, a);   // a verification pass
  else if (a.dtype == TRISPEC_F32) launch_rows<D, float, 3, kOutF32>(st, a);
  else launch_rows<D, bf16, 1, kOutBf16>(st, a);
}
}  // namespace

void launch_mx_attn(hipStream_t st, const MxAttnArgs &a) {
  if (a.head_dim == 128) launch_d<128>(st, a); else launch_d<64>(st, a);
}

}  // namespace ts
