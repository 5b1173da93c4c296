// Attention of 32 query rows over a block of 32 draft nodes, in fp32 from this pass's own projections, and what the
// attention kernels share.
#pragma once

#include <float.h>

#include "device_util.hpp"

namespace ts {

// Maximum, in natural-log units, that a partial is stored with.  -inf marks a partial without keys, which the
// merge skips without reading it; one whose scores are all NaN (fmaxf drops them) or all -inf has to be
// added up all the same, so that the NaN in its sums reaches the row: it is stored with the lowest finite value.
__device__ __forceinline__ float stored_max(float m_log2) { return fmaxf(m_log2 * 0.693147180559945f, -FLT_MAX); }

// e^x through the hardware exp2 (about 1e-7 |x| relative error; the arguments here are <= 0)
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// The draft nodes of one (sequence, kv head): row i of q (first head of the group), k and v
template <typename T>
struct DraftRows {
  const T *q, *k, *v;
  int64_t ld_q, ld_k, ld_v;
};
__device__ __forceinline__ f32x4 load4(const float *p) { return *(const f32x4 *)p; }
__device__ __forceinline__ f32x4 load4(const bf16 *p) {
  const bf16x4 v = *(const bf16x4 *)p;
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}

// Softmax partial of 32 query rows (one wavefront) over the draft nodes 32 kb .. 32 kb + 31: S^T = K Q^T
// and O^T = V^T P^T with fp32 matrix instructions (32x32x2), operands straight from the projections.
// Lane (ln, g) holds features g D/2 .. of key / query row ln for the first product; the scores come out
// with keys 8q + 4g + r in register 4q + r, which is the order in which the second product takes them.
// 128 instructions of 64 cycles, 3.5 us, beside context workgroups that run longer.  Evaluated by the
// merge kernel, where every row fetches its ancestors' keys and values for itself, a chain of 128 nodes
// with 32 heads takes 44 us a layer; the plain merge takes 8.4, the launch before it 18.6 instead of 16.1.
// s_p: 32 x 32 floats of LDS of this wavefront.
// `mask_of` gives a node's root path; part_m, part_l, part_o: this partial's rows.
template <int D, typename T, typename MaskOf>
__device__ void draft_partial(const DraftRows<T> &src, MaskOf mask_of, int M, int group, int kb, int row_block, float *part_m, float *part_l,
                              float *part_o, float *s_p) {
  const int lane = threadIdx.x & 63, ln = lane & 31, g = lane >> 5;
  const int p_rows = group * M;
  const int prow = row_block * 32 + ln;
  if (row_block * 32 >= p_rows) return;   // wave-uniform
  const int pc = min(prow, p_rows - 1), al = pc / M, node = pc - al * M;
  const AncMask mask = mask_of(node);
  const uint32_t mine = (uint32_t)((kb < 2 ? mask.lo : mask.hi) >> (32 * (kb & 1)));   // ancestors in this block
  if (__builtin_amdgcn_ballot_w64(mine != 0) == 0) {   // none for any row
    if (prow < p_rows && g == 0) { part_m[prow] = -INFINITY; part_l[prow] = 0.f; }
    return;
  }
  const T *kp = src.k + min(kb * 32 + ln, M - 1) * src.ld_k + g * (D / 2);
  const T *qp = src.q + node * src.ld_q + al * D + g * (D / 2);
  f32x16 s0, s1;
#pragma unroll
  for (int e = 0; e < 16; ++e) s0[e] = s1[e] = 0.f;
  {
    f32x4 kv[D / 8], qv[D / 8];
#pragma unroll
    for (int t = 0; t < D / 8; ++t) { kv[t] = load4(kp + 4 * t); qv[t] = load4(qp + 4 * t); }
#pragma unroll
    for (int t = 0; t < D / 8; ++t) {
      s0 = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[t][0], qv[t][0], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[t][1], qv[t][1], s1, 0, 0, 0);
      s0 = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[t][2], qv[t][2], s0, 0, 0, 0);
      s1 = __builtin_amdgcn_mfma_f32_32x32x2f32(kv[t][3], qv[t][3], s1, 0, 0, 0);
    }
  }
  const T *vp = src.v;
  float v[16][D / 32];   // all values in one round trip, behind the softmax
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
      v[e][db] = (float)vp[min(kb * 32 + 8 * (e >> 2) + 4 * g + (e & 3), M - 1) * src.ld_v + db * 32 + ln];
  __builtin_amdgcn_sched_barrier(0);
  const float scale = 1.44269504088896f / sqrtf((float)D);
  float p[16], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int key = 8 * (e >> 2) + 4 * g + (e & 3);
    p[e] = (mine >> key) & 1u ? (s0[e] + s1[e]) * scale : -INFINITY;
    m = fmaxf(m, p[e]);
  }
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  const float m_safe = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    p[e] = __builtin_amdgcn_exp2f(p[e] - m_safe);   // 0 for other branches
    l += p[e];
  }
  l += __shfl_xor(l, 32, 64);
  f32x16 o[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
  float finite = 0.f;   // stays 0 while every value is finite
#pragma unroll
  for (int e = 0; e < 16; ++e)
#pragma unroll
    for (int db = 0; db < D / 32; ++db) {
      finite = __builtin_fmaf(v[e][db], 0.f, finite);
      o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(v[e][db], p[e], o[db], 0, 0, 0);
    }
  if (__builtin_amdgcn_ballot_w64(finite != 0.f) != 0) {
    // an infinity or NaN among the values: a weight of 0 would carry it into rows of other branches.
    // Row by row over the ancestors only.
#pragma unroll
    for (int e = 0; e < 16; ++e) s_p[(8 * (e >> 2) + 4 * g + (e & 3)) * 32 + ln] = p[e];
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[db][e] = 0.f;
#pragma unroll 1
    for (int k = 0; k < 32; ++k) {
      if (!((mine >> k) & 1u)) continue;
      const float w = s_p[k * 32 + ln];
      const T *vr = vp + (kb * 32 + k) * src.ld_v + 4 * g;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[db][e] += w * (float)vr[db * 32 + 8 * (e >> 2) + (e & 3)];
    }
  }
  if (prow >= p_rows) return;
  if (g == 0) {
    part_m[prow] = mine != 0 ? stored_max(m) : -INFINITY;
    part_l[prow] = l;
  }
  float *out = part_o + (size_t)prow * D;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *(f32x4 *)(out + db * 32 + 8 * q + 4 * g) = f32x4{o[db][4 * q], o[db][4 * q + 1], o[db][4 * q + 2], o[db][4 * q + 3]};
}


// The same for at most 16 query rows over as many nodes (chains, short trees, single tokens), by one wavefront with 16 x 16 x 4 fp32
// instructions, in half the registers.  Lane (ln, g): features D/4 g .. of node / query row ln for the scores, which come out
// as nodes 4 g + r of row ln; features D/16 ln .. of the nodes 4 g + r for the second product.  s_p: 256 floats of LDS.
template <int D, typename T, typename MaskOf>
__device__ __forceinline__ void draft_partial_small(const DraftRows<T> &src, MaskOf mask_of, int M, int group, float *part_m, float *part_l, float *part_o, float *s_p) {
  const int lane = threadIdx.x & 63, ln = lane & 15, g = lane >> 4;
  const int p_rows = group * M, pc = min(ln, p_rows - 1), al = pc / M, node = pc - al * M;
  const uint32_t mine = (uint32_t)mask_of(node).lo;
  const T *kp = src.k + min(ln, M - 1) * src.ld_k + g * (D / 4), *qp = src.q + node * src.ld_q + al * D + g * (D / 4);
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
  constexpr int F = D / 16;   // features a lane takes
  float v[4][F];
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int f = 0; f < F; f += 4) {
      const f32x4 x = load4(src.v + min(4 * g + r, M - 1) * src.ld_v + ln * F + f);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[r][f + e] = x[e];
    }
  const float scale = 1.44269504088896f / sqrtf((float)D);
  float p[4], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    p[r] = (mine >> (4 * g + r)) & 1u ? (s0[r] + s1[r]) * scale : -INFINITY;
    m = fmaxf(m, p[r]);
  }
  m = fmaxf(m, __shfl_xor(m, 16, 64));
  m = fmaxf(m, __shfl_xor(m, 32, 64));
  const float m_safe = m == -INFINITY ? 0.f : m;
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    p[r] = __builtin_amdgcn_exp2f(p[r] - m_safe);   // 0 for other branches
    l += p[r];
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  f32x4 o[F];
  float finite = 0.f;   // stays 0 while every value is finite
#pragma unroll
  for (int f = 0; f < F; ++f) {
    o[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      finite = __builtin_fmaf(v[r][f], 0.f, finite);
      o[f] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[r][f], p[r], o[f], 0, 0, 0);
    }
  }
  if (__builtin_amdgcn_ballot_w64(finite != 0.f) != 0) {   // as above: over each row's own ancestors only
#pragma unroll
    for (int r = 0; r < 4; ++r) s_p[(4 * g + r) * 16 + ln] = p[r];
    __builtin_amdgcn_s_waitcnt(0);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int f = 0; f < F; ++f) o[f] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int k = 0; k < M; ++k) {
      if (!((mine >> k) & 1u)) continue;
      const float w = s_p[k * 16 + ln];
#pragma unroll
      for (int f = 0; f < F; ++f)
#pragma unroll
        for (int r = 0; r < 4; ++r) o[f][r] += w * (float)src.v[k * src.ld_v + (4 * g + r) * F + f];
    }
  }
  if (ln >= p_rows) return;
  if (g == 0) {
    part_m[ln] = stored_max(m);
    part_l[ln] = l;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int f = 0; f < F; f += 4)
      *(f32x4 *)(part_o + (size_t)ln * D + (4 * g + r) * F + f) = f32x4{o[f][r], o[f + 1][r], o[f + 2][r], o[f + 3][r]};
}

}  // namespace ts
