// Tree-masked grouped-query attention over a context held in 4 bits (layout: mx.hpp) and the draft nodes' own K and V.
//
// For query row r (query head, node) of a kv head: scores s_j = q_r . K_j / sqrt(d) over the context's slots and the row's
// ancestors, one pass over the keys with the running maximum m and l = sum exp(s_j - m), o = sum exp(s_j - m) V_j, result o / l.
// Workgroups take a range of keys each and leave (m, l, o); a second launch adds them up in ascending order.
//
// A wavefront takes 32 keys at a time, straight from the cache to registers: a key's codes are so few bytes that sharing a
// tile through LDS would cost more than converting it once per 16 to 64 query rows.  K Q^T and V^T P^T go through 16 x 16 x 32
// matrix instructions in the transposed form (a query row per lane, so the softmax state is per lane), and the order of the
// reduction is chosen so that nothing moves between lanes: score register e of lane (ln, g) is the key 8 g + e of the
// tile, which is what the second product's operand wants of that lane.  bf16 queries are exact operands and probabilities
// are rounded to bf16, half a step of the result's own type; fp32 ones go as high part + low part, both.
#include "attn_draft.hpp"
#include "mx.hpp"

namespace ts {

namespace {

template <typename T>
struct Parts {   // of an operand
  static constexpr int N = 1;
};
template <>
struct Parts<float> {
  static constexpr int N = 2;
};

// Eight queries as operands: part 0 high, part 1 the rest
__device__ __forceinline__ void query_parts(const bf16 *p, bf16x8 (&q)[1]) { q[0] = *(const bf16x8 *)p; }
__device__ __forceinline__ void query_parts(const float *p, bf16x8 (&q)[2]) {
#pragma unroll
  for (int e = 0; e < 8; e += 4) {
    const f32x4 x = *(const f32x4 *)(p + e);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[0][e + i] = (bf16)x[i];
      q[1][e + i] = (bf16)(x[i] - (float)q[0][e + i]);
    }
  }
}
__device__ __forceinline__ void prob_parts(f32x2 p, bf16x8 (&o)[1], int e) {
  const bf16x2 h = __builtin_convertvector(p, bf16x2);
  o[0][e] = h[0]; o[0][e + 1] = h[1];
}
__device__ __forceinline__ void prob_parts(f32x2 p, bf16x8 (&o)[2], int e) {
  const bf16x2 h = __builtin_convertvector(p, bf16x2);
  const f32x2 rest = {p[0] - (float)h[0], p[1] - (float)h[1]};
  const bf16x2 l = __builtin_convertvector(rest, bf16x2);
  o[0][e] = h[0]; o[0][e + 1] = h[1];
  o[1][e] = l[0]; o[1][e + 1] = l[1];
}

// A wavefront's 32 keys as they lie in the cache.  Lane (ln, g): of key 8 (ln / 4) + 4 t + ln % 4, t = 0, 1, the features
// (D / 4) g .., inside one block; of the keys 8 g .. 8 g + 7 the values of features 64 i + 4 ln .. + 3.
template <int D>
struct KeyCodes {
  uint32_t w[2][D / 32];
  uint32_t scale[2];
};
template <int D>
struct ValueCodes {
  u32x4 w[D / 64];
  u32x2 scale[D / 64];
};

}  // namespace

// RB blocks of 16 query rows a wavefront, RW wavefronts side by side hold the rows of a workgroup and the KG = 4 / RW groups of
// them take every KG-th run of 32 keys; the groups' sums meet in LDS at the end.  Workgroups before the splits take a block of
// 32 draft nodes each; behind them one more a (sequence, kv head) stores the nodes' rows (APPEND), which no other reads.
template <int D, int RB, int RW, typename T, bool PAGED>
__global__ __launch_bounds__(256, RB == 1 ? (D == 128 && Parts<T>::N == 2 ? 3 : 4) : (RB == 2 ? 2 : 1)) void k_mx_attn(MxAttnArgs a) {
  constexpr int KG = 4 / RW, NP = Parts<T>::N, R = 16 * RB * RW, ST = D / 32, NV = D / 64, LD = D + 4;
  constexpr int kMergeBytes = KG > 1 ? 4 * 16 * RB * LD * 4 : 16, kDraftBytes = 4 * 4096 + kMaxNodes * 20;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kMergeBytes > kDraftBytes ? kMergeBytes : kDraftBytes];
  __shared__ float s_m[KG][R], s_l[KG][R];
  const int kvh = blockIdx.y, b = blockIdx.z / a.n_row_groups, rg = blockIdx.z - b * a.n_row_groups;
  const int lane = threadIdx.x & 63, ln = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rw = wave % RW, kg = wave / RW;
  const int M = a.n_nodes, p_rows = a.group * M, n_parts = a.n_splits + a.n_draft;
  const size_t part0 = ((size_t)b * a.c.n_kv + kvh) * n_parts;
  const T *q0 = (const T *)a.q.p + b * a.q.seq + kvh * a.group * D;
  const int ctx = a.ctx.v[b];

  if ((int)blockIdx.x < a.n_draft) {
    // ---- a block of draft nodes: whole 32-row blocks of this row group
    uint64_t *lo = (uint64_t *)(lds + 4 * 4096), *hi = lo + kMaxNodes;
    int32_t *up = (int32_t *)(hi + kMaxNodes);
    if (!a.anc && !a.chain) {   // root paths from the parents: every node takes over what lies above it, twice as far each time
      const int i = threadIdx.x;
      if (i < M) {
        AncMask m = {0, 0};
        m.set(i);
        lo[i] = m.lo; hi[i] = m.hi;
        up[i] = a.parent[b * M + i];
      }
      __syncthreads();
      for (int far = 1; far < M; far *= 2) {
        uint64_t l = 0, h = 0;
        int32_t u = 0;
        if (i < M) { u = up[i]; l = lo[i] | lo[u]; h = hi[i] | hi[u]; u = up[u]; }
        __syncthreads();
        if (i < M) { lo[i] = l; hi[i] = h; up[i] = u; }
        __syncthreads();
      }
    }
    auto mask_of = [&](int node) {
      if (a.anc) return a.anc[b * M + node];
      if (a.chain) return AncMask{node < 63 ? (2ull << node) - 1 : ~0ull, node < 64 ? 0ull : (node < 127 ? (2ull << (node - 64)) - 1 : ~0ull)};
      return AncMask{lo[node], hi[node]};
    };
    const DraftRows<T> src = {q0, (const T *)a.k.p + b * a.k.seq + kvh * D, (const T *)a.v.p + b * a.v.seq + kvh * D, a.q.row, a.k.row, a.v.row};
    const size_t row = (part0 + a.n_splits + blockIdx.x) * p_rows;
    if constexpr (R == 16) {
      if (wave == 0) draft_partial_small<D, T>(src, mask_of, M, a.group, a.part_m + row, a.part_l + row, a.part_o + row * D, (float *)lds);
    } else
      for (int rb = rg * R / 32 + wave; rb * 32 < min((rg + 1) * R, p_rows); rb += 4)
        draft_partial<D>(src, mask_of, M, a.group, blockIdx.x, rb, a.part_m + row, a.part_l + row, a.part_o + row * D, (float *)lds + wave * 1024);
    return;
  }
  const int split = blockIdx.x - a.n_draft;
  if (split >= a.n_splits) {
    if (rg == 0)
      for (int i = (ctx / kMxGroup + wave) * kMxGroup; i < ctx + M; i += 4 * kMxGroup)
        mx_store_group<D, T>(a.c, b, kvh, i, ctx, M, (const T *)a.k.p + b * a.k.seq + kvh * D, a.k.row, (const T *)a.v.p + b * a.v.seq + kvh * D, a.v.row);
    return;
  }

  const size_t part = (part0 + split) * p_rows;
  const int k_begin = split * a.keys_per_split, k_end = min(ctx, k_begin + a.keys_per_split);
  const int row0 = rg * R;
  if (k_begin >= k_end) {   // empty split: neutral partial
    for (int r = threadIdx.x; r < min(R, p_rows - row0); r += 256) {
      a.part_m[part + row0 + r] = -INFINITY;
      a.part_l[part + row0 + r] = 0.f;
    }
    return;
  }

  // past the end a wavefront reads the split's last keys again and leaves all of them out
  const int last = (k_end - 1) & ~31;
  KeyCodes<D> kc;
  ValueCodes<D> vc;
  size_t r_next = a.c.block(b, kvh, min(k_begin + kg * 32, last));
  auto load_k = [&](int k0, size_t r) {
    const int s = PAGED ? k0 % kKvPage : k0;
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int at = s + 8 * (ln >> 2) + 4 * t + (ln & 3);
      const uint8_t *p = a.c.k_codes + MxOffsets<D>::k_codes(a.c, r, at) + g * (D / 8);
      if constexpr (D == 128) {
        const u32x4 w = *(const u32x4 *)p;
#pragma unroll
        for (int i = 0; i < 4; ++i) kc.w[t][i] = w[i];
      } else {
        const u32x2 w = *(const u32x2 *)p;
        kc.w[t][0] = w[0]; kc.w[t][1] = w[1];
      }
      kc.scale[t] = a.c.k_scales[MxOffsets<D>::k_scales(a.c, r, at) + g * (D / 32) / 4];
    }
  };
  auto load_v = [&](int k0, size_t r) {
    const int s = (PAGED ? k0 % kKvPage : k0) + 8 * g;
    const uint8_t *p = a.c.v_codes + MxOffsets<D>::v_codes(a.c, r, s) + ln * 16;
    const uint8_t *ps = a.c.v_scales + MxOffsets<D>::v_scales(a.c, r, s) + (ln >> 3) * 8;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      vc.w[i] = *(const u32x4 *)(p + 256 * i);
      vc.scale[i] = *(const u32x2 *)(ps + 16 * i);
    }
  };
  const int first = k_begin + kg * 32;
  size_t r_v = r_next;
  load_k(min(first, last), r_next);
  load_v(min(first, last), r_v);
  if (PAGED) r_next = a.c.block(b, kvh, min(first + 32 * KG, last));

  // ---- queries: lane (ln, g) features (D / 4) g + 8 t .. of row ln of each block
  bf16x8 qf[RB][ST][NP];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int pc = min(row0 + (rw * RB + rb) * 16 + ln, p_rows - 1), al = pc / M, node = pc - al * M;
    const T *q = q0 + node * a.q.row + al * D + g * (D / 4);
#pragma unroll
    for (int t = 0; t < ST; ++t) query_parts(q + 8 * t, qf[rb][t]);
  }

  const float c = 1.44269504088896f / sqrtf((float)D);   // scores in powers of two
  float m_run[RB], l_run[RB];
  f32x4 o[RB][4 * NV];   // o[rb][4 i + j][r]: feature 64 i + 16 g + 4 r + j of row ln
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    m_run[rb] = -INFINITY;
    l_run[rb] = 0.f;
#pragma unroll
    for (int i = 0; i < 4 * NV; ++i) o[rb][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const bool rows_here = row0 + rw * RB * 16 < p_rows;   // wave-uniform
  if (rows_here)
  for (int k0 = first; k0 < k_end; k0 += 32 * KG) {
    const int next = min(k0 + 32 * KG, last);
    f32x4 s[RB][2];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb][0] = s[rb][1] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x8 kf[2][ST];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < ST; ++i) kf[t][i] = mx_values(kc.w[t][i], mx_scale(kc.scale[t], 0));
    load_k(next, r_next);
#pragma unroll
    for (int i = 0; i < ST; ++i)
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int t = 0; t < 2; ++t) s[rb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[t][i], qf[rb][i][p], s[rb][t], 0, 0, 0);
    const bool ragged = k0 + 32 > k_end;   // the keys end in here
    if (ragged) {
      const int left = k_end - (k0 + 8 * g);   // of this lane's eight keys
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (e >= left) s[rb][e >> 2][e & 3] = -INFINITY;
      // values behind the end: element 0 of the smallest scale, whatever lies there
      const uint64_t keep = left <= 0 ? 0 : (left >= 8 ? ~0ull : (1ull << (8 * left)) - 1);
#pragma unroll
      for (int i = 0; i < NV; ++i) {
        vc.scale[i][0] &= (uint32_t)keep;
        vc.scale[i][1] &= (uint32_t)(keep >> 32);
#pragma unroll
        for (int w = 0; w < 4; ++w) vc.w[i][w] &= (2 * w < left ? 0xffffu : 0u) | (2 * w + 1 < left ? 0xffff0000u : 0u);
      }
    }
    bf16x8 pf[RB][NP];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float top = fmaxf(fmaxf(s[rb][0][0], s[rb][0][1]), fmaxf(s[rb][0][2], s[rb][0][3]));
      top = fmaxf(top, fmaxf(fmaxf(s[rb][1][0], s[rb][1][1]), fmaxf(s[rb][1][2], s[rb][1][3])));
      if (__builtin_amdgcn_ballot_w64(top > m_run[rb]) != 0) {   // the largest score of some row so far: rare on long contexts
        top = fmaxf(top, __shfl_xor(top, 16, 64));
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float m_new = fmaxf(m_run[rb], top);
        const float alpha = __builtin_amdgcn_exp2f((m_run[rb] - (m_new == -INFINITY ? 0.f : m_new)) * c);   // 0 at first
        m_run[rb] = m_new;
        l_run[rb] *= alpha;
#pragma unroll
        for (int i = 0; i < 4 * NV; ++i) o[rb][i] *= alpha;
      }
      const float ref = m_run[rb] == -INFINITY ? 0.f : m_run[rb] * c;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const f32x2 p = {__builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][e >> 2][e & 3], c, -ref)),
                         __builtin_amdgcn_exp2f(__builtin_fmaf(s[rb][e >> 2][(e & 3) + 1], c, -ref))};   // 0 behind the end
        l_run[rb] += p[0] + p[1];
        prob_parts(p, pf[rb], e);
      }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      uint32_t vf[4][4];   // [feature][pair of keys]
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t x = vc.w[i][w];
        const float s0 = mx_scale(vc.scale[i][w >> 1], (2 * w) & 3), s1 = mx_scale(vc.scale[i][w >> 1], (2 * w + 1) & 3);
        union { bf16x2 v; uint32_t u; } a0, a1, b0, b1;   // features 0, 1 and 2, 3 of both keys
        a0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s0, 0); a1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s1, 2);
        b0.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s0, 1); b1.v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, s1, 3);
        vf[0][w] = __builtin_amdgcn_perm(a1.u, a0.u, 0x05040100); vf[1][w] = __builtin_amdgcn_perm(a1.u, a0.u, 0x07060302);
        vf[2][w] = __builtin_amdgcn_perm(b1.u, b0.u, 0x05040100); vf[3][w] = __builtin_amdgcn_perm(b1.u, b0.u, 0x07060302);
      }
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            o[rb][4 * i + j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)vf[j], pf[rb][p], o[rb][4 * i + j], 0, 0, 0);
    }
    load_v(next, r_next);
    if (PAGED) r_next = a.c.block(b, kvh, min(k0 + 64 * KG, last));
  }

#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    l_run[rb] += __shfl_xor(l_run[rb], 16, 64);
    l_run[rb] += __shfl_xor(l_run[rb], 32, 64);
  }
  if constexpr (KG == 1) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = row0 + (rw * RB + rb) * 16 + ln;
      if (row >= p_rows) continue;
      if (g == 0) {
        a.part_m[part + row] = stored_max(m_run[rb] * c);
        a.part_l[part + row] = l_run[rb];
      }
      float *out = a.part_o + (part + row) * D + 16 * g;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(f32x4 *)(out + 64 * i + 4 * r) = f32x4{o[rb][4 * i][r], o[rb][4 * i + 1][r], o[rb][4 * i + 2][r], o[rb][4 * i + 3][r]};
    }
  } else {
    // ---- the key groups' sums through LDS, added in ascending order; a thread then takes four features of some rows
    float *so = (float *)lds;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      if (g == 0) { s_m[kg][(rw * RB + rb) * 16 + ln] = m_run[rb]; s_l[kg][(rw * RB + rb) * 16 + ln] = l_run[rb]; }
      float *w = so + (size_t)(kg * R + (rw * RB + rb) * 16 + ln) * LD + 16 * g;
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *(f32x4 *)(w + 64 * i + 4 * r) = f32x4{o[rb][4 * i][r], o[rb][4 * i + 1][r], o[rb][4 * i + 2][r], o[rb][4 * i + 3][r]};
    }
    __syncthreads();
    for (int x = threadIdx.x; x < min(R, p_rows - row0) * (D / 4); x += 256) {
      const int r = x / (D / 4), f = x % (D / 4) * 4;
      float m = -INFINITY, l = 0.f;
#pragma unroll
      for (int i = 0; i < KG; ++i) m = fmaxf(m, s_m[i][r]);
      const float m_safe = m == -INFINITY ? 0.f : m;
      f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < KG; ++i) {
        const float w = __builtin_amdgcn_exp2f((s_m[i][r] - m_safe) * c);   // 0 for a group without keys
        l += s_l[i][r] * w;
        v += *(const f32x4 *)(so + (size_t)(i * R + r) * LD + f) * w;
      }
      if (f == 0) {
        a.part_m[part + row0 + r] = stored_max(m * c);
        a.part_l[part + row0 + r] = l;
      }
      *(f32x4 *)(a.part_o + (part + row0 + r) * D + f) = v;
    }
  }
}

namespace {
enum { kOutPanels, kOutF32, kOutBf16 };
}

// Combine the partials of one (row, kv head) in ascending order, as k_attn_merge.  A row that saw no key at all (no context, no
// nodes of its own) is 0.
template <int D, int NB, int OUT>
__global__ __launch_bounds__(512) void k_mx_merge(MxAttnArgs a) {
  const int r = blockIdx.x, kvh = blockIdx.y, tid = threadIdx.x;
  const int M = a.n_nodes, group = a.group, b = r / M, node = r - b * M;
  const int p_rows = group * M, n = a.n_splits + a.n_draft;
  const size_t base = ((size_t)b * a.c.n_kv + kvh) * n;
  const int al = tid / (D / 2), f = (tid - al * (D / 2)) * 2;   // head, first feature
  if (al >= group) return;
  const int p = al * M + node;
  float num0 = 0.f, num1 = 0.f, den = 0.f;
  if (n > 0) {
    float pm[NB], pl[NB];
    float2 po[NB];
    auto request = [&](int s0) {
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        const size_t idx = (base + min(s0 + i, n - 1)) * p_rows + p;
        pm[i] = a.part_m[idx];
        pl[i] = a.part_l[idx];
        po[i] = *(const float2 *)(a.part_o + idx * D + f);
      }
    };
    request(0);
    float m_tot = -INFINITY;
#pragma unroll
    for (int i = 0; i < NB; ++i) m_tot = fmaxf(m_tot, i < n ? pm[i] : -INFINITY);
    for (int s0 = NB; s0 < n; s0 += 16) {   // many splits only
      float t[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) t[i] = a.part_m[(base + min(s0 + i, n - 1)) * p_rows + p];
#pragma unroll
      for (int i = 0; i < 16; ++i) m_tot = fmaxf(m_tot, t[i]);
    }
    for (int s0 = 0; s0 < n; s0 += NB) {
      if (s0 > 0) request(s0);
#pragma unroll
      for (int i = 0; i < NB; ++i) {
        if (s0 + i >= n || pm[i] == -INFINITY) continue;   // no key in it: its o was never written
        const float w = fast_exp(pm[i] - m_tot);
        num0 += po[i].x * w;
        num1 += po[i].y * w;
        den += pl[i] * w;
      }
    }
    if (m_tot == -INFINITY) den = 1.f;
  } else {
    den = 1.f;
  }
  const float o0 = num0 / den, o1 = num1 / den;
  const int kk = (kvh * group + al) * D + f;
  if constexpr (OUT == kOutPanels) {   // operand layout of the O projection; both features sit in the same 8-element run
    const bf16 h0 = (bf16)o0, h1 = (bf16)o1;
    bf16 *d0 = (bf16 *)a.out + ol_offset(r, kk, 0, (int)a.out_panel), *d1 = (bf16 *)a.out + ol_offset(r, kk, 1, (int)a.out_panel);
    d0[0] = h0; d0[1] = h1;
    d1[0] = (bf16)(o0 - (float)h0); d1[1] = (bf16)(o1 - (float)h1);
  } else if constexpr (OUT == kOutF32) {
    *(float2 *)((float *)a.out + r * a.out_row + kk) = float2{o0, o1};
  } else {
    *(bf16x2 *)((bf16 *)a.out + r * a.out_row + kk) = bf16x2{(bf16)o0, (bf16)o1};
  }
}

namespace {
template <int D, int OUT>
void launch_merge(hipStream_t st, const MxAttnArgs &a) {
  const int threads = a.group * D / 2 < 64 ? 64 : a.group * D / 2;   // <= 512 (group <= 8, d <= 128)
  const dim3 grid(a.batch * a.n_nodes, a.c.n_kv);
  const int n = a.n_splits + a.n_draft;
  if (n <= 6) hipLaunchKernelGGL((k_mx_merge<D, 6, OUT>), grid, dim3(threads), 0, st, a);
  else if (n <= 12) hipLaunchKernelGGL((k_mx_merge<D, 12, OUT>), grid, dim3(threads), 0, st, a);
  else hipLaunchKernelGGL((k_mx_merge<D, 20, OUT>), grid, dim3(threads), 0, st, a);
}

template <int D, typename T>
void launch_parts(hipStream_t st, const MxAttnArgs &a) {
  const dim3 grid(a.n_draft + a.n_splits + (a.append ? 1 : 0), a.c.n_kv, a.batch * a.n_row_groups);
  if (grid.x == 0) return;
#define TS_MX(RB_, RW_)                                                                                                  \
  do {                                                                                                                   \
    if (a.c.page_table) hipLaunchKernelGGL((k_mx_attn<D, RB_, RW_, T, true>), grid, dim3(256), 0, st, a);                \
    else hipLaunchKernelGGL((k_mx_attn<D, RB_, RW_, T, false>), grid, dim3(256), 0, st, a);                              \
  } while (0)
  const int form = a.row_blocks * 10 + a.row_waves;
  if (form == 11) TS_MX(1, 1);
  else if (form == 21) TS_MX(2, 1);
  else if (form == 22) TS_MX(2, 2);
  else if (form == 24) TS_MX(2, 4);
  else TS_MX(4, 4);
#undef TS_MX
}

template <int D>
void launch_d(hipStream_t st, const MxAttnArgs &a) {
  if (a.dtype == TRISPEC_F32) launch_parts<D, float>(st, a); else launch_parts<D, bf16>(st, a);
  if (a.out_row == 0) launch_merge<D, kOutPanels>(st, a);
  else if (a.dtype == TRISPEC_F32) launch_merge<D, kOutF32>(st, a);
  else launch_merge<D, kOutBf16>(st, a);
}
}  // namespace

void launch_mx_attn(hipStream_t st, const MxAttnArgs &a) {
  if (a.head_dim == 128) launch_d<128>(st, a); else launch_d<64>(st, a);
}

}  // namespace ts
