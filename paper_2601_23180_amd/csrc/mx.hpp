// The cache held in 4 bits: its layout, the conversions, and what its kernels take.
//
// Blocks of 32 features of one head of one slot share a scale 2^(byte - 127); an element is a sign and one of 0, 0.5, 1, 1.5, 2, 3,
// 4, 6 (the MXFP4 format of the OCP microscaling specification).  A value read back is exact in bf16, and gfx950 converts two
// of them, scale included, with one instruction.
// One layer, nkv kv heads, S slots in a block of memory (a sequence's capacity, or a page):
//   K codes  [block][nkv][S][d / 2]            scales [block][nkv][S][d / 32]
//   V codes  [block][nkv][S / 8][d / 4][8][2]  scales [block][nkv][S / 8][d / 32][8]
// K: a lane reads 16 bytes of a key as an operand of the first product (reduction over features).  V: the second product
// reduces over keys, so four features of eight keys lie side by side: 16 bytes hold a lane's operands of four instructions,
// and a row is still written without touching its neighbours' bytes.
#pragma once

#include "device_util.hpp"

namespace ts {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));   // native vectors: stay in registers
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) float f32x2;

__device__ __forceinline__ f32x4 load4(const float *p) { return *(const f32x4 *)p; }
__device__ __forceinline__ f32x4 load4(const bf16 *p) {
  const bf16x4 v = *(const bf16x4 *)p;
  return f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]};
}

constexpr int kMxBlock = 32;   // features that share a scale
constexpr int kMxGroup = 8;    // slots whose values lie side by side

// One layer of the cache.
struct MxMap {
  uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
  const int32_t *page_table;   // device [batch][max_pages], or nullptr: a block per sequence
  int32_t max_pages, n_pages;  // page ids are clamped into [0, n_pages)
  int32_t slots;               // of a block
  int32_t n_kv;
  // row of blocks of (sequence, kv head), and the slot in it: all four arrays are addressed with these two
  __device__ __forceinline__ size_t block(int b, int h, int slot) const {
    if (!page_table) return (size_t)b * n_kv + h;
    const int p = page_table[(size_t)b * max_pages + min(slot / kKvPage, max_pages - 1)];
    return (size_t)min(max(p, 0), n_pages - 1) * n_kv + h;
  }
  __device__ __forceinline__ int in_block(int slot) const { return page_table ? slot % kKvPage : slot; }
};
template <int D>
struct MxOffsets {   // bytes from an array's start of (block row r, slot s of it)
  static __device__ __forceinline__ size_t k_codes(const MxMap &m, size_t r, int s) { return (r * m.slots + s) * (D / 2); }
  static __device__ __forceinline__ size_t k_scales(const MxMap &m, size_t r, int s) { return (r * m.slots + s) * (D / kMxBlock); }
  // V: s a multiple of 8; the group's codes are (D / 4) runs of 16 bytes, its scales D / 32 runs of 8
  static __device__ __forceinline__ size_t v_codes(const MxMap &m, size_t r, int s) { return (r * m.slots + s) * (D / 2); }
  static __device__ __forceinline__ size_t v_scales(const MxMap &m, size_t r, int s) { return (r * m.slots + s) * (D / kMxBlock); }
};

// The conversion instructions take a scale from bits 30..23 of a register and ignore the others; byte 0 is 2^-127, 255 a NaN
// whatever the element.
__device__ __forceinline__ float mx_scale(uint32_t w, int byte) {
  return __uint_as_float(byte == 0 ? w << 23 : byte == 1 ? w << 15 : byte == 2 ? w << 7 : w >> 1);
}
// eight elements of one block
__device__ __forceinline__ bf16x8 mx_values(uint32_t w, float s) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The scale byte of a block whose largest magnitude is `top` (its bits: finite, or not): the largest element ends up
// below 7 times the scale, so that rounding to nearest, 6 included, is all that happens to it.  The largest scale is 2^125:
// 6 times it is finite in bf16, and what lies above is cut off at it.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = (int)((top + 0x00200000u) >> 23) - 2;   // 1.75 and more carries into the exponent
  return (uint32_t)min(max(e, 0), 252);
}

// Rows of K or V, or the like: element (sequence b, row i, head h, feature f) is p[b * seq + i * row + h * d + f].
struct MxRows {
  const void *p;
  int64_t row, seq;
};

// A wavefront takes eight slots (a group) of one kv head: lane (s, c) features 8 c .. 8 c + 7 of slot s, and for d = 128 the
// same of the second half; four lanes side by side hold a block.  16 bytes of bf16 a lane, 128 side by side.
template <int D>
struct MxLane {
  static constexpr int P = D / 64;   // runs of eight features a lane
  int s, c;
  __device__ MxLane(int lane) : s(lane >> 3), c(lane & 7) {}
  __device__ __forceinline__ int feature(int p) const { return 64 * p + 8 * c; }
  __device__ __forceinline__ int scale(int p) const { return 2 * p + (c >> 2); }   // which of the slot's blocks
  __device__ __forceinline__ bool first() const { return (c & 3) == 0; }
};

typedef __attribute__((ext_vector_type(8))) float f32x8;
__device__ __forceinline__ f32x8 load8(const float *p) {
  const f32x4 a = *(const f32x4 *)p, b = *(const f32x4 *)(p + 4);
  return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ f32x8 load8(const bf16 *p) {
  const bf16x8 a = *(const bf16x8 *)p;
  return f32x8{(float)a[0], (float)a[1], (float)a[2], (float)a[3], (float)a[4], (float)a[5], (float)a[6], (float)a[7]};
}
// 16 bytes of a row, past the L2: four fp32 features or eight in bf16, the first of v
__device__ __forceinline__ void stream16(float *p, bf16x8 v) { __builtin_nontemporal_store(f32x4{(float)v[0], (float)v[1], (float)v[2], (float)v[3]}, (f32x4 *)p); }
__device__ __forceinline__ void stream16(bf16 *p, bf16x8 v) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v), (u32x4 *)p); }

// Eight features of a block that four lanes side by side hold: their codes, and the block's scale byte.
__device__ __forceinline__ uint32_t mx_quantise(const f32x8 &x, uint32_t &byte) {
  uint32_t top = 0;   // magnitudes compare as integers; a NaN is above them all
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
  top = max(top, (uint32_t)__shfl_xor((int)top, 1, 64));
  top = max(top, (uint32_t)__shfl_xor((int)top, 2, 64));
  byte = mx_scale_byte(top);
  const float s = __uint_as_float(byte << 23);
  uint32_t w = 0;   // rounds to nearest, ties to the even code, cuts off at 6
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[0], x[1], s, 0);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], s, 1);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], s, 2);
  w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], s, 3);
  return byte == 255 ? 0u : w;
}

// Slots first .. first + n of one (sequence, kv head), of which this wavefront takes the group that starts at `group`
// (a multiple of 8); row i of k and v goes to slot first + i.  Memory is all it costs: the rows once, 0.53 bytes an element.
template <int D, typename T>
__device__ __forceinline__ void mx_store_group(const MxMap &m, int b, int h, int group, int first, int n, const T *k, int64_t k_row, const T *v,
                                               int64_t v_row) {
  using L = MxLane<D>;
  const L l(threadIdx.x & 63);
  const int slot = group + l.s, i = slot - first;
  const bool live = i >= 0 && i < n;
  const int ic = min(max(i, 0), n - 1);
  f32x8 xk[L::P], xv[L::P];
#pragma unroll
  for (int p = 0; p < L::P; ++p) {
    xk[p] = load8(k + (int64_t)ic * k_row + l.feature(p));
    xv[p] = load8(v + (int64_t)ic * v_row + l.feature(p));
  }
  const size_t r = m.block(b, h, group);
  const int at = m.in_block(group);
#pragma unroll
  for (int p = 0; p < L::P; ++p) {
    uint32_t bk, bv;
    const uint32_t wk = mx_quantise(xk[p], bk), wv = mx_quantise(xv[p], bv);
    if (!live) continue;
    *(uint32_t *)(m.k_codes + MxOffsets<D>::k_codes(m, r, at + l.s) + l.feature(p) / 2) = wk;
    uint8_t *vc = m.v_codes + MxOffsets<D>::v_codes(m, r, at) + (l.feature(p) / 4) * 16 + 2 * l.s;
    *(uint16_t *)vc = (uint16_t)wv;
    *(uint16_t *)(vc + 16) = (uint16_t)(wv >> 16);
    if (l.first()) {
      m.k_scales[MxOffsets<D>::k_scales(m, r, at + l.s) + l.scale(p)] = (uint8_t)bk;
      m.v_scales[MxOffsets<D>::v_scales(m, r, at) + 8 * l.scale(p) + l.s] = (uint8_t)bv;
    }
  }
}

struct MxAppendArgs {
  MxMap c;
  MxRows k, v;
  int32_t head_dim, dtype;
  int32_t start[kMaxBatch], count[kMaxBatch];
};
struct MxReadArgs {
  MxMap c;
  void *k, *v;               // either may be nullptr
  int64_t k_row, k_seq, v_row, v_seq;
  int32_t head_dim, dtype;
  int32_t start[kMaxBatch], count[kMaxBatch];
  int32_t first_block;   // of a head's: large ranges go out in several launches
};
void launch_mx_append(hipStream_t st, const MxAppendArgs &a, int batch);
void launch_mx_read(hipStream_t st, const MxReadArgs &a, int batch);
// slots_all: slots of all blocks and kv heads of a layer; layer l lies l * slots_all * (d / 2 or d / 32) bytes behind layer 0
void launch_mx_commit(hipStream_t st, const MxMap &c, int head_dim, size_t slots_all, int n_layers, int batch, const CommitTable &t);

// Whose root paths the nodes have: a device array of masks, the parents by value, or every node's predecessor.
struct MxAttnArgs {
  MxMap c;
  CtxLens ctx;
  MxRows q, k, v;             // k.p == nullptr: the nodes see the cache alone
  const AncMask *anc;         // [batch * n_nodes], or nullptr
  uint8_t parent[kMaxRows];   // of node i > 0 (its own number: the root); read where anc is nullptr and !chain
  int32_t chain;
  int32_t batch, n_nodes, n_q_heads, group, head_dim, dtype;
  int32_t append;             // the nodes' K and V go to slots ctx + i
  int32_t whole, form;        // form: kMxRows*
  int32_t n_row_groups, n_own, keys;       // keys of a split; n_own: partials of a sequence's nodes
  int32_t split0[kMaxBatch + 1];           // splits before those of sequence b
  float *part_o, *part_m, *part_l;         // as in AttnArgs; a sequence's splits, then its nodes
  // rows of partial i and kv head h
  __host__ __device__ size_t part(int i, int h) const { return ((size_t)i * c.n_kv + h) * (group * n_nodes); }
  void *out;                  // rows [batch * n_nodes][n_q_heads * d] in dtype, or operand panels
  int64_t out_row;            // elements between rows; 0: operand panels of out_panel 32-row blocks
  size_t out_panel;
};
void launch_mx_attn(hipStream_t st, const MxAttnArgs &a);

}  // namespace ts
