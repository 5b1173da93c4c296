// Rows into the 4-bit cache, rows out of it, and the move of a verified path inside it (layout: mx.hpp).
#include "mx.hpp"

namespace ts {

// Eight slots of a head a wavefront, as k_mx_read: quantised in registers, the four lanes of a block agree on its largest magnitude.  Bound by memory: 16384
// tokens of 8 heads of 128, 85 MB, in 15 us (5.6 TB/s), fp32 6.3 TB/s; a few tokens are a launch.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_mx_append(MxAppendArgs a) {
  const int h = blockIdx.y, b = blockIdx.z, first = a.start[b], n = a.count[b];
  const int group = (first / kMxGroup + (int)blockIdx.x * 4 + ((int)threadIdx.x >> 6)) * kMxGroup;
  if (group >= first + n) return;
  mx_store_group<D, T>(a.c, b, h, group, first, n, (const T *)a.k.p + (int64_t)b * a.k.seq + h * D, a.k.row,
                       (const T *)a.v.p + (int64_t)b * a.v.seq + h * D, a.v.row);
}

// Eight slots of a head a wavefront, eight lanes a slot; a lane stores 16 bytes at a time, so that the eight write a whole line of 128: fp32 rows in halves of
// lines, 32 bytes a lane, took 83 us instead of 55 (two sequences of 16384 tokens, 8 heads of 128).  What is written is not kept in the L2, where nobody
// reads it again before it is overwritten: 81 -> 50 us for four sequences in bf16 (6.8 TB/s).  Heads change fastest from workgroup to workgroup, as they lie in the rows.
template <int D, typename T>
__global__ __launch_bounds__(256) void k_mx_read(MxReadArgs a) {
  constexpr int N = 16 / sizeof(T), P = D / (8 * N);   // features of a store, stores of a lane
  const int h = blockIdx.x % a.c.n_kv, b = blockIdx.y, first = a.start[b], n = a.count[b], s = threadIdx.x >> 3 & 7, c = threadIdx.x & 7;
  const int group = (first / kMxGroup + (a.first_block + (int)(blockIdx.x / a.c.n_kv)) * 4 + ((int)threadIdx.x >> 6)) * kMxGroup, i = group + s - first;
  if (i < 0 || i >= n) return;
  const size_t r = a.c.block(b, h, group);
  const int at = a.c.in_block(group);
#pragma unroll
  for (int p = 0; p < P; ++p) {
    const int f = 8 * N * p + N * c;
    if (a.k) {
      const uint8_t *kc = a.c.k_codes + MxOffsets<D>::k_codes(a.c, r, at + s) + f / 2;
      const uint32_t w = N == 8 ? *(const uint32_t *)kc : *(const uint16_t *)kc;
      const uint32_t byte = a.c.k_scales[MxOffsets<D>::k_scales(a.c, r, at + s) + f / kMxBlock];
      stream16((T *)a.k + (int64_t)b * a.k_seq + (int64_t)i * a.k_row + h * D + f, mx_values(w, mx_scale(byte, 0)));
    }
    if (a.v) {
      const uint8_t *vc = a.c.v_codes + MxOffsets<D>::v_codes(a.c, r, at) + (f / 4) * 16 + 2 * s;
      const uint32_t w = *(const uint16_t *)vc | (N == 8 ? (uint32_t) * (const uint16_t *)(vc + 16) << 16 : 0u);
      const uint32_t byte = a.c.v_scales[MxOffsets<D>::v_scales(a.c, r, at) + 8 * (f / kMxBlock) + s];
      stream16((T *)a.v + (int64_t)b * a.v_seq + (int64_t)i * a.v_row + h * D + f, mx_values(w, mx_scale(byte, 0)));
    }
  }
}

// workgroups of four groups of 8 slots over the longest sequence's range
template <typename A>
static int mx_groups(const A &a, int batch) {
  int most = 0;
  for (int b = 0; b < batch; ++b)
    if (a.count[b] > 0) most = max(most, (a.start[b] + a.count[b] + kMxGroup - 1) / kMxGroup - a.start[b] / kMxGroup);
  return (most + 3) / 4;
}

void launch_mx_append(hipStream_t st, const MxAppendArgs &a, int batch) {
  const int n = mx_groups(a, batch);
  if (n == 0) return;
  const dim3 grid(n, a.c.n_kv, batch);
  if (a.head_dim == 128) {
    if (a.dtype == TRISPEC_F32) hipLaunchKernelGGL((k_mx_append<128, float>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_mx_append<128, bf16>), grid, dim3(256), 0, st, a);
  } else {
    if (a.dtype == TRISPEC_F32) hipLaunchKernelGGL((k_mx_append<64, float>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_mx_append<64, bf16>), grid, dim3(256), 0, st, a);
  }
}

void launch_mx_read(hipStream_t st, const MxReadArgs &args, int batch) {
  const int n = mx_groups(args, batch), most = (1 << 23) / args.c.n_kv;   // 2^31 threads a launch
  MxReadArgs a = args;
  for (a.first_block = 0; a.first_block < n; a.first_block += most) {
    const dim3 grid(min(n - a.first_block, most) * a.c.n_kv, batch);
    if (a.head_dim == 128) {
      if (a.dtype == TRISPEC_F32) hipLaunchKernelGGL((k_mx_read<128, float>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((k_mx_read<128, bf16>), grid, dim3(256), 0, st, a);
    } else {
      if (a.dtype == TRISPEC_F32) hipLaunchKernelGGL((k_mx_read<64, float>), grid, dim3(256), 0, st, a);
      else hipLaunchKernelGGL((k_mx_read<64, bf16>), grid, dim3(256), 0, st, a);
    }
  }
}

// Commit of a verified path (k_kv_commit) in the 4-bit cache: codes and scales of the path's nodes move from slot
// ctx + node[i] to slot ctx + i, read into registers whole before anything is written.
template <int D>
__global__ __launch_bounds__(256) void k_mx_commit(MxMap m, size_t slots_all, CommitTable t) {
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x;
  const int n = t.n[b], ctx = t.ctx[b];
  if (n == 0) return;   // uniform over the workgroup
  const size_t layer = blockIdx.z * slots_all;
  m.k_codes += layer * (D / 2); m.v_codes += layer * (D / 2);
  m.k_scales += layer * (D / kMxBlock); m.v_scales += layer * (D / kMxBlock);
  constexpr int KW = D / 8, VW = D / 4, SW = D / kMxBlock;   // words of a key, half words of a value, scales of either
  constexpr int KN = kMaxNodes * KW / 256, VN = kMaxNodes * VW / 256, SN = kMaxNodes * SW / 256;
  static_assert(SN >= 1, "every thread a scale");
  auto word = [&](int slot, int w) {
    return (uint32_t *)(m.k_codes + MxOffsets<D>::k_codes(m, m.block(b, h, slot), m.in_block(slot))) + w;
  };
  auto half = [&](int slot, int q) {
    const int s = m.in_block(slot);
    return (uint16_t *)(m.v_codes + MxOffsets<D>::v_codes(m, m.block(b, h, slot), s & ~7)) + q * 8 + (s & 7);
  };
  auto k_scale = [&](int slot, int w) { return m.k_scales + MxOffsets<D>::k_scales(m, m.block(b, h, slot), m.in_block(slot)) + w; };
  auto v_scale = [&](int slot, int w) {
    const int s = m.in_block(slot);
    return m.v_scales + MxOffsets<D>::v_scales(m, m.block(b, h, slot), s & ~7) + 8 * w + (s & 7);
  };
  uint32_t kw[KN];
  uint16_t vw[VN];
  uint8_t ks[SN], vs[SN];
#pragma unroll
  for (int u = 0; u < KN; ++u) {
    const int i = (tid + 256 * u) / KW, w = (tid + 256 * u) % KW;
    if (i < n) kw[u] = *word(ctx + t.node[b][i], w);
  }
#pragma unroll
  for (int u = 0; u < VN; ++u) {
    const int i = (tid + 256 * u) / VW, w = (tid + 256 * u) % VW;
    if (i < n) vw[u] = *half(ctx + t.node[b][i], w);
  }
#pragma unroll
  for (int u = 0; u < SN; ++u) {
    const int i = (tid + 256 * u) / SW, w = (tid + 256 * u) % SW;
    if (i < n) { ks[u] = *k_scale(ctx + t.node[b][i], w); vs[u] = *v_scale(ctx + t.node[b][i], w); }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < KN; ++u) {
    const int i = (tid + 256 * u) / KW, w = (tid + 256 * u) % KW;
    if (i < n) *word(ctx + i, w) = kw[u];
  }
#pragma unroll
  for (int u = 0; u < VN; ++u) {
    const int i = (tid + 256 * u) / VW, w = (tid + 256 * u) % VW;
    if (i < n) *half(ctx + i, w) = vw[u];
  }
#pragma unroll
  for (int u = 0; u < SN; ++u) {
    const int i = (tid + 256 * u) / SW, w = (tid + 256 * u) % SW;
    if (i < n) { *k_scale(ctx + i, w) = ks[u]; *v_scale(ctx + i, w) = vs[u]; }
  }
}

void launch_mx_commit(hipStream_t st, const MxMap &m, int head_dim, size_t slots_all, int n_layers, int batch, const CommitTable &t) {
  const dim3 grid(m.n_kv, batch, n_layers);
  if (head_dim == 128) hipLaunchKernelGGL(k_mx_commit<128>, grid, dim3(256), 0, st, m, slots_all, t);
  else hipLaunchKernelGGL(k_mx_commit<64>, grid, dim3(256), 0, st, m, slots_all, t);
}

}  // namespace ts
