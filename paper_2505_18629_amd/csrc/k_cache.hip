// Operators on the K/V cache: rows appended (per-head norms and rotation on the
// way) and read back, tiles copied between sequences, the ownership table.
#include "rv_internal.h"

namespace {

constexpr int kBlockPos = 32;  // positions per workgroup of append and read: one V block of a bf16 cache

// Workgroup x of a launch over the 32-position blocks of every sequence's rows:
// sequence b with blk0[b] <= x < blk0[b + 1].  The lanes look at all entries at
// once: kernel arguments come from host memory, and a search would wait for one
// after the other.
RV_DEV int find_seq(const int* blk0, int B, int x) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int j = 0; j < RV_MAX_BATCH / 64; ++j) {
    const int b = lane + 64 * j;
    if (64 * j < B) n += __popcll(__ballot(b < B && blk0[b] <= x));
  }
  return n - 1;
}

template <bool ONCE, typename V>
RV_DEV V load_vec(const V* p) {
  return ONCE ? __builtin_nontemporal_load(p) : *p;
}
// 8 consecutive values of a row of fp32 or bf16 as fp32, and back.  ONCE: a row
// that nothing reads after this kernel, past the L2 (see k_append).
template <int IO, bool ONCE = false>
RV_DEV void load8(const void* p, size_t i, float (&x)[8]) {
  if constexpr (IO == RV_F32) {
    const f32x4_t a = load_vec<ONCE>((const f32x4_t*)((const float*)p + i));
    const f32x4_t b = load_vec<ONCE>((const f32x4_t*)((const float*)p + i + 4));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  } else {
    const u32x4 r = load_vec<ONCE>((const u32x4*)((const uint16_t*)p + i));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(r[j] << 16);
      x[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
  }
}
RV_DEV u32x4 pack8(const float (&x)[8]) {
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = f2bf(x[2 * j]) | (uint32_t)f2bf(x[2 * j + 1]) << 16;
  return r;
}
template <int IO>
RV_DEV void store8(void* p, size_t i, const float (&x)[8]) {
  if constexpr (IO == RV_F32) {
    *(f32x4_t*)((float*)p + i) = f32x4_t{x[0], x[1], x[2], x[3]};
    *(f32x4_t*)((float*)p + i + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
  } else {
    *(u32x4*)((uint16_t*)p + i) = pack8(x);
  }
}

// 8 consecutive dims of a K row, or 8 values of one V unit, as the pair of planes.
RV_DEV void store_pair8(void* hi, void* lo, size_t i, const float (&x)[8]) {
  float l[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) l[j] = x[j] - bf2f(f2bf(x[j]));
  *(u32x4*)((uint16_t*)hi + i) = pack8(x);
  *(u32x4*)((uint16_t*)lo + i) = pack8(l);
}
RV_DEV void load_pair8(const void* hi, const void* lo, size_t i, float (&x)[8]) {
  float l[8];
  load8<RV_BF16>(hi, i, x);
  load8<RV_BF16>(lo, i, l);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] += l[j];
}

// Whether keys [k_lo, k_hi) of a V block hold any of slot group g's.
RV_DEV bool group_touched(int g, int k_lo, int k_hi) {
  return (4 * g < k_hi && 4 * g + 4 > k_lo) || (16 + 4 * g < k_hi && 20 + 4 * g > k_lo);
}

// ----------------------------------------------------------- append
// Row r of sequence b at position p = pos[b] + r, per head of q and k:
//   y = x / sqrt(mean(x^2) + eps) * g              (with gains)
//   (o_i, o_{i+hd/2}) = (y_i c - y_{i+hd/2} s, y_{i+hd/2} c + y_i s)   (rotate)
// with c, s of the angle p base^(-2i/hd) from the cache's rotary table; q goes
// to q_out, k and v to the cache.  Statistics and rotation are fp32.
//
// Workgroups: (32-position block of a sequence) x (hpw q or k heads, or one v
// head).  hd / 16 threads per (row, head) own dims d..d+7 and their partners
// d+hd/2..: 16-byte loads and stores throughout, the norm is a sum over those
// threads, and rows are adjacent in a wave, so that a K unit of the bf16 cache
// (16 positions x 32 dims) is written whole.  A thread keeps its row's rotary
// factors for up to kHeadRounds rounds of kHeadBatch heads whose loads it issues
// together.  A V unit holds 8 positions of one dim:
// rows go through LDS and each thread writes the 8 positions of a (dim, slot
// group) with one store -- 2-byte stores of single positions remain for the
// groups that the rows fill in part.
//
// Bound by HBM for prompts: 6 of 300-1100 tokens at the 8B shape in bf16, 148 MB,
// 31 us (4.7 TB/s; 36 with plain loads of the rows, 37 with nontemporal stores of K
// and V, which are read soon; heads four a batch take 2.5 more than two, one a batch
// 0.4).  A verify block (4 x 43 fp32 rows, 14B) takes 6.5 us, a few rows 3.5: launch,
// arguments, row, store.
constexpr int kHeadBatch = 2, kHeadRounds = 4;
template <int DT, int IO, int HD>
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
  constexpr int HALF = HD / 2, TPH = HD / 16;  // threads per (row, head)
  __shared__ float sv[kBlockPos][HD + 1];
  const int x = blockIdx.x, b = find_seq(a.blk0, a.B, x);
  const int pos0 = a.pos[b], n = a.row0[b + 1] - a.row0[b];
  const int blk = pos0 / kBlockPos + (x - a.blk0[b]);
  const int p_lo = max(pos0, blk * kBlockPos), p_hi = min(pos0 + n, (blk + 1) * kBlockPos);
  const int rows = p_hi - p_lo, row_lo = a.row0[b] + (p_lo - pos0);
  const int tid = threadIdx.x;
  const int n_qk = a.n_heads + a.n_kv;

  // q and k heads: thread -> (head of the batch's first, row, part), parts fastest, then rows
  if ((int)blockIdx.y < a.qk_groups) {
    const int h_lo = blockIdx.y * a.hpw, h_end = min(h_lo + a.hpw, n_qk);
    const int per_head = rows * TPH, par = 256 / per_head;  // heads side by side
    if (tid >= par * per_head) return;
    const int r = tid % per_head / TPH, d = tid % TPH * 8, p = p_lo + r;
    float cs[8], sn[8], gq1[8], gq2[8], gk1[8], gk2[8];
    if (a.rotate) {
      load8<RV_F32>(a.rope_cos, (size_t)p * HALF + d, cs);
      load8<RV_F32>(a.rope_sin, (size_t)p * HALF + d, sn);
    }
    if (a.q_gain) {
      load8<RV_F32>(a.q_gain, d, gq1);
      load8<RV_F32>(a.q_gain, HALF + d, gq2);
    }
    if (a.k_gain) {
      load8<RV_F32>(a.k_gain, d, gk1);
      load8<RV_F32>(a.k_gain, HALF + d, gk2);
    }
    for (int h0 = h_lo + tid / per_head; h0 < h_end; h0 += kHeadBatch * par) {
      float y1[kHeadBatch][8], y2[kHeadBatch][8];
#pragma unroll
      for (int u = 0; u < kHeadBatch; ++u) {
        const int h = min(h0 + u * par, h_end - 1);  // past the last: that one again, not stored
        const bool is_q = h < a.n_heads;
        const void* src = is_q ? a.q : a.k;
        const size_t at = (size_t)(row_lo + r) * (is_q ? a.ldq : a.ldk) + (size_t)(is_q ? h : h - a.n_heads) * HD + d;
        load8<IO, true>(src, at, y1[u]);
        load8<IO, true>(src, at + HALF, y2[u]);
      }
#pragma unroll
      for (int u = 0; u < kHeadBatch; ++u) {
        const int h = h0 + u * par;
        if (h >= h_end) break;
        const bool is_q = h < a.n_heads;
        const int hh = is_q ? h : h - a.n_heads;
        if (is_q ? a.q_gain : a.k_gain) {
          float ss = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) ss += y1[u][j] * y1[u][j] + y2[u][j] * y2[u][j];
#pragma unroll
          for (int m = 1; m < TPH; m *= 2) ss += __shfl_xor(ss, m, 64);
          const float rs = 1.0f / sqrtf(ss / (float)HD + a.eps);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            y1[u][j] = y1[u][j] * rs * (is_q ? gq1[j] : gk1[j]);
            y2[u][j] = y2[u][j] * rs * (is_q ? gq2[j] : gk2[j]);
          }
        }
        if (a.rotate) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const float e = y1[u][j], f = y2[u][j];
            y1[u][j] = e * cs[j] - f * sn[j];
            y2[u][j] = f * cs[j] + e * sn[j];
          }
        }
        if (is_q) {
          const size_t o = (size_t)(row_lo + r) * a.ldqo + (size_t)hh * HD + d;
          store8<IO>(a.q_out, o, y1[u]);
          store8<IO>(a.q_out, o + HALF, y2[u]);
        } else {
          const size_t base = (size_t)(b * a.n_kv + hh) * a.kv_len * HD;
          if constexpr (DT == RV_BF16) {
            store_pair8(a.kc, a.kc2, base + k_elem(p, d, HD), y1[u]);
            store_pair8(a.kc, a.kc2, base + k_elem(p, HALF + d, HD), y2[u]);
          } else {
            store8<RV_F32>(a.kc, base + (size_t)p * HD + d, y1[u]);
            store8<RV_F32>(a.kc, base + (size_t)p * HD + HALF + d, y2[u]);
          }
        }
      }
    }
    return;
  }

  // one v head
  const int hh = blockIdx.y - a.qk_groups;
  const size_t base = (size_t)(b * a.n_kv + hh) * a.kv_len * HD;
  for (int i = tid; i < rows * (HD / 8); i += 256) {
    const int r = i / (HD / 8), d = i % (HD / 8) * 8;
    float y[8];
    load8<IO, true>(a.v, (size_t)(row_lo + r) * a.ldv + (size_t)hh * HD + d, y);
    if constexpr (DT == RV_F32) {
      store8<RV_F32>(a.vc, base + (size_t)(p_lo + r) * HD + d, y);
    } else {
      const int kk = p_lo + r - blk * kBlockPos;
#pragma unroll
      for (int j = 0; j < 8; ++j) sv[kk][d + j] = y[j];
    }
  }
  if constexpr (DT == RV_BF16) {
    __syncthreads();
    const int k_lo = p_lo - blk * kBlockPos, k_hi = p_hi - blk * kBlockPos;
    for (int i = tid; i < HD * 4; i += 256) {
      const int g = i / HD, d = i % HD;  // keys 4g..4g+3 and 16+4g..16+4g+3 of the block
      if (!group_touched(g, k_lo, k_hi)) continue;
      const size_t at = base + v_elem(blk * kBlockPos + 4 * g, d, HD);
      float y[8];
      bool all = true;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int kk = 4 * g + (j & 3) + 16 * (j >> 2);
        all = all && kk >= k_lo && kk < k_hi;
        y[j] = sv[kk][d];
      }
      if (all) {
        store_pair8(a.vc, a.vc2, at, y);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int kk = 4 * g + (j & 3) + 16 * (j >> 2);
          if (kk < k_lo || kk >= k_hi) continue;
          const uint16_t hb = f2bf(y[j]);
          ((uint16_t*)a.vc)[at + j] = hb;
          ((uint16_t*)a.vc2)[at + j] = f2bf(y[j] - bf2f(hb));
        }
      }
    }
  }
}

// ----------------------------------------------------------- read
// The inverse for K and V: cached rows as values (hi + lo), wherever the tile
// lies.  Workgroups as above over the k and v heads.  Bound by HBM or the
// last-level cache (the prompts above, just appended, as bf16: 11.5 us).
template <int DT, int IO, int HD>
__global__ __launch_bounds__(256) void k_read(ReadArgs a) {
  __shared__ float sv[kBlockPos][HD + 1];
  const int x = blockIdx.x, b = find_seq(a.blk0, a.B, x);
  const int pos0 = a.pos[b], n = a.row0[b + 1] - a.row0[b];
  const int blk = pos0 / kBlockPos + (x - a.blk0[b]);
  const int p_lo = max(pos0, blk * kBlockPos), p_hi = min(pos0 + n, (blk + 1) * kBlockPos);
  const int rows = p_hi - p_lo, row_lo = a.row0[b] + (p_lo - pos0);
  const int slot = a.own[(size_t)b * (a.kv_len / 64) + blk / 2];
  const int tid = threadIdx.x;
  const int h_lo = blockIdx.y * a.hpw, h_end = min(h_lo + a.hpw, 2 * a.n_kv);

  const int k_end = min(h_end, a.n_kv), per_head = rows * (HD / 8);
  for (int i = tid; i < (k_end - h_lo) * per_head; i += 256) {
    const int h = h_lo + i / per_head, r = i % per_head / (HD / 8), d = i % (HD / 8) * 8, p = p_lo + r;
    const size_t base = (size_t)(slot * a.n_kv + h) * a.kv_len * HD;
    float y[8];
    if constexpr (DT == RV_BF16) load_pair8(a.kc, a.kc2, base + k_elem(p, d, HD), y);
    else load8<RV_F32>(a.kc, base + (size_t)p * HD + d, y);
    store8<IO>(a.k, (size_t)(row_lo + r) * a.ldk + (size_t)h * HD + d, y);
  }
  for (int h = max(h_lo, a.n_kv); h < h_end; ++h) {
    const int hh = h - a.n_kv;
    const size_t base = (size_t)(slot * a.n_kv + hh) * a.kv_len * HD;
    const int k_lo = p_lo - blk * kBlockPos, k_hi = p_hi - blk * kBlockPos;
    if constexpr (DT == RV_BF16) {
      __syncthreads();  // the last head's rows have been read
      for (int i = tid; i < HD * 4; i += 256) {
        const int g = i / HD, d = i % HD;
        if (!group_touched(g, k_lo, k_hi)) continue;
        float y[8];
        load_pair8(a.vc, a.vc2, base + v_elem(blk * kBlockPos + 4 * g, d, HD), y);
#pragma unroll
        for (int j = 0; j < 8; ++j) sv[4 * g + (j & 3) + 16 * (j >> 2)][d] = y[j];
      }
      __syncthreads();
    }
    for (int i = tid; i < rows * (HD / 8); i += 256) {
      const int r = i / (HD / 8), d = i % (HD / 8) * 8;
      float y[8];
      if constexpr (DT == RV_F32) {
        load8<RV_F32>(a.vc, base + (size_t)(p_lo + r) * HD + d, y);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = sv[k_lo + r][d + j];
      }
      store8<IO>(a.v, (size_t)(row_lo + r) * a.ldv + (size_t)hh * HD + d, y);
    }
  }
}

// ----------------------------------------------------------- copy
// The moves of one unit (rv_tiles.h) on values of type V: every load of a batch
// of moves is issued before its first store, N values of stride `step` for each.
// A thread's values belong to it alone, so the units' order is its program order.
template <typename V, int N, typename Addr, typename On>
RV_DEV void run_moves(const CopyProgram& p, int unit, Addr addr, On on, int step, int left) {
  V saved[N];
  const int sv = p.saved[unit];
  if (sv >= 0) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (i * step < left) saved[i] = addr(sv)[i * step];
  }
  const int end = p.unit0[unit + 1];
  for (int m0 = p.unit0[unit]; m0 < end; m0 += kMoveBatch) {
    V v[kMoveBatch][N];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int m = m0 + u;
      if (m >= end || !on(p.len[m])) continue;
      const V* s = addr(p.src[m]);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i * step < left) v[u][i] = p.from_saved[m] ? saved[i] : __builtin_nontemporal_load(s + i * step);
    }
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int m = m0 + u;
      if (m >= end || !on(p.len[m])) continue;
      V* d = addr(p.dst[m]);
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (i * step < left) __builtin_nontemporal_store(v[u][i], d + i * step);
    }
  }
}

// One workgroup per (plane, layer, kv head, tile) and unit of moves; a tile of
// one head is one contiguous span of a slot in every cache layout.  Lengths
// count committed tokens: K and V of positions 0 .. len-2 come in whole tiles,
// the ids 0 .. len-1 one by one (further workgroups, a thread each), and the
// sequence's bad-id flag with them (one more).  Bound by HBM: 16 sequences of
// 512-2048 tokens in a new order, 8 layers of the 8B shape, 2.38 GB read and
// written in 519 us (4.6 TB/s; a large copy reaches 5.5; 546 with kCopyVecs 2, 531 with 8,
// 535 with plain stores).
constexpr int kCopyVecs = 4;  // 16-byte values per thread and move
__global__ __launch_bounds__(256) void k_copy(CopyArgs a) {
  const int unit = blockIdx.y, tid = threadIdx.x;
  int x = blockIdx.x;
  const int tiles = a.tile1 - a.tile0, n_kv_blocks = a.planes * a.layers * a.n_kv * tiles;
  if (x < n_kv_blocks) {
    const int t = a.tile0 + x % tiles;
    x /= tiles;
    const int h = x % a.n_kv, l = x / a.n_kv % a.layers, pl = x / a.n_kv / a.layers;
    u32x4* base = (u32x4*)a.plane[pl] + (size_t)l * a.layer_vecs + (size_t)h * a.head_vecs + (size_t)t * a.tile_vecs;
    auto on = [&](int len) { return t * 64 < len - 1; };
    for (int v0 = tid; v0 < a.tile_vecs; v0 += 256 * kCopyVecs)
      run_moves<u32x4, kCopyVecs>(
          a.p, unit, [&](int s) { return base + (size_t)s * a.slot_vecs + v0; }, on, 256, a.tile_vecs - v0);
    return;
  }
  const int i = (x - n_kv_blocks) * 256 + tid;
  if (i < a.max_len)
    run_moves<int, 1>(
        a.p, unit, [&](int s) { return a.ids + (size_t)s * a.max_len + i; }, [&](int len) { return i < len; }, 1, 1);
  else if (i == a.max_len)
    run_moves<int, 1>(
        a.p, unit, [&](int s) { return a.seq_bad + s; }, [](int) { return true; }, 1, 1);
}

// Ownership rows: sequence seq[y] reads its first `whole` tiles where `src` does
// and the rest in its own slot.
__global__ __launch_bounds__(256) void k_own(OwnArgs a) {
  const int t = blockIdx.x * 256 + threadIdx.x, b = a.seq[blockIdx.y];
  if (t < a.T) a.own[(size_t)b * a.T + t] = t < a.whole ? a.own[(size_t)a.src * a.T + t] : b;
}

template <int DT, int IO>
hipError_t append_hd(const AppendArgs& a, int hd, dim3 grid, hipStream_t st) {
  switch (hd) {
    case 32: k_append<DT, IO, 32><<<grid, 256, 0, st>>>(a); break;
    case 64: k_append<DT, IO, 64><<<grid, 256, 0, st>>>(a); break;
    case 128: k_append<DT, IO, 128><<<grid, 256, 0, st>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}
template <int DT, int IO>
hipError_t read_hd(const ReadArgs& a, int hd, dim3 grid, hipStream_t st) {
  switch (hd) {
    case 32: k_read<DT, IO, 32><<<grid, 256, 0, st>>>(a); break;
    case 64: k_read<DT, IO, 64><<<grid, 256, 0, st>>>(a); break;
    case 128: k_read<DT, IO, 128><<<grid, 256, 0, st>>>(a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

// Heads per workgroup: as many as give its 256 threads one item each.
int heads_per_wg(int max_rows, int threads_per_row, int heads) {
  const int rows = max_rows < kBlockPos ? max_rows : kBlockPos;
  int n = 256 / (rows * threads_per_row);
  if (n < 1) n = 1;
  return n < heads ? n : heads;
}

}  // namespace

int span_blocks(int pos, int rows) { return rows ? (pos + rows - 1) / kBlockPos - pos / kBlockPos + 1 : 0; }

hipError_t launch_append(int dtype, int io, int hd, int max_rows, AppendArgs& a, hipStream_t st) {
  // heads side by side, and as many rounds of them as leave four workgroups to a CU
  const int heads = a.n_heads + a.n_kv, par = heads_per_wg(max_rows, hd / 16, heads);
  int rounds = kHeadRounds;
  while (rounds > 1 && (long long)a.blk0[a.B] * ((heads + par * rounds - 1) / (par * rounds)) < 1024) rounds /= 2;
  a.hpw = par * rounds;
  a.qk_groups = (heads + a.hpw - 1) / a.hpw;
  const dim3 grid(a.blk0[a.B], a.qk_groups + a.n_kv);
  if (dtype == RV_BF16)
    return io == RV_F32 ? append_hd<RV_BF16, RV_F32>(a, hd, grid, st) : append_hd<RV_BF16, RV_BF16>(a, hd, grid, st);
  return io == RV_F32 ? append_hd<RV_F32, RV_F32>(a, hd, grid, st) : append_hd<RV_F32, RV_BF16>(a, hd, grid, st);
}

hipError_t launch_read(int dtype, int io, int hd, int max_rows, ReadArgs& a, hipStream_t st) {
  a.hpw = heads_per_wg(max_rows, hd / 8, 2 * a.n_kv);
  const dim3 grid(a.blk0[a.B], (2 * a.n_kv + a.hpw - 1) / a.hpw);
  if (dtype == RV_BF16)
    return io == RV_F32 ? read_hd<RV_BF16, RV_F32>(a, hd, grid, st) : read_hd<RV_BF16, RV_BF16>(a, hd, grid, st);
  return io == RV_F32 ? read_hd<RV_F32, RV_F32>(a, hd, grid, st) : read_hd<RV_F32, RV_BF16>(a, hd, grid, st);
}

hipError_t launch_copy(const CopyArgs& a, bool with_ids, hipStream_t st) {
  if (!a.p.units) return hipSuccess;
  const size_t blocks = (size_t)a.planes * a.layers * a.n_kv * (a.tile1 - a.tile0) +
                        (with_ids ? (size_t)(a.max_len + 1 + 255) / 256 : 0);
  if (!blocks) return hipSuccess;
  if (blocks > 0x7fffffff) return hipErrorInvalidValue;
  k_copy<<<dim3((unsigned)blocks, a.p.units), 256, 0, st>>>(a);
  return hipGetLastError();
}

hipError_t launch_own(const OwnArgs& a, int n, hipStream_t st) {
  k_own<<<dim3((a.T + 255) / 256, n), 256, 0, st>>>(a);
  return hipGetLastError();
}
