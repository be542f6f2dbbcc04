// Attention of query rows over a K/V cache in which sequences may share tiles.
//
// Row at position p of sequence b attends positions 0..p of b:
//   out = sum_j 2^(s_j - m) v_j / sum_j 2^(s_j - m),  s_j = q.k_j log2(e)/sqrt(hd).
// Tiles that the sequences of a group all read (rv_cache_fork) lie before every
// row of the group, so the queries of all its rows attend them together, without
// a mask, and each tile is read once instead of once per sequence; each
// sequence then attends the rest of its keys by itself, causally.  Runs of keys
// of both parts leave unnormalised partial results, which the last kernel merges
// in a fixed order (shared runs, then own).
#include "rv_internal.h"

namespace {

constexpr int kKB = kTile;

// How a part is computed (kinds of rv_tiles.h): by k_share's workgroups of 512.
enum { KIND_NONE = 0, KIND_FEW = 1, KIND_MANY = 2, KIND_MANY2 = 3, KIND_STREAM = 4 };

// What one workgroup attends: keys [kbeg, kend) as table row `seq` reads them,
// by queries q_begin.. of nq (query slots of one kv head).
struct Unit {
  int seq, kbeg, kend, nq, q_begin, slot, kvh;
  int first, rmax;  // shared part: the group's first member, and as in ShareArgs
  int pos0, row0;   // own part
};

// Query slot q of a unit: its row, head and the last key it may see.
struct Query {
  bool valid;
  int row, head, last;
};

template <int PART>
RV_DEV bool unit_of(const ShareArgs& a, int x, Unit& u) {
  const SharePart& sp = PART ? a.part : a.sh;
  // query groups of one (run, sequence, kv head) are 8 workgroups apart: the
  // same XCD, whose L2 then holds their tiles
  const int j = sp.spread ? x : x / 8, per = j / sp.nqg, qg = j % sp.nqg;
  int i = sp.spread ? per : per * 8 + x % 8;
  const int run = i % sp.ns;
  i /= sp.ns;
  u.kvh = i % a.n_kv;
  i /= a.n_kv;
  const int G = a.n_heads / a.n_kv;
  u.q_begin = qg * sp.qpw;
  if (PART) {
    if (i >= a.nseq) return false;
    if (a.sorted) i = a.order[i];
    u.pos0 = a.seq[i].pos0;
    u.row0 = a.seq[i].row0;
    u.nq = (a.seq[i + 1].row0 - u.row0) * G;
    const int k0 = a.groups ? a.skip[i] * kKB : 0;
    u.seq = i;
    if (u.q_begin >= u.nq) return false;
    const int q_last = min(u.nq, u.q_begin + sp.qpw) - 1;
    u.kbeg = k0 + run * sp.ks;
    u.kend = min(u.pos0 + q_last / G + 1, u.kbeg + sp.ks);
    u.slot = (a.groups ? a.sh.ns : 0) + run;
  } else {
    if (i >= a.groups) return false;
    u.first = a.first[i];
    u.rmax = a.rmax[i];
    u.seq = a.member[u.first];
    u.nq = (u.rmax < 0 ? -u.rmax : (a.first[i + 1] - u.first) * u.rmax) * G;
    if (u.q_begin >= u.nq) return false;
    u.kbeg = run * sp.ks;
    u.kend = min(a.tiles[i] * kKB, u.kbeg + sp.ks);
    u.slot = run;
  }
  return u.kbeg < u.kend;
}

template <int PART>
RV_DEV Query query_of(const ShareArgs& a, const Unit& u, int q) {
  const int G = a.n_heads / a.n_kv;
  Query r;
  const int qc = min(q, u.nq - 1);
  r.head = u.kvh * G + qc % G;
  if (PART) {
    r.valid = q < u.nq;
    r.row = u.row0 + qc / G;
    r.last = u.pos0 + qc / G;
  } else if (u.rmax < 0) {
    r.valid = q < u.nq;
    r.row = a.seq[u.seq].row0 + qc / G;
    r.last = 0x7fffffff;
  } else {
    const int i = qc / G, m = i / u.rmax, seq = a.member[u.first + m];
    const int row0 = a.seq[seq].row0, n = a.seq[seq + 1].row0 - row0, k = i - m * u.rmax;
    r.valid = q < u.nq && k < n;
    r.row = row0 + min(k, n - 1);
    r.last = 0x7fffffff;
  }
  return r;
}

// The last key that every query of a unit sees.
template <int PART>
RV_DEV int first_limit(const ShareArgs& a, const Unit& u) {
  return PART ? u.pos0 + u.q_begin / (a.n_heads / a.n_kv) : 0x7fffffff;
}

// Slot that holds tile t of table row seq, and the tile's first element there in
// a plane of this layer.
RV_DEV int tile_slot(const ShareArgs& a, int seq, int t) {
  return a.own ? a.own[(size_t)seq * (a.kv_len / kKB) + t] : seq;
}
template <int HD>
RV_DEV size_t tile_at(const ShareArgs& a, int slot, int kvh, int t) {
  return ((size_t)(slot * a.n_kv + kvh) * a.kv_len + (size_t)t * kKB) * HD;
}
template <int HD>
RV_DEV size_t tile_base(const ShareArgs& a, int seq, int kvh, int t) {
  return tile_at<HD>(a, __builtin_amdgcn_readfirstlane(tile_slot(a, seq, t)), kvh, t);
}

// B operands of one query: dims 32c + 8g .. +7 of chunk c as hi and lo planes.
template <int HD>
RV_DEV void load_query(const ShareArgs& a, const Query& q, int g, u32x4 (&hi)[HD / 32], u32x4 (&lo)[HD / 32]) {
#pragma unroll
  for (int c = 0; c < HD / 32; ++c) {
    const int d = q.head * HD + 32 * c + 8 * g;
    if (a.q_kind == ROWS_OPERAND) {
      const size_t o = operand_offset(q.row, d, a.n_heads * HD, 2);
      hi[c] = *(const u32x4*)((const char*)a.q + o);
      lo[c] = *(const u32x4*)((const char*)a.q2 + o);
    } else if (a.q_kind == RV_BF16) {
      hi[c] = *(const u32x4*)((const uint16_t*)a.q + (size_t)q.row * a.ldq + d);
      lo[c] = u32x4{0, 0, 0, 0};
    } else {
      const float* p = (const float*)a.q + (size_t)q.row * a.ldq + d;
      const f32x4_t x = *(const f32x4_t*)p, y = *(const f32x4_t*)(p + 4);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float e = j < 2 ? x[2 * j] : y[2 * j - 4], f = j < 2 ? x[2 * j + 1] : y[2 * j - 3];
        const uint16_t eh = f2bf(e), fh = f2bf(f);
        hi[c][j] = eh | (uint32_t)fh << 16;
        lo[c][j] = f2bf(e - bf2f(eh)) | (uint32_t)f2bf(f - bf2f(fh)) << 16;
      }
    }
  }
}

// 4 consecutive dims of a row's head in the output's form.
template <int DT>
RV_DEV void put_out4(const ShareArgs& a, int hd, int row, int head, int d, const f32x4_t& x) {
  const int k = head * hd + d;
  if (a.o_kind == ROWS_OPERAND) {
    put_operand4<DT>(a.out, a.out2, row, k, a.n_heads * hd, x);
  } else if (a.o_kind == RV_BF16) {
    uint16_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) h[j] = f2bf(x[j]);
    memcpy((uint16_t*)a.out + (size_t)row * a.ldo + k, h, 8);
  } else {
    *(f32x4_t*)((float*)a.out + (size_t)row * a.ldo + k) = x;
  }
}

RV_DEV size_t part_index(const ShareArgs& a, int slot, int row, int head) {
  return ((size_t)slot * a.rows + row) * a.n_heads + head;
}

// Softmax weights of one query's scores of NB 16-key blocks: masks keys past
// the limit, adds them to l (this lane's share of the sum) and leaves
// 2^(s - m) in s.  m, the same in the query's four lanes, follows the largest
// score only where one exceeds it by more than kSlack (for the whole wave at
// once): most calls then need neither the lanes' maximum nor a rescale, and
// weights stay below 2^kSlack.  Returns whether *rescale, the factor for what was
// summed before, is to be applied.  A wave whose queries all see nothing yet
// keeps m = -inf, weights 0.
constexpr float kSlack = 6.0f;
template <int NB>
RV_DEV bool softmax_step(f32x4_t (&s)[NB], int k0, int kend, int last, int g, float sc, bool masked, float& m, float& l,
                         float* rescale) {
  float top = -INFINITY;
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (masked) {
        const int key = k0 + 16 * t + 4 * g + i;
        if (!(key < kend && key <= last)) s[t][i] = -INFINITY;
      }
      top = fmaxf(top, s[t][i]);
    }
  const bool grew = __any(top * sc > m + kSlack);
  if (grew) {
    const float m_new = fmaxf(m, rows4_max(top) * sc);
    *rescale = m_new == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - m_new);
    l *= *rescale;
    m = m_new;
  }
  const float base = m == -INFINITY ? 0.f : m;
  float sum = 0.f;
#pragma unroll
  for (int t = 0; t < NB; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[t][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][i], sc, -base));
      sum += s[t][i];
    }
  l += sum;
  return grew;
}

// P of two 16-key blocks as hi and lo B operands.
RV_DEV void split_p(const f32x4_t& s0, const f32x4_t& s1, bf16x8_t& hi, bf16x8_t& lo) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float p = j < 4 ? s0[j] : s1[j - 4];
    const uint16_t h = f2bf(p);
    hi[j] = __builtin_bit_cast(__bf16, h);
    lo[j] = __builtin_bit_cast(__bf16, f2bf(p - bf2f(h)));
  }
}

RV_DEV f32x4_t mfma(const u32x4& x, const bf16x8_t& y, const f32x4_t& acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), y, acc, 0, 0, 0);
}

// A masked key has weight 0, but 0 * inf is NaN: in tiles where some query does
// not see every key, values that are not finite are taken out of the product and
// the queries that see them get NaN instead (what the pair (inf, inf - inf)
// stands for).  v: V operands of a 32-key chunk, vis: per key slot whether the
// lane's query sees it.
// Bits 15 and 31: the two bf16 of x that are not finite (exponent all ones).
RV_DEV uint32_t not_finite2(uint32_t x) { return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u; }
template <int DT>
RV_DEV bool any_not_finite(const u32x4 (&vh)[DT]) {
  uint32_t bad = 0;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j) bad |= not_finite2(vh[d][j]);
  return __any(bad != 0);
}
// O[t][d0 + d] is query tile t's; last[t] the last key its query sees.
template <int ND, int TPW, int DT>
RV_DEV void take_out(u32x4 (&vh)[ND], u32x4 (&vl)[ND], int k0, int kend, const Query (&q)[TPW], int g,
                     f32x4_t (&O)[TPW][DT], int d0) {
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    u32x4 mark;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t bad = not_finite2(vh[d][j]) >> 15;  // 0 or 1 in each half
      const uint32_t keep = ~(bad * 0xffffu);
      mark[j] = bad * 0x3f80u;  // 1.0
      vh[d][j] &= keep;
      vl[d][j] &= keep;
    }
#pragma unroll
    for (int t = 0; t < TPW; ++t) {
      bf16x8_t vis;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = k0 + 4 * g + (j & 3) + 16 * (j >> 2);
        vis[j] = (__bf16)(key < kend && key <= q[t].last ? 1.0f : 0.0f);
      }
      const f32x4_t seen = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, mark), vis,
                                                                   f32x4_t{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (seen[i] > 0.f) O[t][d0 + d][i] = __builtin_nanf("");
    }
    __builtin_amdgcn_sched_barrier(0);  // one d tile's registers at a time
  }
}

// ----------------------------------------------------------- bf16, many queries
// S^T = K Q^T and O^T += V^T P^T on 16x16x32 MFMAs, operands as pairs of planes
// hi = bf16(x), lo = bf16(x - hi), as the cache holds K and V: a pair is within
// 2^-17 of x, and with lo lo dropped (2^-16 of a product) fp32 rows come out
// within 6e-6 of the exact result (fp32 MFMAs would cost 2.6 times these
// products: 153 against 1198 / 3 TFLOP/s in library products).  Three products
// each; queries given in bf16 have no lo plane, two products.  Scores, statistics
// and sums are fp32.  8 waves of TPW 16-query tiles: every K and V operand read
// from LDS serves TPW tiles, and with one LDS reads bound the kernel (512 KiB a
// tile and CU, 4096 cycles, against 192 MFMAs of 16), so calls with more than 128
// queries take two.  The cache holds tiles in operand order (k_elem / v_elem): a
// 64-key tile is four spans that go global -> LDS directly, double-buffered.
// Bound by the matrix cores' power: 64 continuations of 32768 shared keys (70B
// shape, fp32 rows) take 252 us with their own keys and the merge, 1.12 PFLOP/s
// of products in the shared part, where a large library product reaches 1.20.  16
// blocks of 31 rows over 2048 shared keys (8B) 67 us.
template <int HD, int PART, int TPW, bool QLO>
RV_DEV void attend_many(const ShareArgs& a, const Unit& u, uint16_t (&sm0)[4][kKB * HD], uint16_t (&sm1)[4][kKB * HD]) {
  constexpr int NW = 8, DC = HD / 32, DT = HD / 16, SPAN = kKB * HD;
  constexpr int UPW = 4 * SPAN / 512 / NW;  // 1 KiB pieces each wave copies, all of one span
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

  // This wave's share of a tile's copy: UPW pieces of 1 KiB of one span, which go
  // out one by one between the products (all at once they keep the waves from
  // their first products for the 1000 cycles that 64 KiB take to request).  The
  // slot of the tile after the next is looked up a tile ahead.
  const int sp = w / 2, off = (w & 1) * (SPAN / 2);
  const uint16_t* plane = (const uint16_t*)(sp == 0 ? a.kc : sp == 1 ? a.kc2 : sp == 2 ? a.vc : a.vc2) + off;
  const int last_t = (u.kend - 1) / kKB;
  int slot = tile_slot(a, u.seq, u.kbeg / kKB);
  const uint16_t* src = nullptr;  // of the copy under way
  auto next_copy = [&](int k0) {  // the copy of the tile at k0 begins
    src = plane + tile_at<HD>(a, __builtin_amdgcn_readfirstlane(slot), u.kvh, k0 / kKB);
    slot = tile_slot(a, u.seq, min(k0 / kKB + 1, last_t));
  };
  auto copy_piece = [&](uint16_t(&sm)[4][SPAN], int i) {
    __builtin_amdgcn_global_load_lds((const void*)(src + lane * 8 + i * 512),
                                     (__attribute__((address_space(3))) void*)(&sm[0][0] + sp * SPAN + off + i * 512), 16,
                                     0, 0);
  };
  next_copy(u.kbeg);
#pragma unroll
  for (int i = 0; i < UPW; ++i) copy_piece(sm0, i);

  // of the two waves on a SIMD the first goes first, so that its products run
  // while the other computes weights and the other way round
  if (w < 4) __builtin_amdgcn_s_setprio(1);
  const int q0 = u.q_begin + 16 * TPW * w;
  const bool active = q0 < u.nq;
  const int first_last = first_limit<PART>(a, u);
  Query q[TPW];
  u32x4 qh[TPW][DC], ql[TPW][DC];
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    q[t] = query_of<PART>(a, u, q0 + 16 * t + (lane & 15));
    load_query<HD>(a, q[t], g, qh[t], ql[t]);
  }
  float m[TPW], l[TPW];
  f32x4_t O[TPW][DT];
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    m[t] = -INFINITY;
    l[t] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) O[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }

  // 32 keys at a time: scores, weights, products with V
  static_assert(UPW == 2 * DC, "a piece of the copy per 32-dim chunk of each half");
  auto tile = [&](const uint16_t(&sm)[4][SPAN], uint16_t(&other)[4][SPAN], int k_tile) {
    const bool more = k_tile + kKB < u.kend;
    if (more) next_copy(k_tile + kKB);
    if (!active) {
      if (more) {
#pragma unroll
        for (int i = 0; i < UPW; ++i) copy_piece(other, i);
      }
      return;
    }
#pragma unroll 1
    for (int half = 0; half < 2; ++half) {
      const int k0 = k_tile + 32 * half;
      const uint16_t *kp = &sm[0][half * 2 * DC * 512 + lane * 8], *vp = &sm[2][half * DT * 512 + lane * 8];
      f32x4_t s[TPW][2];
#pragma unroll
      for (int t = 0; t < TPW; ++t)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) s[t][kb] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < DC; ++c) {
        u32x4 kh[2], kl[2];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          kh[kb] = *(const u32x4*)(kp + (kb * DC + c) * 512);
          kl[kb] = *(const u32x4*)(kp + SPAN + (kb * DC + c) * 512);
        }
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[t][kb] = mfma(kh[kb], __builtin_bit_cast(bf16x8_t, qh[t][c]), s[t][kb]);
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int kb = 0; kb < 2; ++kb) s[t][kb] = mfma(kl[kb], __builtin_bit_cast(bf16x8_t, qh[t][c]), s[t][kb]);
        if constexpr (QLO) {
#pragma unroll
          for (int t = 0; t < TPW; ++t)
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) s[t][kb] = mfma(kh[kb], __builtin_bit_cast(bf16x8_t, ql[t][c]), s[t][kb]);
        }
        if (more) copy_piece(other, half * DC + c);
      }
      const bool masked = PART && (k0 + 32 > u.kend || k0 + 31 > first_last);
      bf16x8_t ph[TPW], pl[TPW];
#pragma unroll
      for (int t = 0; t < TPW; ++t) {
        float rescale;
        if (softmax_step<2>(s[t], k0, u.kend, q[t].last, g, a.scale_log2, masked, m[t], l[t], &rescale)) {
#pragma unroll
          for (int d = 0; d < DT; ++d) O[t][d] *= rescale;
        }
        split_p(s[t][0], s[t][1], ph[t], pl[t]);
      }
      // four d tiles at a time: their operands, then the products in passes, so
      // that dependent MFMAs are 4 TPW apart
      constexpr int ND = DT < 4 ? DT : 4;
#pragma unroll
      for (int d0 = 0; d0 < DT; d0 += ND) {
        u32x4 vh[ND], vl[ND];
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          vh[d] = *(const u32x4*)(vp + (d0 + d) * 512);
          vl[d] = *(const u32x4*)(vp + SPAN + (d0 + d) * 512);
        }
        if (masked && any_not_finite<ND>(vh)) take_out<ND, TPW, DT>(vh, vl, k0, u.kend, q, g, O, d0);
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int d = 0; d < ND; ++d) O[t][d0 + d] = mfma(vh[d], ph[t], O[t][d0 + d]);
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int d = 0; d < ND; ++d) O[t][d0 + d] = mfma(vh[d], pl[t], O[t][d0 + d]);
#pragma unroll
        for (int t = 0; t < TPW; ++t)
#pragma unroll
          for (int d = 0; d < ND; ++d) O[t][d0 + d] = mfma(vl[d], ph[t], O[t][d0 + d]);
      }
    }
  };

  // at the top of each step only the copy of the tile about to be used is in
  // flight; after the barrier every wave has finished the one before, whose
  // buffer takes the next
  for (int k0 = u.kbeg; k0 < u.kend; k0 += 2 * kKB) {
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    tile(sm0, sm1, k0);
    if (k0 + kKB >= u.kend) break;
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    tile(sm1, sm0, k0 + kKB);
  }

  // lane holds O^T[d = 16t + 4g + i][query lane%16]
#pragma unroll
  for (int t = 0; t < TPW; ++t) {
    l[t] = rows4_sum(l[t]);
    if (!q[t].valid) continue;
    if (a.direct) {
      const float inv = 1.0f / l[t];
#pragma unroll
      for (int d = 0; d < DT; ++d) put_out4<RV_BF16>(a, HD, q[t].row, q[t].head, 16 * d + 4 * g, O[t][d] * inv);
      continue;
    }
    const size_t e = part_index(a, u.slot, q[t].row, q[t].head);
#pragma unroll
    for (int d = 0; d < DT; ++d) *(f32x4_t*)(a.part_o + e * HD + 16 * d + 4 * g) = O[t][d];
    if (g == 0) {
      a.part_ml[2 * e] = m[t];
      a.part_ml[2 * e + 1] = l[t];
    }
  }
}

// ----------------------------------------------------------- bf16, at most 16 queries
// Decode steps: the 8 waves share the 16 queries and split the keys, wave w
// taking tiles w, w + 8, ... of KT keys straight to registers; their states
// merge in LDS.  Bound by what a CU draws from HBM: 640 keys of one kv head in 19 us
// (34 GB/s a CU), 64 sequences of 16-2000 keys 94 us with the merge (5.9 TB/s); one
// sequence of 1024 keys 8 us, latency.  STREAM: nontemporal loads, for calls whose keys exceed the
// last-level cache anyway (64 sequences of 1000 keys, 524 MB: 110 -> 98 us at the
// 70B shape, 101 -> 91 at 8B; with 112 MB, 33.2 -> 34.8).
// red: 8 x 16 x HD values in LDS, 16-byte columns xor-ed with the query so that
// the 16 queries of a column lie in different banks; red_ml: 2 x 8 x 16.
template <int HD, int PART, bool QLO, bool STREAM>
RV_DEV void attend_few(const ShareArgs& a, const Unit& u, float* red, float* red_ml) {
  constexpr int KT = HD == 128 ? 32 : 64, NW = 8, NB = KT / 16, NC = KT / 32, DC = HD / 32, DT = HD / 16;
  constexpr int COLS = HD / 4 < 16 ? HD / 4 : 16;  // columns that the xor permutes
  auto at_red = [&](int wave, int query, int col) {
    return (f32x4_t*)(red + ((wave * 16 + query) * (HD / 4) + (col ^ (query & (COLS - 1)))) * 4);
  };
  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);

  const Query q[1] = {query_of<PART>(a, u, u.q_begin + (lane & 15))};
  const int first_last = first_limit<PART>(a, u);
  u32x4 qh[DC], ql[DC];
  load_query<HD>(a, q[0], g, qh, ql);

  u32x4 k[2][NB][DC], v[2][NC][DT];
  // tiles past the last load that one again and are not used
  const int last_tile = u.kbeg + (u.kend - 1 - u.kbeg) / KT * KT;
  // (uniform offsets: the loads then need one lane offset and no 64-bit addresses)
  auto at = [&](int k0) { return tile_base<HD>(a, u.seq, u.kvh, k0 / kKB) + (size_t)(k0 % kKB) * HD; };
  const unsigned lane16 = lane * 16;
  auto load = [](const char* p) {
    return STREAM ? __builtin_nontemporal_load((const u32x4*)p) : *(const u32x4*)p;
  };
  auto load_k = [&](size_t o) {
#pragma unroll
    for (int pl = 0; pl < 2; ++pl)
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int c = 0; c < DC; ++c)
          k[pl][t][c] = load((const char*)((const uint16_t*)(pl ? a.kc2 : a.kc) + o + (t * DC + c) * 512) + lane16);
  };
  auto load_v = [&](size_t o) {
#pragma unroll
    for (int pl = 0; pl < 2; ++pl)
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int d = 0; d < DT; ++d)
          v[pl][c][d] = load((const char*)((const uint16_t*)(pl ? a.vc2 : a.vc) + o + (c * DT + d) * 512) + lane16);
  };
  int k0 = u.kbeg + w * KT;
  size_t next = at(min(k0, last_tile));
  if (k0 >= u.kend) next = at(last_tile);  // a wave without tiles loads the last one and uses it not
  // the order of the loop: K, then V, so that the wait for K leaves V in flight
  load_k(next);
  __builtin_amdgcn_sched_barrier(0);
  load_v(next);
  __builtin_amdgcn_sched_barrier(0);
  next = at(min(k0 + NW * KT, last_tile));
  float m = -INFINITY, l = 0.f;
  f32x4_t O[1][DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) O[0][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};

  for (; k0 < u.kend; k0 += NW * KT) {
    f32x4_t s[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < DC; ++c) {
      const bf16x8_t h = __builtin_bit_cast(bf16x8_t, qh[c]), lo = __builtin_bit_cast(bf16x8_t, ql[c]);
#pragma unroll
      for (int t = 0; t < NB; ++t) s[t] = mfma(k[0][t][c], h, s[t]);
      if constexpr (QLO) {
#pragma unroll
        for (int t = 0; t < NB; ++t) s[t] = mfma(k[0][t][c], lo, s[t]);
      }
#pragma unroll
      for (int t = 0; t < NB; ++t) s[t] = mfma(k[1][t][c], h, s[t]);
    }
    __builtin_amdgcn_sched_barrier(0);  // the next operands replace these: none are loaded before their last use
    load_k(next);
    const bool masked = k0 + KT > u.kend || k0 + KT - 1 > first_last;
    float rescale;
    if (softmax_step<NB>(s, k0, u.kend, q[0].last, g, a.scale_log2, masked, m, l, &rescale)) {
#pragma unroll
      for (int d = 0; d < DT; ++d) O[0][d] *= rescale;
    }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      bf16x8_t ph, pl;
      split_p(s[2 * c], s[2 * c + 1], ph, pl);
      if (masked && any_not_finite<DT>(v[0][c])) 
        take_out<DT, 1, DT>(v[0][c], v[1][c], k0 + 32 * c, u.kend, q, g, O, 0);
#pragma unroll
      for (int d = 0; d < DT; ++d) O[0][d] = mfma(v[0][c][d], ph, O[0][d]);
#pragma unroll
      for (int d = 0; d < DT; ++d) O[0][d] = mfma(v[0][c][d], pl, O[0][d]);
#pragma unroll
      for (int d = 0; d < DT; ++d) O[0][d] = mfma(v[1][c][d], ph, O[0][d]);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_v(next);
    next = at(min(k0 + 2 * NW * KT, last_tile));
  }

  // merge the waves: one without tiles has m = -inf, l = 0, O = 0
  l = rows4_sum(l);
#pragma unroll
  for (int d = 0; d < DT; ++d) *at_red(w, lane & 15, 4 * d + g) = O[0][d];
  if (g == 0) {
    red_ml[w * 16 + (lane & 15)] = m;
    red_ml[(NW + w) * 16 + (lane & 15)] = l;
  }
  __syncthreads();
  const int oq = tid / (HD / 4), od = tid % (HD / 4) * 4;
  if (oq >= 16) return;
  const Query oqr = query_of<PART>(a, u, u.q_begin + oq);
  if (!oqr.valid) return;
  float M = -INFINITY, L = 0.f;
#pragma unroll
  for (int i = 0; i < NW; ++i) M = fmaxf(M, red_ml[i * 16 + oq]);
  f32x4_t x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NW; ++i) {
    const float f = red_ml[i * 16 + oq] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(red_ml[i * 16 + oq] - M);
    L += red_ml[(NW + i) * 16 + oq] * f;
    x += *at_red(i, oq, od / 4) * f;
  }
  if (a.direct) {
    put_out4<RV_BF16>(a, HD, oqr.row, oqr.head, od, x * (1.0f / L));
    return;
  }
  const size_t e = part_index(a, u.slot, oqr.row, oqr.head);
  *(f32x4_t*)(a.part_o + e * HD + od) = x;
  if (od == 0) {
    a.part_ml[2 * e] = M;
    a.part_ml[2 * e + 1] = L;
  }
}

// ----------------------------------------------------------- bf16, one launch for both parts
// Shared keys are compute (many queries a key), own keys of decode steps HBM (few
// queries a key), so workgroups of the two parts run side by side.  Where the own
// part fits beside the last round of the shared part, the shared part goes first;
// else half of the chip starts with the one and half with the other (runs of 8
// workgroups, one per XCD: lead_sh of the shared part, lead_own of the own, the
// rest of the shared, the rest of the own).  SH, OW: kinds of the parts.
template <int HD, int KIND, int PART, bool QLO>
RV_DEV void attend_part(const ShareArgs& a, int x, uint16_t (&sm0)[4][kKB * HD], uint16_t (&sm1)[4][kKB * HD]) {
  Unit u;
  if (!unit_of<PART>(a, x, u)) return;
  if constexpr (KIND == KIND_FEW || KIND == KIND_STREAM)
    attend_few<HD, PART, QLO, KIND == KIND_STREAM>(a, u, (float*)&sm0[0][0], (float*)&sm1[0][0]);
  else if constexpr (KIND == KIND_MANY) attend_many<HD, PART, 1, QLO>(a, u, sm0, sm1);
  else if constexpr (KIND == KIND_MANY2) attend_many<HD, PART, 2, QLO>(a, u, sm0, sm1);
}
template <int HD, int SH, int OW, bool QLO>
__global__ __launch_bounds__(512, HD <= 64 && (OW == KIND_MANY || OW == KIND_NONE) && SH != KIND_MANY2 ? 4 : 2) void k_share(ShareArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t sm0[4][kKB * HD];
  __shared__ __attribute__((aligned(16))) uint16_t sm1[4][kKB * HD];
  int x = blockIdx.x;
  if constexpr (SH != KIND_NONE) {
    const int j = x / 8, lead = a.lead_sh + a.lead_own;
    const bool sh = j < a.lead_sh || (j >= lead && j < a.runs_sh + a.lead_own);
    const int run = j < a.lead_sh ? j : j < lead ? j - a.lead_sh : sh ? j - a.lead_own : j - a.runs_sh;
    x = run * 8 + x % 8;
    if (sh) {
      attend_part<HD, SH, 0, QLO>(a, x, sm0, sm1);
      return;
    }
  }
  attend_part<HD, OW, 1, QLO>(a, x, sm0, sm1);
}

// As take_out, for four keys of an fp32 cache, where infinities keep their sign:
// an infinity that a query sees is added to its output as it is.
template <int DC>
RV_DEV void take_out_f32(float (&v)[DC], bool vis, f32x4_t (&o)[DC]) {
  const f32x4_t zero = {0.f, 0.f, 0.f, 0.f};
  const float see = vis ? 1.f : 0.f;
#pragma unroll
  for (int e = 0; e < DC; ++e) {
    const uint32_t b = __float_as_uint(v[e]), inf = 0x7f800000u;
    const bool odd = (b & inf) == inf, is_nan = odd && (b & 0x007fffffu);
    // counts of what each query sees: 1 for +inf, 2^10 for -inf, 2^20 for NaN (at most 4 keys each)
    const float mark = !odd ? 0.f : is_nan ? 1048576.f : (int)b < 0 ? 1024.f : 1.f;
    const f32x4_t seen = __builtin_amdgcn_mfma_f32_16x16x4f32(mark, see, zero, 0, 0, 0);
    v[e] = odd ? 0.f : v[e];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int n = (int)seen[i];
      float add = n & 1023 ? INFINITY : 0.f;
      add -= (n >> 10) & 1023 ? INFINITY : 0.f;
      add += n >> 20 ? __builtin_nanf("") : 0.f;
      o[e][i] += add;
    }
  }
}

// ----------------------------------------------------------- fp32
// One wave per (16 queries, run, kv head) on 16x16x4 fp32 MFMAs; K and V come
// straight from the row-major cache.  The k slots of an MFMA may hold any four
// dims that both operands agree on, so a lane's 16-byte load of dims
// 16c + 4(l/16) .. +3 feeds four MFMAs, and P comes straight from the scores.
// Bound by latency: all loads of KT keys, K and V, are issued together (four blocks
// of 21 rows over 128 shared keys, 8 heads of 64: 8.5 us).
template <int HD, int PART>
RV_DEV void attend_f32(const ShareArgs& a, const Unit& u) {
  constexpr int DC = HD / 16, KT = HD == 128 ? 32 : 64, NB = KT / 16;
  const int lane = threadIdx.x, g = lane >> 4, c16 = lane & 15;
  const Query q = query_of<PART>(a, u, u.q_begin + c16);
  const int first_last = first_limit<PART>(a, u);
  f32x4_t qv[DC];
#pragma unroll
  for (int c = 0; c < DC; ++c) {
    const int d = q.head * HD + 16 * c + 4 * g;
    if (a.q_kind == ROWS_OPERAND) {
      qv[c] = *(const f32x4_t*)((const char*)a.q + operand_offset(q.row, d, a.n_heads * HD, 4));
    } else if (a.q_kind == RV_F32) {
      qv[c] = *(const f32x4_t*)((const float*)a.q + (size_t)q.row * a.ldq + d);
    } else {
      uint16_t h[4];
      memcpy(h, (const uint16_t*)a.q + (size_t)q.row * a.ldq + d, 8);
#pragma unroll
      for (int j = 0; j < 4; ++j) qv[c][j] = bf2f(h[j]);
    }
  }
  f32x4_t o[DC];
#pragma unroll
  for (int t = 0; t < DC; ++t) o[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  float m = -INFINITY, l = 0.f;

  for (int k0 = u.kbeg; k0 < u.kend; k0 += KT) {
    const size_t base = tile_base<HD>(a, u.seq, u.kvh, k0 / kKB) + (size_t)(k0 % kKB) * HD;
    const float* kb = (const float*)a.kc + base;
    const float* vb = (const float*)a.vc + base;
    f32x4_t kv[NB][DC];
    float v[NB][4][DC];
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int c = 0; c < DC; ++c) kv[t][c] = *(const f32x4_t*)(kb + (16 * t + c16) * HD + 4 * g + 16 * c);
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float* vr = vb + (16 * t + 4 * g + i) * HD + c16 * DC;
        if constexpr (DC == 2) {
          const float2 x = *(const float2*)vr;
          v[t][i][0] = x.x;
          v[t][i][1] = x.y;
        } else {
#pragma unroll
          for (int e = 0; e < DC; e += 4) {
            const f32x4_t x = *(const f32x4_t*)(vr + e);
#pragma unroll
            for (int f = 0; f < 4; ++f) v[t][i][e + f] = x[f];
          }
        }
      }
    f32x4_t s[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) s[t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    // the key blocks side by side: dependent MFMAs are NB apart
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int t = 0; t < NB; ++t)
          s[t] = __builtin_amdgcn_mfma_f32_16x16x4f32(kv[t][c][i], qv[c][i], s[t], 0, 0, 0);
    const bool masked = k0 + KT > u.kend || k0 + KT - 1 > first_last;
    float rescale;
    if (softmax_step<NB>(s, k0, u.kend, q.last, g, a.scale_log2, masked, m, l, &rescale)) {
#pragma unroll
      for (int t = 0; t < DC; ++t) o[t] *= rescale;
    }
    bool bad = false;
    if (masked) {
      uint32_t bits = 0;  // bit 31: an exponent of all ones
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < DC; ++e) bits |= (__float_as_uint(v[t][i][e]) & 0x7f800000u) + 0x00800000u;
      bad = __any((int)bits < 0);
    }
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (bad) {
          const int key = k0 + 16 * t + 4 * g + i;
          take_out_f32<DC>(v[t][i], key < u.kend && key <= q.last, o);
        }
#pragma unroll
        for (int e = 0; e < DC; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v[t][i][e], s[t][i], o[e], 0, 0, 0);
      }
  }
  l = rows4_sum(l);
  if (!q.valid) return;
  // lane holds dims (4g + i) DC + t of its query: a run of 4 DC
  const size_t e = part_index(a, u.slot, q.row, q.head);
  const float inv = a.direct ? 1.0f / l : 1.0f;
#pragma unroll
  for (int y = 0; y < DC; ++y) {
    f32x4_t x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = o[(4 * y + j) % DC][(4 * y + j) / DC] * inv;
    if (a.direct) put_out4<RV_F32>(a, HD, q.row, q.head, 4 * g * DC + 4 * y, x);
    else *(f32x4_t*)(a.part_o + e * HD + 4 * g * DC + 4 * y) = x;
  }
  if (!a.direct && g == 0) {
    a.part_ml[2 * e] = m;
    a.part_ml[2 * e + 1] = l;
  }
}
template <int HD>
__global__ __launch_bounds__(64) void k_share_f32(ShareArgs a) {
  const int x = blockIdx.x, n = a.runs_sh * 8;
  Unit u;
  if (x < n) {
    if (unit_of<0>(a, x, u)) attend_f32<HD, 0>(a, u);
  } else if (unit_of<1>(a, x - n, u)) {
    attend_f32<HD, 1>(a, u);
  }
}

// ----------------------------------------------------------- merge
// hd / 4 lanes per (row, head), a workgroup per row and 1024 / hd heads: one pass
// over the runs that had keys for the row, shared runs first, in batches whose
// loads are issued together.  Latency bound for few rows (4 us), else by its bytes
// (16 x 31 rows x 4 runs, 8B: 33 MB, 9 us).
template <int DT, int HD>
__global__ __launch_bounds__(256) void k_share_merge(ShareArgs a, int head_groups) {
  constexpr int LPQ = HD / 4, BATCH = 8;
  const int row = blockIdx.x / head_groups, lane = threadIdx.x & 63;
  int b = -1;  // the last sequence that starts at the row or before
#pragma unroll
  for (int j = 0; j < RV_MAX_BATCH / 64; ++j)
    if (64 * j < a.nseq) b += __popcll(__ballot(lane + 64 * j < a.nseq && a.seq[lane + 64 * j].row0 <= row));
  const int head = blockIdx.x % head_groups * (256 / LPQ) + threadIdx.x / LPQ, d = threadIdx.x % LPQ * 4;
  if (head >= a.n_heads) return;
  const int r = row - a.seq[b].row0;
  const int k0 = a.groups ? a.skip[b] * kKB : 0;
  const int n_sh = k0 ? (k0 + a.sh.ks - 1) / a.sh.ks : 0;
  const int n_own = (a.seq[b].pos0 + r - k0) / a.part.ks + 1;
  const int skip = (a.groups ? a.sh.ns : 0) - n_sh;  // slots of shared runs that this row has not
  const size_t e0 = part_index(a, 0, row, head), stride = (size_t)a.rows * a.n_heads;
  float M = -INFINITY, L = 0.f;
  f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < n_sh + n_own; s0 += BATCH) {
    float m[BATCH], l[BATCH];
    f32x4_t x[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const int s = min(s0 + u, n_sh + n_own - 1);  // past the last: that one again, weight 0
      const size_t e = e0 + (size_t)(s < n_sh ? s : s + skip) * stride;
      m[u] = a.part_ml[2 * e];
      l[u] = a.part_ml[2 * e + 1];
      x[u] = *(const f32x4_t*)(a.part_o + e * HD + d);
    }
    float top = M;
#pragma unroll
    for (int u = 0; u < BATCH; ++u) top = fmaxf(top, m[u]);
    const float base = top == -INFINITY ? 0.f : top, keep = __builtin_amdgcn_exp2f(M - base);
    L *= keep;
    acc *= keep;
#pragma unroll
    for (int u = 0; u < BATCH; ++u) {
      const float f = s0 + u < n_sh + n_own ? __builtin_amdgcn_exp2f(m[u] - base) : 0.f;
      L += l[u] * f;
      acc += x[u] * f;
    }
    M = top;
  }
  put_out4<DT>(a, HD, row, head, d, acc * (1.0f / L));
}

template <int HD, int SH, int OW>
void launch_kinds(const ShareArgs& a, hipStream_t st) {
  const unsigned grid = (unsigned)(a.runs_sh + a.runs_own) * 8;
  if (a.q_kind == RV_BF16) k_share<HD, SH, OW, false><<<grid, 512, 0, st>>>(a);
  else k_share<HD, SH, OW, true><<<grid, 512, 0, st>>>(a);
}

int kind_of(const SharePart& p) { return p.qpw == 16 ? KIND_FEW : p.qpw == 128 ? KIND_MANY : KIND_MANY2; }

// Workgroups of a part, in runs of 8.
size_t part_runs(const SharePart& p, int n, int n_kv) {
  const size_t units = (size_t)p.ns * n_kv * n;
  return p.spread ? (units * p.nqg + 7) / 8 : (units + 7) / 8 * p.nqg;
}

template <int HD>
hipError_t launch_all(int dtype, ShareArgs& a, hipStream_t st) {
  a.direct = a.groups == 0 && a.part.ns == 1;
  const size_t sh = a.groups ? part_runs(a.sh, a.groups, a.n_kv) : 0, own = part_runs(a.part, a.nseq, a.n_kv);
  if ((sh + own) * 8 > 0x7fffffff) return hipErrorInvalidValue;
  a.runs_sh = (int)sh;
  a.runs_own = (int)own;
  a.lead_sh = a.own_last ? a.runs_sh : std::min(a.runs_sh, 16);
  a.lead_own = a.own_last ? 0 : a.runs_own / 2;
  if (dtype == RV_F32) {
    k_share_f32<HD><<<(unsigned)(a.runs_sh + a.runs_own) * 8, 64, 0, st>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  } else {
    const int kinds = a.stream ? KIND_NONE * 8 + KIND_STREAM : (sh ? kind_of(a.sh) : KIND_NONE) * 8 + kind_of(a.part);
    switch (kinds) {
      case KIND_NONE * 8 + KIND_FEW: launch_kinds<HD, KIND_NONE, KIND_FEW>(a, st); break;
      case KIND_NONE * 8 + KIND_STREAM: launch_kinds<HD, KIND_NONE, KIND_STREAM>(a, st); break;
      case KIND_FEW * 8 + KIND_FEW: launch_kinds<HD, KIND_FEW, KIND_FEW>(a, st); break;
      case KIND_MANY * 8 + KIND_FEW: launch_kinds<HD, KIND_MANY, KIND_FEW>(a, st); break;
      case KIND_MANY2 * 8 + KIND_FEW: launch_kinds<HD, KIND_MANY2, KIND_FEW>(a, st); break;
      case KIND_NONE * 8 + KIND_MANY: launch_kinds<HD, KIND_NONE, KIND_MANY>(a, st); break;
      case KIND_MANY * 8 + KIND_MANY: launch_kinds<HD, KIND_MANY, KIND_MANY>(a, st); break;
      case KIND_MANY2 * 8 + KIND_MANY: launch_kinds<HD, KIND_MANY2, KIND_MANY>(a, st); break;
      case KIND_NONE * 8 + KIND_MANY2: launch_kinds<HD, KIND_NONE, KIND_MANY2>(a, st); break;
      case KIND_MANY2 * 8 + KIND_MANY2: launch_kinds<HD, KIND_MANY2, KIND_MANY2>(a, st); break;
      default: return hipErrorInvalidValue;
    }
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  if (a.direct) return hipSuccess;
  constexpr int per = 256 / (HD / 4);
  const int head_groups = (a.n_heads + per - 1) / per;
  if ((size_t)a.rows * head_groups > 0x7fffffff) return hipErrorInvalidValue;
  const unsigned grid = (unsigned)a.rows * head_groups;
  if (dtype == RV_BF16) k_share_merge<RV_BF16, HD><<<grid, 256, 0, st>>>(a, head_groups);
  else k_share_merge<RV_F32, HD><<<grid, 256, 0, st>>>(a, head_groups);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_share(int dtype, int hd, ShareArgs& a, hipStream_t st) {
  switch (hd) {
    case 32: return launch_all<32>(dtype, a, st);
    case 64: return launch_all<64>(dtype, a, st);
    case 128: return launch_all<128>(dtype, a, st);
  }
  return hipErrorInvalidValue;
}
