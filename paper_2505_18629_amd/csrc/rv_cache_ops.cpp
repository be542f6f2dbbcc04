// Host side of the operators on the K/V cache: appending and reading rows,
// copying and forking sequences, attention over a layer.
#include <cmath>

#include "rv_state.h"

namespace {

// The row spans of a call: sequence b has h_rows[b] rows at positions h_pos[b] ..,
// n_rows together.  Fills pos, row0 and (blk0 not NULL) blk0; *max_rows the longest span.
rv_status check_spans(const rv_cache* c, int32_t batch, const int32_t* h_pos, const int32_t* h_rows, int64_t n_rows,
                      int* pos, int* row0, int* blk0, int* max_rows) {
  if (batch != c->B) return rv_fail(RV_E_ARG, "positions and counts of %d sequences, the cache has %d", batch, c->B);
  long long rows = 0, blocks = 0;
  *max_rows = 0;
  for (int b = 0; b < c->B; ++b) {
    const int n = h_rows[b], p = h_pos[b];
    if (n < 0) return rv_fail(RV_E_ARG, "rows[%d] = %d is negative", b, n);
    if (n > 0 && (p < 0 || (long long)p + n > c->max_len))
      return rv_fail(RV_E_RANGE, "sequence %d: %d rows at position %d outside [0, max_len=%d)", b, n, p, c->max_len);
    row0[b] = (int)rows;
    pos[b] = n ? p : 0;
    if (blk0) blk0[b] = (int)blocks;
    rows += n;
    blocks += span_blocks(n ? p : 0, n);
    if (rows > 0x7fffffff) return rv_fail(RV_E_CAPACITY, "more than 2^31 - 1 rows");
    if (n > *max_rows) *max_rows = n;
  }
  row0[c->B] = (int)rows;
  if (blk0) blk0[c->B] = (int)blocks;
  if (rows != n_rows) return rv_fail(RV_E_ARG, "counts add up to %lld rows, given are %lld", rows, (long long)n_rows);
  return RV_OK;
}

rv_status check_layer(const rv_cache* c, int32_t layer) {
  if (layer < 0 || layer >= c->m->cfg.n_layers)
    return rv_fail(RV_E_ARG, "layer %d outside [0, %d)", layer, c->m->cfg.n_layers);
  return RV_OK;
}

// Rows that the kernels read and write 16 bytes at a time.
rv_status check_rows(const char* what, const void* d, int64_t ld, int64_t width, int want, int io) {
  if (width != want) return rv_fail(RV_E_ARG, "%s: rows of %lld values, the model's have %d", what, (long long)width, want);
  if (!d) return rv_fail(RV_E_ARG, "%s rows are NULL", what);
  const int per16 = io == RV_F32 ? 4 : 8;
  if (ld < width) return rv_fail(RV_E_ARG, "%s: row stride %lld below the width %d", what, (long long)ld, want);
  if (((uintptr_t)d & 15) || ld % per16)
    return rv_fail(RV_E_ARG, "%s: rows must start at multiples of 16 bytes", what);
  return RV_OK;
}

struct Planes {
  char *kc, *vc, *kc2, *vc2;
};
Planes layer_planes(const rv_cache* c, int layer) {
  const size_t lo = (size_t)layer * c->kv_layer_elems * c->m->es;
  const bool pair = c->m->es == 2;
  return Planes{c->kc + lo, c->vc + lo, pair ? c->kc2 + lo : nullptr, pair ? c->vc2 + lo : nullptr};
}

// Destinations of a copy or fork: in range, distinct, and not read by a sequence
// that the call leaves alone.
rv_status check_dsts(const rv_cache* c, int n, const int32_t* h_dst, bool* gone) {
  for (int b = 0; b < c->B; ++b) gone[b] = false;
  for (int i = 0; i < n; ++i) {
    if (h_dst[i] < 0 || h_dst[i] >= c->B)
      return rv_fail(RV_E_ARG, "destination %d outside [0, batch=%d)", h_dst[i], c->B);
    if (gone[h_dst[i]]) return rv_fail(RV_E_ARG, "sequence %d is written twice", h_dst[i]);
    gone[h_dst[i]] = true;
  }
  const int r = c->tiles.reader_of(gone);
  if (r >= 0) return rv_fail(RV_E_STATE, "sequence %d reads tiles of a sequence that would be overwritten", r);
  return RV_OK;
}

CopyArgs copy_args(const rv_cache* c) {
  const rv_config& mc = c->m->cfg;
  CopyArgs a{};
  const size_t es = c->m->es, head = (size_t)c->kv_len * mc.head_dim * es / 16;
  a.plane[0] = c->kc;
  a.plane[1] = c->vc;
  a.plane[2] = c->kc2;
  a.plane[3] = c->vc2;
  a.planes = es == 2 ? 4 : 2;
  a.layers = mc.n_layers;
  a.n_kv = mc.n_kv_heads;
  a.max_len = c->max_len;
  a.head_vecs = head;
  a.slot_vecs = head * mc.n_kv_heads;
  a.layer_vecs = a.slot_vecs * c->B;
  a.tile_vecs = (int)(kTile * mc.head_dim * es / 16);
  a.ids = c->ids;
  a.seq_bad = c->seq_bad;
  return a;
}

int kv_tiles(int len) { return (len - 1 + kTile - 1) / kTile; }

}  // namespace

rv_status reset_owners(rv_cache* c, hipStream_t st) {
  if (!c->tiles.foreign) return RV_OK;
  OwnArgs o{};
  o.own = c->tile_own;
  o.T = c->tiles.T;
  for (int b = 0; b < c->B; ++b) o.seq[b] = (uint8_t)b;
  HIP_TRY(launch_own(o, c->B, st), "tile owners");
  c->tiles.reset();
  return RV_OK;
}

rv_status check_writable(const rv_cache* c, int b, int pos, int rows) {
  if (!c->tiles.foreign || rows <= 0) return RV_OK;
  const int t = c->tiles.first_shared(b, pos / kTile, (pos + rows - 1) / kTile + 1);
  if (t >= 0)
    return rv_fail(RV_E_STATE, "sequence %d: positions %d.. are shared with another sequence and cannot be written", b,
                   std::max(pos, t * kTile));
  return RV_OK;
}

void plan_attend(const rv_cache* c, const int* pos0, const int* row0, ShareArgs& a) {
  const rv_config& mc = c->m->cfg;
  a.own = c->tiles.foreign ? c->tile_own : nullptr;
  a.part_o = c->part_o;
  a.part_ml = c->part_ml;
  a.n_heads = mc.n_heads;
  a.n_kv = mc.n_kv_heads;
  a.kv_len = c->kv_len;
  a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)mc.head_dim));
  SharePlan p;
  plan_share(c->tiles, mc.dtype == RV_BF16, pos0, row0, mc.n_heads, mc.n_kv_heads, mc.head_dim, c->part_entries, p);
  a.nseq = p.nseq;
  a.rows = p.rows;
  a.groups = p.groups;
  a.sh = p.sh;
  a.part = p.own;
  a.own_last = p.own_last;
  a.stream = p.stream;
  a.sorted = p.sorted;
  if (p.sorted) std::copy(p.order, p.order + c->B, a.order);
  for (int b = 0; b < c->B; ++b) {
    a.seq[b] = ShareSeq{pos0[b], row0[b]};
    a.skip[b] = p.group_of[b] == 255 ? 0 : (uint16_t)p.tiles[p.group_of[b]];
  }
  a.seq[c->B].row0 = row0[c->B];
  if (p.groups) {
    std::copy(p.member, p.member + c->B, a.member);
    std::copy(p.first, p.first + p.groups + 1, a.first);
    std::copy(p.tiles, p.tiles + p.groups, a.tiles);
    for (int g = 0; g < p.groups; ++g) a.rmax[g] = p.dense[g] ? -p.dense[g] : p.rmax[g];
  }
}

extern "C" {

rv_status rv_model_qk_norm(rv_model* m, const float* d_q_gain, const float* d_k_gain, int64_t count) {
  if (!m) return rv_fail(RV_E_ARG, "model is NULL");
  if (!d_q_gain != !d_k_gain) return rv_fail(RV_E_ARG, "gains of queries and keys come together");
  if (d_q_gain && count != (int64_t)m->cfg.n_layers * m->cfg.head_dim)
    return rv_fail(RV_E_ARG, "%lld gains, the model has %d layers of head_dim %d", (long long)count, m->cfg.n_layers,
                   m->cfg.head_dim);
  if (((uintptr_t)d_q_gain | (uintptr_t)d_k_gain) & 15) return rv_fail(RV_E_ARG, "gains must start at multiples of 16 bytes");
  m->q_gain = d_q_gain;
  m->k_gain = d_k_gain;
  return RV_OK;
}

rv_status rv_cache_dims(const rv_cache* c, int32_t* h_dims) {
  if (!c || !h_dims) return rv_fail(RV_E_ARG, "cache and dims must not be NULL");
  const rv_config& mc = c->m->cfg;
  h_dims[0] = c->B;
  h_dims[1] = mc.n_heads;
  h_dims[2] = mc.n_kv_heads;
  h_dims[3] = mc.head_dim;
  return RV_OK;
}

rv_status rv_cache_append(rv_cache* c, int32_t layer, int32_t batch, const int32_t* h_pos, const int32_t* h_rows,
                          const rv_rows* rows, void* stream) {
  if (!c || !h_pos || !h_rows || !rows) return rv_fail(RV_E_ARG, "cache, positions, counts and rows must not be NULL");
  if (rv_status s = check_layer(c, layer); s != RV_OK) return s;
  const rv_config& mc = c->m->cfg;
  const int io = rows->dtype, qd = mc.n_heads * mc.head_dim, kvd = mc.n_kv_heads * mc.head_dim;
  if (io != RV_F32 && io != RV_BF16) return rv_fail(RV_E_ARG, "rows must be RV_F32 or RV_BF16");
  AppendArgs a{};
  int max_rows = 0;
  if (rv_status s = check_spans(c, batch, h_pos, h_rows, rows->n_rows, a.pos, a.row0, a.blk0, &max_rows); s != RV_OK)
    return s;
  for (int b = 0; b < c->B; ++b)
    if (rv_status s = check_writable(c, b, h_pos[b], h_rows[b]); s != RV_OK) return s;
  if (!max_rows) return RV_OK;
  if (rv_status s = check_rows("k", rows->d_k, rows->ld_k, rows->kv_width, kvd, io); s != RV_OK) return s;
  if (rv_status s = check_rows("v", rows->d_v, rows->ld_v, rows->kv_width, kvd, io); s != RV_OK) return s;
  if (!rows->d_q != !rows->d_q_out) return rv_fail(RV_E_ARG, "q and its output come together");
  if (rows->d_q) {
    if (rv_status s = check_rows("q", rows->d_q, rows->ld_q, rows->q_width, qd, io); s != RV_OK) return s;
    if (rv_status s = check_rows("q output", rows->d_q_out, rows->ld_q_out, rows->q_width, qd, io); s != RV_OK) return s;
    if (rows->d_q_out == rows->d_q && rows->ld_q_out != rows->ld_q) return rv_fail(RV_E_ARG, "q in place with two row strides");
  }
  if (((uintptr_t)rows->d_q_gain | (uintptr_t)rows->d_k_gain) & 15)
    return rv_fail(RV_E_ARG, "gains must start at multiples of 16 bytes");
  const Planes p = layer_planes(c, layer);
  a.q = rows->d_q;
  a.k = rows->d_k;
  a.v = rows->d_v;
  a.q_out = rows->d_q_out;
  a.ldq = rows->ld_q;
  a.ldk = rows->ld_k;
  a.ldv = rows->ld_v;
  a.ldqo = rows->ld_q_out;
  a.q_gain = rows->d_q_gain;
  a.k_gain = rows->d_k_gain;
  a.eps = mc.rms_eps;
  a.rotate = rows->rotate != 0;
  a.rope_cos = c->rope_cos;
  a.rope_sin = c->rope_sin;
  a.kc = p.kc;
  a.vc = p.vc;
  a.kc2 = p.kc2;
  a.vc2 = p.vc2;
  a.n_heads = rows->d_q ? mc.n_heads : 0;
  a.n_kv = mc.n_kv_heads;
  a.kv_len = c->kv_len;
  a.B = c->B;
  HIP_TRY(launch_append(mc.dtype, io, mc.head_dim, max_rows, a, (hipStream_t)stream), "append");
  return RV_OK;
}

rv_status rv_cache_read(const rv_cache* c, int32_t layer, int32_t batch, const int32_t* h_pos, const int32_t* h_rows,
                        int32_t dtype, int64_t n_rows, int64_t width, void* d_k, int64_t ld_k, void* d_v, int64_t ld_v,
                        void* stream) {
  if (!c || !h_pos || !h_rows) return rv_fail(RV_E_ARG, "cache, positions and counts must not be NULL");
  if (rv_status s = check_layer(c, layer); s != RV_OK) return s;
  const rv_config& mc = c->m->cfg;
  if (dtype != RV_F32 && dtype != RV_BF16) return rv_fail(RV_E_ARG, "rows must be RV_F32 or RV_BF16");
  ReadArgs a{};
  int max_rows = 0;
  if (rv_status s = check_spans(c, batch, h_pos, h_rows, n_rows, a.pos, a.row0, a.blk0, &max_rows); s != RV_OK)
    return s;
  if (!max_rows) return RV_OK;
  const int kvd = mc.n_kv_heads * mc.head_dim;
  if (rv_status s = check_rows("k", d_k, ld_k, width, kvd, dtype); s != RV_OK) return s;
  if (rv_status s = check_rows("v", d_v, ld_v, width, kvd, dtype); s != RV_OK) return s;
  const Planes p = layer_planes(c, layer);
  a.k = d_k;
  a.v = d_v;
  a.ldk = ld_k;
  a.ldv = ld_v;
  a.kc = p.kc;
  a.vc = p.vc;
  a.kc2 = p.kc2;
  a.vc2 = p.vc2;
  a.own = c->tile_own;
  a.n_kv = mc.n_kv_heads;
  a.kv_len = c->kv_len;
  a.B = c->B;
  HIP_TRY(launch_read(mc.dtype, dtype, mc.head_dim, max_rows, a, (hipStream_t)stream), "read");
  return RV_OK;
}

rv_status rv_cache_copy(rv_cache* c, int32_t n, const int32_t* h_src, const int32_t* h_dst, const int32_t* h_len,
                        void* stream) {
  if (!c || n < 0 || (n > 0 && (!h_src || !h_dst || !h_len)))
    return rv_fail(RV_E_ARG, "cache, sources, destinations and lengths must not be NULL and n not negative");
  if (n > c->B) return rv_fail(RV_E_ARG, "%d moves into %d sequences", n, c->B);
  int tiles = 0;
  for (int i = 0; i < n; ++i) {
    if (h_src[i] < 0 || h_src[i] >= c->B) return rv_fail(RV_E_ARG, "source %d outside [0, batch=%d)", h_src[i], c->B);
    if (h_len[i] < 1 || h_len[i] > c->max_len)
      return rv_fail(RV_E_RANGE, "length %d outside [1, max_len=%d]", h_len[i], c->max_len);
    tiles = std::max(tiles, kv_tiles(h_len[i]));
  }
  bool gone[RV_MAX_BATCH];
  if (rv_status s = check_dsts(c, n, h_dst, gone); s != RV_OK) return s;
  if (!n) return RV_OK;
  hipStream_t st = (hipStream_t)stream;
  CopyArgs a = copy_args(c);
  uint8_t src[RV_MAX_BATCH], from[RV_MAX_BATCH], dst[RV_MAX_BATCH];
  for (int i = 0; i < n; ++i) {
    src[i] = (uint8_t)h_src[i];
    dst[i] = (uint8_t)h_dst[i];
  }
  // The ids and flags move as asked; a tile of a forked source comes from the slot
  // that holds it, so the moves of K and V are planned for each range of tiles
  // whose sources lie in the same slots (one range where nothing is shared).
  bool ids_done = false;
  for (int t0 = 0; t0 < tiles;) {
    int t1 = tiles;
    bool same = true;
    for (int i = 0; i < n; ++i) {
      from[i] = (uint8_t)c->tiles.at(src[i], t0);
      same = same && from[i] == src[i];
    }
    if (c->tiles.foreign) {
      for (t1 = t0 + 1; t1 < tiles; ++t1) {
        bool stays = true;
        for (int i = 0; i < n && stays; ++i) stays = c->tiles.at(src[i], t1) == from[i];
        if (!stays) break;
      }
    }
    plan_copy(n, from, dst, h_len, a.p);
    a.tile0 = t0;
    a.tile1 = t1;
    HIP_TRY(launch_copy(a, same && !ids_done, st), "copy");
    ids_done = ids_done || same;
    t0 = t1;
  }
  if (!ids_done) {
    plan_copy(n, src, dst, h_len, a.p);
    a.tile0 = a.tile1 = 0;
    HIP_TRY(launch_copy(a, true, st), "copy");
  }
  if (c->tiles.foreign) {
    OwnArgs o{};
    o.own = c->tile_own;
    o.T = c->tiles.T;
    int m = 0;
    for (int i = 0; i < n; ++i)
      if (!c->tiles.private_row(dst[i])) o.seq[m++] = dst[i];
    if (m) HIP_TRY(launch_own(o, m, st), "tile owners");
    for (int i = 0; i < m; ++i) c->tiles.make_private(o.seq[i]);
  }
  return RV_OK;
}

rv_status rv_cache_fork(rv_cache* c, int32_t src, int32_t len, int32_t n, const int32_t* h_dst, void* stream) {
  if (!c || n < 0 || (n > 0 && !h_dst)) return rv_fail(RV_E_ARG, "cache and destinations must not be NULL and n not negative");
  if (src < 0 || src >= c->B) return rv_fail(RV_E_ARG, "source %d outside [0, batch=%d)", src, c->B);
  if (len < 1 || len > c->max_len) return rv_fail(RV_E_RANGE, "length %d outside [1, max_len=%d]", len, c->max_len);
  if (n > c->B) return rv_fail(RV_E_ARG, "%d destinations of %d sequences", n, c->B);
  bool gone[RV_MAX_BATCH];
  if (rv_status s = check_dsts(c, n, h_dst, gone); s != RV_OK) return s;
  if (!n) return RV_OK;
  if (gone[src]) return rv_fail(RV_E_ARG, "sequence %d cannot be forked onto itself", src);
  hipStream_t st = (hipStream_t)stream;
  const int whole = (len - 1) / kTile, tail = kv_tiles(len);
  // the ids, and the tile that the fork's next positions share with its last ones
  CopyArgs a = copy_args(c);
  uint8_t from[RV_MAX_BATCH], dst[RV_MAX_BATCH];
  int32_t lens[RV_MAX_BATCH];
  const int slot = tail > whole ? c->tiles.at(src, whole) : src;
  for (int i = 0; i < n; ++i) {
    from[i] = (uint8_t)slot;
    dst[i] = (uint8_t)h_dst[i];
    lens[i] = len;
  }
  a.tile0 = whole;
  a.tile1 = tail;
  plan_copy(n, from, dst, lens, a.p);
  HIP_TRY(launch_copy(a, slot == src, st), "copy");
  if (slot != src) {
    for (int i = 0; i < n; ++i) from[i] = (uint8_t)src;
    plan_copy(n, from, dst, lens, a.p);
    a.tile0 = a.tile1 = 0;
    HIP_TRY(launch_copy(a, true, st), "copy");
  }
  OwnArgs o{};
  o.own = c->tile_own;
  o.T = c->tiles.T;
  o.src = src;
  o.whole = whole;
  for (int i = 0; i < n; ++i) o.seq[i] = dst[i];
  HIP_TRY(launch_own(o, n, st), "tile owners");
  for (int i = 0; i < n; ++i) {
    c->tiles.make_private(dst[i]);
    for (int t = 0; t < whole; ++t) c->tiles.set(dst[i], t, c->tiles.at(src, t));
  }
  return RV_OK;
}

rv_status rv_cache_attend(const rv_cache* c, int32_t layer, int32_t batch, const int32_t* h_pos, const int32_t* h_rows,
                          int32_t dtype, int64_t n_rows, int64_t width, const void* d_q, int64_t ld_q, void* d_out,
                          int64_t ld_out, void* stream) {
  if (!c || !h_pos || !h_rows) return rv_fail(RV_E_ARG, "cache, positions and counts must not be NULL");
  if (rv_status s = check_layer(c, layer); s != RV_OK) return s;
  const rv_config& mc = c->m->cfg;
  if (dtype != RV_F32 && dtype != RV_BF16) return rv_fail(RV_E_ARG, "rows must be RV_F32 or RV_BF16");
  int pos[RV_MAX_BATCH], row0[RV_MAX_BATCH + 1], max_rows = 0;
  if (rv_status s = check_spans(c, batch, h_pos, h_rows, n_rows, pos, row0, nullptr, &max_rows); s != RV_OK)
    return s;
  if (!max_rows) return RV_OK;
  if (row0[c->B] > c->rows_cap)
    return rv_fail(RV_E_CAPACITY, "%d rows, the cache's workspace holds %d", row0[c->B], c->rows_cap);
  const int qd = mc.n_heads * mc.head_dim;
  if (rv_status s = check_rows("q", d_q, ld_q, width, qd, dtype); s != RV_OK) return s;
  if (rv_status s = check_rows("output", d_out, ld_out, width, qd, dtype); s != RV_OK) return s;
  if (d_out == d_q && ld_out != ld_q) return rv_fail(RV_E_ARG, "q in place with two row strides");
  ShareArgs a{};
  plan_attend(c, pos, row0, a);
  const Planes p = layer_planes(c, layer);
  a.kc = p.kc;
  a.vc = p.vc;
  a.kc2 = p.kc2;
  a.vc2 = p.vc2;
  a.q = d_q;
  a.out = d_out;
  a.ldq = ld_q;
  a.ldo = ld_out;
  a.q_kind = a.o_kind = dtype;
  HIP_TRY(launch_share(mc.dtype, mc.head_dim, a, (hipStream_t)stream), "attention");
  return RV_OK;
}

rv_status rv_debug_cache_span(const rv_cache* c, int32_t which, size_t* offset, size_t* bytes) {
  if (!c || !offset || !bytes) return rv_fail(RV_E_ARG, "arguments must not be NULL");
  const size_t plane = c->kv_layer_elems * c->m->cfg.n_layers * c->m->es;
  const void* p = nullptr;
  size_t n = plane;
  switch (which) {
    case RV_SPAN_K: p = c->kc; break;
    case RV_SPAN_V: p = c->vc; break;
    case RV_SPAN_K_LO: p = c->kc2; break;
    case RV_SPAN_V_LO: p = c->vc2; break;
    case RV_SPAN_IDS:
      p = c->ids;
      n = (size_t)c->B * c->max_len * 4;
      break;
    default: return rv_fail(RV_E_ARG, "unknown span %d", which);
  }
  if ((which == RV_SPAN_K_LO || which == RV_SPAN_V_LO) && c->m->es != 2)
    return rv_fail(RV_E_ARG, "only caches of bf16 models have low planes");
  *offset = (size_t)((const char*)p - c->base);
  *bytes = n;
  return RV_OK;
}

}  // extern "C"
