// CPU check of the bookkeeping of rv_tiles.h and of the entry points that use it
// (rv_cache_ops.cpp), on a cache whose "device" memory is host memory and whose
// kernels are replaced by the plainest loops that do what their comments say.
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../../paper_2505_18629_amd/csrc/rv_cache_ops.cpp"

#define CHECK(x)                                                       \
  do {                                                                 \
    if (!(x)) {                                                        \
      printf("%s:%d: %s\n", __FILE__, __LINE__, #x);                   \
      exit(1);                                                         \
    }                                                                  \
  } while (0)

static char g_msg[512];
rv_status rv_fail(rv_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_msg, sizeof g_msg, fmt, ap);
  va_end(ap);
  return s;
}

int span_blocks(int pos, int rows) { return rows ? (pos + rows - 1) / 32 - pos / 32 + 1 : 0; }

// One value of each slot, moved as the kernel moves it: units in any order (the
// last first), every batch read before it is written.
template <typename V>
static void run_units(const CopyProgram& p, V* base, size_t stride, bool (*on)(int, int), int at) {
  for (int u = p.units - 1; u >= 0; --u) {
    V saved = p.saved[u] >= 0 ? base[p.saved[u] * stride] : V();
    for (int m0 = p.unit0[u]; m0 < p.unit0[u + 1]; m0 += kMoveBatch) {
      const int end = std::min<int>(m0 + kMoveBatch, p.unit0[u + 1]);
      V v[kMoveBatch];
      for (int m = m0; m < end; ++m) v[m - m0] = p.from_saved[m] ? saved : base[p.src[m] * stride];
      for (int m = m0; m < end; ++m)
        if (on(at, p.len[m])) base[p.dst[m] * stride] = v[m - m0];
    }
  }
}
static bool tile_on(int t, int len) { return t * 64 < len - 1; }
static bool id_on(int i, int len) { return i < len; }
static bool always(int, int) { return true; }

struct Vec {
  uint32_t x[4];
};
hipError_t launch_copy(const CopyArgs& a, bool with_ids, hipStream_t) {
  for (int pl = 0; pl < a.planes; ++pl)
    for (int l = 0; l < a.layers; ++l)
      for (int h = 0; h < a.n_kv; ++h)
        for (int t = a.tile0; t < a.tile1; ++t)
          for (int v = 0; v < a.tile_vecs; ++v)
            run_units(a.p, (Vec*)a.plane[pl] + l * a.layer_vecs + h * a.head_vecs + (size_t)t * a.tile_vecs + v,
                      a.slot_vecs, tile_on, t);
  if (!with_ids) return hipSuccess;
  for (int i = 0; i < a.max_len; ++i) run_units(a.p, a.ids + i, a.max_len, id_on, i);
  run_units(a.p, a.seq_bad, 1, always, 0);
  return hipSuccess;
}
hipError_t launch_own(const OwnArgs& a, int n, hipStream_t) {
  for (int i = 0; i < n; ++i)
    for (int t = 0; t < a.T; ++t)
      a.own[a.seq[i] * a.T + t] = t < a.whole ? a.own[a.src * a.T + t] : a.seq[i];
  return hipSuccess;
}
static int g_launches;
static ShareArgs g_share;
hipError_t launch_append(int, int, int, int, AppendArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_read(int, int, int, int, ReadArgs&, hipStream_t) { return ++g_launches, hipSuccess; }
hipError_t launch_share(int, int, ShareArgs& a, hipStream_t) {
  g_share = a;
  return ++g_launches, hipSuccess;
}

// A cache of one layer, one kv head and head_dim 32 in host memory.
struct Host {
  rv_model m{};
  rv_cache c{};
  std::vector<uint32_t> k, v;
  std::vector<int> own, ids, bad;
  Host(int B, int max_len, int heads = 4) {
    m.cfg = rv_config{1, 256, heads, 1, 32, 128, 16, RV_F32, 1e-5f, 10000.f, 0.02f};
    m.es = 4;
    c.m = &m;
    c.B = B;
    c.max_len = max_len;
    c.kv_len = (max_len + 63) / 64 * 64;
    c.kv_layer_elems = (size_t)B * c.kv_len * 32;
    c.rows_cap = 2048;
    c.part_entries = (size_t)2048 * heads * 8;
    k.resize(c.kv_layer_elems);
    v.resize(c.kv_layer_elems);
    c.tiles.create(B, c.kv_len / 64);
    own.assign(c.tiles.own.begin(), c.tiles.own.end());
    ids.resize((size_t)B * max_len);
    bad.resize(B);
    c.base = c.kc = (char*)k.data();
    c.vc = (char*)v.data();
    c.tile_own = own.data();
    c.ids = ids.data();
    c.seq_bad = bad.data();
  }
  // the value of K at position p as sequence b reads it
  uint32_t& at(std::vector<uint32_t>& x, int slot, int p) { return x[((size_t)slot * c.kv_len + p) * 32]; }
  uint32_t read(std::vector<uint32_t>& x, int b, int p) { return at(x, own[(size_t)b * c.tiles.T + p / 64], p); }
  void check_tables() {
    std::vector<int> refs((size_t)c.B * c.tiles.T);
    int foreign = 0;
    for (int b = 0; b < c.B; ++b)
      for (int t = 0; t < c.tiles.T; ++t) {
        const int o = c.tiles.at(b, t);
        CHECK(o == own[(size_t)b * c.tiles.T + t]);
        if (o != b) ++foreign, ++refs[(size_t)o * c.tiles.T + t];
      }
    CHECK(foreign == c.tiles.foreign);
    for (size_t i = 0; i < refs.size(); ++i) CHECK(refs[i] == c.tiles.refs[i]);
  }
};

// Sequences as plain lists of (K, V, id), against the cache after random copies,
// forks and writes.
static void walk(int B, int max_len, int steps, unsigned seed) {
  Host h(B, max_len);
  std::mt19937 r(seed);
  auto pick = [&](int n) { return (int)(r() % n); };
  struct Seq {
    int len = 1;
    std::vector<uint32_t> k, v;
    std::vector<int> ids;
    int bad = 0;
  };
  std::vector<Seq> s(B);
  uint32_t stamp = 1;
  auto write = [&](int b, int p, int n) {  // as rv_cache_append would
    if (check_writable(&h.c, b, p, n) != RV_OK) {
      // refused exactly where a tile is shared
      bool shared = false;
      for (int t = p / 64; t <= (p + n - 1) / 64; ++t)
        for (int x = 0; x < B; ++x)
          shared |= x != b ? h.own[(size_t)x * h.c.tiles.T + t] == b : h.own[(size_t)b * h.c.tiles.T + t] != b;
      CHECK(shared);
      return;
    }
    for (int q = p; q < p + n; ++q) {
      CHECK(h.own[(size_t)b * h.c.tiles.T + q / 64] == b);
      h.at(h.k, b, q) = s[b].k[q] = stamp++;
      h.at(h.v, b, q) = s[b].v[q] = stamp++;
    }
  };
  for (int b = 0; b < B; ++b) {
    s[b].k.assign(max_len, 0);
    s[b].v.assign(max_len, 0);
    s[b].ids.resize(max_len);
    for (int i = 0; i < max_len; ++i) h.ids[(size_t)b * max_len + i] = s[b].ids[i] = (int)stamp++;
    h.bad[b] = s[b].bad = pick(2);
    write(b, 0, max_len);
    s[b].len = max_len;
  }
  for (int step = 0; step < steps; ++step) {
    const int what = pick(4);
    if (what == 0) {
      const int b = pick(B), p = pick(max_len), n = 1 + pick(std::min(90, max_len - p));
      write(b, p, n);
    } else {
      std::vector<int32_t> dst(B), src(B), len(B);
      for (int b = 0; b < B; ++b) dst[b] = b;
      std::shuffle(dst.begin(), dst.end(), r);
      const int n = what == 1 ? 1 + pick(B) : 1 + pick(std::max(1, B - 1));
      std::vector<Seq> was = s;
      rv_status st;
      if (what < 3) {
        for (int i = 0; i < n; ++i) {
          src[i] = pick(4) ? pick(B) : dst[(i + 1) % n];
          len[i] = 1 + pick(s[src[i]].len);
        }
        st = rv_cache_copy(&h.c, n, src.data(), dst.data(), len.data(), nullptr);
      } else {
        src.assign(B, pick(B));
        len.assign(B, 1 + pick(s[src[0]].len));
        st = rv_cache_fork(&h.c, src[0], len[0], n, dst.data(), nullptr);
      }
      std::vector<bool> gone(B);
      for (int i = 0; i < n; ++i) gone[dst[i]] = true;
      bool blocked = false;
      for (int b = 0; b < B; ++b)
        for (int t = 0; t < h.c.tiles.T && !gone[b]; ++t) {
          if (st == RV_OK) CHECK(!gone[h.own[(size_t)b * h.c.tiles.T + t]] || what == 3);
          blocked |= gone[h.own[(size_t)b * h.c.tiles.T + t]];
        }
      if (st == RV_E_STATE) CHECK(blocked);
      else if (st == RV_E_ARG) CHECK(what == 3 && gone[src[0]]);
      else {
        CHECK(st == RV_OK);
        for (int i = 0; i < n; ++i) {
          Seq& d = s[dst[i]];
          const Seq& f = was[src[i]];
          const int keep = (len[i] - 1 + 63) / 64 * 64;
          // beyond the copied tiles the destination's own slot shows through
          for (int p = 0; p < max_len; ++p) {
            const bool in = p < std::min(keep, max_len);
            d.k[p] = in ? f.k[p] : h.at(h.k, dst[i], p);
            d.v[p] = in ? f.v[p] : h.at(h.v, dst[i], p);
          }
          for (int j = 0; j < len[i]; ++j) d.ids[j] = f.ids[j];
          d.bad = f.bad;
          d.len = len[i];
          if (what < 3) CHECK(h.c.tiles.private_row(dst[i]));
        }
      }
    }
    h.check_tables();
    for (int b = 0; b < B; ++b) {
      for (int p = 0; p < s[b].len - 1; ++p) {
        CHECK(h.read(h.k, b, p) == s[b].k[p]);
        CHECK(h.read(h.v, b, p) == s[b].v[p]);
      }
      for (int i = 0; i < max_len; ++i) CHECK(h.ids[(size_t)b * max_len + i] == s[b].ids[i]);
      CHECK(h.bad[b] == s[b].bad);
    }
  }
}

// Units touch nothing that another writes, for the most awkward sets of moves.
static void programs() {
  std::mt19937 r(7);
  for (int it = 0; it < 4000; ++it) {
    const int B = 1 + r() % 256, n = 1 + r() % B;
    std::vector<uint8_t> slots(B), src(n), dst(n);
    std::vector<int32_t> len(n);
    for (int b = 0; b < B; ++b) slots[b] = (uint8_t)b;
    std::shuffle(slots.begin(), slots.end(), r);
    for (int i = 0; i < n; ++i) {
      dst[i] = slots[i];
      src[i] = it % 3 == 0 ? slots[(i + 1) % n] : it % 3 == 1 ? slots[r() % B] : slots[r() % std::min(B, 3)];
      len[i] = 1 + r() % 300;
    }
    CopyProgram p;
    plan_copy(n, src.data(), dst.data(), len.data(), p);
    int moves = 0;
    for (int i = 0; i < n; ++i) moves += src[i] != dst[i];
    CHECK(p.n == moves && p.unit0[p.units] == p.n && p.units <= n);
    std::vector<int> writer(256, -1);
    for (int u = 0; u < p.units; ++u) {
      CHECK(p.unit0[u] < p.unit0[u + 1]);
      for (int m = p.unit0[u]; m < p.unit0[u + 1]; ++m) {
        CHECK(writer[p.dst[m]] < 0);
        writer[p.dst[m]] = u;
      }
    }
    for (int u = 0; u < p.units; ++u)
      for (int m = p.unit0[u]; m < p.unit0[u + 1]; ++m) CHECK(writer[p.src[m]] < 0 || writer[p.src[m]] == u);
    for (int t = 0; t < 5; ++t) {
      std::vector<int> x(256), want(256);
      for (int b = 0; b < 256; ++b) x[b] = want[b] = b;
      for (int i = 0; i < n; ++i)
        if (tile_on(t, len[i])) want[dst[i]] = src[i];
      run_units(p, x.data(), 1, tile_on, t);
      CHECK(x == want);
    }
  }
}

// Every key that a row may see falls into exactly one run that its merge reads,
// and every result has a place in the partial buffer.
static void shares() {
  std::mt19937 r(11);
  int grouped = 0, dense = 0, strided = 0;
  for (int it = 0; it < 600; ++it) {
    const int B = 1 + r() % 40, max_len = 64 + r() % 3000, G = 1 + r() % 8, n_kv = 1 + r() % 3;
    TileOwners tl;
    tl.create(B, (max_len + 63) / 64);
    const int forks = r() % 6;
    for (int f = 0; f < forks; ++f) {
      const int src = r() % B, whole = r() % tl.T;
      for (int b = 0; b < B; ++b)
        if (b != src && r() % 2)
          for (int t = 0; t < tl.T; ++t) tl.set(b, t, t < whole ? tl.at(src, t) : b);
    }
    int pos[256], row0[257] = {0};
    const int longest = 1 + r() % (it % 4 ? 5 : 60);
    for (int b = 0; b < B; ++b) {
      const int n = std::min<int>(it % 5 ? longest : r() % (longest + 1), max_len);
      pos[b] = n ? r() % (max_len - n + 1) : 0;
      row0[b + 1] = row0[b] + n;
    }
    if (!row0[B]) continue;
    const bool bf16 = it % 2;
    const int heads = G * n_kv;
    const size_t entries = (size_t)std::max(row0[B], 64) * heads * 8;
    SharePlan p;
    plan_share(tl, bf16, pos, row0, heads, n_kv, 32 << r() % 3, entries, p);
    grouped += p.groups;
    CHECK((size_t)p.slots() * p.rows * heads <= entries && p.slots() <= kMergeSlots);
    CHECK(p.own.ks > 0 && p.own.ks % 64 == 0 && p.own.ns > 0 && p.own.nqg > 0);
    CHECK(!p.groups || (p.sh.ks > 0 && p.sh.ks % 64 == 0 && p.sh.ns > 0 && p.sh.nqg > 0));
    std::vector<int> seen(B);
    for (int g = 0; g < p.groups; ++g) {
      CHECK(p.first[g + 1] - p.first[g] >= 2 && p.tiles[g] >= 1);
      CHECK(p.tiles[g] * 64 <= p.sh.ks * p.sh.ns);
      CHECK(p.slot_rows(g) * G <= p.sh.qpw * p.sh.nqg);
      int rows = 0, next = row0[p.member[p.first[g]]];
      bool follow = true;
      for (int i = p.first[g]; i < p.first[g + 1]; ++i) {
        const int b = p.member[i];
        follow = follow && row0[b] == next;
        next = row0[b + 1];
        rows += row0[b + 1] - row0[b];
      }
      CHECK(p.dense[g] == (follow ? rows : 0));
      (follow ? dense : strided) += 1;
      for (int i = p.first[g]; i < p.first[g + 1]; ++i) {
        const int b = p.member[i];
        CHECK(p.group_of[b] == g && !seen[b]++);
        CHECK(row0[b + 1] - row0[b] <= p.rmax[g] && row0[b + 1] > row0[b]);
        CHECK(p.tiles[g] * 64 <= pos[b]);
        for (int t = 0; t < p.tiles[g]; ++t) CHECK(tl.at(b, t) == tl.at(p.member[p.first[g]], t));
      }
    }
    for (int b = 0; b < B; ++b) {
      CHECK((p.group_of[b] == 255) == !seen[b]);
      const int n = row0[b + 1] - row0[b], k0 = seen[b] ? p.tiles[p.group_of[b]] * 64 : 0;
      if (!n) continue;
      CHECK(n * G <= p.own.qpw * p.own.nqg);
      CHECK(pos[b] + n - k0 <= p.own.ks * p.own.ns);  // the merge's last run exists
    }
  }
  CHECK(grouped > 200 && dense > 20 && strided > 20);
}

// Many sequences: the order of the own part's workgroups names each once, most keys first.
static void orders() {
  std::mt19937 r(5);
  int sorted = 0;
  for (int it = 0; it < 60; ++it) {
    const int B = 2 + r() % 255, n_kv = 8;
    TileOwners tl;
    tl.create(B, 40);
    if (it % 2)
      for (int b = 1; b < B; ++b)
        for (int t = 0; t < 20; ++t) tl.set(b, t, 0);
    int pos[256], row0[257] = {0};
    for (int b = 0; b < B; ++b) {
      const int n = r() % 8 ? 1 : 0;
      pos[b] = n ? 20 * 64 + r() % (20 * 64) : 0;
      row0[b + 1] = row0[b] + n;
    }
    if (!row0[B]) continue;
    SharePlan p;
    plan_share(tl, it % 3, pos, row0, 32, n_kv, 128, (size_t)2048 * 32 * 8, p);
    if (!p.sorted) continue;
    ++sorted;
    std::vector<int> met(B);
    int before = 0x7fffffff;
    for (int i = 0; i < B; ++i) {
      const int b = p.order[i], n = row0[b + 1] - row0[b];
      const int keys = n ? pos[b] + n - (p.group_of[b] == 255 ? 0 : p.tiles[p.group_of[b]] * 64) : 0;
      CHECK(!met[b]++ && keys <= before);
      before = keys;
    }
  }
  CHECK(sorted > 20);
}

alignas(16) static char mem[64];
static void refusals() {
  Host h(4, 200);
  rv_cache* c = &h.c;
  int32_t pos[4] = {0, 0, 0, 0}, n[4] = {1, 0, 2, 0};
  rv_rows ok{RV_F32, 1, 3, 128, 32, mem, mem, mem, mem, 128, 32, 32, 128, nullptr, nullptr};
  auto append = [&](rv_rows r, int layer = 0) { return rv_cache_append(c, layer, 4, pos, n, &r, nullptr); };
  CHECK(append(ok) == RV_OK && g_launches == 1);
  g_launches = 0;
  rv_rows r;
  CHECK(rv_cache_append(nullptr, 0, 4, pos, n, &ok, nullptr) == RV_E_ARG);
  CHECK(rv_cache_append(c, 0, 4, nullptr, n, &ok, nullptr) == RV_E_ARG);
  CHECK(rv_cache_append(c, 0, 4, pos, n, nullptr, nullptr) == RV_E_ARG);
  CHECK(append(ok, 1) == RV_E_ARG && append(ok, -1) == RV_E_ARG);
  CHECK((r = ok, r.dtype = 2, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.d_k = nullptr, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.d_v = mem + 8, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.ld_k = 31, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.ld_v = 34, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.dtype = RV_BF16, r.ld_q = 132, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.d_q_out = nullptr, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.ld_q_out = 127, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.ld_q_out = 132, append(r)) == RV_E_ARG);  // in place with another stride
  CHECK((r = ok, r.n_rows = 2, append(r)) == RV_E_ARG && (r = ok, r.q_width = 96, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.kv_width = 28, append(r)) == RV_E_ARG);
  CHECK((r = ok, r.d_k_gain = (const float*)(mem + 4), append(r)) == RV_E_ARG);
  CHECK(rv_cache_append(c, 0, 3, pos, n, &ok, nullptr) == RV_E_ARG);
  auto read = [&](int64_t rows, int io = RV_F32, void* v = mem, int w = 32, int batch = 4) {
    return rv_cache_read(c, 0, batch, pos, n, io, rows, w, mem, 32, v, 32, nullptr);
  };
  auto attend = [&](int64_t rows, int io = RV_F32, void* o = mem, int w = 128, int64_t ld = 128, int batch = 4) {
    return rv_cache_attend(c, 0, batch, pos, n, io, rows, w, mem, ld, o, 128, nullptr);
  };
  auto spans = [&](int p2, int n2) {
    pos[2] = p2;
    n[2] = n2;
    const rv_status a = (r = ok, r.n_rows = 1LL + n2, append(r)), b = read(1LL + n2), d = attend(1LL + n2);
    CHECK(a == b && b == d);
    pos[2] = 0;
    n[2] = 2;
    return a;
  };
  CHECK(spans(199, 2) == RV_E_RANGE && spans(-1, 1) == RV_E_RANGE && spans(0, -1) == RV_E_ARG);
  CHECK(spans(0x7fffffff, 0x7fffffff) == RV_E_RANGE && g_launches == 0);
  CHECK(spans(199, 1) == RV_OK && spans(-5, 0) == RV_OK);
  g_launches = 0;
  CHECK(read(3, 7) == RV_E_ARG && read(3, RV_F32, nullptr) == RV_E_ARG && read(3, RV_F32, mem, 64) == RV_E_ARG);
  CHECK(read(4) == RV_E_ARG && read(3, RV_F32, mem, 32, 5) == RV_E_ARG);
  CHECK(attend(3, 7) == RV_E_ARG && attend(3, RV_F32, nullptr) == RV_E_ARG && attend(2) == RV_E_ARG);
  CHECK(attend(3, RV_F32, mem, 64) == RV_E_ARG && attend(3, RV_F32, mem, 128, 64) == RV_E_ARG);
  CHECK(attend(3, RV_F32, mem, 128, 128, 1) == RV_E_ARG);
  CHECK(attend(3, RV_F32, mem, 128, 132) == RV_E_ARG);  // in place with another stride
  CHECK(g_launches == 0);
  const int32_t none[4] = {0, 0, 0, 0};
  CHECK(rv_cache_attend(c, 0, 4, pos, none, RV_F32, 0, 128, nullptr, 0, nullptr, 0, nullptr) == RV_OK && g_launches == 0);
  c->rows_cap = 2;
  CHECK(attend(3) == RV_E_CAPACITY);
  c->rows_cap = 2048;

  const int32_t s01[2] = {0, 1}, d23[2] = {2, 3}, d22[2] = {2, 2}, d24[2] = {2, 4}, l[2] = {100, 200}, l0[2] = {0, 1},
                l9[2] = {100, 201}, two[1] = {2}, zero[1] = {0}, one[1] = {1}, l1[1] = {100};
  CHECK(rv_cache_copy(nullptr, 2, s01, d23, l, nullptr) == RV_E_ARG);
  CHECK(rv_cache_copy(c, -1, s01, d23, l, nullptr) == RV_E_ARG && rv_cache_copy(c, 5, s01, d23, l, nullptr) == RV_E_ARG);
  CHECK(rv_cache_copy(c, 2, s01, d22, l, nullptr) == RV_E_ARG && rv_cache_copy(c, 2, s01, d24, l, nullptr) == RV_E_ARG);
  CHECK(rv_cache_copy(c, 2, d24, s01, l, nullptr) == RV_E_ARG);
  CHECK(rv_cache_copy(c, 2, s01, d23, l0, nullptr) == RV_E_RANGE && rv_cache_copy(c, 2, s01, d23, l9, nullptr) == RV_E_RANGE);
  CHECK(rv_cache_copy(c, 0, nullptr, nullptr, nullptr, nullptr) == RV_OK);
  CHECK(rv_cache_fork(c, 4, 100, 2, d23, nullptr) == RV_E_ARG && rv_cache_fork(c, 0, 0, 2, d23, nullptr) == RV_E_RANGE);
  CHECK(rv_cache_fork(c, 2, 100, 2, d23, nullptr) == RV_E_ARG && rv_cache_fork(c, 0, 201, 2, d23, nullptr) == RV_E_RANGE);
  CHECK(rv_cache_fork(c, 0, 100, 2, d22, nullptr) == RV_E_ARG);
  h.check_tables();

  // 2 and 3 read tile 0 of slot 0
  CHECK(rv_cache_fork(c, 0, 100, 2, d23, nullptr) == RV_OK);
  CHECK(check_writable(c, 0, 0, 1) == RV_E_STATE && check_writable(c, 2, 63, 2) == RV_E_STATE);
  CHECK(check_writable(c, 0, 64, 100) == RV_OK && check_writable(c, 3, 64, 1) == RV_OK && check_writable(c, 1, 0, 200) == RV_OK);
  CHECK(append(ok) == RV_E_STATE);
  CHECK(rv_cache_copy(c, 1, one, zero, l1, nullptr) == RV_E_STATE);  // 2 and 3 would lose their prompt
  CHECK(rv_cache_fork(c, 1, 100, 1, zero, nullptr) == RV_E_STATE);
  CHECK(rv_cache_copy(c, 1, two, two, l1, nullptr) == RV_OK && c->tiles.private_row(2) && !c->tiles.private_row(3));
  CHECK(check_writable(c, 2, 0, 1) == RV_OK && check_writable(c, 0, 0, 1) == RV_E_STATE);
  h.check_tables();
  CHECK(reset_owners(c, nullptr) == RV_OK && check_writable(c, 0, 0, 200) == RV_OK);
  h.check_tables();

  size_t off = 9, bytes = 9;
  CHECK(rv_debug_cache_span(c, RV_SPAN_K, &off, &bytes) == RV_OK && off == 0 && bytes == h.k.size() * 4);
  CHECK(rv_debug_cache_span(c, RV_SPAN_K_LO, &off, &bytes) == RV_E_ARG && rv_debug_cache_span(c, 9, &off, &bytes) == RV_E_ARG);
  CHECK(rv_model_qk_norm(nullptr, nullptr, nullptr, 0) == RV_E_ARG);
  CHECK(rv_model_qk_norm(&h.m, (const float*)mem, nullptr, 32) == RV_E_ARG);
  CHECK(rv_model_qk_norm(&h.m, (const float*)(mem + 4), (const float*)mem, 32) == RV_E_ARG);
  CHECK(rv_model_qk_norm(&h.m, (const float*)mem, (const float*)mem, 64) == RV_E_ARG);
  CHECK(rv_model_qk_norm(&h.m, (const float*)mem, (const float*)mem, 32) == RV_OK && h.m.q_gain);
  CHECK(rv_model_qk_norm(&h.m, nullptr, nullptr, 0) == RV_OK && !h.m.q_gain);
  int32_t dims[4];
  CHECK(rv_cache_dims(c, dims) == RV_OK && dims[0] == 4 && dims[1] == 4 && dims[2] == 1 && dims[3] == 32);
}

int main() {
  orders();
  refusals();
  programs();
  for (unsigned s = 0; s < 12; ++s) walk(2 + s % 6, s % 3 ? 64 * (1 + s % 4) + s : 64 * (1 + s % 3), 250, s);
  walk(40, 130, 60, 99);
  shares();
  puts("all moves, tables and plans as they should be");
  return 0;
}
