// Host-side bookkeeping of the operators on the K/V cache: which slot holds
// each 64-position tile of each sequence, the order in which a copy moves
// tiles, and the launch shape of attention over tiles that sequences share.
// Plain arithmetic with no HIP types, so the same code also builds for the CPU
// alone (the host checks under tests/).
#pragma once
#include <algorithm>
#include <cmath>
#include <cstddef>
#include <cstdint>
#include <cstring>
#include <vector>

constexpr int kTile = 64;       // positions per tile
constexpr int kMaxSlots = 256;  // sequences of a cache (RV_MAX_BATCH)

// ---------------------------------------------------------------- ownership
// Tile t of sequence b lies in the slot of sequence at(b, t): its own unless b
// was forked from a sequence whose tile it reads.  A tile is only ever read at
// its own index t, so a slot's number says where it lies.  A sequence writes
// only to tiles of its own slot that no other sequence reads.
struct TileOwners {
  int B = 0, T = 0;
  int foreign = 0;             // (b, t) with at(b, t) != b
  std::vector<uint8_t> own;    // [B][T]
  std::vector<uint16_t> refs;  // [B][T]: other sequences that read tile t of slot b

  void create(int batch, int tiles) {
    B = batch;
    T = tiles;
    own.resize((size_t)B * T);
    refs.resize((size_t)B * T);
    reset();
  }
  void reset() {
    foreign = 0;
    for (int b = 0; b < B; ++b) std::fill_n(own.begin() + (size_t)b * T, T, (uint8_t)b);
    std::fill(refs.begin(), refs.end(), (uint16_t)0);
  }
  int at(int b, int t) const { return own[(size_t)b * T + t]; }
  void set(int b, int t, int slot) {
    uint8_t& o = own[(size_t)b * T + t];
    if (o != b) {
      --refs[(size_t)o * T + t];
      --foreign;
    }
    o = (uint8_t)slot;
    if (slot != b) {
      ++refs[(size_t)slot * T + t];
      ++foreign;
    }
  }
  void make_private(int b) {
    for (int t = 0; foreign && t < T; ++t) set(b, t, b);
  }
  bool private_row(int b) const {
    const uint8_t* o = own.data() + (size_t)b * T;
    for (int t = 0; t < T; ++t)
      if (o[t] != b) return false;
    return true;
  }
  // First tile of [t0, t1) that b may not write (-1: none).
  int first_shared(int b, int t0, int t1) const {
    if (!foreign) return -1;
    for (int t = t0; t < t1; ++t)
      if (at(b, t) != b || refs[(size_t)b * T + t]) return t;
    return -1;
  }
  // A sequence outside `gone` that reads a tile of a slot in it, or -1.
  int reader_of(const bool* gone) const {
    if (!foreign) return -1;
    for (int b = 0; b < B; ++b) {
      if (gone[b]) continue;
      for (int t = 0; t < T; ++t)
        if (gone[at(b, t)]) return b;
    }
    return -1;
  }
  // Leading tiles, at most cap, that a and b read from the same slots.
  int common(int a, int b, int cap) const {
    const uint8_t *x = own.data() + (size_t)a * T, *y = own.data() + (size_t)b * T;
    int t = 0;
    for (; t + 8 <= cap; t += 8) {
      uint64_t u, v;
      memcpy(&u, x + t, 8);
      memcpy(&v, y + t, 8);
      if (u != v) break;
    }
    while (t < cap && x[t] == y[t]) ++t;
    return t;
  }
};

// ---------------------------------------------------------------- copying
// Moves between slots that all read what was there before any of them wrote.
// A unit is a list of moves that one thread executes in order, batch of
// kMoveBatch by batch (it reads the whole batch before it writes it); different
// units touch no slot that another writes.  The order within a unit:
// a slot is overwritten once every move that reads it has been executed; what
// then remains is one cycle, which is opened by saving the slot that its first
// move overwrites, for its last move (from_saved) to write.
constexpr int kMoveBatch = 4;
constexpr int kFanMoves = 8;  // moves of one source per unit where nothing overwrites it

struct CopyProgram {
  int n = 0, units = 0;
  uint8_t src[kMaxSlots], dst[kMaxSlots];
  int32_t len[kMaxSlots];
  uint8_t from_saved[kMaxSlots];
  int16_t unit0[kMaxSlots + 1];   // first move of each unit
  int16_t saved[kMaxSlots];       // slot that the unit saves at its start, or -1
};

// h_src / h_dst: slots of the moves (destinations distinct), h_len what each brings.
inline void plan_copy(int n, const uint8_t* h_src, const uint8_t* h_dst, const int32_t* h_len, CopyProgram& p) {
  int16_t mover[kMaxSlots], readers[kMaxSlots], parent[kMaxSlots];
  for (int s = 0; s < kMaxSlots; ++s) {
    mover[s] = -1;
    readers[s] = 0;
    parent[s] = (int16_t)s;
  }
  auto root = [&](int s) {
    while (parent[s] != s) s = parent[s] = parent[parent[s]];
    return s;
  };
  for (int i = 0; i < n; ++i)
    if (h_src[i] != h_dst[i]) mover[h_dst[i]] = (int16_t)i;
  for (int i = 0; i < n; ++i) {
    if (h_src[i] == h_dst[i]) continue;
    ++readers[h_src[i]];
    if (mover[h_src[i]] >= 0) parent[root(h_src[i])] = (int16_t)root(h_dst[i]);  // must be ordered
  }
  // a source that is overwritten ties together every move that reads it (above);
  // one that is not leaves its moves free
  p.n = p.units = 0;
  int16_t open_saved = -1;
  int unit_first = 0;
  auto close = [&]() {
    if (p.n == unit_first) return;
    p.unit0[p.units] = (int16_t)unit_first;
    p.saved[p.units] = open_saved;
    ++p.units;
    unit_first = p.n;
    open_saved = -1;
  };
  auto push = [&](int i, bool from_saved) {
    p.src[p.n] = h_src[i];
    p.dst[p.n] = h_dst[i];
    p.len[p.n] = h_len[i];
    p.from_saved[p.n] = from_saved;
    ++p.n;
  };
  // free moves: by source, in units of up to kFanMoves
  bool done[kMaxSlots];
  for (int i = 0; i < n; ++i) done[i] = h_src[i] == h_dst[i];
  for (int i = 0; i < n; ++i) {
    if (done[i] || mover[h_src[i]] >= 0 || readers[h_dst[i]]) continue;
    for (int j = i; j < n; ++j) {
      if (done[j] || h_src[j] != h_src[i] || readers[h_dst[j]]) continue;
      push(j, false);
      done[j] = true;
      if (p.n - unit_first == kFanMoves) close();
    }
    close();
  }
  // ordered moves: one unit per set of slots tied together
  for (int r = 0; r < kMaxSlots; ++r) {
    if (root(r) != r) continue;
    bool again = true;
    while (again) {  // moves whose destination nothing still reads
      again = false;
      for (int i = 0; i < n; ++i) {
        if (done[i] || root(h_dst[i]) != r || readers[h_dst[i]]) continue;
        push(i, false);
        done[i] = true;
        --readers[h_src[i]];
        again = true;
      }
    }
    for (int i = 0; i < n; ++i) {
      if (done[i] || root(h_dst[i]) != r) continue;
      // the rest is one cycle: dst(i) <- src(i) <- ... <- dst(i)
      open_saved = h_dst[i];
      for (int j = i;;) {
        done[j] = true;
        const int next = mover[h_src[j]];
        push(j, next == i);
        if (next == i) break;
        j = next;
      }
      break;
    }
    close();
  }
  p.unit0[p.units] = (int16_t)p.n;
}

// ---------------------------------------------------------------- attention
// Query rows of one call: sequence b has rows row0[b] .. row0[b+1]-1 at
// positions pos0[b] ...  Sequences that read the same leading tiles form a
// group; its shared keys 0 .. 64*tiles-1 lie before every row of it, and are
// attended by the queries of all its rows together: one query slot for each
// (row, head of the kv head) where the members' rows follow each other in the call,
// else for each (member, row < rmax, head), so that slots of a member with fewer
// rows stay empty (12 continuations of 3030 tokens, 12-36 rows each, 70B shape:
// 147 us by rows, 181 by members).  Every sequence then attends its remaining keys alone.
// Both parts are split into runs of keys; the results of a row's runs (slots
// 0 .. sh.ns-1 of the shared part, then those of its own) are merged afterwards.
constexpr double kStreamBytes = 256e6;  // of the last-level cache
constexpr int kShareGroups = 32;
constexpr int kMergeSlots = 96;

struct SharePart {
  int qpw = 0;   // queries per workgroup
  int nqg = 0;   // query groups of the largest unit
  int ks = 0;    // keys per run (multiple of 64)
  int ns = 0;    // runs of the longest unit
  // query groups of one (run, sequence, kv head) lie on one XCD (8 workgroups apart),
  // unless that would leave a quarter of the XCDs' turns empty: one group over 2 kv
  // heads, 165 query groups, on 2 of the 8 XCDs take 31 us, spread 19 (fp32)
  bool spread = false;
  void place(int units) { spread = (units + 7) / 8 * 8 - units > (units + 7) / 8 * 2; }
};

struct SharePlan {
  int nseq = 0, rows = 0, groups = 0;
  bool stream = false;           // nothing shared, 16 queries to a kv head at most, keys beyond kStreamBytes
  bool own_last = false;         // the own part fits beside the last round of the shared part
  SharePart sh, own;
  // more workgroups of the own part than run at once: they start in `order`, long ones
  // first (64 sequences of 16-2000 keys, one row each, 8B: 104.2 -> 94.1 us; without
  // need the lookup costs 0.5 us of 37)
  bool sorted = false;
  uint8_t order[kMaxSlots];      // sequences by their own keys, most first
  uint8_t group_of[kMaxSlots];   // 255: none
  uint8_t member[kMaxSlots];     // members, group after group
  int16_t first[kShareGroups + 1];
  int32_t tiles[kShareGroups], rmax[kShareGroups];
  int32_t dense[kShareGroups];   // rows of a group whose rows follow each other, else 0
  int slot_rows(int g) const { return dense[g] ? dense[g] : (first[g + 1] - first[g]) * rmax[g]; }
  int slots() const { return (groups ? sh.ns : 0) + own.ns; }
};

// Groups of sequences that share leading tiles (all tables as described above).
// A sequence belongs to the group that saves the most tile reads among those
// still free; slots of a group are at most twice its queries.
inline void plan_groups(const TileOwners& tl, const int32_t* pos0, const int32_t* row0, SharePlan& p) {
  const int B = tl.B;
  p.groups = 0;
  p.first[0] = 0;
  memset(p.group_of, 255, sizeof p.group_of);
  if (!tl.foreign) return;
  bool free_[kMaxSlots];
  for (int b = 0; b < B; ++b) free_[b] = row0[b + 1] > row0[b] && pos0[b] >= kTile;
  for (int b = 0; b < B && p.groups < kShareGroups; ++b) {
    if (!free_[b]) continue;
    // leading tiles that each free sequence has in common with b
    int c[kMaxSlots], order[kMaxSlots], m = 0;
    for (int x = b; x < B; ++x) {
      if (!free_[x] || tl.at(x, 0) != tl.at(b, 0)) continue;
      c[x] = tl.common(b, x, std::min(pos0[b], pos0[x]) / kTile);
      if (c[x] > 0) order[m++] = x;
    }
    if (m < 2) continue;
    std::sort(order, order + m, [&](int x, int y) { return c[x] != c[y] ? c[x] > c[y] : x < y; });
    long long best = 0;
    int take = 0;
    for (int i = 1; i < m; ++i)
      if ((long long)c[order[i]] * i > best) {
        best = (long long)c[order[i]] * i;
        take = i + 1;
      }
    long long sum = 0;
    int rmax = 0;
    for (int i = 0; i < take; ++i) {
      const int r = row0[order[i] + 1] - row0[order[i]];
      sum += r;
      rmax = std::max(rmax, r);
    }
    const int shared = c[order[take - 1]];
    std::sort(order, order + take);
    const bool dense = row0[order[take - 1] + 1] - row0[order[0]] == sum;
    if (!dense && (long long)take * rmax > 2 * sum) continue;
    const int g = p.groups++, f = p.first[g];
    p.tiles[g] = shared;
    p.rmax[g] = rmax;
    p.dense[g] = dense ? (int32_t)sum : 0;
    for (int i = 0; i < take; ++i) {
      p.member[f + i] = (uint8_t)order[i];
      p.group_of[order[i]] = (uint8_t)g;
      free_[order[i]] = false;
    }
    p.first[g + 1] = (int16_t)(f + take);
  }
}

// One unit of a part before it is cut into runs: `keys` keys against `queries`
// queries of a kv head.
struct ShareUnit {
  int keys, queries;
};

// A part cut into `ns` runs of ks keys: its workgroups, the sum of their times
// and the longest (us).
struct ShareCut {
  int ks, ns;
  long long wgs;
  double sum, longest;
};

constexpr int kCutCounts[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 80};
constexpr int kCuts = sizeof kCutCounts / sizeof kCutCounts[0];

// The own part's workgroups take this much longer beside the shared part's (64
// continuations of 32768 keys, about 1000 own keys each: 160 workgroups of the
// shared part leave the other CUs enough time, 253 us; 192 do not, 296).
constexpr double kBeside = 1.35;

// Two workgroups share a CU where registers and LDS hold them (head_dim 64 and less,
// 128 queries a workgroup), and do this much more than one.  (16 sequences of
// 300-1900 keys, 1-9 rows each at the 1B shape: 2 runs, one workgroup per CU, 26.8 us;
// 3: 24.0, 4: 22.4, 6: 25.7, 8: 26.4.)
constexpr double kPair = 1.25;

// us of a workgroup that attends `keys` keys: prologue, epilogue and latencies,
// then the keys at its rate (head_dim 128; others in proportion).
inline double share_wg_us(bool bf16, int qpw, int keys, int hd) {
  const double f = hd / 128.0;
  // a wave of 16 queries, latency and products in turn (1024 keys, one row: head_dim 64
  // 52 us in one run, 13.5 in 8; 128: 92 and 19)
  if (!bf16) return 3.5 + (keys + kTile - 1) / kTile * (0.6 + 5.2 * f);
  if (qpw == 16) return 4.0 + keys * 8.0 * hd / 4.0e4;               // what one CU draws
  return 5.0 + (keys + kTile - 1) / kTile * (qpw == 128 ? 2.6 : 5.3) * f;
}

// The cuts of a part worth trying, within max_ns runs; their number.
inline int cut_part(bool bf16, const ShareUnit* u, int n, int n_kv, int hd, int qpw, int max_ns, ShareCut* out) {
  int kmax = 0, m = 0;
  for (int i = 0; i < n; ++i) kmax = std::max(kmax, u[i].keys);
  for (int ns : kCutCounts) {
    if (ns > max_ns || (ns > 1 && (ns - 1) * kTile >= kmax)) break;
    ShareCut c{};
    c.ks = ((kmax + ns - 1) / ns + kTile - 1) / kTile * kTile;
    c.ns = (kmax + c.ks - 1) / c.ks;
    if (m && out[m - 1].ns == c.ns) continue;
    const double whole = share_wg_us(bf16, qpw, c.ks, hd);
    for (int i = 0; i < n; ++i) {
      const long long w = (long long)((u[i].queries + qpw - 1) / qpw) * n_kv;
      const int full = u[i].keys / c.ks, rest = u[i].keys % c.ks;
      c.wgs += w * (full + (rest > 0));
      c.sum += (double)w * (full * whole + (rest ? share_wg_us(bf16, qpw, rest, hd) : 0));
    }
    c.longest = share_wg_us(bf16, qpw, std::min(c.ks, kmax), hd);
    out[m++] = c;
  }
  return m;
}

// Launch shape of a call.  part_entries: (run, row, head) results that the
// partial buffer holds; n_heads * rows <= part_entries / 2 always fits.  Both
// parts run in one launch.  The shared part's workgroups are
// the long ones: they take whole rounds of the CUs, the own part's fill what
// those leave and then add their share and half of one; every run costs its
// results' write and the merge's read.  (64 continuations of 32768 keys at the
// 70B shape: one round of 256 workgroups; with one and a half, 384, the same
// work took 253 instead of 184 us.)
inline void plan_share(const TileOwners& tl, bool bf16, const int32_t* pos0, const int32_t* row0, int n_heads, int n_kv,
                       int hd, size_t part_entries, SharePlan& p) {
  const int B = tl.B, G = n_heads / n_kv;
  p.nseq = B;
  p.rows = row0[B];
  plan_groups(tl, pos0, row0, p);
  const int fit = (int)std::min<size_t>(kMergeSlots, part_entries / ((size_t)p.rows * n_heads));
  ShareUnit own[kMaxSlots], sh[kShareGroups];
  int n = 0, most = 0, most_sh = 0, keys[kMaxSlots] = {};  // of each sequence's own part
  long long bytes = 0;
  for (int b = 0; b < B; ++b) {
    const int r = row0[b + 1] - row0[b];
    if (!r) continue;
    const int t0 = p.group_of[b] == 255 ? 0 : p.tiles[p.group_of[b]];
    keys[b] = pos0[b] + r - t0 * kTile;
    own[n++] = ShareUnit{keys[b], r * G};
    most = std::max(most, r * G);
    bytes += keys[b];
  }
  for (int g = 0; g < p.groups; ++g) {
    sh[g] = ShareUnit{p.tiles[g] * kTile, p.slot_rows(g) * G};
    most_sh = std::max(most_sh, sh[g].queries);
    bytes += sh[g].keys;
  }
  // queries per workgroup: never fewer of the shared part than of the own part
  auto qpw = [&](int q) { return !bf16 || q <= 16 ? 16 : q <= 128 ? 128 : 256; };
  p.own = p.sh = SharePart{};
  p.own.qpw = qpw(most);
  p.sh.qpw = std::max(p.own.qpw, qpw(most_sh));
  p.own.nqg = (most + p.own.qpw - 1) / p.own.qpw;
  p.sh.nqg = (most_sh + p.sh.qpw - 1) / p.sh.qpw;
  p.stream = bf16 && !p.groups && p.own.qpw == 16 && (double)bytes * n_kv * 8 * hd > kStreamBytes;
  ShareCut a[kCuts], c[kCuts];
  const int na = p.groups ? cut_part(bf16, sh, p.groups, n_kv, hd, p.sh.qpw, std::max(1, fit / 2), a) : 1;
  if (!p.groups) a[0] = ShareCut{};
  const int nc = cut_part(bf16, own, n, n_kv, hd, p.own.qpw, std::max(1, fit - (p.groups ? 1 : 0)), c);
  const bool pair = bf16 && hd <= 64 && p.own.qpw == 128 && p.sh.qpw == 128;
  const double stream = (double)bytes * n_kv * 8 * hd / 5.2e6, slots = bf16 ? pair ? 512 : 256 : 1024;
  double best = 0;
  for (int i = 0; i < na; ++i)
    for (int j = 0; j < nc; ++j) {
      const int runs = a[i].ns + c[j].ns;
      if (runs > fit && (i || j)) continue;
      const double rounds = std::ceil(a[i].wgs / slots), gap = rounds * slots * a[i].longest - a[i].sum;
      const double beside = c[j].sum * kBeside;
      double t = rounds * a[i].longest;
      if (!rounds) t = c[j].wgs <= slots ? c[j].longest : c[j].sum / slots + c[j].longest / 2;
      else if (beside > gap) t += (beside - gap) / slots + c[j].longest / 2;
      t = std::max(std::max(t, c[j].longest), stream);
      if (pair) t = std::max(t, (a[i].sum + c[j].sum) / (256 * kPair));
      if (runs > 1) t += 5.0 + 0.1 * runs + (double)runs * p.rows * n_heads * hd * 8 / 3.5e6;
      if ((!i && !j) || t < best) {
        best = t;
        p.sh.ks = a[i].ks;
        p.sh.ns = a[i].ns;
        p.own.ks = c[j].ks;
        p.own.ns = c[j].ns;
        p.own_last = beside <= gap;
        p.sorted = c[j].wgs > slots;
      }
    }
  p.sh.place(p.sh.ns * n_kv * p.groups);
  p.own.place(p.own.ns * n_kv * B);
  if (!p.sorted) return;
  for (int b = 0; b < B; ++b) p.order[b] = (uint8_t)b;
  std::sort(p.order, p.order + B, [&](int x, int y) { return keys[x] != keys[y] ? keys[x] > keys[y] : x < y; });
}
