// Host side of include/catekv_paged.h: argument checks, plans and launches.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <exception>
#include <functional>
#include <queue>
#include <utility>
#include <vector>

#include "paged.h"

namespace {

using namespace catekv;

constexpr uint64_t kPagedMagic = 0x6361746570616765ull;
constexpr int64_t kMaxViews = (int64_t)1 << 20;
constexpr int64_t kMaxTokens = (int64_t)1 << 26;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return host_error(code, buf);
}

int hip_fail(hipError_t e, const char* what) { return fail(CATEKV_ERR_HIP, "%s: %s", what, hipGetErrorString(e)); }

size_t a256(size_t x) { return (x + 255) & ~(size_t)255; }

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

int check_cache(const catekv_paged_cache* c) {
  if (!c) return fail(CATEKV_ERR_INVALID_ARG, "null cache");
  if (!c->k || !c->v || !c->table || !c->lens || !c->refs || !c->free_bits)
    return fail(CATEKV_ERR_INVALID_ARG, "null pointer in the cache");
  if (!aligned16(c->k) || !aligned16(c->v)) return fail(CATEKV_ERR_INVALID_ARG, "pages are not on a 16-byte border");
  if (c->dtype != CATEKV_F32 && c->dtype != CATEKV_BF16) return fail(CATEKV_ERR_UNSUPPORTED, "dtype %d unsupported", c->dtype);
  const int p = c->page;
  if (p != 16 && p != 32 && p != 64 && p != 128 && p != 256)
    return fail(CATEKV_ERR_INVALID_ARG, "pages of %d rows (16, 32, 64, 128 or 256)", p);
  if (c->n_pages < 1 || c->n_slots < 1 || c->hkv < 1 || c->max_pages < 1)
    return fail(CATEKV_ERR_INVALID_ARG, "n_pages=%d n_slots=%d hkv=%d max_pages=%d must be >= 1", c->n_pages, c->n_slots,
                c->hkv, c->max_pages);
  if (c->hkv > kPagedMaxHkv || (int64_t)c->n_slots * c->hkv > kMaxViews)
    return fail(CATEKV_ERR_UNSUPPORTED, "n_slots=%d hkv=%d: more than 2^20 views, or %d of a slot", c->n_slots, c->hkv,
                kPagedMaxHkv);
  if ((int64_t)c->max_pages * p > kPagedMaxRows)
    return fail(CATEKV_ERR_UNSUPPORTED, "max_pages=%d of %d rows: more than 2^26 rows in a view", c->max_pages, p);
  return CATEKV_OK;
}

PagedCache kernel_cache(const catekv_paged_cache* c) {
  PagedCache k{};
  k.k = static_cast<char*>(c->k);
  k.v = static_cast<char*>(c->v);
  k.table = c->table;
  k.lens = c->lens;
  k.refs = c->refs;
  k.bits = c->free_bits;
  k.n_pages = c->n_pages;
  k.n_slots = c->n_slots;
  k.hkv = c->hkv;
  k.max_pages = c->max_pages;
  k.page_log = __builtin_ctz((unsigned)c->page);
  k.row_bytes = kD * (c->dtype == CATEKV_BF16 ? 2 : 4);
  return k;
}

// Slots in range; `distinct`: none twice.
int check_slots(const catekv_paged_cache* c, const int32_t* slots, int n, bool distinct, const char* name) {
  std::vector<char> seen(distinct ? c->n_slots : 0);
  for (int i = 0; i < n; ++i) {
    if (slots[i] < 0 || slots[i] >= c->n_slots)
      return fail(CATEKV_ERR_INVALID_ARG, "%s slot %d outside [0, %d)", name, slots[i], c->n_slots);
    if (distinct && seen[slots[i]]++) return fail(CATEKV_ERR_INVALID_ARG, "%s slot %d listed twice", name, slots[i]);
  }
  return CATEKV_OK;
}

int device_cus() {
  int dev = 0, n = 0;
  if (hipGetDevice(&dev) != hipSuccess ||
      hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n < 1)
    n = 256;
  return n;
}

// ---- the plan ------------------------------------------------------------------

struct Plan {
  int64_t n_tokens = 0, takes = 0;
  std::vector<PagedSeq> seqs;
  std::vector<PagedPiece> tiles;    // pieces of many new rows, by worker, and
  std::vector<int32_t> tile_workers;   // the first of every worker
  std::vector<PagedPiece> segs;     // of few: the stream workers' segments, and
  std::vector<int32_t> workers;     // the first of every worker
  std::vector<PagedJoin> joins;
  int64_t slot16 = 0;               // 16-byte units of partial slots
  int tile_joins = 0;               // joins of tiles, which come first
  int tile_parts = 0, few_parts = 0;   // the most parts of one join
  size_t seqs_off = 0, toks_off = 0, views_off = 0, takes_off = 0, tiles_off = 0, tile_workers_off = 0, segs_off = 0, workers_off = 0, joins_off = 0, slots_off = 0, total = 0;
};

// ---- tiles of many new rows --------------------------------------------------------
// Cut into pieces and dealt out to workgroups here, as many as the GPU holds at once: the
// GPU deals workgroups to its engines in turn and lets one engine's compute units stand
// idle while another's queue (2048 tokens at 32K in 376 pieces of unequal length: 1280 us
// where its longest share takes 890).
//
// What the ways to cut are compared by, in us as measured: a unit (64 cached rows; fp32: 32,
// with two workgroups to a compute unit), a piece's way in and out, the joining launch
// and a partial result's way to memory and back.
struct TileCosts {
  double unit, piece, join, slot;
  double apart;                        // of a unit's, for tiles of a view that do not run side by side
};
constexpr TileCosts kTileCosts = {1.8, 7.0, 6.0, 0.07, 0.08}, kTileCostsF32 = {7.5, 12.0, 6.0, 0.035, 0.0};
constexpr int kGang = 4;               // tiles of a view side by side, at most
constexpr int kXcds = 8;               // a worker's engine is its number modulo this

struct Tile {
  PagedPiece p;
  int64_t rows, units;
};

struct Cut {
  int tile;
  int64_t u0, u1;                      // units
  int worker;
};

struct Deal {
  std::vector<Cut> cuts;
  double cost = 0;
};

void price(Deal& d, const std::vector<Tile>& tiles, int workers, const TileCosts& k) {
  std::vector<double> load(workers, 0.0);
  double most = 0;
  int64_t slots = 0;
  for (const Cut& c : d.cuts) {
    load[c.worker] += k.unit * (double)(c.u1 - c.u0) + k.piece;
    most = std::max(most, load[c.worker]);
    slots += c.u1 - c.u0 < tiles[c.tile].units;
  }
  d.cost = most + (slots > 0 ? k.join + k.slot * (double)slots : 0.0);
}

// Tiles in parts of at most `share` units (0: whole), the longest first, each to the
// worker with least to do; one of the engine that has the view's other pieces (its cache
// holds what they read) if that costs little.
Deal deal(const std::vector<Tile>& tiles, int64_t share, int workers, const TileCosts& k) {
  Deal d;
  for (size_t i = 0; i < tiles.size(); ++i) {
    const int64_t u = tiles[i].units, parts = share ? (u + share - 1) / share : 1;
    for (int64_t s = 0; s < parts; ++s) d.cuts.push_back({(int)i, u * s / parts, u * (s + 1) / parts, 0});
  }
  std::stable_sort(d.cuts.begin(), d.cuts.end(), [](const Cut& x, const Cut& y) { return x.u1 - x.u0 > y.u1 - y.u0; });
  using Load = std::pair<double, int>;
  std::vector<std::priority_queue<Load, std::vector<Load>, std::greater<Load>>> engines(kXcds);
  for (int w = 0; w < workers; ++w) engines[w % kXcds].push({0.0, w});
  double total = 0;
  for (const Cut& c : d.cuts) total += k.unit * (double)(c.u1 - c.u0) + k.piece;
  const double slack = total / workers / 64;
  for (Cut& c : d.cuts) {
    int best = -1;
    for (int x = 0; x < kXcds; ++x)
      if (!engines[x].empty() && (best < 0 || engines[x].top() < engines[best].top())) best = x;
    const int own = tiles[c.tile].p.view % kXcds;
    if (!engines[own].empty() && engines[own].top().first <= engines[best].top().first + slack) best = own;
    const Load l = engines[best].top();
    engines[best].pop();
    engines[best].push({l.first + k.unit * (double)(c.u1 - c.u0) + k.piece, l.second});
    c.worker = l.second;
  }
  price(d, tiles, workers, k);
  return d;
}

// What a deal in parts of at most `share` units costs at least: no less than on average, and
// where there are more than j workers' worth of parts, one worker has j + 1 of the longest.
double least_cost(const std::vector<Tile>& tiles, int64_t share, int workers, const TileCosts& k) {
  int64_t units = 0, pieces = 0, slots = 0;
  std::vector<std::pair<int64_t, int64_t>> parts;      // length (rounded down), how many
  parts.reserve(tiles.size());
  for (const Tile& t : tiles) {
    const int64_t n = share ? (t.units + share - 1) / share : 1;
    parts.push_back({t.units / n, n});
    units += t.units;
    pieces += n;
    slots += n > 1 ? n : 0;
  }
  double most = (k.unit * (double)units + k.piece * (double)pieces) / workers;
  std::sort(parts.begin(), parts.end(), std::greater<>());
  int64_t before = 0, j = 0;
  for (const auto& p : parts)
    for (before += p.second; before > j * workers; ++j) most = std::max(most, (double)(j + 1) * (k.unit * (double)p.first + k.piece));
  return most + (slots ? k.join + k.slot * (double)slots : 0.0);
}

// All tiles end to end, cut into shares that take as long; neighbours lie in one engine.  No
// part is shorter than half a piece's way in and out.  `gang` neighbouring tiles of a view are
// cut at the same rows and given to workers of one engine, which read them at the same time:
// its cache is asked for them by all and the memory by one (8 tiles each of 16 views of 8498
// and 22747 rows: 347 us with shares of single tiles, which drift apart and read 1000 MB
// for 136; 331 in twos, 321 in fours).
Deal deal_line(const std::vector<Tile>& tiles, int workers, TileCosts k, int gang) {
  Deal d;
  struct Group {
    size_t first, n;
    int64_t units;
  };
  std::vector<Group> groups;
  int64_t units = 0;
  for (size_t i = 0; i < tiles.size();) {
    size_t n = 1;
    while (n < (size_t)gang && i + n < tiles.size() && tiles[i + n].p.view == tiles[i].p.view) ++n;
    groups.push_back({i, n, tiles[i + n - 1].units});  // later tiles see more
    units += groups.back().units;
    i += n;
  }
  // what smaller gangs than the views have tiles for lose, as measured
  size_t views = 1;
  for (size_t i = 1; i < tiles.size(); ++i) views += tiles[i].p.view != tiles[i - 1].p.view;
  const double width = std::min<double>(kGang, (double)tiles.size() / (double)views);
  if (width > gang) k.unit *= 1.0 + k.apart * (width - gang) / (width - 1.0);
  int gangs = workers / gang, per = gangs / kXcds;
  if (gang > 1) gangs = per * kXcds;
  if (gangs == 0) {
    d.cost = HUGE_VAL;
    return d;
  }
  const double share = (k.unit * (double)units + k.piece * (double)(groups.size() + gangs)) / gangs;
  const int64_t least = std::max<int64_t>(1, (int64_t)(k.piece / k.unit / 2));
  double spent = 0;
  size_t i = 0;
  int64_t off = 0;
  for (int s = 0; s < gangs && i < groups.size(); ++s) {
    const bool last = s == gangs - 1;
    while (i < groups.size()) {
      const int64_t room = (int64_t)std::floor(((s + 1) * share - spent - k.piece) / k.unit + 0.5);
      if (room < least && !last) break;
      const int64_t rest = groups[i].units - off, take = last || rest <= room + least ? rest : room;
      for (size_t j = 0; j < groups[i].n; ++j) {
        const int64_t end = std::min(off + take, tiles[groups[i].first + j].units);
        const int w = gangs % kXcds == 0 ? (int)((s % per * gang + j) * kXcds + s / per) : s;
        if (off < end) d.cuts.push_back({(int)(groups[i].first + j), off, end, w});
      }
      spent += k.piece + k.unit * (double)take;
      off += take;
      if (off == groups[i].units) {
        ++i;
        off = 0;
      }
    }
  }
  price(d, tiles, workers, k);
  return d;
}

// bf16 batches of both kinds run in one launch: as many of the compute units for the few-token
// sequences as end both at about the same time.  A compute unit reads 64 rows of K and V in 1.2 us
// (1.5 with all of them at it), and a share's start, joining of waves and way out take 8; a
// tile's unit takes 2.2 beside them.  (16 sequences of 4096 to 32768 rows, two of them with 512 new
// tokens: 455 us with 96 of 256, 564 with 64, 490 with 112; as launches one after the other 476.)
int few_workers(int64_t tile_units, int64_t n_tiles, int64_t few_units, int cus) {
  const TileCosts& k = kTileCosts;
  int best = 1;
  double least = HUGE_VAL;
  for (int w = 8; w < cus; w += w < 32 ? 8 : 32) {     // whole gangs are left in every engine
    const double tiles = (2.2 * (double)tile_units + k.piece * (double)std::max<int64_t>(n_tiles, cus - w)) / (cus - w);
    const double few = 8.0 + 1.2 * (double)((few_units + w - 1) / w);
    if (std::max(tiles, few) < least) {
      least = std::max(tiles, few);
      best = w;
    }
  }
  return best;
}

int build_plan(const catekv_paged_cache* c, const int32_t* slots, const int32_t* n_new, const int64_t* max_rows, int n_seqs,
               int hq, Plan& P) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!slots || !n_new || !max_rows) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  if (n_seqs < 1) return fail(CATEKV_ERR_INVALID_ARG, "n_seqs=%d must be >= 1", n_seqs);
  rc = host_check_heads(hq, c->hkv, kD);
  if (!rc) rc = check_slots(c, slots, n_seqs, true, "sequence's");
  if (rc) return rc;
  const int hkv = c->hkv, G = hq / hkv;
  int64_t tokens = 0;
  for (int i = 0; i < n_seqs; ++i) {
    if (n_new[i] < 0) return fail(CATEKV_ERR_INVALID_ARG, "sequence %d has %d new tokens", i, n_new[i]);
    if (n_new[i] > kMaxTokens || tokens + n_new[i] > kMaxTokens) return fail(CATEKV_ERR_UNSUPPORTED, "more than 2^26 new tokens");
    P.seqs.push_back({slots[i], n_new[i], (int32_t)tokens, 0});
    tokens += n_new[i];
    P.takes += (int64_t)hkv * ((n_new[i] + c->page - 1) / c->page + 1);
  }
  for (int64_t v = 0; v < (int64_t)n_seqs * hkv; ++v) {
    if (max_rows[v] < 0) return fail(CATEKV_ERR_INVALID_ARG, "max_rows=%lld of a view below 0", (long long)max_rows[v]);
    if (max_rows[v] > kPagedMaxRows) return fail(CATEKV_ERR_UNSUPPORTED, "max_rows=%lld of a view above 2^26", (long long)max_rows[v]);
  }
  P.n_tokens = tokens;
  // launches of 256 threads: rows (16 or 32 lanes each) and views of the append; query rows of a join
  const int lanes = c->dtype == CATEKV_BF16 ? 16 : 32;
  if (!launch_fits((tokens * hkv * lanes + 255) / 256 + (int64_t)n_seqs * hkv, 256) || P.takes > INT32_MAX)
    return fail(CATEKV_ERR_UNSUPPORTED, "%lld tokens of %d heads: too many for one launch", (long long)tokens, hkv);

  // Work counts in units of kPagedUnit cached rows, fp32 tiles' in halves of that.  A view's new rows are one piece of
  // the stream kernel if they are few, or tiles of the other one.
  const int R = paged_tile_rows(c->dtype), cus = device_cus();
  auto few = [&](int i) { return (int64_t)n_new[i] * G <= kStreamRows; };
  auto rows_seen = [&](int i, int h, int64_t row0, int rows) {       // by the piece's last token
    const int64_t last = std::min<int64_t>(row0 + rows, (int64_t)n_new[i] * G) - 1;
    return std::max<int64_t>(0, max_rows[(int64_t)i * hkv + h] - n_new[i] + 1 + last / G);
  };
  const int unit = c->dtype == CATEKV_BF16 ? kPagedUnit : kPagedUnit / 2;
  auto units_of = [](int64_t rows, int each) { return std::max<int64_t>(1, (rows + each - 1) / each); };
  auto piece = [&](int i, int h, int64_t row0) {
    PagedPiece p{};
    p.view = slots[i] * hkv + h;
    p.tok0 = P.seqs[i].tok0;
    p.n_new = n_new[i];
    p.row0 = (int32_t)row0;
    p.max_rows = (int32_t)max_rows[(int64_t)i * hkv + h];
    return p;
  };
  auto join = [&](const PagedPiece& p, int64_t parts, int rows) {    // slots for the parts of p
    if (parts < 2) return;
    P.joins.push_back({p.view, p.tok0, p.n_new, p.row0, (int32_t)P.slot16, (int32_t)parts, rows, 0});
    int& most = rows == kStreamRows ? P.few_parts : P.tile_parts;
    most = std::max(most, (int)parts);
    P.slot16 += parts * (int64_t)(paged_slot_floats(rows) / 4);
  };
  int64_t tile_units = 0, n_tiles = 0, few_units = 0;
  for (int i = 0; i < n_seqs; ++i)
    for (int h = 0; n_new[i] > 0 && h < hkv; ++h) {
      if (few(i)) {
        few_units += units_of(rows_seen(i, h, 0, kStreamRows), kPagedUnit);
        continue;
      }
      for (int64_t r = 0; r < (int64_t)n_new[i] * G; r += R, ++n_tiles) tile_units += units_of(rows_seen(i, h, r, R), unit);
    }
  if (n_tiles > (int64_t)1 << 22) return fail(CATEKV_ERR_UNSUPPORTED, "%lld tiles of new rows: too many for one launch", (long long)n_tiles);

  int few_cus = cus;                                   // compute units of the few-token sequences
  // tiles: whole, or cut at some share of the work, whichever is done first
  if (n_tiles > 0) {
    std::vector<Tile> tiles;
    tiles.reserve(n_tiles);
    for (int i = 0; i < n_seqs; ++i)
      for (int h = 0; n_new[i] > 0 && !few(i) && h < hkv; ++h)
        for (int64_t r = 0; r < (int64_t)n_new[i] * G; r += R) {
          const int64_t rows = rows_seen(i, h, r, R);
          tiles.push_back({piece(i, h, r), rows, units_of(rows, unit)});
        }
    const bool half = c->dtype == CATEKV_BF16;
    const TileCosts& costs = half ? kTileCosts : kTileCostsF32;
    const int workers = !half ? 2 * cus : few_units > 0 ? std::max(1, cus - few_workers(tile_units, n_tiles, few_units, cus)) : cus;
    if (half && few_units > 0) few_cus = std::max(1, cus - workers);
    Deal best = deal(tiles, 0, workers, costs);
    // (a whole tile's way is not left for less than a twentieth)
    const double even_cost = (costs.unit * (double)tile_units + costs.piece * (double)n_tiles) / workers;
    if (n_tiles < 8 * (int64_t)workers && best.cost > 1.05 * even_cost) {
      const int64_t even = (tile_units + workers - 1) / workers;
      int64_t longest = 0;
      for (const Tile& t : tiles) longest = std::max(longest, t.units);
      Deal d;
      for (int gang = half ? kGang : 1; gang >= 1; gang /= 2) {
        d = deal_line(tiles, workers, costs, gang);
        if (d.cost < best.cost) best = std::move(d);
      }
      for (int k = 2; k <= 8; ++k) {                 // shares of 2 to 1/2 of an equal one
        const int64_t share = std::max<int64_t>(1, (4 * even + k - 1) / k);
        if (share >= longest || least_cost(tiles, share, workers, costs) >= best.cost) continue;
        d = deal(tiles, share, workers, costs);
        if (d.cost < best.cost) best = std::move(d);
      }
    }
    std::vector<int> parts(tiles.size(), 0);
    for (const Cut& c : best.cuts) ++parts[c.tile];
    std::vector<int64_t> slot(tiles.size(), -1);
    const int64_t each = (int64_t)(paged_slot_floats(R) / 4);
    for (size_t i = 0; i < tiles.size(); ++i)
      if (parts[i] > 1) {
        slot[i] = P.slot16;
        join(tiles[i].p, parts[i], R);
        if (P.slot16 > INT32_MAX) return fail(CATEKV_ERR_UNSUPPORTED, "too many partial results");
      }
    std::stable_sort(best.cuts.begin(), best.cuts.end(), [](const Cut& x, const Cut& y) { return x.worker < y.worker; });
    P.tile_workers.assign(1, 0);
    for (const Cut& c : best.cuts) {
      while ((int)P.tile_workers.size() <= c.worker) P.tile_workers.push_back((int32_t)P.tiles.size());
      PagedPiece p = tiles[c.tile].p;
      p.t0 = (int32_t)(c.u0 * unit);
      p.t1 = (int32_t)std::min<int64_t>(tiles[c.tile].rows, c.u1 * unit);
      p.slot = -1;
      if (parts[c.tile] > 1) {
        p.slot = (int32_t)slot[c.tile];
        slot[c.tile] += each;
      }
      P.tiles.push_back(p);
    }
    P.tile_workers.push_back((int32_t)P.tiles.size());
  }
  P.tile_joins = (int)P.joins.size();

  // the rest laid end to end and cut into equal shares, one per workgroup
  if (few_units > 0) {
    const int64_t W = std::min<int64_t>(few_cus, few_units);
    int64_t w = 0, left = 0, done = 0;            // the share being filled, units left of it, units given out
    P.workers.push_back(0);
    auto open = [&] {
      left = (w + 1) * few_units / W - done;
    };
    open();
    for (int i = 0; i < n_seqs; ++i)
      for (int h = 0; n_new[i] > 0 && few(i) && h < hkv; ++h) {
        const int64_t rows = rows_seen(i, h, 0, kStreamRows), u = units_of(rows, kPagedUnit);
        const size_t begin = P.segs.size();
        PagedPiece p = piece(i, h, 0);
        for (int64_t off = 0; off < u;) {
          const int64_t n = std::min(left, u - off);
          p.t0 = (int32_t)(off * kPagedUnit);
          p.t1 = (int32_t)std::min<int64_t>(rows, (off + n) * kPagedUnit);
          p.slot = -1;
          P.segs.push_back(p);
          off += n;
          left -= n;
          done += n;
          if (left == 0 && ++w < W) {
            P.workers.push_back((int32_t)P.segs.size());
            open();
          }
        }
        const int64_t parts = (int64_t)(P.segs.size() - begin), slot = P.slot16;
        join(p, parts, kStreamRows);
        if (P.slot16 > INT32_MAX) return fail(CATEKV_ERR_UNSUPPORTED, "too many partial results");
        for (int64_t s = 0; parts > 1 && s < parts; ++s)
          P.segs[begin + s].slot = (int32_t)(slot + s * (int64_t)(paged_slot_floats(kStreamRows) / 4));
      }
    P.workers.push_back((int32_t)P.segs.size());
  }
  if (!launch_fits((int64_t)P.joins.size() * std::max(R, kStreamRows), kJoinThreads))
    return fail(CATEKV_ERR_UNSUPPORTED, "%zu views' results to join: too many for one launch", P.joins.size());

  size_t at = 0;
  auto put = [&](size_t& off, size_t bytes) {
    off = at;
    at += a256(bytes);
  };
  put(P.seqs_off, P.seqs.size() * sizeof(PagedSeq));
  put(P.toks_off, (size_t)tokens * sizeof(int32_t));
  put(P.tiles_off, P.tiles.size() * sizeof(PagedPiece));
  put(P.tile_workers_off, P.tile_workers.size() * sizeof(int32_t));
  put(P.segs_off, P.segs.size() * sizeof(PagedPiece));
  put(P.workers_off, P.workers.size() * sizeof(int32_t));
  put(P.joins_off, P.joins.size() * sizeof(PagedJoin));
  put(P.views_off, (size_t)n_seqs * hkv * sizeof(PagedTake));     // from here on: written by the calls
  put(P.takes_off, (size_t)P.takes * sizeof(int32_t));
  put(P.slots_off, (size_t)P.slot16 * 16);
  P.total = std::max<size_t>(at, 256);
  return CATEKV_OK;
}

int check_plan(const catekv_paged_cache* c, const catekv_paged_plan_t* plan, const void* ws, size_t ws_bytes) {
  int rc = check_cache(c);
  if (rc) return rc;
  if (!plan || plan->magic != kPagedMagic) return fail(CATEKV_ERR_INVALID_ARG, "plan missing or not built by catekv_paged_plan");
  if (plan->hkv != c->hkv || plan->n_slots != c->n_slots || plan->page != c->page || plan->dtype != c->dtype)
    return fail(CATEKV_ERR_INVALID_ARG, "the cache (hkv=%d n_slots=%d page=%d dtype=%d) differs from the plan's (%d, %d, %d, %d)",
                c->hkv, c->n_slots, c->page, c->dtype, plan->hkv, plan->n_slots, plan->page, plan->dtype);
  return host_check_ws(ws, ws_bytes, plan->ws_bytes);
}

template <typename F>
int guarded(F f) {                  // no exception leaves a C entry
  try {
    return f();
  } catch (const std::exception& e) {
    return fail(CATEKV_ERR_HIP, "host memory: %s", e.what());
  }
}

int64_t compact_takes(const catekv_paged_cache* c, int n_sel, int b, int cs, int tail) {
  return (int64_t)n_sel * (((int64_t)b * cs + tail + c->page - 1) / c->page);
}

int check_compact(const catekv_paged_cache* c, int n_sel, int b, int cs, int tail) {
  const int rc = check_cache(c);
  if (rc) return rc;
  if (n_sel < 1 || n_sel > kPagedMaxHeads) return fail(CATEKV_ERR_INVALID_ARG, "n_sel=%d outside [1, %d]", n_sel, kPagedMaxHeads);
  if (b < 1 || cs < 1 || tail < 0) return fail(CATEKV_ERR_INVALID_ARG, "b=%d, cs=%d must be >= 1, tail=%d >= 0", b, cs, tail);
  if ((int64_t)n_sel * b > 1 << 24 || (int64_t)b * cs + tail > kPagedMaxRows || compact_takes(c, n_sel, b, cs, tail) > INT32_MAX)
    return fail(CATEKV_ERR_UNSUPPORTED, "n_sel=%d, b=%d, cs=%d, tail=%d: too large for one call", n_sel, b, cs, tail);
  return CATEKV_OK;
}

size_t compact_bytes(const catekv_paged_cache* c, int n_sel, int b, int cs, int tail) {
  return a256((size_t)n_sel * b * sizeof(int32_t)) + a256((size_t)n_sel * sizeof(PagedTake)) +
         a256((size_t)compact_takes(c, n_sel, b, cs, tail) * sizeof(int32_t));
}

}  // namespace

extern "C" {

int catekv_paged_init(const catekv_paged_cache* cache, void* stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  const hipError_t e = launch_paged_init(kernel_cache(cache), reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "paged_init launch");
}

size_t catekv_paged_workspace(const catekv_paged_cache* cache, const int32_t* slots_host, const int32_t* new_host,
                              const int64_t* max_rows_host, int n_seqs, int hq) {
  size_t bytes = 0;
  guarded([&] {
    Plan P;
    const int rc = build_plan(cache, slots_host, new_host, max_rows_host, n_seqs, hq, P);
    if (!rc) bytes = P.total;
    return rc;
  });
  return bytes;
}

int catekv_paged_plan(const catekv_paged_cache* cache, const int32_t* slots_host, const int32_t* new_host,
                      const int64_t* max_rows_host, int n_seqs, int hq, catekv_paged_plan_t* plan, void* ws,
                      size_t ws_bytes, void* stream) {
  return guarded([&]() -> int {
    if (!plan) return fail(CATEKV_ERR_INVALID_ARG, "null plan");
    Plan P;
    int rc = build_plan(cache, slots_host, new_host, max_rows_host, n_seqs, hq, P);
    if (!rc) rc = host_check_ws(ws, ws_bytes, P.total);
    if (rc) return rc;
    std::vector<unsigned char> host(P.views_off, 0);
    auto copy = [&](size_t off, const void* from, size_t bytes) {
      if (bytes) std::memcpy(host.data() + off, from, bytes);
    };
    copy(P.seqs_off, P.seqs.data(), P.seqs.size() * sizeof(PagedSeq));
    for (size_t i = 0; i < P.seqs.size(); ++i)
      for (int t = 0; t < P.seqs[i].n_new; ++t) {
        const int32_t s = (int32_t)i;
        std::memcpy(host.data() + P.toks_off + ((size_t)P.seqs[i].tok0 + t) * sizeof s, &s, sizeof s);
      }
    copy(P.tiles_off, P.tiles.data(), P.tiles.size() * sizeof(PagedPiece));
    copy(P.tile_workers_off, P.tile_workers.data(), P.tile_workers.size() * sizeof(int32_t));
    copy(P.segs_off, P.segs.data(), P.segs.size() * sizeof(PagedPiece));
    copy(P.workers_off, P.workers.data(), P.workers.size() * sizeof(int32_t));
    copy(P.joins_off, P.joins.data(), P.joins.size() * sizeof(PagedJoin));
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    hipError_t e = hipMemcpyAsync(ws, host.data(), host.size(), hipMemcpyHostToDevice, s);
    if (e != hipSuccess) return hip_fail(e, "paged_plan upload");
    e = hipStreamSynchronize(s);
    if (e != hipSuccess) return hip_fail(e, "paged_plan synchronize");
    std::memset(plan, 0, sizeof *plan);
    plan->magic = kPagedMagic;
    plan->n_seqs = n_seqs;
    plan->n_tokens = (int32_t)P.n_tokens;
    plan->hq = hq;
    plan->hkv = cache->hkv;
    plan->n_slots = cache->n_slots;
    plan->page = cache->page;
    plan->dtype = cache->dtype;
    plan->n_tile = P.tile_workers.empty() ? 0 : (int32_t)P.tile_workers.size() - 1;
    plan->n_workers = P.workers.empty() ? 0 : (int32_t)P.workers.size() - 1;
    plan->n_joins = (int32_t)P.joins.size();
    plan->tile_joins = P.tile_joins;
    plan->tile_parts = P.tile_parts;
    plan->few_parts = P.few_parts;
    plan->seqs_off = P.seqs_off;
    plan->toks_off = P.toks_off;
    plan->tiles_off = P.tiles_off;
    plan->tile_workers_off = P.tile_workers_off;
    plan->segs_off = P.segs_off;
    plan->workers_off = P.workers_off;
    plan->joins_off = P.joins_off;
    plan->views_off = P.views_off;
    plan->takes_off = P.takes_off;
    plan->slots_off = P.slots_off;
    plan->ws_bytes = P.total;
    return host_ok();
  });
}

int catekv_paged_append(const catekv_paged_cache* cache, const catekv_paged_plan_t* plan, const void* k_new,
                        const void* v_new, int64_t tok_stride, int64_t head_stride, int32_t* overflow, void* ws,
                        size_t ws_bytes, void* stream) {
  const int rc = check_plan(cache, plan, ws, ws_bytes);
  if (rc) return rc;
  if ((!k_new || !v_new) && plan->n_tokens > 0) return fail(CATEKV_ERR_INVALID_ARG, "null tensor pointer");
  const int64_t size = cache->dtype == CATEKV_BF16 ? 2 : 4;
  if (!aligned16(k_new) || !aligned16(v_new)) return fail(CATEKV_ERR_INVALID_ARG, "k_new or v_new is not on a 16-byte border");
  if (tok_stride < 0 || head_stride < 0 || tok_stride * size % 16 || head_stride * size % 16 || tok_stride > (int64_t)1 << 40 ||
      head_stride > (int64_t)1 << 40)
    return fail(CATEKV_ERR_INVALID_ARG, "strides %lld, %lld: not multiples of 16 bytes from 0 to 2^40 elements",
                (long long)tok_stride, (long long)head_stride);
  char* w = static_cast<char*>(ws);
  PagedAppend a{};
  a.c = kernel_cache(cache);
  a.seqs = reinterpret_cast<const PagedSeq*>(w + plan->seqs_off);
  a.tok_seq = reinterpret_cast<const int32_t*>(w + plan->toks_off);
  a.views = reinterpret_cast<PagedTake*>(w + plan->views_off);
  a.takes = reinterpret_cast<int32_t*>(w + plan->takes_off);
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.tok_bytes = tok_stride * size;
  a.head_bytes = head_stride * size;
  a.overflow = overflow;
  a.n_seqs = plan->n_seqs;
  a.n_tokens = plan->n_tokens;
  const hipError_t e = launch_paged_append(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "paged_append launch");
}

int catekv_paged_attn(const catekv_paged_cache* cache, const catekv_paged_plan_t* plan, const void* q, float scale,
                      void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  const int rc = check_plan(cache, plan, ws, ws_bytes);
  if (rc) return rc;
  if ((!q || !out) && plan->n_tokens > 0) return fail(CATEKV_ERR_INVALID_ARG, "null tensor pointer");
  if (!aligned16(q) || !aligned16(out)) return fail(CATEKV_ERR_INVALID_ARG, "q or out is not on a 16-byte border");
  if (!(scale > 0.f) || !std::isfinite(scale))
    return fail(CATEKV_ERR_INVALID_ARG, "scale=%g must be positive and finite", (double)scale);
  char* w = static_cast<char*>(ws);
  PagedAttn a{};
  a.c = kernel_cache(cache);
  a.q = static_cast<const char*>(q);
  a.out = static_cast<char*>(out);
  a.lse = lse;
  a.joins = reinterpret_cast<const PagedJoin*>(w + plan->joins_off);
  a.slots = reinterpret_cast<float*>(w + plan->slots_off);
  a.hq = plan->hq;
  a.scale = scale;
  // fp32 queries are scaled on their way in, bf16 scores behind their products
  a.log2_scale = 1.4426950408889634f * (cache->dtype == CATEKV_BF16 ? scale : 1.f);
  a.rise = 8.f / a.log2_scale;
  const int G = plan->hq / plan->hkv;
  const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
  hipError_t e = hipSuccess;
  a.pieces = reinterpret_cast<const PagedPiece*>(w + plan->tiles_off);
  a.workers = reinterpret_cast<const int32_t*>(w + plan->tile_workers_off);
  a.n = plan->n_tile;
  a.segs = reinterpret_cast<const PagedPiece*>(w + plan->segs_off);
  a.seg_workers = reinterpret_cast<const int32_t*>(w + plan->workers_off);
  a.n_few = plan->n_workers;
  if (a.n > 0 && a.n_few > 0 && cache->dtype == CATEKV_BF16) {
    e = launch_paged_mixed(G, a, s);
  } else {
    if (a.n > 0) e = cache->dtype == CATEKV_BF16 ? launch_paged_tile(G, a, s) : launch_paged_tile_f32(G, a, s);
    if (e == hipSuccess && a.n_few > 0) e = launch_paged_stream(cache->dtype, G, a, s);
  }
  if (e != hipSuccess) return hip_fail(e, "paged_attn launch");
  e = launch_paged_join(cache->dtype, G, a, paged_join_shape(plan->tile_joins, paged_tile_rows(cache->dtype), plan->tile_parts),
                        paged_join_shape(plan->n_joins - plan->tile_joins, kStreamRows, plan->few_parts), s);
  if (e != hipSuccess) return hip_fail(e, "paged_attn join launch");
  return host_ok();
}

int catekv_paged_fork(const catekv_paged_cache* cache, const int32_t* src_host, const int32_t* dst_host, int n,
                      int32_t* refused, void* stream) {
  return guarded([&]() -> int {
    int rc = check_cache(cache);
    if (rc) return rc;
    if (!src_host || !dst_host) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
    if (n < 1) return fail(CATEKV_ERR_INVALID_ARG, "n=%d must be >= 1", n);
    rc = check_slots(cache, src_host, n, false, "source");
    if (!rc) rc = check_slots(cache, dst_host, n, true, "destination");
    if (rc) return rc;
    std::vector<char> is_src(cache->n_slots);
    for (int i = 0; i < n; ++i) is_src[src_host[i]] = 1;
    for (int i = 0; i < n; ++i)
      if (is_src[dst_host[i]]) return fail(CATEKV_ERR_INVALID_ARG, "slot %d is a source and a destination", dst_host[i]);
    PagedFork a{};
    a.c = kernel_cache(cache);
    a.refused = refused;
    for (int i = 0; i < n; i += a.n) {             // no pair depends on another
      a.n = std::min(n - i, kPagedMaxList);
      std::copy(src_host + i, src_host + i + a.n, a.src);
      std::copy(dst_host + i, dst_host + i + a.n, a.dst);
      const hipError_t e = launch_paged_fork(a, reinterpret_cast<hipStream_t>(stream));
      if (e != hipSuccess) return hip_fail(e, "paged_fork launch");
    }
    return host_ok();
  });
}

int catekv_paged_drop(const catekv_paged_cache* cache, const int64_t* rows, void* stream) {
  const int rc = check_cache(cache);
  if (rc) return rc;
  if (!rows) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  const hipError_t e = launch_paged_drop(kernel_cache(cache), rows, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "paged_drop launch");
}

size_t catekv_paged_compact_workspace(const catekv_paged_cache* cache, int n_sel, int b, int cs, int tail) {
  return check_compact(cache, n_sel, b, cs, tail) ? 0 : compact_bytes(cache, n_sel, b, cs, tail);
}

int catekv_paged_compact(const catekv_paged_cache* cache, int slot, const int32_t* heads_host, int n_sel,
                         const int32_t* idx, int b, int cs, int tail, int32_t* overflow, void* ws, size_t ws_bytes,
                         void* stream) {
  int rc = check_compact(cache, n_sel, b, cs, tail);
  if (rc) return rc;
  if (!heads_host || !idx) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  rc = check_slots(cache, &slot, 1, false, "the");
  if (rc) return rc;
  PagedCompact a{};
  for (int s = 0; s < n_sel; ++s) {
    if (heads_host[s] < 0 || heads_host[s] >= cache->hkv)
      return fail(CATEKV_ERR_INVALID_ARG, "head %d outside [0, %d)", heads_host[s], cache->hkv);
    for (int t = 0; t < s; ++t)
      if (heads_host[t] == heads_host[s]) return fail(CATEKV_ERR_INVALID_ARG, "head %d listed twice", heads_host[s]);
    a.heads[s] = heads_host[s];
  }
  rc = host_check_ws(ws, ws_bytes, compact_bytes(cache, n_sel, b, cs, tail));
  if (rc) return rc;
  char* w = static_cast<char*>(ws);
  a.c = kernel_cache(cache);
  a.idx = idx;
  a.offs = reinterpret_cast<int32_t*>(w);
  w += a256((size_t)n_sel * b * sizeof(int32_t));
  a.views = reinterpret_cast<PagedTake*>(w);
  w += a256((size_t)n_sel * sizeof(PagedTake));
  a.takes = reinterpret_cast<int32_t*>(w);
  a.overflow = overflow;
  a.slot = slot;
  a.n_sel = n_sel;
  a.b = b;
  a.cs = cs;
  a.tail = tail;
  const hipError_t e = launch_paged_compact(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "paged_compact launch");
}

int catekv_paged_gather(const catekv_paged_cache* cache, const int32_t* slots_host, int n,
                        const catekv_kv_ptrs* kv_out, int64_t max_rows, void* stream) {
  int rc = check_cache(cache);
  if (rc) return rc;
  if (!slots_host || !kv_out) return fail(CATEKV_ERR_INVALID_ARG, "null pointer");
  if (n < 1 || n > kPagedMaxList) return fail(CATEKV_ERR_INVALID_ARG, "n=%d outside [1, %d]", n, kPagedMaxList);
  if (max_rows < 1) return fail(CATEKV_ERR_INVALID_ARG, "max_rows=%lld must be >= 1", (long long)max_rows);
  rc = check_slots(cache, slots_host, n, false, "the");
  if (rc) return rc;
  PagedGather a{};
  a.c = kernel_cache(cache);
  a.out = kv_out;
  a.max_rows = std::min<int64_t>(max_rows, (int64_t)cache->max_pages * cache->page);   // no view has more
  if (!launch_fits(paged_gather_groups(a.max_rows, a.c.row_bytes) * n * cache->hkv, kGatherThreads))
    return fail(CATEKV_ERR_UNSUPPORTED, "n=%d of max_rows=%lld: too many rows for one launch", n, (long long)max_rows);
  a.n = n;
  std::copy(slots_host, slots_host + n, a.slots);
  const hipError_t e = launch_paged_gather(a, reinterpret_cast<hipStream_t>(stream));
  return e == hipSuccess ? host_ok() : hip_fail(e, "paged_gather launch");
}

}  // extern "C"
