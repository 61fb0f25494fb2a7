// Host half of dlfp_cache.h: the checks of the rotating appends, and the metadata
// and work list of attention with a window.  Plain C++ (no HIP calls), so it also
// builds with a host compiler and its sanitizers.
#include <algorithm>
#include <cstdint>
#include <cstring>
#include <limits>
#include <new>
#include <vector>

#include "dlfp_cache.h"
#include "dlfp_internal.h"

namespace {

constexpr int64_t PAGE = DLFP_PAGE_SIZE;
constexpr int64_t I32_MAX = std::numeric_limits<int32_t>::max();

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round_up(int64_t a, int64_t b) { return ceil_div(a, b) * b; }
// Floats of one partial result: O (rows x 128), m[rows], l[rows], padded to 256 bytes.
int64_t slot_floats(int64_t rows) { return round_up(rows * (DLFP_HEAD_DIM + 2), 64); }

struct Unit {
  int32_t f[DLFP_WORK_INTS];
};
static_assert(sizeof(Unit) == DLFP_WORK_INTS * sizeof(int32_t), "work records are packed");

// The rows of a unit before its keys are split, and the keys that it reads.
struct Rows {
  int32_t seq, t0, nt;
  int64_t gap;   // pages left out
  int64_t keys;  // keys read, the gap left out
};

bool aligned16(const void* p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool good_stride(int64_t ld, int64_t heads) {
  return ld % 8 == 0 && ld >= heads * DLFP_HEAD_DIM;
}

}  // namespace

namespace dlfp {

int check_rope_append(const dlfp_dims* dims, const dlfp_rope* rope, int32_t num_tokens,
                      const int32_t* positions, const int32_t* slot_mapping, const void* q,
                      int64_t ldq, const void* k_new, int64_t ldk, const void* v_new, int64_t ldv,
                      const void* q_out, int64_t ldo, const void* k_cache, const void* v_cache,
                      int32_t num_blocks) {
  const int st = check_dims(dims, nullptr);
  if (st != DLFP_OK) return st;
  if (!rope || num_tokens < 0 || num_blocks < 0) return DLFP_EINVAL;
  if (rope->rotary_dim != 32 && rope->rotary_dim != 64 && rope->rotary_dim != 128)
    return DLFP_EUNSUPPORTED;
  if (rope->interleaved != 0 && rope->interleaved != 1) return DLFP_EINVAL;
  const int64_t hq = dims->num_q_heads, hkv = dims->num_kv_heads;
  // A launch has fewer than 2^32 threads: workgroups of 256 for 16 tokens (4 of up to 512)
  // of a KV head and for 4 tokens' group of 16 query heads, the most of either append.
  const int64_t chunks = ceil_div(hq, 16);
  if (num_tokens * (hkv + chunks) > I32_MAX / 4 ||
      ceil_div(num_tokens, num_tokens <= 512 ? 4 : 16) * hkv + ceil_div(num_tokens * chunks, 4) >=
          1 << 24)
    return DLFP_ERANGE;
  if (!good_stride(ldq, hq) || !good_stride(ldo, hq) || !good_stride(ldk, hkv) ||
      !good_stride(ldv, hkv))
    return DLFP_EINVAL;
  if (num_tokens == 0) return DLFP_OK;
  if (!rope->table || rope->positions <= 0) return DLFP_EINVAL;
  if (!positions || !slot_mapping || !q || !k_new || !v_new || !q_out || !k_cache || !v_cache)
    return DLFP_EINVAL;
  if (!aligned16(rope->table) || !aligned16(q) || !aligned16(k_new) || !aligned16(v_new) ||
      !aligned16(q_out) || !aligned16(k_cache) || !aligned16(v_cache))
    return DLFP_EINVAL;
  return DLFP_OK;
}

}  // namespace dlfp

namespace {

int build(const dlfp_dims* dims, const dlfp_tuning* tuning, const dlfp_window* win,
          int32_t num_seqs, const int32_t* q_len, const int32_t* kv_len,
          const int32_t* block_table, int32_t max_blocks, int32_t num_blocks, dlfp_meta* meta) {
  int g = 0;
  const int st = dlfp::check_dims(dims, &g);
  if (st != DLFP_OK) return st;
  if (!meta || num_seqs < 0 || num_blocks < 0) return DLFP_EINVAL;
  if (num_seqs > 0 && (!q_len || !kv_len || !block_table || max_blocks <= 0)) return DLFP_EINVAL;
  if (win && (win->window < 1 || win->sinks < 0)) return DLFP_EINVAL;
  dlfp_tuning tn = {0, 0, 0, 0, 0, 0};
  if (tuning) tn = *tuning;
  if (tn.prefill_lead_units < -1) return DLFP_EINVAL;
  if (tn.decode_pages_in_flight < 0 || tn.decode_pages_in_flight > 2) return DLFP_EINVAL;
  if (tn.decode_split_tokens < 0 || tn.decode_split_tokens % PAGE ||
      tn.decode_split_tokens > DLFP_MAX_DECODE_UNIT_KEYS)
    return DLFP_EINVAL;
  if (tn.prefill_split_tokens < 0 || tn.prefill_split_tokens % 64 ||
      tn.prefill_split_tokens > DLFP_MAX_PREFILL_UNIT_KEYS)
    return DLFP_EINVAL;
  if (tn.target_units < 0) return DLFP_EINVAL;
  if (tn.prefill_tile_tokens < 0 || tn.prefill_tile_tokens > DLFP_TILE_ROWS / g)
    return DLFP_EINVAL;
  if ((int64_t)num_blocks * PAGE > I32_MAX && num_seqs > 0) return DLFP_ERANGE;
  const int64_t resident = tn.target_units ? tn.target_units : DLFP_DEFAULT_RESIDENT_WAVES;
  const int64_t slots = std::max<int64_t>(1, resident / 4);  // workgroups resident together
  const int64_t cus = std::max<int64_t>(1, resident / 8);
  const int64_t hkv = dims->num_kv_heads;
  const int64_t window = win ? win->window : I32_MAX;
  const int64_t sinks = win ? win->sinks : 0;

  // Pages of a range of rows at positions first .. last: all from page 0, or the
  // sink pages and, past a gap, those from the first row's window on.
  auto rows_of = [&](int32_t s, int64_t t0, int64_t nt) {
    const int64_t first = (int64_t)kv_len[s] - q_len[s] + t0, last = first + nt - 1;
    const int64_t low = std::max<int64_t>(0, first - window + 1) / PAGE;
    const int64_t sunk = ceil_div(std::min(sinks, last + 1), PAGE);
    const int64_t gap = std::max<int64_t>(0, low - sunk);
    return Rows{s, (int32_t)t0, (int32_t)nt, gap, last + 1 - PAGE * gap};
  };

  // Validate the sequences and the pages they use.
  int64_t tokens = 0;
  std::vector<int32_t> prompts, decoders;
  for (int s = 0; s < num_seqs; ++s) {
    const int32_t ql = q_len[s], kl = kv_len[s];
    if (ql < 1 || kl < ql) return DLFP_EINVAL;
    const int64_t pages = ceil_div(kl, PAGE);
    if (pages > max_blocks) return DLFP_ERANGE;
    const int32_t* row = block_table + (int64_t)s * max_blocks;
    const Rows r = rows_of(s, 0, ql);
    if (r.keys > I32_MAX - 64) return DLFP_ERANGE;  // kernels look 64 keys past a unit's end
    // Pages before and past the gap of the sequence's first row.
    const int64_t sunk = r.gap ? ceil_div(sinks, PAGE) : 0;
    int32_t lo = std::numeric_limits<int32_t>::max(), hi = std::numeric_limits<int32_t>::min();
    for (int64_t p = 0; p < sunk; ++p) lo = std::min(lo, row[p]), hi = std::max(hi, row[p]);
    for (int64_t p = sunk + r.gap; p < pages; ++p)
      lo = std::min(lo, row[p]), hi = std::max(hi, row[p]);
    if (lo < 0 || hi >= num_blocks) return DLFP_ERANGE;
    tokens += ql;
    (ql == 1 ? decoders : prompts).push_back(s);
  }
  if (tokens > I32_MAX) return DLFP_ERANGE;

  std::vector<Rows> tiles, ones;
  int64_t one_keys = 0, one_longest = 0;
  for (int32_t s : decoders) {
    ones.push_back(rows_of(s, 0, 1));
    one_keys += ones.back().keys;
    one_longest = std::max(one_longest, ones.back().keys);
  }
  // A range longer than the split is cut into equal parts.
  auto cut = [](int64_t keys, int64_t split, int64_t granule) {
    const int64_t n = ceil_div(keys, split);
    return round_up(ceil_div(keys, n), granule);
  };
  // Units of ranges cut at `split`: their count, keys of all, of the longest and of
  // the range with the shortest, parts of the longest range.
  struct Cut {
    int64_t units, keys, longest, shortest, parts;
  };
  auto cuts = [&](const std::vector<Rows>& ranges, int64_t split) {
    Cut c = {0, 0, 0, I32_MAX, 1};
    for (const Rows& r : ranges) {
      const int64_t part = cut(r.keys, split, 64), n = ceil_div(r.keys, part);
      c.units += n * hkv;
      c.keys += r.keys * hkv;
      c.longest = std::max(c.longest, std::min(part, r.keys));
      c.shortest = std::min(c.shortest, std::min(part, r.keys));
      c.parts = std::max(c.parts, n);
    }
    return c;
  };
  auto split_tiles = [&](int64_t tokens_each) {
    std::vector<Rows> t;
    for (int32_t s : prompts)
      for (int64_t t0 = 0; t0 < q_len[s]; t0 += tokens_each)
        t.push_back(rows_of(s, t0, std::min<int64_t>(tokens_each, q_len[s] - t0)));
    return t;
  };

  // Decode split: an n-th of the longest range, the n that minimises an estimate of
  // the decode share's time in us: full rounds of units and the rest of the last one
  // stream at 6.2 TB/s (256 bytes a key, those of 8-bit pages), no unit faster
  // than 6.3 ns a key (10.8 where some compute units have two); a full round
  // takes 3.5 us more, a merge 3 and 0.1 for each part.
  int64_t split_d = tn.decode_split_tokens;
  if (!split_d && !ones.empty()) {
    // Beside a prefill share for every compute unit: one slot of each, and a round
    // costs more (whole 8-bit contexts beside 1999 tokens, 4096-key units 403 us,
    // of 2752 keys 445).
    const bool beside = (int64_t)split_tiles(std::max(1, DLFP_TILE_ROWS / g)).size() * hkv >= cus;
    const int64_t room = beside ? std::max<int64_t>(1, slots - cus) : slots;
    const double round = beside ? 8. : 3.5;
    double best = 0.;
    // (A range that takes more than 256 units at the longest unit is cut into those.)
    const int64_t fewest = ceil_div(one_longest, DLFP_MAX_DECODE_UNIT_KEYS);
    for (int64_t n = fewest; n <= std::max<int64_t>(fewest, 256); ++n) {
      const int64_t split = std::max<int64_t>(round_up(ceil_div(one_longest, n), 64), 128);
      const Cut c = cuts(ones, split);
      const double keys_us = 6.2e6 / 256, mean = (double)c.keys / c.units;
      const int64_t full = c.units / room, rest = c.units % room;
      // The longest units come first, so a last round after full ones has the short
      // ones.
      const double least = full ? c.shortest * 6.3e-3
                                : c.longest * (rest > cus ? 10.8e-3 : 6.3e-3);
      const double stream = full * room * mean / keys_us + round * full +
                            (rest ? std::max(least, rest * mean / keys_us) : 0.);
      const double est = std::max(stream, c.longest * (c.units > cus ? 10.8e-3 : 6.3e-3)) +
                         (c.parts > 1 ? 3. + 0.1 * c.parts : 0.);
      if (!split_d || est < best) {
        best = est;
        split_d = split;
      }
      if (split == 128) break;
    }
  }

  // Prefill tiles and split: tiles of 128 rows, or of 32 whose units split their
  // keys over the wavefronts, and a number of equal parts, by an estimate of the
  // prefill share's time in us.  A unit of 128 rows takes 22.7 ns a key with a
  // compute unit to itself and 30.5 beside another one, one of 32 rows 9.2 and 13.5;
  // its start and end 4.5 and 8, 5 and 6; a further round 6 and 4, with partial
  // results 7 and 2 more; a merge 5 and 3, and 0.9 and 0.4 for each part, twice that
  // where a decode share leaves few slots.  The units of a decode share have a slot
  // each, up to one on every compute unit, for 6 us and 16 ns a key, and prefill units
  // that find none left wait so long.  (Tiles of 128 and of 32 rows, 8 KV heads, bf16
  // pages: 64 tokens of 16 heads over 264 keys 12.2 and 8.7 us, 1024 over 2024 33.6 and
  // 27.3, 2048 over 4048 68 and 86; of 64 heads, 256 over 1256 25.7 and 21.3, 1024 over
  // 2024 64 and 93.  Whole and in two parts: 2 x 1365 tokens of 32 heads over windows
  // of 1870 keys 115 and 144.)
  int64_t split_p = tn.prefill_split_tokens, tile_tokens = tn.prefill_tile_tokens;
  if (!prompts.empty()) {
    struct Height {
      int64_t rows;
      double alone, beside, start, start2, round, merge, part, partial;
    };
    constexpr Height heights[] = {{DLFP_TILE_ROWS, 22.7e-3, 30.5e-3, 4.5, 8., 6., 5., 0.9, 7.},
                                  {DLFP_SMALL_ROWS, 9.2e-3, 13.5e-3, 5., 6., 4., 3., 0.4, 2.}};
    const int64_t fixed_tile = tile_tokens, fixed_split = split_p;
    const Cut d = cuts(ones, split_d);
    const int64_t taken = std::min(d.units, cus);
    const double held = taken ? 6. * ceil_div(d.units, cus) + 16e-3 * d.keys / taken : 0.;
    double best = 0.;
    bool found = false;
    for (const Height& h : heights) {
      const int64_t each = fixed_tile ? fixed_tile : std::max<int64_t>(1, h.rows / g);
      if (fixed_tile && (each * g <= DLFP_SMALL_ROWS) != (h.rows == DLFP_SMALL_ROWS)) continue;
      std::vector<Rows> t = split_tiles(each);
      int64_t whole = 0;
      for (const Rows& r : t) whole = std::max(whole, r.keys);
      const int64_t most = each * g <= DLFP_SMALL_ROWS ? DLFP_MAX_DECODE_UNIT_KEYS
                                                       : DLFP_MAX_PREFILL_UNIT_KEYS;
      bool better = false;
      for (int64_t n = ceil_div(whole, most); n <= ceil_div(whole, most) + 15; ++n) {
        const int64_t split = fixed_split ? fixed_split
                                          : std::max<int64_t>(round_up(ceil_div(whole, n), 64), 256);
        const Cut c = cuts(t, split);
        const double mean = (double)c.keys / c.units;
        const int64_t full = (c.units - 1) / slots, rest = c.units - full * slots;
        const bool two = taken + c.units > cus;
        const double crowd = taken > 0 && taken + c.units > slots * 3 / 4 ? 2. : 1.;
        // Keys of the busiest slot: longest units first, the shortest fill the end.
        const double keys = full ? (double)c.keys / slots + c.shortest * (1. - (double)rest / slots)
                                 : two ? 0.5 * (mean + c.longest) : (double)c.longest;
        const double est = (two ? h.start2 : h.start) + h.round * full +
                           keys * (two ? h.beside : h.alone) +
                           (taken + c.units > slots ? held : 0.) +
                           (c.parts > 1 ? crowd * (h.merge + h.part * c.parts) + h.partial * full : 0.);
        if (!found || est < best) {
          best = est;
          split_p = split;
          found = better = true;
        }
        if (fixed_split || split == 256) break;
      }
      if (better) tiles = std::move(t);
    }
  }
  int64_t tile_keys = 0;
  for (const Rows& r : tiles) tile_keys += r.keys;
  auto longest_first = [](const Rows& x, const Rows& y) { return x.keys > y.keys; };
  std::stable_sort(tiles.begin(), tiles.end(), longest_first);
  std::stable_sort(ones.begin(), ones.end(), longest_first);

  std::vector<Unit> units;
  int64_t groups = 0, off = DLFP_WORKSPACE_PARTIALS / 4;
  int64_t group_bytes = 0;  // of the largest group's partial results
  auto emit = [&](const Rows& r, int64_t kh, int64_t split, int64_t granule, int32_t kind) {
    // Units of few rows keep their block ids where decode units do.
    if ((int64_t)r.nt * g <= DLFP_SMALL_ROWS)
      split = std::min<int64_t>(split, DLFP_MAX_DECODE_UNIT_KEYS);
    const int64_t part = cut(r.keys, split, granule);
    const int64_t parts = ceil_div(r.keys, part);
    const int64_t floats = slot_floats((int64_t)r.nt * g);
    for (int64_t j = 0; j < parts; ++j) {
      Unit u;
      std::memset(&u, 0, sizeof(u));
      u.f[DLFP_W_SEQ] = r.seq;
      u.f[DLFP_W_KVHEAD] = (int32_t)kh;
      u.f[DLFP_W_QTOK0] = r.t0;
      u.f[DLFP_W_QNTOK] = r.nt;
      u.f[DLFP_W_KVBEGIN] = (int32_t)(j * part);
      u.f[DLFP_W_KVEND] = (int32_t)std::min(r.keys, (j + 1) * part);
      u.f[DLFP_W_GROUP] = parts > 1 ? (int32_t)groups : -1;
      u.f[DLFP_W_SPLIT] = (int32_t)j;
      u.f[DLFP_W_NSPLITS] = (int32_t)parts;
      u.f[DLFP_W_WINDOW] = (int32_t)window;
      u.f[DLFP_W_WSGROUP] = parts > 1 ? (int32_t)std::min(off, I32_MAX) : 0;
      u.f[DLFP_W_KIND] = kind;
      u.f[DLFP_W_QROW0] = r.t0;  // the sequence's first row is added below
      u.f[DLFP_W_QPOS0] = kv_len[r.seq] - q_len[r.seq] + r.t0;
      u.f[DLFP_W_SINKS] = (int32_t)std::min<int64_t>(sinks, I32_MAX - PAGE);
      u.f[DLFP_W_GAP] = (int32_t)r.gap;
      units.push_back(u);
    }
    if (parts > 1) {
      ++groups;
      off += parts * floats;
      group_bytes = std::max(group_bytes, 4 * parts * floats);
    }
  };
  // Prefill units of one KV head together: the launch gives each XCD a contiguous
  // range of them, so that units reading the same keys share an L2.
  for (int64_t kh = 0; kh < hkv; ++kh)
    for (const Rows& r : tiles) emit(r, kh, split_p, 64, DLFP_KIND_PREFILL);
  const int64_t num_prefill = (int64_t)units.size();
  for (const Rows& r : ones)
    for (int64_t kh = 0; kh < hkv; ++kh) emit(r, kh, split_d, 64, DLFP_KIND_DECODE);
  std::stable_sort(units.begin() + num_prefill, units.end(), [](const Unit& x, const Unit& y) {
    return x.f[DLFP_W_KVEND] - x.f[DLFP_W_KVBEGIN] > y.f[DLFP_W_KVEND] - y.f[DLFP_W_KVBEGIN];
  });
  const int64_t n_units = (int64_t)units.size();
  auto longest = [](auto first, auto last) {
    int32_t n = 0;
    for (; first != last; ++first) n = std::max(n, first->f[DLFP_W_KVEND] - first->f[DLFP_W_KVBEGIN]);
    return n;
  };
  // (A launch addresses the partial results of a group in 31 bits.)
  if (n_units > I32_MAX / DLFP_WORK_INTS || groups > DLFP_MAX_GROUPS || off > I32_MAX ||
      group_bytes > I32_MAX)
    return DLFP_ERANGE;

  meta->num_seqs = num_seqs;
  meta->num_tokens = (int32_t)tokens;
  meta->num_units = (int32_t)n_units;
  meta->num_prefill_units = (int32_t)num_prefill;
  meta->num_groups = (int32_t)groups;
  meta->decode_split_tokens = longest(units.begin() + num_prefill, units.end());
  meta->prefill_split_tokens = longest(units.begin(), units.begin() + num_prefill);
  meta->workspace_bytes = 4 * off;
  meta->num_append = 0;
  meta->num_waiting_units =
      num_prefill ? (int32_t)std::min<int64_t>(1024 * one_keys / std::max<int64_t>(tile_keys, 1), I32_MAX) : 0;
  // With more prefill units than compute units, one for each of those leads and
  // the decode units follow, so that the two shares run side by side.
  int64_t lead = num_prefill;
  if (tn.prefill_lead_units > 0)
    lead = std::min<int64_t>(tn.prefill_lead_units, num_prefill);
  else if (tn.prefill_lead_units == 0 && n_units > num_prefill && num_prefill > cus)
    lead = cus;
  meta->prefill_lead_units = (int32_t)lead;
  meta->decode_pages_in_flight = DLFP_WINDOW_META;
  if (meta->cap_seqs < num_seqs || meta->cap_tokens < tokens || meta->cap_work < n_units)
    return DLFP_ENOSPC;
  if ((num_seqs > 0 && (!meta->cu_q || !meta->q_pos0)) || (tokens > 0 && !meta->slot_mapping) ||
      (n_units > 0 && !meta->work))
    return DLFP_EINVAL;
  if (meta->cu_q) meta->cu_q[0] = 0;
  int64_t t = 0;
  for (int s = 0; s < num_seqs; ++s) {
    const int32_t pos0 = kv_len[s] - q_len[s];
    meta->q_pos0[s] = pos0;
    const int32_t* row = block_table + (int64_t)s * max_blocks;
    for (int32_t i = 0; i < q_len[s]; ++i) {
      const int32_t p = pos0 + i;
      meta->slot_mapping[t++] = row[p / PAGE] * (int32_t)PAGE + p % (int32_t)PAGE;
    }
    meta->cu_q[s + 1] = (int32_t)t;
  }
  for (Unit& u : units) u.f[DLFP_W_QROW0] += meta->cu_q[u.f[DLFP_W_SEQ]];
  if (!units.empty()) std::memcpy(meta->work, units.data(), units.size() * sizeof(Unit));
  return DLFP_OK;
}

}  // namespace

extern "C" int dlfp_build_window_meta(const dlfp_dims* dims, const dlfp_tuning* tuning,
                                      const dlfp_window* window, int32_t num_seqs,
                                      const int32_t* q_len, const int32_t* kv_len,
                                      const int32_t* block_table, int32_t max_blocks,
                                      int32_t num_blocks, dlfp_meta* meta) {
  try {
    return build(dims, tuning, window, num_seqs, q_len, kv_len, block_table, max_blocks, num_blocks,
                 meta);
  } catch (const std::bad_alloc&) {
    return DLFP_ENOSPC;
  }
}
