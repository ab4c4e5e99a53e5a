// Which waves of the 8-bit fill take which blocks of the sequences (plain C++,
// host and device).
#pragma once
#include <stdint.h>

namespace lat {

constexpr int CACHE8_BLOCK = 16;                   // slots that share a scale

// A sequence's items are its blocks of 16 slots, each `sides` times.  They are taken by
// per_seq waves of a group that goes through the sequences, or, where it has `large` rows
// or more, by those waves behind the groups (from wave `behind` on) whose row it holds:
// `sides` waves for each packed row that is a multiple of `tile`.
struct Fill8Plan { int per_seq, groups, behind, tile, sides, large, waves; };

// per_seq is a wave an item where a sequence has the batch's mean length.  A sequence of
// more than FILL8_DEEP times that many blocks would be many rounds of a few waves: it goes
// behind, where a wave has at most 7 items whatever the mean (a tile is four blocks).
// Where no sequence can have so many (a ring that is not that much longer than the mean, or
// a bound of the lengths that says so) there are no waves behind.
// bf16, heads of 64, 2 key heads, one long history among shorter ones, rings that hold it,
// us with the groups alone / here / with tiles of 32 / of 128: 32000 among 3000 of 20 (4100
// slots) 195 / 17 / 19 / 18; 2000 among 1000 of 30 63 / 15 / 12 / 21; 8000 among 1000 of 500
// 77 / 83 / 92 / 89; 100000 among 100 of 1000 90 / 35 / 35 / 41; 60000 among 100 of 4000
// 77 / 78 / 83 / 83.  FILL8_DEEP of 4 or 16: the same within 2%.
constexpr int FILL8_TILE = 64, FILL8_DEEP = 8;
constexpr int64_t FILL8_WAVES = (int64_t)1 << 22;  // of either kind, at most

inline Fill8Plan fill8_plan(int64_t rows, int num_seqs, int64_t max_len, int64_t cap, int sides) {
  Fill8Plan p;
  const int64_t mean = (rows + num_seqs - 1) / num_seqs;
  const int64_t per_seq = ((mean < cap ? mean : cap) / CACHE8_BLOCK + 1) * sides;
  p.per_seq = (int)(per_seq < 4096 ? per_seq : 4096);
  int64_t n = (int64_t)p.per_seq * num_seqs;
  if (n > FILL8_WAVES) n = FILL8_WAVES;
  p.groups = (int)(n / p.per_seq);
  p.behind = p.waves = (int)((n + 3) & ~(int64_t)3);
  p.sides = sides;
  p.tile = FILL8_TILE;
  if (rows * sides > FILL8_WAVES * p.tile) p.tile = (int)((rows * sides + FILL8_WAVES - 1) / FILL8_WAVES);
  int64_t large = (int64_t)FILL8_DEEP * (p.per_seq / sides) * CACHE8_BLOCK;
  if (large < 2 * (int64_t)p.tile) large = 2 * (int64_t)p.tile;
  const int64_t longest = max_len > 0 && max_len < rows ? max_len : rows;
  p.large = 0x7fffffff;
  if (large <= longest && large <= cap) {
    p.large = (int)large;
    p.waves += (int)((rows + p.tile - 1) / p.tile) * sides;
  }
  return p;
}

// What a wave takes: of sequences s, s + ds, .. (those that are large, or those that are
// not) the items it0, it0 + dit, ..
struct Fill8Share { int64_t s, ds, it0, dit; bool behind; };

// off(i): offsets[i].  False: nothing.
template <typename Off>
__host__ __device__ inline bool fill8_share(const Fill8Plan& p, int wave, int rows, int num_seqs, Off off, Fill8Share* w) {
  w->behind = wave >= p.behind;
  w->s = wave / p.per_seq;
  w->ds = p.groups;
  w->it0 = wave % p.per_seq;
  w->dit = p.per_seq;
  if (!w->behind) return w->s < p.groups;            // (a rest that makes no whole group)
  const int64_t row = (int64_t)((wave - p.behind) / p.sides) * p.tile;
  if (row >= rows) return false;
  int lo = 0, hi = num_seqs - 1;                     // the last sequence that starts at or before the row
  while (lo < hi) {
    const int m = lo + (hi - lo + 1) / 2;
    if (off(m) <= row) lo = m; else hi = m - 1;
  }
  const int64_t a = off(lo), b = off(lo + 1), e = b < rows ? b : rows;
  if (a < 0 || row < a || row >= e) return false;
  const int64_t t0 = (a + p.tile - 1) / p.tile;      // the sequence's first such row
  w->it0 = (row / p.tile - t0) * p.sides + (wave - p.behind) % p.sides;
  w->dit = ((e - 1) / p.tile - t0 + 1) * p.sides;
  w->s = lo;
  w->ds = num_seqs;
  return true;
}

}  // namespace lat
