// Which memory the rows of a tensor of heads take, and whether those of two tensors meet (host code of api.hip).
#pragma once

#include <stdint.h>

namespace adakv {

// `count` steps `by` bytes apart, twice over, and `bytes` bytes at each: rows of heads, or (counts of 1) one piece.
struct Places {
  struct Steps { long long count, by; };
  uintptr_t at;
  long long bytes;
  Steps steps[2];

  Places(uintptr_t x, long long piece) : at(x), bytes(piece), steps{{1, 0}, {1, 0}} {}
  Places(uintptr_t x, long long piece, Steps outer, Steps inner) : at(x), bytes(piece), steps{outer, inner} {
    for (int turn = 0; turn < 2; ++turn)       // pieces one behind the other are one piece
      for (Steps &s : steps) {
        if (s.count == 1 || s.by != bytes) continue;
        bytes *= s.count;
        s = {1, 0};
      }
  }
  bool none() const { return bytes == 0 || steps[0].count < 1 || steps[1].count < 1; }
};

__extension__ typedef __int128 wide;           // counts up to 2^40 of steps up to 2^43 bytes apart

// Sum of floor((a i + b) / m) over i < n, for a, b >= 0 and m > 0.  Beyond the whole parts of a / m and b / m it counts the pairs (i, j), j >= 1, with
// j m <= a i + b, and the other way round, for every j <= k = floor((a (n - 1) + b) / m), the i that are too small: n k less the sum
// of ceil((j m - b) / a), a problem of the same kind with a and m in each other's place.
inline wide floors(wide n, wide m, wide a, wide b) {
  if (n <= 0) return 0;
  const wide whole = n * (n - 1) / 2 * (a / m) + n * (b / m);
  a %= m;
  b %= m;
  const wide k = (a * (n - 1) + b) / m;
  return whole + (k ? n * k - floors(k, a, m, m - b + a - 1) : 0);
}
// Pairs (x, y), x < X, y < Y, with b y <= a x + c.
inline wide pairs_up_to(wide c, wide a, wide X, wide b, wide Y) {
  const auto first = [&](wide v) {             // the first x with a x + c >= v
    const wide x = v <= c ? 0 : (v - c + a - 1) / a;
    return x < X ? x : X;
  };
  const wide some = first(0), all = first((Y - 1) * b), here = a * some + c;
  return (X - all) * Y + (all > some ? all - some + floors(all - some, b, a, here) : 0);
}
// Whether lo <= c + a x - b y <= hi for some x < X, y < Y.
inline bool any_between(wide lo, wide hi, wide c, wide a, wide X, wide b, wide Y) {
  if (c + a * (X - 1) < lo || c - b * (Y - 1) > hi) return false;
  if (X == 1 && Y == 1) return true;
  if (X == 1) a = b;
  if (Y == 1) b = a;
  if (a == b) {                                // x - y is any number from 1 - Y to X - 1: the least that is not too small
    wide k = lo - c > 0 ? (lo - c + a - 1) / a : -((c - lo) / a);
    if (k < 1 - Y) k = 1 - Y;
    return k < X && c + a * k <= hi;
  }
  return pairs_up_to(c - lo, a, X, b, Y) > pairs_up_to(c - hi - 1, a, X, b, Y);
}

enum class Meet { NO, YES, UNKNOWN };          // (UNKNOWN: it would take too long)
inline Meet meet_places(const Places &p, const Places &o) {
  if (p.none() || o.none()) return Meet::NO;
  const auto end = [](const Places &x) {
    return (wide)x.at + (wide)(x.steps[0].count - 1) * x.steps[0].by + (wide)(x.steps[1].count - 1) * x.steps[1].by + x.bytes;
  };
  if (end(p) <= (wide)o.at || end(o) <= (wide)p.at) return Meet::NO;
  // One of either tensor's steps goes by arithmetic, the others one after the other: those of which there are the fewest, and if they
  // are alike it is their difference that counts.
  const auto turns = [&](int i, int j) {
    const Places::Steps &s = p.steps[i], &t = o.steps[j];
    return s.by == t.by || s.count == 1 || t.count == 1 ? (wide)s.count + t.count - 1 : (wide)s.count * t.count;
  };
  int i = 0, j = 0;
  for (int x = 0; x < 4; ++x)
    if (turns(x / 2, x % 2) < turns(i, j)) i = x / 2, j = x % 2;
  if (turns(i, j) > 1 << 20) return Meet::UNKNOWN;
  const Places::Steps &s = p.steps[i], &t = o.steps[j], &u = p.steps[1 - i], &v = o.steps[1 - j];
  const wide apart = (wide)p.at - (wide)o.at;  // two pieces meet where they begin less than the second's bytes later or the first's earlier
  const auto look = [&](wide more) { return any_between(1 - p.bytes, o.bytes - 1, apart + more, u.by, u.count, v.by, v.count); };
  if (s.by == t.by || s.count == 1 || t.count == 1) {
    const wide by = s.count > 1 ? s.by : t.by;
    for (long long k = 1 - t.count; k < s.count; ++k)
      if (look(by * k)) return Meet::YES;
    return Meet::NO;
  }
  for (long long x = 0; x < s.count; ++x)
    for (long long y = 0; y < t.count; ++y)
      if (look((wide)s.by * x - (wide)t.by * y)) return Meet::YES;
  return Meet::NO;
}

}  // namespace adakv
