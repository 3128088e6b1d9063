// Attention of a block's rows over the paged cache (lsv_attend_paged).
//
// The query vectors of a kv head are the block's rows times the head's group of query heads: vector
// v of a sequence is row v / group, head kvh * group + v % group.  Tiles of them share the keys and
// values that they read.  Scores are formed transposed, S^T = K Q^T, so that a lane holds the keys of one
// query: the softmax statistics are one lane's (and its partners') and the probabilities are, in
// the registers they were formed in, the operand of O^T = V^T P^T, since a page keeps V transposed with
// its keys in that order (LSV_V_COLUMN).
//
//  * stream kernel: few query vectors per sequence (tiles of 16 or 32), where reading K and V is the
//    work; and every fp32 call.  Equal shares of one line of all the call's pages go to workgroups of two
//    waves, each with a page (fp32: half of one) of its own in LDS.
//  * tile kernel (bf16): 128 query vectors, 32 a wave, over pages that the workgroup shares in
//    LDS, the next page's direct loads in flight.
//  * merge kernels: join the sums of tiles whose pages were cut over workgroups.
//
// Pages go to LDS by direct loads, whole lines of 16 bytes a lane: fragments of 64 bytes loaded straight into
// operands reach 4.4 to 5.1 TB/s, these 6.2 (64 ragged sequences, 1.08 GB: 246 -> 183 us by this alone, 170 with what
// followed).
#include <math.h>

#include "lsv_attn.h"
#include "lsv_ops.h"

namespace lsv {

typedef float f32x16_t __attribute__((ext_vector_type(16)));

constexpr int kPage = LSV_KV_PAGE;
constexpr int kStreamWaves = 2;  // waves of a stream kernel's workgroup
constexpr float kLog2e = 1.4426950408889634f;

// How the tile kernel's units -- (sequence, tile, split of its pages, kv head) -- are cut.  Either a sequence's
// tiles are split by its length, `pps` pages a split (whole = all); or, with pps no limit, the first
// `whole` tiles of the call stay whole and the rest, which would fill a last round of workgroups badly, are cut
// into `rest` parts each.
struct TileCut {
  int pps, whole, rest;
  LSV_DEV bool none() const { return pps == kNoLimit && rest == 1; }
  static constexpr int kNoLimit = 1 << 28;
};
// How a call is cut.  Kernels take their sequences' real lengths; the host has the bounds.
struct AttendPlan {
  int group;    // query heads per kv head
  int tile;     // query vectors per tile
  int target;   // workgroups that fill the chip; shares of the stream kernel's line
  int least;    // pages of a share at least
  int slots;    // partial results that the workspace holds
  float* o;     // [slots][tile][hd] sums of p v
  float* ml;    // [slots][tile][2] maximum (log2 units), sum of p
  // cap * tanh(x), x = s * cap_ratio, is in log2 units s * poly(x^2) up to |s| = cap_limit, half of the cap: tanh(x) / x
  // in x^2 to 5.5e-7, fitted over [0, 1/4], times the scale.  The powers of the ratio are folded into the coefficients,
  // poly then takes s^2 (poly_ratio 1), but where they would leave fp32's range (poly_ratio is the ratio).  A page whose
  // scores all lie below fold_limit, the limit where they are folded, takes the polynomial without that multiplication
  // (256 positions of window: 53 -> 51 us); a score gets the same bits on either way.
  float cap_ratio, cap_limit, poly_ratio, cap_poly[4], fold_limit;
  TileCut* how; // written by the tile kernel for the merge
  int* parts;   // stream kernel: arrivals of a cut chain's parts [target][n_kv], zero between calls; NULL:
                // the merge kernel joins them
};

// One (sequence, tile, kv head, split) of the main kernels.
struct Unit {
  int b, t, kvh, s, splits, slot;  // slot: of split 0's partial result (slots of a tile are nkv apart)
  int C, rows, r0;
};

// Lane b's part of the cut: sequence b's tiles and pages; walk: the pages that one tile walks at most.
struct Cut {
  SeqRows s;
  int tiles, pages, walk, splits;
};

LSV_DEV Cut cut_of(const AttendArgs& a, const AttendPlan& pl) {
  Cut c;
  c.s = seq_rows(a.rows);
  c.tiles = (c.s.rows * pl.group + pl.tile - 1) / pl.tile;
  const int first = a.window ? max(0, c.s.C - a.window + 1) / kPage : 0;  // what the first row sees at least
  c.pages = c.s.rows > 0 ? (c.s.C + c.s.rows + kPage - 1) / kPage - first : 0;
  c.walk = c.pages;
  if (a.window && !a.prefix_len) c.walk = min(c.pages, (a.window + (pl.tile - 1) / pl.group + kPage - 1) / kPage + 1);
  c.splits = 1;
  return c;
}

// The stream kernel's work is one line of pages: the chains (sequence, tile), each as long as the
// sequence's pages, one after another, the same line for every kv head.  Share w of it goes to
// the workgroups w * n_kv + kv head: all shares are equal, whatever chains they meet, and the workgroups of a
// share walk the same pages, whose kv heads lie side by side.  A share's ends cut chains, whose parts
// the merge kernel joins.
struct Line {
  Cut c;
  int end;    // lane b: where sequence b's chains end
  int share;  // pages of a share
};
LSV_DEV Line line_of(const AttendArgs& a, const AttendPlan& pl) {
  Line l;
  l.c = cut_of(a, pl);
  // a chain is as long as whole least shares, so that these never hold more than one chain
  l.c.pages = (l.c.pages + pl.least - 1) / pl.least * pl.least;
  l.end = wave_scan_sum(l.c.tiles * l.c.pages);
  const int total = __builtin_amdgcn_readlane(l.end, a.rows.batch - 1);
  // whole least shares again (least is 1 or 2), so that both waves have as many pages: 40.9 -> 36.4 us for four rows behind
  // each of four contexts of 8192, 32 query vectors and shares of ten pages instead of nine
  l.share = max(pl.least, ((total + pl.target - 1) / pl.target + pl.least - 1) & -pl.least);
  return l;
}
// The part of the chain at place `g` of the line that a share holds from there on; len 0 past the line.
struct Part {
  int b, t, C, rows, r0;
  int chain;   // the chain's pages
  int at;      // pages of the chain before this part
  int len;
};
LSV_DEV Part part_at(const Line& l, int g) {
  Part p{};
  const int share_end = (g / l.share + 1) * l.share;
  const unsigned long long past = __ballot(l.end > g);
  if (!past) return p;
  p.b = __builtin_amdgcn_readfirstlane(__ffsll((long long)past) - 1);
  p.C = __builtin_amdgcn_readlane(l.c.s.C, p.b);
  p.rows = __builtin_amdgcn_readlane(l.c.s.rows, p.b);
  p.r0 = __builtin_amdgcn_readlane(l.c.s.r0, p.b);
  p.chain = __builtin_amdgcn_readlane(l.c.pages, p.b);
  const int local = g - (__builtin_amdgcn_readlane(l.end, p.b) - __builtin_amdgcn_readlane(l.c.tiles, p.b) * p.chain);
  p.t = local / p.chain;
  p.at = local - p.t * p.chain;
  p.len = min(p.chain - p.at, share_end - g);
  return p;
}
// The partial result of a part that starts (`first`) or continues a chain in share w.
LSV_DEV int slot_of(int w, bool first, int nkv, int kvh) { return (2 * w + (first ? 1 : 0)) * nkv + kvh; }

// The cheapest of sixteen cuts of either kind, one a lane: rounds of workgroups times their longest walk, three pages'
// time for what a workgroup does besides.  (556 units of 18 pages at head dimension 64, capped scores: 57 us whole
// in two rounds of 512, 49 with the last 44 in parts.)
LSV_DEV TileCut tile_cut(const AttendArgs& a, const AttendPlan& pl, const Cut& c) {
  const int lane = threadIdx.x & 63, longest = wave_max_int(c.walk), k = (lane & 15) + 1;
  if (longest <= 4) return TileCut{TileCut::kNoLimit, 1 << 30, 1};
  const int pps = max(4, (longest + k - 1) / k);
  int units = 0, split = 0, tiles = 0;
  for (int b = 0; b < a.rows.batch; ++b) {
    const int t = __builtin_amdgcn_readlane(c.tiles, b), pages = __builtin_amdgcn_readlane(c.walk, b);
    const int n = t * ((pages + pps - 1) / pps);
    tiles += t;
    units += n;
    split += pages > pps ? n : 0;
  }
  const int rounds = tiles * a.nkv / pl.target, whole = rounds * pl.target / a.nkv, rest = (tiles - whole) * k * a.nkv;
  int cost = min((units * a.nkv + pl.target - 1) / pl.target, 1 << 14) * min(pps + 3, 1 << 16);
  if (k > 1 && split * a.nkv > pl.slots) cost = 0x7fffffff;
  if (lane & 16) {
    cost = min(rounds, 1 << 13) * min(longest + 3, 1 << 16) + min((rest + pl.target - 1) / pl.target, 1 << 13) * min(pps + 3, 1 << 16);
    if (k == 1 || rest > pl.slots || pps * (k - 1) >= longest) cost = 0x7fffffff;
  }
  const int best = wave_min_int(cost), at = __ffsll((long long)__ballot(cost == best)) - 1;
  if (at & 16) return TileCut{TileCut::kNoLimit, __builtin_amdgcn_readlane(whole, at), (at & 15) + 1};
  return TileCut{(at & 15) == 0 ? TileCut::kNoLimit : __builtin_amdgcn_readlane(pps, at), 1 << 30, 1};
}

// The unit that workgroup `i` takes; false: none is left.  Units go by sequence, tile (the last, which sees
// most, first), split, kv head: neighbouring workgroups read neighbouring memory, and with eight kv heads an XCD
// keeps one head's pages in its L2.
LSV_DEV bool unit_of(const AttendArgs& a, const AttendPlan& pl, Cut c, const TileCut& cut, int i, Unit& u) {
  u.kvh = i % a.nkv;
  int line = i / a.nkv;  // the tile's place among all, counting every split (by length) as one
  c.splits = max(1, (c.walk + cut.pps - 1) / cut.pps);
  const int units = c.tiles * c.splits, held = c.splits > 1 ? units : 0;
  const int sum = wave_scan_sum(units), slots = wave_scan_sum(held);
  const int whole = __builtin_amdgcn_readlane(sum, 63), lines = whole <= cut.whole ? whole : cut.whole + (whole - cut.whole) * cut.rest;
  // where all units are on the chip at once, those that join others on their compute units go the other way, a long
  // walk beside a short one (512 units of 94 to 126 pages: 250 -> 243 us)
  const int half = pl.target / 2 / a.nkv;
  if (line >= half && line < lines && lines <= 2 * half) line = half + lines - 1 - line;
  u.s = 0;
  u.splits = 1;
  if (line >= cut.whole) {
    u.s = (line - cut.whole) % cut.rest;
    u.splits = cut.rest;
    line = cut.whole + (line - cut.whole) / cut.rest;
  }
  u.slot = (line - cut.whole) * cut.rest * a.nkv + u.kvh;
  const unsigned long long past = __ballot(sum > line);
  if (!past) return false;
  const int b = __builtin_amdgcn_readfirstlane(__ffsll((long long)past) - 1);
  u.b = b;
  u.C = __builtin_amdgcn_readlane(c.s.C, b);
  u.rows = __builtin_amdgcn_readlane(c.s.rows, b);
  u.r0 = __builtin_amdgcn_readlane(c.s.r0, b);
  int local = line - __builtin_amdgcn_readlane(sum - units, b);
  const int tiles = __builtin_amdgcn_readlane(c.tiles, b), by_length = __builtin_amdgcn_readlane(c.splits, b);
  if (by_length > 1) {
    u.splits = by_length;
    u.s = local % by_length;
    u.slot = (__builtin_amdgcn_readlane(slots - held, b) + local - u.s) * a.nkv + u.kvh;
    local /= by_length;
  }
  u.t = tiles - 1 - local;
  return true;
}

// What one query vector sees and how its scores are changed.
struct Query {
  int lo, hi;   // visible keys; nothing: lo = INT_MAX, hi = 0
  int pos;
  float slope;  // log2 units
};
template <typename U> LSV_DEV Query query_of(const AttendArgs& a, const U& u, int kvh, int group, int qv, int nqv) {
  Query q{0x7fffffff, 0, 0, 0.f};
  if (qv >= nqv) return q;
  const int row = qv / group, L = u.C + u.rows;
  q.pos = u.C + row;
  int hi = q.pos + 1, lo = 0;
  if (a.prefix_len) hi = max(hi, GL(a.prefix_len)[u.b]);
  hi = min(hi, L);
  if (a.window) lo = max(lo, q.pos - a.window + 1);
  if (a.key_start) lo = max(lo, GL(a.key_start)[u.r0 + row]);
  if (a.slopes) q.slope = kLog2e * GL(a.slopes)[kvh * group + qv % group];
  if (lo < hi) {
    q.lo = lo;
    q.hi = hi;
  }
  return q;
}

// A tile's keys over its valid vectors: [lo_min, hi_max) has what some vector sees, [lo_max, hi_min)
// what every one does.
struct Range {
  int lo_min, lo_max, hi_min, hi_max;
};
LSV_DEV void add_query(Range& r, const Query& q, bool valid) {
  if (!valid) return;
  r.lo_min = min(r.lo_min, q.lo);
  r.lo_max = max(r.lo_max, q.lo);
  r.hi_min = min(r.hi_min, q.hi);
  r.hi_max = max(r.hi_max, q.hi);
}
LSV_DEV Range wave_range(Range r) {
  return Range{wave_min_int(r.lo_min), wave_max_int(r.lo_max), wave_min_int(r.hi_min), wave_max_int(r.hi_max)};
}

// The pages of split s of `splits` of a tile that sees keys [lo, hi).
LSV_DEV void split_pages(int lo, int hi, int s, int splits, int& pa, int& pb) {
  pa = pb = 0;
  if (lo >= hi) return;
  const int first = lo / kPage, n = (hi + kPage - 1) / kPage - first, each = (n + splits - 1) / splits;
  pa = first + min(s * each, n);
  pb = first + min((s + 1) * each, n);
}

// Page p of the sequence as buffer resources of its K and V blocks of one kv head; a page outside
// the pool has no bytes and reads as zeros.  The table goes through the scalar cache: a vector load
// would have to wait for the K and V loads issued before it.
LSV_DEV int page_at(const AttendArgs& a, int b, int p) {
  return ((const __attribute__((address_space(4))) int32_t*)a.kv.pages)[(size_t)b * a.kv.max_pages + p];
}
template <typename T, int HD>
LSV_DEV __amdgpu_buffer_rsrc_t page_rsrc(const AttendArgs& a, const void* pool, int page, int kvh) {
  const bool there = page >= 0 && page < a.kv.n_pages;
  const T* base = (const T*)pool + ((size_t)(there ? page : 0) * a.nkv + kvh) * kPage * HD;
  return stream_rsrc(base, there ? kPage * HD * sizeof(T) : 0);
}

// A call's scores: plain, capped, biased by distance, or both.
enum { kPlain = 0, kCapped = 1, kBiased = 2 };

LSV_DEV float cap_poly(const float (&c)[4], float s, float y) { return s * fmaf(fmaf(fmaf(c[3], y, c[2]), y, c[1]), y, c[0]); }
// A score in log2 units from the product q.k; key: its position.
// cap * tanh(x) = cap - 2 cap / (exp(2 x) + 1): right at both ends, off by some 2^-23 of the cap; so the polynomial
// below half of it, or a cap far above the scores would leave nothing of them.  fp32 takes the library's tanh.
template <typename T, int MOD> LSV_DEV float capped_of(const AttendArgs& a, const AttendPlan& pl, float s) {
  if constexpr (!(MOD & kCapped)) {
    return s * (a.scale * kLog2e);
  } else if constexpr (sizeof(T) == 4) {
    return a.softcap * kLog2e * tanhf(s * a.scale / a.softcap);
  } else {
    const float cap = a.softcap * kLog2e;
    const float e = __builtin_amdgcn_exp2f(s * (2.f * kLog2e * pl.cap_ratio));
    const float big = fmaf(-2.f * cap, __builtin_amdgcn_rcpf(e + 1.f), cap);
    const float x = s * pl.poly_ratio;
    return fabsf(s) <= pl.cap_limit ? cap_poly(pl.cap_poly, s, x * x) : big;
  }
}
LSV_DEV float biased_of(const Query& q, float s, int key) { return fmaf(-q.slope, fabsf((float)(q.pos - key)), s); }
template <typename T, int MOD> LSV_DEV float score_of(const AttendArgs& a, const AttendPlan& pl, const Query& q, float s, int key) {
  s = capped_of<T, MOD>(a, pl, s);
  if constexpr (MOD & kBiased) s = biased_of(q, s, key);
  return s;
}

// Values that are not finite stay out of the product with V where some rows do not see them (0 times
// infinity is NaN): they are cleared, and two products over the rows' visibility then count, for each element of
// the output, the seen values that are infinite upwards and downwards, NaN among both.
constexpr float kMaxFloat = 3.4028234663852886e38f;
template <typename T> LSV_DEV uint32_t clean(uint32_t u) {
  auto kept = [](uint32_t x, uint32_t y) { return fabsf(__uint_as_float(x)) <= kMaxFloat ? y : 0u; };
  if constexpr (sizeof(T) == 4) return kept(u, u);
  return kept(u & 0xffff0000u, u & 0xffff0000u) | kept(u << 16, u & 0xffffu);
}
// 1 for each value that is NaN or infinite upwards (`down`: downwards), else 0.
template <typename T> LSV_DEV u32x4_t class_of(u32x4_t f, bool down) {
  auto counts = [&](uint32_t x, uint32_t one) {
    const float v = __uint_as_float(x);
    return (down ? v >= -kMaxFloat : v <= kMaxFloat) ? 0u : one;
  };
  u32x4_t c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (sizeof(T) == 4) c[i] = counts(f[i], 0x3f800000u);
    else c[i] = counts(f[i] & 0xffff0000u, 0x3f800000u) | counts(f[i] << 16, 0x3f80u);
  }
  return c;
}
LSV_DEV float infinite_part(uint32_t up, uint32_t down) {  // bit 0 of each
  return (up & 1u ? INFINITY : 0.f) + (down & 1u ? -INFINITY : 0.f);
}
// Gathers in `bits` whether a fragment of V holds such a value: an exponent of ones carries into the sign's place.
template <typename T> constexpr uint32_t kSigns = sizeof(T) == 4 ? 0x80000000u : 0x80008000u;
template <typename T> LSV_DEV void gather_not_finite(u32x4_t f, uint32_t& bits) {
  constexpr uint32_t one = sizeof(T) == 4 ? 0x00800000u : 0x00800080u;
#pragma unroll
  for (int i = 0; i < 4; ++i) bits |= (f[i] & ~kSigns<T>) + one;
}
template <typename T> LSV_DEV void clean_fragment(u32x4_t& f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = clean<T>(f[i]);
}

// ------------------------------------------------------------------ stream kernel
// One pass over a chain's pages with the running maximum m and sum l of the softmax: for a step's scores s_j (in log2
// units), m' = max(m, s_j), p_j = 2^(s_j - m'), l' = l 2^(m - m') + sum p_j and o' = o 2^(m - m') + sum p_j v_j; a row's
// result is o / l and m + log2 l.  Parts of a chain join by the same rule, so its pages may be cut anywhere.
// Exponentials are the hardware's 2^x, in fp32 too: off by 2^-22 of a probability, where the score that it comes from is off
// by up to HD 2^-24 of its largest products.
// Reading K and V bounds it, once each: a page meets every query vector of its tile.  Measured: 64 sequences of one
// token behind 200 to 8000 positions, 1.08 GB in 170 us (6.3 TB/s; four waves a workgroup that took whole sequences:
// 257); two of four tokens behind 100K to 131K, 0.95 GB in 150 us + 10 for the merge; one token behind 2047, 8.4 MB: 10.7 us,
// a chain of dependent loads (row offsets, page table, K, V, the other parts' sums).

// A wave's step: 16 KT keys, whose K rows and V^T rows (of KP and VP 16-byte pieces) it holds in LDS.
// Pieces are exchanged within a row -- piece c of row r stands at c ^ turn(r) -- so that the sixteen rows
// that a read touches at once lie on separate banks; direct loads to LDS allow no padding.
template <int PIECES> LSV_DEV int turn_of(int row) { return PIECES >= 16 ? row & 15 : (row >> 1) & 7; }

template <typename T, int HD> struct Stream;
template <int HD> struct Stream<bf16_t, HD> {
  static constexpr int KT = 4, KP = HD / 8, VP = 8;
  // pieces of Q (and of a K row) that a lane group takes: 32 f + 8 g4 .. + 7
  static constexpr int QF = HD / 32;
  LSV_DEV static int q_piece(int f, int g4) { return 4 * f + g4; }
  LSV_DEV static int v_piece(int i, int g4) { return 4 * i + g4; }  // keys of the 32 i: columns 32 i + 8 g4 .. + 7
  LSV_DEV static f32x4_t score(u32x4_t k, u32x4_t q, f32x4_t s) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k), __builtin_bit_cast(bf16x8_t, q), s, 0, 0, 0);
  }
  // P^T as an operand: rounded to bf16, so that the product runs on the matrix cores at their bf16 rate.  An output
  // is off by up to 2^-8 of the mean |v| for it (1.2 to 1.4 times the error of rounding the output alone, over random
  // values); l sums the probabilities as they were.
  struct P {
    bf16x8_t p[2];
  };
  LSV_DEV static P pack(const f32x4_t (&sc)[KT]) {
    P r;
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        r.p[k][i] = (__bf16)sc[2 * k][i];
        r.p[k][4 + i] = (__bf16)sc[2 * k + 1][i];
      }
    return r;
  }
  LSV_DEV static f32x4_t product(u32x4_t v, const P& p, int i, f32x4_t o) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v), p.p[i], o, 0, 0, 0);
  }
};
template <int HD> struct Stream<float, HD> {
  static constexpr int KT = 2, KP = HD / 4, VP = 8;  // half a page: 32 columns of V^T
  // a piece holds four of a row's dimensions, one for each of four products: lane group g4 has
  // dimensions 16 f + 4 g4 + e in product e, in K and Q alike
  static constexpr int QF = HD / 16;
  LSV_DEV static int q_piece(int f, int g4) { return 4 * f + g4; }
  LSV_DEV static int v_piece(int i, int g4) { return 2 * g4 + i; }  // keys 16 i + 4 g4 .. + 3: columns 8 g4 + 4 i .. + 3
  LSV_DEV static f32x4_t score(u32x4_t k, u32x4_t q, f32x4_t s) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), __uint_as_float(q[e]), s, 0, 0, 0);
    return s;
  }
  struct P {
    f32x4_t p[2];
  };
  LSV_DEV static P pack(const f32x4_t (&sc)[KT]) { return P{{sc[0], sc[1]}}; }
  LSV_DEV static f32x4_t product(u32x4_t v, const P& p, int i, f32x4_t o) {
#pragma unroll
    for (int e = 0; e < 4; ++e) o = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[e]), p.p[i][e], o, 0, 0, 0);
    return o;
  }
};

template <typename T> LSV_DEV void store4(T* p, f32x4_t v) {
  if constexpr (sizeof(T) == 4) {
    *(GLOBAL f32x4_t*)(GLOBAL T*)GL(p) = v;
  } else {
    *(GLOBAL u32x2_t*)(GLOBAL T*)GL(p) =
        u32x2_t{(uint32_t)f2bf(v[0]) | ((uint32_t)f2bf(v[1]) << 16), (uint32_t)f2bf(v[2]) | ((uint32_t)f2bf(v[3]) << 16)};
  }
}
// The factor on sums under maximum m when they join others under maximum top >= m.  Equal ones, two
// empty ones (-inf) too, take 1; sums that are NaN stay NaN under any factor.
LSV_DEV float rescale(float m, float top) { return m == top ? 1.f : __builtin_amdgcn_exp2f(m - top); }
// A row's result from its sums: nothing seen gives 0 and -inf.
LSV_DEV float factor_of(float l) { return l == 0.f ? 0.f : 1.f / l; }
LSV_DEV float lse_of(float m, float l) { return l == 0.f ? -INFINITY : (m + log2f(l)) * (1.f / kLog2e); }

// Partial results that another workgroup of the same launch reads: relaxed atomic stores and loads of the
// agent's scope go past the L2 of the XCD, so that no fence has to write it back and drop it (with fences
// 64 ragged sequences take 296 us instead of 176).  The stores are waited for before the arrival is counted.
LSV_DEV void put_agent(float* p, f32x2_t v) {
  __hip_atomic_store((uint64_t*)p, __builtin_bit_cast(uint64_t, v), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
LSV_DEV f32x2_t get_agent(const float* p) {
  return __builtin_bit_cast(f32x2_t, __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// Sums of a query vector that are being joined, four dimensions of them.
struct Joined {
  float m = -INFINITY, den = 0.f;
  f32x4_t num = {0.f, 0.f, 0.f, 0.f};
};
// Join parts s0 .. s0 + NB - 1 with their loads in flight together; those past the last part repeat it.  SAME: the parts
// are of this launch.
template <int HD, int NB, bool SAME, typename SlotAt>
LSV_DEV void join_some(Joined& j, const AttendPlan& pl, int s0, int parts, SlotAt slot_at, int in_tile, int d) {
  f32x2_t ml[NB];
  f32x4_t ov[NB];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    const size_t at = (size_t)slot_at(min(s0 + k, parts - 1)) * pl.tile + in_tile;
    if constexpr (SAME) {
      const f32x2_t lo = get_agent(pl.o + at * HD + d), hi = get_agent(pl.o + at * HD + d + 2);
      ml[k] = get_agent(pl.ml + at * 2);
      ov[k] = f32x4_t{lo[0], lo[1], hi[0], hi[1]};
    } else {
      ml[k] = *(const GLOBAL f32x2_t*)(GL(pl.ml) + at * 2);
      ov[k] = *(const GLOBAL f32x4_t*)(GL(pl.o) + at * HD + d);
    }
  }
  float top = j.m;
#pragma unroll
  for (int k = 0; k < NB; ++k) top = fmaxf(top, ml[k][0]);
  const float f = rescale(j.m, top);
  j.num *= f;
  j.den *= f;
  j.m = top;
#pragma unroll
  for (int k = 0; k < NB; ++k)
    if (s0 + k < parts) {
      const float w = rescale(ml[k][0], top);
      j.num += ov[k] * w;
      j.den += ml[k][1] * w;
    }
}
// Join the `parts` partial results of a query vector, in tile place in_tile of their slots, and write dimensions
// d .. d + 3 of its row.  Sixteen at a time, the rest by eight or four: 24 sequences of one token behind some 900 positions
// 22.5 -> 21.6 us (sixteen at a time throughout; always eight in the merge kernels cost 15.6 us for 15.0 with masked fp32 rows,
// always sixteen 44.3 for 41.4 with 1000 rows in few parts).
template <typename T, int HD, bool SAME, typename SlotAt>
LSV_DEV void join_parts(const AttendArgs& a, const AttendPlan& pl, int parts, SlotAt slot_at, int in_tile, int d, int row, int head) {
  Joined j;
  int s = 0;
  for (; parts - s > 8; s += 16) join_some<HD, 16, SAME>(j, pl, s, parts, slot_at, in_tile, d);
  if (parts - s > 4) join_some<HD, 8, SAME>(j, pl, s, parts, slot_at, in_tile, d);
  else if (parts - s > 0) join_some<HD, 4, SAME>(j, pl, s, parts, slot_at, in_tile, d);
  store4<T>((T*)a.out + (int64_t)row * a.os + (int64_t)head * HD + d, j.num * factor_of(j.den));
  if (a.lse && d == 0) GL(a.lse)[(int64_t)row * a.nq + head] = lse_of(j.m, j.den);
}

template <typename T, int HD, int NQ, int MOD>
__global__ void __launch_bounds__(64 * kStreamWaves, 1) attend_stream_kernel(AttendArgs a, AttendPlan pl) {
  using St = Stream<T, HD>;
  constexpr int KT = St::KT, KP = St::KP, VP = St::VP, SUB = kPage / (16 * KT);  // steps per page
  constexpr int N = 16 * KT * KP;  // pieces of a step's K, and of its V^T
  constexpr int LOADS = N / 64;    // direct loads for either
  constexpr int PITCH = HD / 2 + 4;  // of the sums' rows in LDS: sixteen lanes' pieces on separate banks
  static_assert(N == HD * VP && kStreamWaves == 2, "two waves exchange halves of their sums");
  // each wave's own step; K and V are variables of their own, so that the compiler sees that the reads
  // of one need not wait for the direct loads to the other
  __shared__ __align__(16) u32x4_t kl[kStreamWaves * N];
  __shared__ __align__(16) u32x4_t vl[kStreamWaves * N];
  __shared__ __align__(16) float os[kStreamWaves][16 * PITCH];
  __shared__ float ms[kStreamWaves][16], ls[kStreamWaves][16];
  __shared__ int flag;

  const Line line = line_of(a, pl);
  if (a.status && blockIdx.x == 0 && (int)threadIdx.x < a.rows.batch) a.status[threadIdx.x] = line.c.s.status;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g4 = lane >> 4, l16 = lane & 15;
  const int w = blockIdx.x / a.nkv, kvh = blockIdx.x - w * a.nkv;
  int g = w * line.share;
  Part part = part_at(line, g);
  if (!part.len) return;
  const int share_end = g + line.share;

  // LDS piece i of a step is piece (i % P) ^ turn of row i / P
  const int mine = wave * N;
  auto load_k = [&](int page, int half) {
    const __amdgpu_buffer_rsrc_t rs = page_rsrc<T, HD>(a, a.k_pool, page, kvh);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = i * 64 + lane;
      load_lds<kBufferStream>(rs, &kl[mine + i * 64], ((at & ~(KP - 1)) + ((at % KP) ^ turn_of<KP>(at / KP))) * 16, half * N * 16);
    }
  };
  auto load_v = [&](int page, int half) {
    const __amdgpu_buffer_rsrc_t rs = page_rsrc<T, HD>(a, a.v_pool, page, kvh);
#pragma unroll
    for (int i = 0; i < LOADS; ++i) {
      const int at = i * 64 + lane, row = at / VP;
      load_lds<kBufferStream>(rs, &vl[mine + i * 64], (row * (VP * SUB) + ((at % VP) ^ turn_of<VP>(row))) * 16, half * VP * 16);
    }
  };
  const int krow = mine + l16 * KP, vrow = mine + l16 * VP, kturn = turn_of<KP>(l16), vturn = turn_of<VP>(l16);
  auto v_frag = [&](int d, int i) { return vl[vrow + 16 * d * VP + (St::v_piece(i, g4) ^ vturn)]; };
  // The pages [pa, pb) of a part that its tile sees, as far as lengths, prefix and window tell.
  struct Pages {
    int pa, pb;
  };
  auto pages_of = [&](const Part& p) {
    if (!p.len) return Pages{0, 0};
    const int row0 = p.t * pl.tile / pl.group, row1 = (min((p.t + 1) * pl.tile, p.rows * pl.group) - 1) / pl.group;
    int hi = p.C + row1 + 1, lo = 0, first = 0;
    if (a.prefix_len) hi = max(hi, __builtin_amdgcn_readfirstlane(GL(a.prefix_len)[p.b]));
    hi = min(hi, p.C + p.rows);
    if (a.window) {
      lo = max(0, p.C + row0 - a.window + 1) / kPage;
      first = max(0, p.C - a.window + 1) / kPage;
    }
    first += p.at;
    return Pages{max(first, lo), min(first + p.len, (hi + kPage - 1) / kPage)};
  };
  // The page of step i of pages `p`; behind the last step a page outside the pool: the loads are then issued
  // without a branch around them, and the compiler counts them exactly.
  auto step_page = [&](const Part& part, const Pages& p, int i) {
    return p.pa + i / SUB < p.pb ? page_at(a, part.b, p.pa + i / SUB) : -1;
  };
  auto load_q = [&](const Part& p, u32x4_t (&qf)[NQ][St::QF]) {
    const int nqv = p.rows * pl.group;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {  // an invalid column repeats the last vector, its result is dropped
      const int qv = min(p.t * pl.tile + 16 * t + l16, nqv - 1);
      const T* src = (const T*)a.q + (int64_t)(p.r0 + qv / pl.group) * a.qs + (int64_t)(kvh * pl.group + qv % pl.group) * HD;
#pragma unroll
      for (int f = 0; f < St::QF; ++f) qf[t][f] = ((const GLOBAL u32x4_t*)(const GLOBAL T*)GL(src))[St::q_piece(f, g4)];
    }
  };
  auto meet = [] {  // a barrier that leaves direct loads in flight
    wait_loads<63>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };

  // Rows with starts of their own (key_start) show what a tile sees only when they are loaded: its pages
  // are then asked for at the start of the part, else during the part before.
  u32x4_t qf[NQ][St::QF];
  load_q(part, qf);
  Pages pages = pages_of(part);
  if (!a.key_start) {
    const int page = step_page(part, pages, wave);
    load_k(page, wave % SUB);
    load_v(page, wave % SUB);
  }
  while (true) {
    Part next{};
    if (g + part.len < share_end) next = part_at(line, g + part.len);
    const Pages next_pages = pages_of(next);
    const int nqv = part.rows * pl.group, v0 = part.t * pl.tile;
    u32x4_t qn[NQ][St::QF] = {};
    if (next.len) load_q(next, qn);
    Query q[NQ];
    Range range{0x7fffffff, 0, 0x7fffffff, 0};
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      q[t] = query_of(a, part, kvh, pl.group, v0 + 16 * t + l16, nqv);
      add_query(range, q[t], v0 + 16 * t + l16 < nqv);
    }
    int all_lo = 0, all_hi = part.C + v0 / pl.group + 1;  // keys that every row of the tile sees
    if (a.key_start) {
      range = wave_range(range);
      all_lo = range.lo_max;
      pages.pa = max(pages.pa, range.lo_min / kPage);
      const int page = step_page(part, pages, wave);
      load_k(page, wave % SUB);
      load_v(page, wave % SUB);
    } else if (a.window) {
      all_lo = max(0, part.C + (min(v0 + pl.tile, nqv) - 1) / pl.group - a.window + 1);
    }

    f32x4_t o[NQ][HD / 16];
    float mrun[NQ], lrun[NQ];
    uint32_t infinite[NQ][2] = {};  // per element of o: whether it sums a value infinite upwards, downwards
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      mrun[t] = -INFINITY;
      lrun[t] = 0.f;
#pragma unroll
      for (int d = 0; d < HD / 16; ++d) o[t][d] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int steps = max(0, pages.pb - pages.pa) * SUB;
    for (int i = wave; i < steps; i += kStreamWaves) {
      int k0 = (pages.pa + i / SUB) * kPage + i % SUB * (16 * KT);
      const bool last = i + kStreamWaves >= steps;
      const int to = last ? wave : i + kStreamWaves;
      const int next_page = !last ? step_page(part, pages, to) : a.key_start ? -1 : step_page(next, next_pages, to);
      const bool full = k0 >= all_lo && k0 + 16 * KT <= all_hi;
      wait_loads<LOADS>();  // K has landed; V may be on its way
      f32x4_t sc[NQ][KT];
#pragma unroll
      for (int k = 0; k < KT; ++k) {
#pragma unroll
        for (int t = 0; t < NQ; ++t) sc[t][k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int f = 0; f < St::QF; ++f) {
          const u32x4_t x = kl[krow + 16 * k * KP + (St::q_piece(f, g4) ^ kturn)];
#pragma unroll
          for (int t = 0; t < NQ; ++t) sc[t][k] = St::score(x, qf[t][f], sc[t][k]);
        }
      }
      wait_loads<63>();  // every read of K has returned
      load_k(next_page, to % SUB);
      typename St::P p[NQ];
#pragma unroll
      for (int t = 0; t < NQ; ++t) {
        float mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const int key = k0 + 16 * k + 4 * g4 + r;
            float v = score_of<T, MOD>(a, pl, q[t], sc[t][k][r], key);
            if (!full) v = key >= q[t].lo && key < q[t].hi ? v : -INFINITY;
            sc[t][k][r] = v;
            mx = fmaxf(mx, v);
          }
        mx = fmaxf(mx, __shfl_xor(mx, 16, kWave));
        mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
        const float mnew = fmaxf(mrun[t], mx);
        const float ref = mnew == -INFINITY ? 0.f : mnew;  // nothing seen yet: every probability is 2^-inf
        const float alpha = __builtin_amdgcn_exp2f(mrun[t] - ref);
        float sum = 0.f;
#pragma unroll
        for (int k = 0; k < KT; ++k)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            sc[t][k][r] = __builtin_amdgcn_exp2f(sc[t][k][r] - ref);
            sum += sc[t][k][r];
          }
        mrun[t] = mnew;
        lrun[t] = lrun[t] * alpha + sum;
        p[t] = St::pack(sc[t]);
#pragma unroll
        for (int d = 0; d < HD / 16; ++d) o[t][d] *= alpha;
      }
      wait_loads<LOADS>();  // V has landed; the next K may be on its way
      if (!full) {  // a key that some row does not see may hold anything
        uint32_t bits = 0;
#pragma unroll
        for (int j = 0; j < LOADS; ++j) gather_not_finite<T>(vl[mine + j * 64 + lane], bits);
        if (__any((bits & kSigns<T>) != 0)) {
          asm volatile("" : "+v"(k0));  // keeps what follows out of the loop's registers
#pragma unroll
          for (int t = 0; t < NQ; ++t) {
#pragma unroll
            for (int k = 0; k < KT; ++k)
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const int key = k0 + 16 * k + 4 * g4 + r;
                sc[t][k][r] = key >= q[t].lo && key < q[t].hi ? 1.f : 0.f;
              }
            const typename St::P seen = St::pack(sc[t]);
#pragma unroll
            for (int d = 0; d < HD / 16; ++d)
#pragma unroll
              for (int down = 0; down < 2; ++down) {
                __builtin_amdgcn_sched_barrier(0);
                f32x4_t n = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 2; ++j) n = St::product(class_of<T>(v_frag(d, j), down), seen, j, n);
#pragma unroll
                for (int r = 0; r < 4; ++r) infinite[t][down] |= (n[r] > 0.f ? 1u : 0u) << (4 * d + r);
              }
          }
#pragma unroll
          for (int j = 0; j < LOADS; ++j) clean_fragment<T>(vl[mine + j * 64 + lane]);
          wait_loads<63>();
        }
      }
#pragma unroll
      for (int d = 0; d < HD / 16; ++d)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4_t v = v_frag(d, j);
#pragma unroll
          for (int t = 0; t < NQ; ++t) o[t][d] = St::product(v, p[t], j, o[t][d]);
        }
      wait_loads<63>();  // every read of V has returned
      load_v(next_page, to % SUB);
    }
    if (wave >= steps) {  // no step for this wave: the next part's first one is still to be asked for
      const int page = a.key_start ? -1 : step_page(next, next_pages, wave);
      load_k(page, wave % SUB);
      load_v(page, wave % SUB);
    }

    // The waves exchange halves of their sums, sixteen query vectors at a time: each joins and writes half
    // of the head.
    const bool whole = part.len == part.chain;
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
      if (__any((infinite[t][0] | infinite[t][1]) != 0)) {
#pragma unroll
        for (int d = 0; d < HD / 16; ++d)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            o[t][d][r] += infinite_part(infinite[t][0] >> (4 * d + r), infinite[t][1] >> (4 * d + r));
      }
      float l = lrun[t];
      const float m = mrun[t];
      l += __shfl_xor(l, 16, kWave);
      l += __shfl_xor(l, 32, kWave);
      if (t) meet();
#pragma unroll
      for (int d = 0; d < HD / 32; ++d)
        *(f32x4_t*)&os[wave][l16 * PITCH + 16 * d + 4 * g4] = wave ? o[t][d] : o[t][HD / 32 + d];
      if (g4 == 0) {
        ms[wave][l16] = m;
        ls[wave][l16] = l;
      }
      meet();
      const int in_tile = 16 * t + l16, qv = v0 + in_tile, other = wave ^ 1;
      const float mo = ms[other][l16], top = fmaxf(m, mo), f0 = rescale(m, top), f1 = rescale(mo, top);
      l = l * f0 + ls[other][l16] * f1;
      const float f = factor_of(l);
      if (qv < nqv) {
        const int row = part.r0 + qv / pl.group, head = kvh * pl.group + qv % pl.group;
        const size_t slot = (size_t)slot_of(w, part.at == 0, a.nkv, kvh) * pl.tile + in_tile;
        T* const out = (T*)a.out + (int64_t)row * a.os + (int64_t)head * HD;
#pragma unroll
        for (int d = 0; d < HD / 32; ++d) {
          const f32x4_t mine_ = wave ? o[t][HD / 32 + d] : o[t][d];
          const f32x4_t x = mine_ * f0 + *(const f32x4_t*)&os[other][l16 * PITCH + 16 * d + 4 * g4] * f1;
          const int dim = wave * (HD / 2) + 16 * d + 4 * g4;
          if (whole) store4<T>(out + dim, x * f);
          else {
            put_agent(pl.o + slot * HD + dim, f32x2_t{x[0], x[1]});
            put_agent(pl.o + slot * HD + dim + 2, f32x2_t{x[2], x[3]});
          }
        }
        if (wave == 0 && g4 == 0) {
          if (!whole) put_agent(pl.ml + slot * 2, f32x2_t{top, l});
          else if (a.lse) GL(a.lse)[(int64_t)row * a.nq + head] = lse_of(top, l);
        }
      }
    }
    if (!whole && pl.parts) {  // the last part of the chain to arrive joins them all
      const int w0 = (g - part.at) / line.share, parts = (g - part.at + part.chain - 1) / line.share - w0 + 1;
      int* const arrived = pl.parts + w0 * a.nkv + kvh;
      wait_loads<0>();  // this wave's stores have reached memory
      meet();
      if (threadIdx.x == 0) flag = __hip_atomic_fetch_add(arrived, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == parts - 1;
      meet();
      if (flag) {
        reset_counter(arrived);
        const int d = threadIdx.x % (HD / 4) * 4;
        for (int in_tile = threadIdx.x / (HD / 4); in_tile < pl.tile && v0 + in_tile < nqv; in_tile += 256 * kStreamWaves / HD) {
          const int qv = v0 + in_tile;
          join_parts<T, HD, true>(a, pl, parts, [&](int i) { return slot_of(w0 + i, i == 0, a.nkv, kvh); }, in_tile, d,
                                  part.r0 + qv / pl.group, kvh * pl.group + qv % pl.group);
        }
      }
    }
    if (!next.len) break;
    meet();  // the exchange's space is free again
    g += part.len;
    part = next;
    pages = next_pages;
#pragma unroll
    for (int t = 0; t < NQ; ++t)
#pragma unroll
      for (int f = 0; f < St::QF; ++f) qf[t][f] = qn[t][f];
  }
  wait_loads<0>();  // the loads behind the last step have ended before the workgroup's LDS is given back
}

// ------------------------------------------------------------------ tile kernel
// The same recurrence with a page's 64 keys a step, and 32 query vectors a wave, on 32x32x16 products: S^T = K Q^T
// of 64 keys, and O^T += V^T P^T.  A workgroup's four waves share a page's K and V in LDS, so that it is
// loaded once for 128 query vectors; two workgroups a compute unit fill each other's waits.
// The matrix cores and the exponentials bound it, and for long calls the power that both draw: 4096 rows behind
// 4000, 64 heads: 759 us, 1.07 PFLOP/s, the matrix cores busy 54 % and the vector units 48 % of the cycles at a clock that
// falls to 1.85 GHz (a plain product of 8192^3 reaches 1.19 PFLOP/s); 2047 rows behind 6001, 32 heads: 231 us.  At head
// dimension 64 a score costs as many vector instructions for half the products: capped scores in a window of 1000,
// four sequences of 700 to 1500 rows, 16 heads: 48 us, 0.34 PFLOP/s, the clock at 2.6 GHz.
constexpr int kTileQ = 128;  // query vectors of a workgroup, 32 a wave

template <int HD, int MOD>
__global__ void __launch_bounds__(256, 2) attend_tile_kernel(AttendArgs a, AttendPlan pl) {
  constexpr int KP = HD / 8, VP = kPage / 8;  // pieces of a K row, of a V^T row
  constexpr int N = kPage * HD / 8;           // pieces of a page's K, and of its V
  // Two buffers of a page's K and V^T.  They are variables of their own, and the loop names them in turn:
  // the compiler then sees that the reads of one need not wait for the direct loads to the other.
  __shared__ __align__(16) u32x4_t even[2 * N];
  __shared__ __align__(16) u32x4_t odd[2 * N];
  __shared__ Range span[4];
  __shared__ int bad_page;

  const Cut cut = cut_of(a, pl);
  if (a.status && blockIdx.x == 0 && (int)threadIdx.x < a.rows.batch) a.status[threadIdx.x] = cut.s.status;
  const TileCut how = tile_cut(a, pl, cut);
  if (blockIdx.x == 0 && threadIdx.x == 0) *pl.how = how;
  Unit u;
  if (!unit_of(a, pl, cut, how, blockIdx.x, u)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int h = lane >> 5, l32 = lane & 31;
  const int nqv = u.rows * pl.group, qv = u.t * kTileQ + 32 * wave + l32;
  const bool valid = qv < nqv;

  const Query q = query_of(a, u, u.kvh, pl.group, qv, nqv);
  Range range{0x7fffffff, 0, 0x7fffffff, 0};
  add_query(range, q, valid);
  range = wave_range(range);
  const int row = u.r0 + (valid ? qv : 0) / pl.group, head = u.kvh * pl.group + (valid ? qv : 0) % pl.group;
  bf16x8_t qf[HD / 16];
  {
    const bf16_t* src = (const bf16_t*)a.q + (int64_t)row * a.qs + (int64_t)head * HD;
#pragma unroll
    for (int f = 0; f < HD / 16; ++f) {
      const u32x4_t x = *(const GLOBAL u32x4_t*)(const GLOBAL bf16_t*)GL(src + 16 * f + 8 * h);
      qf[f] = __builtin_bit_cast(bf16x8_t, valid ? x : u32x4_t{0u, 0u, 0u, 0u});
    }
  }
  if (lane == 0) span[wave] = range;
  if (threadIdx.x == 0) bad_page = 0;
  __syncthreads();
  Range all = range;
  for (int w = 0; w < 4; ++w) {
    all.lo_min = min(all.lo_min, span[w].lo_min);
    all.lo_max = max(all.lo_max, span[w].lo_max);
    all.hi_min = min(all.hi_min, span[w].hi_min);
    all.hi_max = max(all.hi_max, span[w].hi_max);
  }
  all = Range{__builtin_amdgcn_readfirstlane(all.lo_min), __builtin_amdgcn_readfirstlane(all.lo_max),
              __builtin_amdgcn_readfirstlane(all.hi_min), __builtin_amdgcn_readfirstlane(all.hi_max)};
  int pa, pb;
  split_pages(all.lo_min, all.hi_max, u.s, u.splits, pa, pb);

  f32x16_t o[HD / 32];
#pragma unroll
  for (int d = 0; d < HD / 32; ++d) o[d] = f32x16_t{};
  float mrun = -INFINITY, lrun = 0.f;  // the reference of the probabilities, their sum
  // plain scores stay unscaled (their factor is positive) until the exponent's multiply-add
  const float c = MOD ? 1.f : a.scale * kLog2e;
  float slack = 8.f / c;  // of the reference; -inf for a row whose scores are far from 0 (below)
  // a score times its factor, rounded as it is, in no multiply-add
  auto scaled = [&](float s) {
#pragma clang fp contract(off)
    return s * c;
  };
  uint32_t infinite[2][HD / 64] = {};  // per element of o: whether it sums a value infinite upwards, downwards

  // this lane's source pieces of the direct loads: piece i of a page's block goes to LDS slot i, which
  // holds piece (i % P) ^ turn of row i / P
  auto issue = [&](int p, u32x4_t* to) {
    const int page = page_at(a, u.b, p);
    const __amdgpu_buffer_rsrc_t kr = page_rsrc<bf16_t, HD>(a, a.k_pool, page, u.kvh);
    const __amdgpu_buffer_rsrc_t vr = page_rsrc<bf16_t, HD>(a, a.v_pool, page, u.kvh);
#pragma unroll
    for (int i = 0; i < N / 256; ++i) {
      const int base = (i * 4 + wave) * 64, at = base + lane;
      load_lds<0>(kr, to + base, ((at & ~(KP - 1)) + ((at % KP) ^ turn_of<KP>(at / KP))) * 16, 0);
      load_lds<0>(vr, to + N + base, ((at & ~(VP - 1)) + ((at % VP) ^ turn_of<VP>(at / VP))) * 16, 0);
    }
  };

  // K rows are read with bits 3 and 4 of the row exchanged: register r of S^T in lane half h is then
  // key 16 (r / 4 % 2) + 8 (r / 8) + 4 h + r % 4 of its 32, and registers 8 t .. 8 t + 7 are the keys of
  // V columns 8 (2 t + h) .. + 7
  const int krow = (l32 & 7) | ((l32 & 8) << 1) | ((l32 & 16) >> 1);
  const int kturn = turn_of<KP>(krow) ^ h, vturn = turn_of<VP>(l32) ^ h;

  auto page_step = [&](const u32x4_t* K, const u32x4_t* V, int p, bool full) {
    f32x16_t sc[2] = {};
#pragma unroll
    for (int f = 0; f < HD / 16; ++f)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
        sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8_t, K[(32 * kb + krow) * KP + ((2 * f) ^ kturn)]), qf[f], sc[kb], 0, 0, 0);
    // six reads of K ahead of the products: left to itself the compiler waits for each pair (hd 64: 48.5 -> 48.0 us;
    // hd 128 has the same time either way, its clock falls instead)
    constexpr int AHEAD = 6, READS = 0x100, PRODUCTS = 0x8;
    __builtin_amdgcn_sched_group_barrier(READS, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < HD / 8 - AHEAD; ++i) {
      __builtin_amdgcn_sched_group_barrier(PRODUCTS, 1, 0);
      __builtin_amdgcn_sched_group_barrier(READS, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(PRODUCTS, AHEAD, 0);
    int k0 = p * kPage + 4 * h;
    asm volatile("" : "+v"(k0));  // else every key's comparison takes registers of the loop
    auto key_of = [&](int kb, int r) { return k0 + 32 * kb + 16 * (r / 4 % 2) + 8 * (r / 8) + r % 4; };
    bool small = false;
    if constexpr (MOD & kCapped) {  // most calls' scores stay below half of their cap: no transcendentals for it
      float most = 0.f;
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(sc[kb][r]));
      small = __all(most <= pl.fold_limit);
      if (small) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[kb][r] = cap_poly(pl.cap_poly, sc[kb][r], sc[kb][r] * sc[kb][r]);
      }
    }
    if (MOD && !(MOD == kCapped && small)) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          if (!small) sc[kb][r] = capped_of<bf16_t, MOD>(a, pl, sc[kb][r]);
          if constexpr (MOD & kBiased) sc[kb][r] = biased_of(q, sc[kb][r], key_of(kb, r));
        }
    }
    if (!full) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          sc[kb][r] = key_of(kb, r) >= q.lo && key_of(kb, r) < q.hi ? sc[kb][r] : -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sc[kb][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, kWave));
    // The reference follows a row's maximum only when that has outgrown it 2^8 times (a probability is then at most
    // 256 and rounded like any other): else one of 32 rows raises its own on most pages and every sum is scaled
    // (4096 rows behind 4000: 811 -> 781 us).  Each row goes by its own scores, or its rounding would depend on
    // what the others see.
    const bool within = mx <= mrun + slack;
    if (!__all(within)) {
      const float mnew = within ? mrun : fmaxf(mrun, mx);
      const float alpha = mnew == mrun ? 1.f : __builtin_amdgcn_exp2f(scaled(mrun) - scaled(mnew));
      mrun = mnew;
      lrun *= alpha;
#pragma unroll
      for (int d = 0; d < HD / 32; ++d) o[d] *= alpha;
      // The exponent's multiply-add is off by the rounding of the reference: half a unit at 2^24, past all of fp32's
      // exponents from 2^31 on.  A row that far comes here for each page: its scores are rounded like the reference and their
      // differences handed on, in units of the scores, under a reference of 0.
      if constexpr (!MOD) {
        const float from = scaled(mrun), back = 1.f / c;
        const bool far = fabsf(from) >= 0x1p24f && mrun != -INFINITY;
        slack = far ? -INFINITY : 8.f / c;
        if (__any(far)) {
#pragma unroll
          for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) sc[kb][r] = far ? (scaled(sc[kb][r]) - from) * back : sc[kb][r];
        }
      }
    }
    // nothing seen yet: every probability is 2^-inf
    const float ref = mrun == -INFINITY || slack == -INFINITY ? 0.f : scaled(mrun);
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        sc[kb][r] = __builtin_amdgcn_exp2f(fmaf(sc[kb][r], c, -ref));
        sum += sc[kb][r];
      }
    lrun += sum;
    bf16x8_t pb8[2][2];  // the probabilities as an operand: rounded to bf16, as in the stream kernel
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int e = 0; e < 8; ++e) pb8[kb][t][e] = (__bf16)sc[kb][8 * t + e];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < HD / 32; ++d)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
              __builtin_bit_cast(bf16x8_t, V[(32 * d + l32) * VP + ((4 * kb + 2 * t) ^ vturn)]), pb8[kb][t], o[d], 0, 0, 0);
  };
  auto meet = [] {  // a barrier that leaves the next page's loads in flight
    wait_loads<63>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // A page that some row of the workgroup does not see whole may hold anything there: the waves look over a
  // quarter of its V each.  If something is not finite, it is counted for the rows that see it and cleared.
  auto screen = [&](u32x4_t* V, int p) {
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < N / 256; ++i) gather_not_finite<bf16_t>(V[i * 256 + threadIdx.x], bits);
    if (__any((bits & kSigns<bf16_t>) != 0) && lane == 0) bad_page = p + 1;
    meet();
    if (bad_page != p + 1) return;
    int k0 = p * kPage + 4 * h;
    asm volatile("" : "+v"(k0));  // keeps what follows out of the page loop's registers
    bf16x8_t seen[2][2];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int key = k0 + 32 * kb + 16 * (r / 4 % 2) + 8 * (r / 8) + r % 4;
        seen[kb][r / 8][r % 8] = (__bf16)(key >= q.lo && key < q.hi ? 1.f : 0.f);
      }
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int down = 0; down < 2; ++down) {
        f32x16_t n = {};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          __builtin_amdgcn_sched_barrier(0);
          const u32x4_t c = class_of<bf16_t>(V[(32 * d + l32) * VP + ((2 * i) ^ vturn)], down);
          n = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, c), seen[i / 2][i % 2], n, 0, 0, 0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) infinite[down][d / 2] |= (n[r] > 0.f ? 1u : 0u) << (16 * (d % 2) + r);
      }
    meet();
#pragma unroll
    for (int i = 0; i < N / 256; ++i) clean_fragment<bf16_t>(V[i * 256 + threadIdx.x]);
    meet();
  };

  auto step = [&](u32x4_t* cur, u32x4_t* next, int p) {
    wait_loads<0>();               // this wave's part of page p has landed
    __builtin_amdgcn_s_barrier();  // every wave's part, and every wave is done with the other buffer
    asm volatile("" ::: "memory");
    if (p + 1 < pb) issue(p + 1, next);
    const int k0 = p * kPage;
    if (k0 < all.lo_max || k0 + kPage > all.hi_min) screen(cur + N, p);
    if (k0 < range.hi_max && k0 + kPage > range.lo_min)  // else the wave sees none of it
      page_step(cur, cur + N, p, k0 >= range.lo_max && k0 + kPage <= range.hi_min);
  };
  if (pa < pb) issue(pa, even);
  for (int p = pa; p < pb; p += 2) {
    step(even, odd, p);
    if (p + 1 < pb) step(odd, even, p + 1);
  }
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r)
      o[d][r] += infinite_part(infinite[0][d / 2] >> (16 * (d % 2) + r), infinite[1][d / 2] >> (16 * (d % 2) + r));

  const float l = lrun + __shfl_xor(lrun, 32, kWave);
  const float m = scaled(mrun);
  auto part_of = [&](int d, int r) { return f32x4_t{o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]}; };
  if (u.splits > 1) {
    if (!valid) return;
    const size_t slot = (size_t)(u.slot + u.s * a.nkv) * kTileQ + 32 * wave + l32;
    float* const out = pl.o + slot * HD + 4 * h;
#pragma unroll
    for (int d = 0; d < HD / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) *(GLOBAL f32x4_t*)GL(out + 32 * d + 2 * r) = part_of(d, r);
    if (h == 0) *(GLOBAL f32x2_t*)(GL(pl.ml) + slot * 2) = f32x2_t{m, l};
    return;
  }
  // Rows leave through LDS, whole lines a store: a lane's own eight bytes of 32 rows at a time keep the address
  // unit busy for 2 us.  The wave's 32 rows lie where page buffers were, pieces exchanged as those of K.
  if (valid && a.lse && h == 0) GL(a.lse)[(int64_t)row * a.nq + head] = lse_of(m, l);
  meet();  // every wave is done with the pages
  u32x4_t* const rows = even + wave * (32 * KP);
  long long* const ends = (long long*)odd + wave * 32;
  const float f = factor_of(l);
#pragma unroll
  for (int d = 0; d < HD / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      const f32x4_t x = part_of(d, r) * f;
      ((u32x2_t*)&rows[l32 * KP + ((4 * d + r / 4) ^ turn_of<KP>(l32))])[h] =
          u32x2_t{(uint32_t)f2bf(x[0]) | ((uint32_t)f2bf(x[1]) << 16), (uint32_t)f2bf(x[2]) | ((uint32_t)f2bf(x[3]) << 16)};
    }
  if (h == 0) ends[l32] = valid ? (int64_t)row * a.os + (int64_t)head * HD : -1;
  wait_loads<63>();
#pragma unroll
  for (int i = 0; i < 32 * KP / 64; ++i) {
    const int r = i * (64 / KP) + lane / KP, piece = lane % KP;
    const long long at = ends[r];
    const u32x4_t x = rows[r * KP + (piece ^ turn_of<KP>(r))];
    if (at >= 0) *(GLOBAL u32x4_t*)(GLOBAL bf16_t*)GL((bf16_t*)a.out + at + 8 * piece) = x;
  }
}

// ------------------------------------------------------------------ merge kernels
// Bound by the chain of loads that finds a part, and by the sums: at most 1024 slots of 32 x HD (16.8 MB at 128) of the
// stream kernel, 512 of 128 x HD (33.6 MB) of the tile kernel.  Two sequences of four tokens behind 100K to 131K: 8.7 MB in
// 9.3 us; nothing to join: 4.2.
// The stream kernel's chains: blockIdx.x + 1 is a share whose start lies inside a chain; the first such share
// of a chain joins its parts.  blockIdx.y: the query vectors in lots of 1024 / HD, four dimensions a lane;
// blockIdx.z: the kv head.
template <typename T, int HD>
__global__ void __launch_bounds__(256) attend_merge_line_kernel(AttendArgs a, AttendPlan pl) {
  const Line l = line_of(a, pl);
  const int w = blockIdx.x + 1, g = w * l.share, kvh = blockIdx.z;
  const Part p = part_at(l, g);
  if (!p.len || p.at == 0 || p.at > l.share) return;
  const int in_tile = blockIdx.y * (1024 / HD) + threadIdx.x / (HD / 4), d = threadIdx.x % (HD / 4) * 4;
  const int qv = p.t * pl.tile + in_tile;
  if (in_tile >= pl.tile || qv >= p.rows * pl.group) return;
  const int parts = (g - p.at + p.chain - 1) / l.share - (w - 1) + 1;
  join_parts<T, HD, false>(a, pl, parts, [&](int i) { return slot_of(w - 1 + i, i == 0, a.nkv, kvh); }, in_tile, d,
                    p.r0 + qv / pl.group, kvh * pl.group + qv % pl.group);
}

// The tile kernel's cut tiles: a workgroup takes 1024 / HD query vectors of one at a time, and leaves at once where
// nothing was cut.
constexpr int kMergeGroups = 1024;
template <int HD>
__global__ void __launch_bounds__(256) attend_merge_tiles_kernel(AttendArgs a, AttendPlan pl) {
  constexpr int LOT = 1024 / HD, LOTS = kTileQ / LOT;
  const TileCut how = *pl.how;
  if (how.none()) return;
  const Cut c = cut_of(a, pl);
  const bool by_length = how.pps != TileCut::kNoLimit;  // then tiles of long walks are cut, else those from `whole` on
  const int splits = by_length ? max(1, (c.walk + how.pps - 1) / how.pps) : how.rest;
  const int mine = by_length && splits == 1 ? 0 : c.tiles;
  const int sum = wave_scan_sum(mine), slots = wave_scan_sum(mine * splits), skip = by_length ? 0 : how.whole;
  const int items = (__builtin_amdgcn_readlane(sum, 63) - skip) * a.nkv * LOTS;
  for (int i = blockIdx.x; i < items; i += kMergeGroups) {
    const int tile = i / LOTS / a.nkv, kvh = i / LOTS % a.nkv, at = tile + skip;
    const int b = __builtin_amdgcn_readfirstlane(__ffsll((long long)__ballot(sum > at)) - 1);
    const int local = at - __builtin_amdgcn_readlane(sum - mine, b), parts = __builtin_amdgcn_readlane(splits, b);
    const int slot = (by_length ? __builtin_amdgcn_readlane(slots - mine * splits, b) + local * parts : tile * parts) * a.nkv + kvh;
    const int t = __builtin_amdgcn_readlane(c.tiles, b) - 1 - local;
    const int in_tile = i % LOTS * LOT + threadIdx.x / (HD / 4), d = threadIdx.x % (HD / 4) * 4, qv = t * kTileQ + in_tile;
    if (qv < __builtin_amdgcn_readlane(c.s.rows, b) * pl.group)
      join_parts<bf16_t, HD, false>(a, pl, parts, [&](int k) { return slot + k * a.nkv; }, in_tile, d,
                                    __builtin_amdgcn_readlane(c.s.r0, b) + qv / pl.group, kvh * pl.group + qv % pl.group);
  }
}

// ------------------------------------------------------------------ host
namespace {
// The workspace begins with the tile kernel's cut and the arrival counters, which stay zero between calls: they lie
// apart from the partial results, wherever those begin and end under a call's bounds.
constexpr int kMostUnits = 1024;
constexpr size_t kHead = 256 + 4 * kMostUnits;
constexpr int kLongF32 = 512;  // query vectors
struct HostPlan {
  bool tiles;       // the tile kernel
  bool join;        // the stream kernel joins cut chains itself
  int tile, target, least, slots;
  long long units;  // workgroups of the main kernel at most
  long long walk;   // pages of its tiles, as the kernels count them in 32 bits
};

// The stream kernel takes calls of at most 32 query vectors per sequence and kv head, and fp32.
HostPlan host_plan(int dtype, int hd, int nq, int nkv, int batch, int max_rows, int max_rows_per_seq, int max_ctx) {
  HostPlan p{};
  const long long group = nq / nkv, per_seq = max_rows_per_seq * group;
  p.tiles = dtype == LSV_DTYPE_BF16 && per_seq > 32;
  // fp32 is bound by its matrix instructions: two tiles a wave pay from long chunks on, at head dimension 128
  // (300 rows behind 3000, group 4: 65 us against 70; 8 rows: 24 against 20; head dimension 64: 41 against 29)
  const bool two = dtype == LSV_DTYPE_BF16 ? per_seq > 16 : hd == 128 && per_seq > kLongF32;
  p.tile = p.tiles ? kTileQ : two ? 32 : 16;
  p.target = p.tiles || hd == 128 ? 512 : 1024;  // the workgroups that the chip holds at once
  p.least = dtype == LSV_DTYPE_BF16 ? kStreamWaves : 1;  // a step for each wave
  // tiles of sequences that share max_rows rows, each sequence's last one begun
  const long long seqs = batch < max_rows ? batch : max_rows, pages = (max_ctx + kPage - 1) / kPage;
  const long long by_rows = max_rows * group / p.tile + seqs, by_seq = seqs * ((per_seq + p.tile - 1) / p.tile);
  const long long tiles = by_rows < by_seq ? by_rows : by_seq;
  const long long chain = p.tiles ? pages * nkv : (pages + p.least - 1) / p.least * p.least;
  p.walk = tiles * chain;
  if (p.tiles) {
    const long long most_splits = (pages + 3) / 4, held = p.target;  // four pages a split at least, one round of splits
    p.slots = (int)(most_splits == 1 ? 0 : tiles * nkv * most_splits < held ? tiles * nkv * most_splits : held);
    p.units = tiles * nkv + p.slots;  // unsplit sequences have one unit a tile; the others' are bounded by the slots
  } else {
    const long long shares = tiles * ((pages + p.least - 1) / p.least), fill = p.target / nkv > 1 ? p.target / nkv : 1;
    p.target = (int)(shares < fill ? shares : fill);
    p.units = (long long)p.target * nkv;
    p.slots = (int)(p.target > 1 ? 2 * p.units : 0);  // a share cuts two chains at most
    // few query vectors: the last workgroup of a cut chain joins it, which spares a launch (one token behind 2,047
    // positions: 12.4 -> 11.3 us); with 32 of them it has too much to read (128K contexts: 161 -> 201 us)
    p.join = p.slots && per_seq <= 8 && p.units <= kMostUnits;
  }
  return p;
}
size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
}  // namespace

size_t attend_workspace_bytes(const Shape& s, int batch, int max_rows, int max_rows_per_seq, int max_ctx) {
  // fewer rows per sequence may take smaller tiles and more partial results: the largest of the kinds
  const int group = s.nq / s.nkv;
  size_t most = 0;
  for (const int rows : {16 / group, 32 / group, kLongF32 / group, max_rows_per_seq}) {
    if (rows < 1 || rows > max_rows_per_seq) continue;
    const HostPlan p = host_plan(s.dtype, s.hd, s.nq, s.nkv, batch, max_rows, rows, max_ctx);
    const size_t n = kHead + align256((size_t)p.slots * p.tile * s.hd * 4) + align256((size_t)p.slots * p.tile * 8);
    most = n > most ? n : most;
  }
  return most;
}

template <typename T, int HD, int MOD>
static void launch_main(const AttendArgs& a, const HostPlan& p, const AttendPlan& pl, hipStream_t st) {
  const dim3 units((unsigned)p.units);
  if constexpr (sizeof(T) == 2) {
    if (p.tiles) hipLaunchKernelGGL((attend_tile_kernel<HD, MOD>), units, dim3(256), 0, st, a, pl);
  }
  if constexpr (sizeof(T) == 2 || HD == 128) {  // as in host_plan
    if (p.tile == 32) hipLaunchKernelGGL((attend_stream_kernel<T, HD, 2, MOD>), units, dim3(64 * kStreamWaves), 0, st, a, pl);
  }
  if (p.tile == 16) hipLaunchKernelGGL((attend_stream_kernel<T, HD, 1, MOD>), units, dim3(64 * kStreamWaves), 0, st, a, pl);
}

template <typename T, int HD>
static int launch_hd(const AttendArgs& a, const HostPlan& p, const AttendPlan& pl, hipStream_t st) {
  // the tile kernel's plain scores need a positive factor; another goes with a bias of no slopes
  const int mod = (a.softcap > 0.f ? kCapped : 0) | (a.slopes || !(a.scale > 0.f) ? kBiased : 0);
  if (mod == kPlain) launch_main<T, HD, kPlain>(a, p, pl, st);
  else if (mod == kCapped) launch_main<T, HD, kCapped>(a, p, pl, st);
  else if (mod == kBiased) launch_main<T, HD, kBiased>(a, p, pl, st);
  else launch_main<T, HD, kCapped | kBiased>(a, p, pl, st);
  if (p.slots && !p.join) {
    const int lot = 1024 / HD;
    const unsigned lots = (unsigned)((p.tile + lot - 1) / lot);
    if (!p.tiles)
      hipLaunchKernelGGL((attend_merge_line_kernel<T, HD>), dim3((unsigned)p.target - 1, lots, (unsigned)a.nkv), dim3(256), 0, st, a, pl);
    else if constexpr (sizeof(T) == 2)
      hipLaunchKernelGGL((attend_merge_tiles_kernel<HD>), dim3(kMergeGroups), dim3(256), 0, st, a, pl);
  }
  return hipGetLastError() == hipSuccess ? LSV_OK : LSV_ERR_HIP;
}

bool attend_fits(const Shape& s, int batch, int max_rows, int max_rows_per_seq, int max_ctx) {
  const HostPlan p = host_plan(s.dtype, s.hd, s.nq, s.nkv, batch, max_rows, max_rows_per_seq, max_ctx);
  return p.walk < 1ll << 30 && p.units < 1ll << 24 && (long long)max_rows * (s.nq / s.nkv) < 1ll << 30;
}

int launch_attend(int dtype, const AttendArgs& a, void* ws, hipStream_t st) {
  const HostPlan p = host_plan(dtype, a.hd, a.nq, a.nkv, a.rows.batch, a.rows.max_rows, a.rows.max_rows_per_seq, a.rows.max_ctx);
  AttendPlan pl{};
  pl.group = a.nq / a.nkv;
  pl.tile = p.tile;
  pl.target = p.target;
  pl.least = p.least;
  pl.slots = p.slots;
  if (a.softcap > 0.f) {
    const double fit[4] = {0.999999456, -0.33326318, 0.131902968, -0.0444022301};
    const double ratio = (double)a.scale / a.softcap;
    auto near_one = [](double x, double far) { return fabs(x) >= 1.0 / far && fabs(x) <= far; };
    const bool fold = near_one(ratio, 1e5) && near_one(a.scale, 1e7);
    for (int i = 0; i < 4; ++i) pl.cap_poly[i] = (float)(fit[i] * a.scale * kLog2e * (fold ? pow(ratio, 2 * i) : 1.0));
    pl.cap_ratio = (float)ratio;
    pl.poly_ratio = fold ? 1.f : pl.cap_ratio;
    pl.cap_limit = (float)fmin(0.5 / fabs(ratio), 1e30);  // infinities are above it
    pl.fold_limit = fold ? pl.cap_limit : -1.f;
  }
  pl.how = (TileCut*)ws;
  pl.parts = p.join ? (int*)((char*)ws + 256) : nullptr;
  pl.o = (float*)((char*)ws + kHead);
  pl.ml = (float*)((char*)pl.o + align256((size_t)p.slots * p.tile * a.hd * 4));
  if (dtype == LSV_DTYPE_BF16)
    return a.hd == 128 ? launch_hd<bf16_t, 128>(a, p, pl, st) : launch_hd<bf16_t, 64>(a, p, pl, st);
  return a.hd == 128 ? launch_hd<float, 128>(a, p, pl, st) : launch_hd<float, 64>(a, p, pl, st);
}

}  // namespace lsv
