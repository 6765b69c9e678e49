// Attention of a step's rows over a paged cache (gfx950).
//
// A row r of sequence s at position p sees a key at position j of the cache if
//   j < len(s),  (j <= p or j < prefix(s)),  p - j < window,  j >= first(r),
// and with a tree mask, of the keys that this step appended (from ctx on),
// those of its mask's bits, which stand at the positions of their depth.  With
//   x = scale * q.k,  x = cap * tanh(x / cap),  x = x - slope(h) * |p - j|
// the row's output is sum_j exp(x_j) v_j / sum_j exp(x_j), 0 where it sees none.
//
// Scores, their maximum, sums and outputs are 32-bit; the weights are rounded to
// the cache's type for the product with V (an fp16 weight is scaled by 2^7, so
// that weights down to 2^-21 of the largest keep all its bits), not for the sum.
//
// The G query heads of a key head and the rows of a sequence are one list of
// columns, column m = row m / G, head m % G: the products are transposed,
//   S^T = K Q^T (keys x columns),  O^T = V^T P^T (head dim x columns),
// so that a lane holds one column: its maximum, sum and rescaling need no other
// lane but the one 32 away, and S^T's accumulators are, rounded, P^T's operand
// as they lie (a 32x32 accumulator's lane has keys 8i + 4h + 0..3; V's operand
// takes its keys in that order, by LDS reads that transpose).
//
// K and V go from the cache to LDS without registers (global_load_lds), in
// tiles whose 16-byte pieces are XOR-swizzled by key for both kinds of read.
#include "common.h"
#include "kernels.h"
#include "rows.h"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace hvd {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kFar = 4096.f;   // larger maxima are taken off the scores themselves (base 2)
constexpr float kCancels = 64.f;
constexpr int kNoKey = 0x7fffffff;

template <bool BF16>
struct Half;
template <>
struct Half<false> {
  static constexpr float kShift = 7.f;
  static constexpr float kLazy = 8.f;  // the running maximum may lag by this (base 2): weights stay below 2^16
  static constexpr uint32_t kInf = 0x04000400u;  // 0x8000 - the exponent of infinities and NaNs
  __device__ static f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
  __device__ static uint16_t bits(float v) { return f2h(v); }
};
template <>
struct Half<true> {
  static constexpr float kShift = 0.f;
  // Rounding is as fine at any scale, but a largest weight of 1 has none: packed prompts of
  // 256-wide heads with a bias 172 us and off by 2.2e-3, with 8 177 and 2.1e-3, with 0 191 and 1.9e-3.
  static constexpr float kLazy = 16.f;
  static constexpr uint32_t kInf = 0x00800080u;
  __device__ static f32x16 mfma(s16x8 a, s16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
  __device__ static uint16_t bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
};

// A value of the lane 32 away.
__device__ __forceinline__ float other_half_max(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

template <int CTRL>
__device__ __forceinline__ int dpp(int v) {
  return __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, false);
}
// f over all lanes of a wave (one that does not mind a value twice)
template <class F>
__device__ __forceinline__ int wave_all(int v, F f) {
  v = f(v, dpp<0xB1>(v));
  v = f(v, dpp<0x4E>(v));
  v = f(v, dpp<0x141>(v));
  v = f(v, dpp<0x140>(v));
  const auto x = __builtin_amdgcn_permlane16_swap((uint32_t)v, (uint32_t)v, false, false);
  v = f((int)x[0], (int)x[1]);
  const auto y = __builtin_amdgcn_permlane32_swap((uint32_t)v, (uint32_t)v, false, false);
  return __builtin_amdgcn_readfirstlane(f((int)y[0], (int)y[1]));
}

// How the work is cut: columns per tile; workgroups that the card holds at once, or
// 0: no tile's keys are split; the fewest keys of a split; the items there is
// room for.
struct Cut {
  int cols, slots, min_chunk, items;
  float item, split;  // what they cost, in keys
};

// One item: columns [col0, col0 + cols) of sequence s over the keys of split
// `split` of its tile.
struct Item {
  int s, row0, n, ctx, len, tile, split, splits, chunk;
};

// A sequence's rows, context, keys and tiles; how many keys one of its tiles spans at
// most, and in the mean (about).
struct Load {
  int row0, n, ctx, len, tiles, range;
  float mean;
};
__device__ __forceinline__ Load seq_load(const AttendArgs& a, const Cut& c, int s) {
  Load d{};
  if (s > a.b.S) return d;
  int e, len = 0;
  seq_rows(a.b, s, d.row0, e);
  if (s < a.b.S) len = a.b.lengths[s];
  d.n = e - d.row0;
  d.ctx = len - d.n;
  d.len = min(max(len, 0), a.b.P << a.page_shift);
  const int G = a.Hq / a.H;
  d.tiles = (int)(((int64_t)d.n * G + c.cols - 1) / c.cols);
  const bool chain = !a.b.tree && !a.prefix;
  const int rows = chain ? min(d.n, (c.cols + G - 1) / G + 1) : d.n;  // behind the first one's last key
  d.range = d.len;
  if (a.window > 0 && a.window < kNoKey - rows) d.range = min(d.len, a.window + rows);
  d.mean = (float)d.range;
  // (a chain's first tiles end before its last keys)
  if (chain && d.range == d.len && d.tiles > 1) d.mean = fmaxf((float)d.len - 0.5f * (float)d.n, 0.5f * (float)d.len);
  return d;
}

// A tile of up to `range` keys in even splits of at most `chunk`.
__device__ __forceinline__ int splits_of(int range, int chunk) { return max(1, (int)(((int64_t)range + 63 + chunk - 1) / chunk)); }
__device__ __forceinline__ int even_chunk(int range, int splits) { return (int)((((int64_t)range + 63 + splits - 1) / splits + 63) & ~63ll); }

// The most keys of one split, the same in every workgroup.  Up to 63 sequences: the
// best of 16 lengths, a lane each and the first so long that nothing is split, by
// when the last workgroup would be done -- its items in rounds of equal length or
// one after the other, whichever is sooner.  (8 trees over 8192 keys 162 us when
// it came, with 3 items for 2 slots throughout 178; one tree over 16384 keys 36 and 49.)
// The other 15 are 0.43 to 2.25 of a slot's share of the keys, in even steps: from more
// than two rounds of items to less than half of one.
constexpr int kWhole = 1 << 30;
constexpr float kStore = 60.f;  // keys' time that the last stores of a split take (with 0 all cases timed stayed within 1%)
__device__ __forceinline__ int chunk_of(const AttendArgs& a, const Cut& c, const Load& first) {
  if (c.slots == 0) return kWhole;
  const int lane = threadIdx.x & 63;
  const float slots = (float)c.slots / (float)a.H;
  float worst = 0.f, total = 0.f;
  int count = 0, longest = 0;
  for (int s = 0; s <= a.b.S; s += 64) {
    const Load d = s == 0 ? first : seq_load(a, c, s + lane);
    worst += (float)d.tiles * (float)d.range;
    total += (float)d.tiles * d.mean;
    count += d.tiles;
    longest = max(longest, d.tiles > 0 ? d.range : 0);
  }
  worst = wave_sum(worst);
  // 3 items for 2 slots: there is room for them, whatever the lengths
  const int usual = __builtin_amdgcn_readfirstlane(max(((int)fminf(worst / (1.5f * slots), 1.0e9f) + 127) & ~63, c.min_chunk));
  if (a.b.S >= 64) {  // whole where the tiles fill the card and none is much longer than a slot's share
    for (int o = 32; o > 0; o >>= 1) {
      count += __shfl_xor(count, o);
      longest = max(longest, __shfl_xor(longest, o));
    }
    return (float)count * 8.f >= slots * 7.f && (float)longest * slots <= 1.2f * worst ? kWhole : usual;
  }
  // long tiles that are few: as many splits as there may be (one token over 2048 keys
  // 14.6 -> 12.0 us: what follows is a long way through instructions not fetched yet)
  if (usual == c.min_chunk && !__builtin_amdgcn_ballot_w64(first.range > 0 && first.range < 8 * c.min_chunk)) return usual;
  const float share = wave_sum(total) / slots;
  const int pick = lane & 15;
  const int mine = pick == 0 ? kWhole : max(((int)fminf(share * (0.3f + 0.13f * (float)pick), 1.0e9f) + 127) & ~63, c.min_chunk);
  const float inv = 1.f / (float)mine;
  float items = 0.f, most = 0.f;
  for (int s = 0; s <= a.b.S; ++s) {
    const int tiles = __builtin_amdgcn_readlane(first.tiles, s);
    if (tiles == 0) continue;
    const float range = (float)(__builtin_amdgcn_readlane(first.range, s) + 63);
    const float mean = 63.f + __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(first.mean), s));
    const float splits = fmaxf(1.f, ceilf(range * inv - 0.001f)), each = range * __builtin_amdgcn_rcpf(splits);
    items += (float)tiles * (mean < range ? fminf(splits, mean * __builtin_amdgcn_rcpf(each) + 0.5f) : splits);
    most = fmaxf(most, each);
  }
  const float turns = items / slots, path = most + c.item + (pick ? kStore : 0.f);
  float end = share + turns * c.item + (turns > 1.f ? most : 0.f);
  end = fmaxf(fminf(end, ceilf(turns - 0.001f) * path), path) + (pick ? turns * c.split : 0.f);
  // Whole tiles unless splits are clearly sooner: with 1 in place of both factors 4
  // prompts 148 -> 188 us and packed prompts of documents 173 -> 206.  Documents' tiles are
  // shorter than their range, by how much only their rows tell: with 0.95 they are split
  // (207 us); other batches with a `first` came out the same with either.
  if (pick == 0) end *= a.first ? 0.7f : 0.95f;
  const int best = wave_all((int)((__float_as_uint(end) & ~15u) | pick), [](int x, int y) { return x < y ? x : y; }) & 15;
  const int chunk = __builtin_amdgcn_readlane(mine, best);
  const float all = wave_sum((float)first.tiles * (float)splits_of(first.range, chunk));
  return all <= (float)c.items ? chunk : usual;
}

// Item number `idx`; false past the last one.
__device__ __forceinline__ bool find_item(const AttendArgs& a, const Cut& c, int idx, Item& it) {
  const int lane = threadIdx.x & 63;
  const Load first = seq_load(a, c, lane);
  const int chunk = chunk_of(a, c, first);
  int base = 0;
  for (int s = 0; s <= a.b.S; s += 64) {
    const Load d = s == 0 ? first : seq_load(a, c, s + lane);
    const int splits = splits_of(d.range, chunk), mine = d.tiles * splits;
    const int upto = wave_scan(mine);
    const uint64_t past = __builtin_amdgcn_ballot_w64(base + upto > idx);
    if (past) {
      const int l = __builtin_ctzll(past);
      it.s = s + l;
      it.row0 = __builtin_amdgcn_readlane(d.row0, l);
      it.n = __builtin_amdgcn_readlane(d.n, l);
      it.ctx = __builtin_amdgcn_readlane(d.ctx, l);
      it.len = __builtin_amdgcn_readlane(d.len, l);
      it.splits = __builtin_amdgcn_readlane(splits, l);
      const int at = idx - base - __builtin_amdgcn_readlane(upto - mine, l);
      // the last tiles of a sequence see the most keys: they go first
      const int t = at / it.splits;
      it.tile = __builtin_amdgcn_readlane(d.tiles, l) - 1 - t;
      it.split = at - t * it.splits;
      it.chunk = even_chunk(__builtin_amdgcn_readlane(d.range, l), it.splits);
      return true;
    }
    base += __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// What a column sees: keys [lo, hi), and of the keys from ctx on (tree only)
// those of `see`.
struct Column {
  int row, head;  // row of the batch (-1: none)
  int pos, lo, hi, ctx;
  uint64_t path;  // the tree mask
  uint64_t see;   // its bits that window, first and len leave
};
__device__ __forceinline__ Column column_of(const AttendArgs& a, const Item& it, int m, int head0) {
  Column c;
  const int G = a.Hq / a.H;
  const int i = m / G;
  const bool on = i < it.n, in_seq = it.s < a.b.S;
  c.row = on ? it.row0 + i : -1;
  c.head = head0 + (m - i * G);
  c.ctx = it.ctx;
  c.path = c.see = 0;
  c.pos = c.ctx + i;
  const int first = on && a.first ? max(a.first[c.row], 0) : 0;
  if (a.b.tree) {
    if (on && in_seq) c.path = (uint64_t)a.b.tree[c.row];
    const int depth = __builtin_popcountll(c.path);
    c.pos = c.ctx + depth - 1;
    c.see = c.path;
    if (a.window > 0)
      for (int drop = depth - a.window; drop > 0; --drop) c.see &= c.see - 1;  // positions rise with the bits
    const int64_t from = max((int64_t)first - c.ctx, (int64_t)-c.ctx), to = (int64_t)it.len - c.ctx;
    if (from > 0) c.see = from < 64 ? c.see >> from << from : 0;
    if (to < 64) c.see = to > 0 ? c.see & ((1ull << to) - 1) : 0;
  }
  c.lo = first;
  if (a.window > 0) c.lo = (int)max((int64_t)c.lo, (int64_t)c.pos - a.window + 1);
  c.hi = c.pos + 1;
  if (a.b.tree) c.hi = c.ctx;
  else if (a.prefix && in_seq) c.hi = max(c.hi, a.prefix[it.s]);
  c.hi = min(c.hi, it.len);
  if (!on || !in_seq || c.hi <= c.lo) c.hi = c.lo = 0;
  if (!on || !in_seq) c.see = 0;
  return c;
}

// The keys that some column of a wave sees lie in [lo, hi); all columns (that
// exist) see all keys of [all_lo, all_hi).
struct Span {
  int lo, hi, all_lo, all_hi;
};
__device__ __forceinline__ Span span_of(const AttendArgs& a, const Column& c) {
  const auto least = [](int x, int y) { return x < y ? x : y; };
  const auto most = [](int x, int y) { return x > y ? x : y; };
  int lo = c.hi > c.lo ? c.lo : kNoKey, hi = c.hi;
  if (c.see) {
    lo = min(lo, c.ctx + __builtin_ctzll(c.see));
    hi = max(hi, c.ctx + 64 - __builtin_clzll(c.see));
  }
  Span s;
  s.lo = wave_all(lo, least);
  s.hi = wave_all(hi, most);
  s.all_lo = wave_all(c.row >= 0 ? c.lo : 0, most);
  s.all_hi = wave_all(c.row >= 0 ? c.hi : kNoKey, least);
  return s;
}

template <int DHP>
struct Geo {
  static constexpr int CH = DHP / 8;   // 16-byte pieces of a key
  static constexpr int KPI = 64 / CH;  // keys of one copy instruction
  static constexpr int ROW = DHP * 2;  // bytes of a key
  // Piece c of key k lies at piece c ^ swz(k): four successive keys (a transposing
  // read takes 64 bytes of each) and sixteen keys (a row read takes one piece
  // of each) fall on different banks; with 8 pieces two keys share 256 bytes.
  __device__ static constexpr int swz(int k) {
    return CH == 8 ? ((k >> 1 & 1) << 2) | (k >> 2 & 3) : ((k & 3) << 2) | (k >> 2 & 3);
  }
};

// Where 64 groups of 16 keys lie in the cache, one per lane (group l starts at key
// `key` of lane l): the addresses of their first keys and values of one head, and
// which of them have a page -- none past `end`, and none that the cache does not
// have.
struct Pages {
  uint32_t k_lo, k_hi, v_lo, v_hi;
  uint64_t has;
};
__device__ __forceinline__ Pages pages_of(const AttendArgs& a, const int32_t* table, int kvh, int key, int end) {
  const int pi = key >> a.page_shift, tok = key & ((1 << a.page_shift) - 1);
  const int p = key < end && pi < a.b.P ? table[pi] : -1;
  const bool in = (unsigned)p < (unsigned)a.n_pages;
  const uint64_t k = (uint64_t)((const uint16_t*)a.k.p + kvh * a.k.head + (in ? p * a.k.page + tok * a.k.tok : 0));
  const uint64_t v = (uint64_t)((const uint16_t*)a.v.p + kvh * a.v.head + (in ? p * a.v.page + tok * a.v.tok : 0));
  return Pages{(uint32_t)k, (uint32_t)(k >> 32), (uint32_t)v, (uint32_t)(v >> 32), __builtin_amdgcn_ballot_w64(in)};
}
__device__ __forceinline__ const char* address_of(uint32_t lo, uint32_t hi, int lane) {
  return (const char*)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(hi, lane) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, lane));
}

// Which of a tile's NK keys have a page: group g0 is the tile's first.
template <int NK>
__device__ __forceinline__ uint64_t good_keys(uint64_t has, int g0, int key0, int end) {
  constexpr uint64_t kAll = NK == 64 ? ~0ull : (1ull << NK) - 1, kGroups = (1 << (NK / 16)) - 1;
  const uint64_t mine = has >> g0 & kGroups;
  if (mine == kGroups && key0 + NK <= end) return kAll;
  uint64_t good = 0;
#pragma unroll
  for (int g = 0; g < NK / 16; ++g) good |= mine >> g & 1 ? 0xffffull << (16 * g) : 0;
  const int n = end - key0;
  return n >= NK ? good : n > 0 ? good & ((1ull << n) - 1) : 0;
}

// The same value, which the compiler takes for a new one each time: addresses built
// from it are not kept in registers (which the accumulators need) over the loop.
__device__ __forceinline__ int afresh(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// 16 bytes per lane from base + off (bytes; a wave-uniform base, 32 bits per lane)
// to LDS at dst + 16 * lane.  In assembly because the compiler, which cannot tell
// the tiles apart, would have a transposing read of one tile wait for the
// copies to the other; the waits are the callers'.  (m0 holds the place: an operand, so
// that the compiler writes it and knows of it; it takes a cycle to arrive.)
__device__ __forceinline__ void copy_to_lds(const char* base, uint32_t off, uint32_t dst) {
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"{m0}"(dst), "v"(off), "s"(base) : "memory");
}

// Copies of N * KPI keys of a tile to LDS, K and V: whole groups of 16, or a part
// of one.  KEEP: each copy's place is kept in registers, where there are some left.
template <int DHP, int N, bool KEEP>
struct Copies {
  using G = Geo<DHP>;
  static constexpr int PER = N * G::KPI < 16 ? N : 16 / G::KPI;  // copies per group
  int place;  // of this lane: its piece of the first key, in bytes
  uint32_t k_off[KEEP ? PER : 1], v_off[KEEP ? PER : 1];  // from the first key's place

  // k0: the first key's place in the tile (of a group, or of this part of one)
  __device__ __forceinline__ void init(const AttendArgs& a, int k0) {
    const int lane = threadIdx.x & 63, kk = lane / G::CH;
    place = ((lane % G::CH) ^ G::swz(k0 + kk)) * 16;
#pragma unroll
    for (int i = 0; i < (KEEP ? PER : 1); ++i) {
      k_off[i] = 2u * (uint32_t)((i * G::KPI + kk) * (int)a.k.tok) + (KEEP ? piece(i) : 0);
      v_off[i] = 2u * (uint32_t)((i * G::KPI + kk) * (int)a.v.tok) + (KEEP ? piece(i) : 0);
    }
  }
  // The lane's piece in copy i of a group (a key's swizzle is linear in its bits).
  __device__ __forceinline__ uint32_t piece(int i) const {
    return (uint32_t)((KEEP ? place : afresh(place)) ^ (G::swz(i * G::KPI) * 16));
  }
  // Copy i of keys or values: from `from`, a group's first key.
  __device__ __forceinline__ void copy(int i, const char* from, int64_t tok, const uint32_t* off, uint32_t to) const {
    if constexpr (KEEP) copy_to_lds(from, off[i], to);
    else copy_to_lds(from + 2u * i * G::KPI * (uint32_t)tok, off[0] + piece(i), to);
  }

  // The tile begins with key0; group g0 of `pg` is its first, `good` its keys that
  // have a page.  Returns false if fewer than N copies (of each) were asked for.
  template <bool K = true, bool V = true>
  __device__ __forceinline__ bool issue(const AttendArgs& a, int k0, const Pages& pg, int g0,
                                        uint64_t good, unsigned char* smem, uint32_t lk, uint32_t lv) const {
    constexpr uint64_t kMine = N * G::KPI >= 64 ? ~0ull : (1ull << (N * G::KPI & 63)) - 1;
    const bool full = (good >> k0 & kMine) == kMine, whole = full && a.D == DHP;
    const uint32_t base = (uint32_t)(uintptr_t)(lds_void*)smem;
#pragma unroll
    for (int f = 0; f < N; f += PER) {
      const int first = k0 + f * G::KPI, g = g0 + (first >> 4);  // wave-uniform
      const uint32_t in_group = PER * G::KPI < 16 ? first & 15 : 0;
      const char* kp = address_of(pg.k_lo, pg.k_hi, g) + 2u * in_group * (uint32_t)a.k.tok;
      const char* vp = address_of(pg.v_lo, pg.v_hi, g) + 2u * in_group * (uint32_t)a.v.tok;
      if (whole) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const uint32_t at = (first + i * G::KPI) * G::ROW;
          if constexpr (K) copy(i, kp, a.k.tok, k_off, base + lk + at);
          if constexpr (V) copy(i, vp, a.v.tok, v_off, base + lv + at);
        }
      } else {
        // pieces past the head dimension stay zero, keys without a page become it
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const uint32_t at = (first + i * G::KPI) * G::ROW;
          const bool in = (int)piece(i) < 2 * a.D, ok = good >> (first + i * G::KPI + lane / G::CH) & 1;
          if (in && ok) {
            if constexpr (K) copy(i, kp, a.k.tok, k_off, base + lk + at);
            if constexpr (V) copy(i, vp, a.v.tok, v_off, base + lv + at);
          }
          if (in && !ok) {
            if constexpr (K) *(uint4*)(smem + lk + at + lane * 16) = uint4{0, 0, 0, 0};
            if constexpr (V) *(uint4*)(smem + lv + at + lane * 16) = uint4{0, 0, 0, 0};
          }
        }
      }
    }
    if (!full) __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0): the zeros are there before the barrier
    return full;  // (a narrower head's copies have lanes with a piece each all the same)
  }
};

__device__ __forceinline__ s16x8 join4(s16x4 x, s16x4 y) {
  return s16x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// The lowest n bits (none for n <= 0, all for n >= 64).
__device__ __forceinline__ uint64_t below(int n) { return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1; }

// The state of a wave's 32 columns; NB blocks of 32 keys per step.  TURN: scores
// are made exponents one by one (a cap, a bias, a scale that is not positive).
template <int DHP, bool BF16, int NB, bool TURN>
struct Wave {
  using G = Geo<DHP>;
  using H = Half<BF16>;
  s16x8 q[DHP / 16];
  f32x16 o[DHP / 32];
  float m, l;   // of the scores times `c`; l of this lane's half of the keys
  float c;      // the scores' factor to base-2 exponents

  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  }
  __device__ __forceinline__ void init(const AttendArgs& a, const Column& col, int h) {
    reset();
    c = TURN ? 1.f : a.scale * kLog2e;
    const uint16_t* src = (const uint16_t*)a.q + (int64_t)max(col.row, 0) * a.q_row + (col.row >= 0 ? col.head : 0) * a.q_head;
#pragma unroll
    for (int s = 0; s < DHP / 16; ++s) {
      const int d = s * 16 + h * 8;
      q[s] = s16x8{0, 0, 0, 0, 0, 0, 0, 0};
      if (col.row >= 0 && d < a.D) q[s] = *(const s16x8*)(src + d);
    }
  }

  // Scores become base-2 exponents (with a factor c of 1) by a cap and a bias.
  __device__ __forceinline__ void turn(const AttendArgs& a, const Column& col, int key0, float slope, f32x16 (&s)[NB]) {
    const int h = (threadIdx.x & 63) >> 5;
    if (a.cap > 0.f) {
      // tanh y = 1 - 2 / (exp 2y + 1).  Near 0 that cancels: off by 2^-22, which up to
      // this cap is 2^-16 of a weight; past it the series takes over there
      const float cl = a.cap * kLog2e, inv = fminf(fmaxf(a.scale / a.cap, -1e38f), 1e38f);
      const float two = inv * (2.f * kLog2e);
      if (a.cap <= kCancels) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i)
            s[b][i] = __builtin_fmaf(-2.f * cl, __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[b][i] * two) + 1.f), cl);
      } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float y = s[b][i] * inv, y2 = y * y;
            const float far = 1.f - 2.f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(s[b][i] * two) + 1.f);
            const float near = 1.f + y2 * (-1.f / 3.f + y2 * (2.f / 15.f - y2 * (17.f / 315.f)));  // of y
            s[b][i] = fabsf(y) < 0.25f ? s[b][i] * (a.scale * kLog2e) * near : cl * far;
          }
      }
    } else {
      const float f = a.scale * kLog2e;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] *= f;
    }
    if (a.slopes) {
      const float apart = (float)(col.pos - key0 - 4 * h);
      if (a.b.tree && key0 + 32 * NB > col.ctx) {  // this step's keys stand at the positions of their depth
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int k = 32 * b + 8 * (i >> 2) + (i & 3), j = key0 + 4 * h + k - col.ctx;
            const int d = col.pos - col.ctx - __builtin_popcountll(col.path & below(j));
            s[b][i] -= slope * fabsf(j >= 0 ? (float)d : apart - (float)k);
          }
      } else {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[b][i] -= slope * fabsf(apart - (float)(32 * b + 8 * (i >> 2) + (i & 3)));
      }
    }
  }

  // -inf for keys that the column does not see.
  __device__ __forceinline__ void hide(const AttendArgs& a, const Column& col, int key0, uint64_t good, f32x16 (&s)[NB]) {
    const int h = (threadIdx.x & 63) >> 5;
    // bit k: key k of the tile is seen
    uint64_t see = below(col.hi - key0) & ~below(col.lo - key0);
    if (a.b.tree) {
      const int from = key0 - col.ctx;
      see |= from >= 64 || from <= -64 ? 0 : from >= 0 ? col.see >> from : col.see << -from;
    }
    see = (see & good) >> (4 * h);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        s[b][i] = ((uint32_t)(see >> (32 * b)) & 1u << (8 * (i >> 2) + (i & 3))) ? s[b][i] : -INFINITY;
  }

  // Has the maximum and the sums up to date with a tile's scores; what they lack to a
  // weight's exponent.  That is the maximum times c, rounded: by at most 2^-13 up to kFar, but
  // by more than an exponent may hold for scores past 2^30.  EXACT: a larger maximum
  // is taken off the scores here, which leaves what is near it exact; a column with a smaller
  // one has the same bits as without.
  template <bool APART, bool EXACT>
  __device__ __forceinline__ float follow(f32x16 (&s)[NB]) {
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
    top = other_half_max(top);
    // The maximum lags until a weight would pass 2^kLazy: most tiles rescale nothing
    // (a column's own scores alone decide: what other rows see leaves its bits)
    const bool lags = EXACT && fabsf(m * c) > kFar ? (top - m) * c > H::kLazy : top * c > m * c + H::kLazy;
    if (__builtin_amdgcn_ballot_w64(lags)) {
      if constexpr (APART) keep_apart();
      const float mn = lags ? top : m;
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m - mn) * c);
      l *= f;
#pragma unroll
      for (int d = 0; d < DHP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
      if constexpr (APART) keep_apart();
      m = mn;
    }
    if constexpr (EXACT) {
      const bool far = m > -INFINITY && fabsf(m * c) > kFar;
      const float base = far ? m : 0.f;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] -= base;
      if (far) return -H::kShift;
    }
    return (m == -INFINITY ? 0.f : m * c) - H::kShift;
  }
  // The weights, and their sum.
  __device__ __forceinline__ void weigh(f32x16 (&s)[NB], float mc, s16x8 (&p)[2 * NB]) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][i], c, -mc));
        l += s[b][i];
      }
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t)
#pragma unroll
      for (int j = 0; j < 8; ++j) p[t][j] = (short)H::bits(s[t >> 1][8 * (t & 1) + j]);
  }

  // The keys' operand of a tile.  (Piece 2t + h of key 32b + r: the key's swizzle does
  // not depend on b, nor its low bit on t.)
  __device__ __forceinline__ void read_keys(const unsigned char* lk, s16x8 (&kf)[DHP / 16][NB]) {
    const int lane = threadIdx.x & 63, h = lane >> 5, r = lane & 31;
    const unsigned char* kr = lk + r * G::ROW;
    const int kx = afresh((h ^ G::swz(r)) * 16);
#pragma unroll
    for (int t = 0; t < DHP / 16; ++t)
#pragma unroll
      for (int b = 0; b < NB; ++b) kf[t][b] = *(const s16x8*)(kr + (kx ^ (32 * t)) + 32 * b * G::ROW);
  }

  // One tile: keys key0 .. key0 + 32 NB - 1.  masked: some column does not see some
  // key of it.  CAREFUL: with what is not finite in V, and scores of any size, taken care
  // of.
  // The operands of a product are read from LDS before it begins (and half of V
  // before the softmax), which the barriers for the scheduler say: left to
  // itself it reads each just before its use.
  template <bool CAREFUL>
  __device__ __forceinline__ void step(const AttendArgs& a, const Column& col, const unsigned char* lk, const unsigned char* lv,
                                       int key0, uint64_t good, bool masked, float slope) {
    const int h = (threadIdx.x & 63) >> 5;
    f32x16 s[NB];
    {
      s16x8 kf[DHP / 16][NB];
      read_keys(lk, kf);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
      // products go before another wave's softmax (2048-row prompt 548 -> 533 us)
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < DHP / 16; ++t)
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b] = H::mfma(kf[t][b], q[t], s[b]);
      __builtin_amdgcn_s_setprio(0);
    }
    s16x8 vf[2 * NB][DHP / 32];
    constexpr int AHEAD = TURN && NB == 2 && DHP == 128 ? 0 : NB;  // (no registers are left: 161 us, 158 without)
    const uint32_t values = values_at(lv);
    if constexpr (!CAREFUL) {
      read_values<0, AHEAD>(values, vf);
      __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (TURN) turn(a, col, key0, slope, s);
    if (masked) hide(a, col, key0, good, s);
    const float mc = follow<false, CAREFUL>(s);
    s16x8 p[2 * NB];
    weigh(s, mc, p);
    if constexpr (CAREFUL) {
      add_not_finite(lv, p, h);
    } else {
      __builtin_amdgcn_sched_barrier(0);
      read_values<AHEAD, 2 * NB>((uint32_t)afresh((int)values), vf);
      __builtin_amdgcn_sched_barrier(0);
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int t = 0; t < 2 * NB; ++t)
#pragma unroll
        for (int d = 0; d < DHP / 32; ++d) o[d] = H::mfma(vf[t][d], p[t], o[d]);
      __builtin_amdgcn_s_setprio(0);
    }
  }

  // The same with the products of one tile between the softmax of another, for a
  // wave that has its vector unit to itself.  `s` are the tile's scores, turned;
  // they become those of the next tile, whose keys lie at lk.
  __device__ __forceinline__ void first_scores(const AttendArgs& a, const Column& col, const unsigned char* lk, int key0, float slope,
                                               f32x16 (&s)[NB]) {
    s16x8 kf[DHP / 16][NB];
    read_keys(lk, kf);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
    for (int t = 0; t < DHP / 16; ++t)
#pragma unroll
      for (int b = 0; b < NB; ++b) s[b] = H::mfma(kf[t][b], q[t], s[b]);
    if constexpr (TURN) turn(a, col, key0, slope, s);
  }
  __device__ __forceinline__ void piped_step(const AttendArgs& a, const Column& col, const unsigned char* lk, const unsigned char* lv,
                                             int key0, uint64_t good, bool masked, float slope, f32x16 (&s)[NB]) {
    static_assert(NB == 1);
    s16x8 kf[DHP / 16][NB], vf[2 * NB][DHP / 32], p[2 * NB];
    read_keys(lk, kf);
    __builtin_amdgcn_sched_barrier(0);
    if (masked) hide(a, col, key0, good, s);
    const float mc = follow<true, false>(s);
    __builtin_amdgcn_sched_barrier(0);
    read_values<0, 2 * NB>(values_at(lv), vf);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 n[NB];
#pragma unroll
    for (int i = 0; i < 16; ++i) n[0][i] = 0.f;
#pragma unroll
    for (int t = 0; t < DHP / 16; ++t) n[0] = H::mfma(kf[t][0], q[t], n[0]);
    asm volatile("" : "+v"(n[0]));  // (not among the accumulation registers: vector operations follow)
    weigh(s, mc, p);
#pragma unroll
    for (int t = 0; t < DHP / 16; ++t) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // a matrix product,
      __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);  // vector operations,
      __builtin_amdgcn_sched_group_barrier(0x400, 1, 0);  // an exponential
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2 * NB; ++t)
#pragma unroll
      for (int d = 0; d < DHP / 32; ++d) o[d] = H::mfma(vf[t][d], p[t], o[d]);
    s[0] = n[0];
    if constexpr (TURN) turn(a, col, key0 + 32 * NB, slope, s);
  }

  // Has the sums of a wide head in accumulation registers here, and so from step to
  // step: the compiler would else move all of them for the rare rescaling.
  __device__ __forceinline__ void keep_apart() {
    if constexpr (DHP == 256) {
#pragma unroll
      for (int d = 0; d < DHP / 32; ++d) asm volatile("" : "+a"(o[d]));
    }
  }

  // Whether some dimension of some column came out as a NaN, or its scores were too
  // large for what was taken off them: then the item is done once more with care, which
  // takes about three times as long (2048 rows over 4048 keys 124 -> 464 us in all); a branch
  // per tile in its place cost ordinary scores up to 3%.
  __device__ __forceinline__ bool doubtful() const {
    bool bad = m > -INFINITY && fabsf(m * c) > kFar;
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) bad = bad || o[d][i] != o[d][i];
    return __builtin_amdgcn_ballot_w64(bad) != 0;
  }

  // V's operand of 32 dimensions (from 32 d) for the 16 keys of P's operand t: keys
  // 16t + 4h .. + 3 and the four 8 further on.  Sixteen lanes read four keys' 16
  // dimensions, and each gets one dimension's four keys.  (The keys' swizzle
  // does not depend on t.)
  __device__ __forceinline__ s16x8 read_v8(const unsigned char* lv, int t, int h, int d) {
    const int lane = threadIdx.x & 63;
    const int key = 4 * h + (lane >> 2 & 3), dim = (lane & 16) + (lane & 3) * 4;
    const unsigned char* p = lv + key * G::ROW + (dim & 7) * 2 + 16 * t * G::ROW;
    const int x = afresh(((dim >> 3) ^ G::swz(key)) * 16);  // (key + 8: another piece, two away)
    return join4(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (x ^ (64 * d)))),
                 __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + (x ^ (64 * d) ^ 32) + 8 * G::ROW)));
  }

  // The same for 16-key operands T0 .. T1 - 1 and all dimensions: a tile begins at a
  // multiple of 1024, so an XOR of a lane's place gives each dimension's.
  __device__ __forceinline__ uint32_t values_at(const unsigned char* lv) {
    const int lane = threadIdx.x & 63, h = lane >> 5;
    const int key = 4 * h + (lane >> 2 & 3), dim = (lane & 16) + (lane & 3) * 4;
    return (uint32_t)(uintptr_t)(lds_void*)lv + (key * G::ROW + (dim & 7) * 2 + (((dim >> 3) ^ G::swz(key)) * 16));
  }
  template <int T0, int T1>
  __device__ __forceinline__ void read_values(uint32_t p, s16x8 (&vf)[2 * NB][DHP / 32]) {
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d) {
      const uint32_t one = p ^ (64 * d), two = p ^ (64 * d) ^ 32;
#pragma unroll
      for (int t = T0; t < T1; ++t)
        vf[t][d] = join4(__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(one + 16 * t * G::ROW)),
                         __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(uintptr_t)(two + (16 * t + 8) * G::ROW)));
    }
  }

  // A value that a column does not see must not reach it, and 0 times an infinity
  // or a NaN would.  So where a result is a NaN, the item is done once more with
  // this: such values are taken out of V and counted, by weight, where they are;
  // a dimension's count makes it infinite, both signs' (a NaN is both) a NaN.
  __device__ __forceinline__ void add_not_finite(const unsigned char* lv, const s16x8 (&p)[2 * NB], int h) {
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d) {
#pragma unroll
      for (int sign = 0; sign < 2; ++sign) {
        f32x16 there;
#pragma unroll
        for (int i = 0; i < 16; ++i) there[i] = 0.f;
#pragma unroll
        for (int t = 0; t < 2 * NB; ++t) {
          __builtin_amdgcn_sched_barrier(0);  // one operand at a time: this path may not cost the other one registers
          const u32x4 v = __builtin_bit_cast(u32x4, read_v8(lv, t, h, d));
          u32x4 finite, u;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t mag = (v[j] & 0x7fff7fffu) + H::kInf;  // bit 15 of a half: not finite
            const uint32_t not_finite = mag & 0x80008000u, nan = (mag - 0x00010001u) & 0x80008000u;
            finite[j] = v[j] & ~(not_finite | (not_finite - (not_finite >> 15)));
            u[j] = (nan | (not_finite & (sign ? v[j] : ~v[j]))) >> 1;  // 2 in either type
          }
          if (sign == 0) o[d] = H::mfma(__builtin_bit_cast(s16x8, finite), p[t], o[d]);
          there = H::mfma(__builtin_bit_cast(s16x8, u), p[t], there);
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] += there[i] > 0.f ? (sign ? -INFINITY : INFINITY) : 0.f;
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
};

// Four successive dimensions of a row's result.
template <bool BF16>
__device__ __forceinline__ void store_out(const AttendArgs& a, int row, int head, int dim, float x, float y, float z, float w) {
  if (dim >= a.D) return;
  using H = Half<BF16>;
  uint16_t* p = (uint16_t*)a.out + (int64_t)row * a.out_row + head * a.out_head + dim;
  *(uint2*)p = uint2{(uint32_t)H::bits(x) | (uint32_t)H::bits(y) << 16, (uint32_t)H::bits(z) | (uint32_t)H::bits(w) << 16};
}

// Partial results of the items (a.part): [blocks][cols][DHP] sums, [blocks][cols][2]
// maxima (base 2) and weights' sums; and for each row and head the place of its
// first split and how many there are (1: its result is written already).
struct Part {
  float *o, *ml;
  int2* where;
};
__device__ __forceinline__ Part part_of(const AttendArgs& a, int blocks, int cols, int dhp) {
  Part p;
  p.o = a.part;
  p.ml = a.part + (size_t)blocks * cols * dhp;
  p.where = (int2*)(p.ml + (size_t)blocks * cols * 2);
  return p;
}

// Cuts an item down to the keys [k0, k1) it is to look at; false: none.  live: the
// splits of its tile that have keys.
__device__ __forceinline__ bool cut_keys(const Item& it, int lo, int hi, int& k0, int& k1, int& live) {
  const int base = lo == kNoKey ? 0 : lo & ~63;
  hi = max(hi, base);
  live = max(1, (int)(((int64_t)hi - base + it.chunk - 1) / it.chunk));
  if (it.split >= live) return false;
  k0 = base + it.split * it.chunk;
  k1 = (int)min((int64_t)hi, (int64_t)k0 + it.chunk);
  return true;
}
// The first split says where the results of a column (of its lane) are.
__device__ __forceinline__ void tell_where(const AttendArgs& a, const Part& part, const Item& it, const Column& col, int at, int live) {
  if (a.part && it.split == 0 && col.row >= 0) part.where[(int64_t)col.row * a.Hq + col.head] = int2{at, live};
}

// Many columns: four waves of 32 share the tiles of 64 keys, one being copied while
// one is worked on.  Bound by the matrix cores and what is issued beside them, two
// workgroups a CU: 2048 rows of 32 heads of 128 over 16384 keys 517 to 549 us, from
// card to card, 0.94 to 1.0 PFLOP/s (a large product: 1.2 to 1.36).  Where a key is 256 wide a wave has its vector unit
// to itself, and a tile is two steps of 32 keys whose softmax goes on beside the next
// one's products: 1500 rows of 16 heads over 3500 keys 147 us (296 one after
// the other).
constexpr int kWideCols = 128;
template <int DHP>
constexpr int wide_blocks() { return DHP == 256 ? 1 : 2; }
template <int DHP>
constexpr int wide_lds() { return 2 * 2 * 64 * DHP * 2; }

template <int DHP, bool BF16, bool TURN>
__global__ __launch_bounds__(256, DHP == 256 ? 1 : 2) void attend_wide(AttendArgs a, Cut cut, int blocks) {
  extern __shared__ __align__(1024) unsigned char tiles[];  // (addresses in them are made by XOR)
  unsigned char* const smem = tiles;
  __shared__ int red[4][2];
  using G = Geo<DHP>;
  constexpr int NB = wide_blocks<DHP>(), KT = 32 * NB, TILE = KT * G::ROW;
  constexpr uint64_t kAll = KT == 64 ? ~0ull : 0xffffffffull;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = blockIdx.x / a.H, kvh = blockIdx.x - idx * a.H;
  Item it;
  if (!find_item(a, cut, idx, it)) return;
  const Column col = column_of(a, it, it.tile * kWideCols + wave * 32 + (lane & 31), kvh * (a.Hq / a.H));
  const Span sp = span_of(a, col);
  if (lane == 0) {
    red[wave][0] = sp.lo;
    red[wave][1] = sp.hi;
  }
  __syncthreads();
  const int lo = min(min(red[0][0], red[1][0]), min(red[2][0], red[3][0]));
  const int hi = max(max(red[0][1], red[1][1]), max(red[2][1], red[3][1]));
  const Part part = part_of(a, blocks, kWideCols, DHP);
  int k0, k1, live;
  if (!cut_keys(it, lo, hi, k0, k1, live)) return;
  if (lane < 32) tell_where(a, part, it, col, blockIdx.x * kWideCols + wave * 32 + lane, live);
  Wave<DHP, BF16, NB, TURN> w;
  w.init(a, col, lane >> 5);
  const float slope = a.slopes && col.row >= 0 ? a.slopes[col.head] * kLog2e : 0.f;
  if (k0 < k1) {
    if (a.D < DHP) {
      for (int i = tid; i < wide_lds<DHP>() / 16; i += 256) ((uint4*)smem)[i] = uint4{0, 0, 0, 0};
      __syncthreads();
    }
    const int32_t* table = a.b.pages + (it.s < a.b.S ? it.s : 0) * a.b.pages_stride;
    const int end = min(hi, it.len);
    constexpr int N = KT / G::KPI / 4;
    const int mine = wave * N * G::KPI;
    Copies<DHP, N, DHP <= 128> copies;
    copies.init(a, mine);
    const auto run = [&](auto careful) __attribute__((always_inline)) {
      Pages pg = pages_of(a, table, kvh, k0 + lane * 16, end);
      uint64_t good = good_keys<KT>(pg.has, 0, k0, end), next_good = 0;
      copies.issue(a, mine, pg, 0, good, smem, 0, TILE);
      int key = k0, t = 0;
      // waits for this tile and begins to copy the next one
      const auto next = [&]() __attribute__((always_inline)) {
        vm_wait<0>();
        block_barrier();
        if (key + KT < k1) {
          const int g = (t + 1) * (KT / 16) & 63;
          if (g == 0) pg = pages_of(a, table, kvh, key + KT + lane * 16, end);
          next_good = good_keys<KT>(pg.has, g, key + KT, end);
          const uint32_t to = ((t + 1) & 1) * 2 * TILE;
          copies.issue(a, mine, pg, g, next_good, smem, to, to + TILE);
        }
      };
      const auto skip = [&](int until) __attribute__((always_inline)) {
        for (; key < until; key += KT, ++t) {
          next();
          good = next_good;
        }
      };
      // tiles that this wave's columns see, those before and after them only copied
      // (three loops: a branch around the step has the compiler move its accumulators)
      skip(min(k1, sp.lo - (KT - 1)));
      for (; key < min(k1, sp.hi); key += KT, ++t) {
        next();
        unsigned char* now = smem + (t & 1) * 2 * TILE;
        w.template step<decltype(careful)::value>(a, col, now, now + TILE, key, good,
                                                  key < sp.all_lo || key + KT > sp.all_hi || good != kAll, slope);
        good = next_good;
      }
      skip(k1);
    };
    if constexpr (DHP == 256) {
      // Two steps a round, the scores of each made a step ahead: the keys that are
      // copied for a round begin 32 after its values.
      constexpr int KW = 2 * KT, WIDE = 2 * TILE;
      const int my = 2 * mine;
      Copies<DHP, 2 * N, false> two;
      two.init(a, my);
      Pages pv = pages_of(a, table, kvh, k0 + lane * 16, end), pk = pages_of(a, table, kvh, k0 + KT + lane * 16, end);
      uint64_t good = good_keys<KW>(pv.has, 0, k0, end);
      copies.template issue<true, false>(a, mine, pv, 0, good & kAll, smem, 2 * WIDE, 0);
      two.template issue<false, true>(a, my, pv, 0, good, smem, 0, WIDE);
      two.template issue<true, false>(a, my, pk, 0, good_keys<KW>(pk.has, 0, k0 + KT, end), smem, 0, 0);
      vm_wait<0>();
      block_barrier();
      f32x16 s[NB];
      w.first_scores(a, col, smem + 2 * WIDE, k0, slope, s);
      for (int key = k0, t = 0; key < k1; key += KW, ++t) {
        const uint32_t now = (t & 1) * 2 * WIDE, next = ((t + 1) & 1) * 2 * WIDE;
        vm_wait<0>();
        block_barrier();
        uint64_t coming = 0;
        if (key + KW < k1) {
          const int g = (t + 1) * (KW / 16) & 63;
          if (g == 0) {
            pv = pages_of(a, table, kvh, key + KW + lane * 16, end);
            pk = pages_of(a, table, kvh, key + KW + KT + lane * 16, end);
          }
          coming = good_keys<KW>(pv.has, g, key + KW, end);
          two.template issue<false, true>(a, my, pv, g, coming, smem, 0, next + WIDE);
          two.template issue<true, false>(a, my, pk, g, good_keys<KW>(pk.has, g, key + KW + KT, end), smem,
                                          next, 0);
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int at = key + u * KT;
          const uint64_t there = good >> (32 * u) & 0xffffffffull;
          w.piped_step(a, col, smem + now + u * TILE, smem + now + WIDE + u * TILE, at, there,
                       at < sp.all_lo || at + KT > sp.all_hi || there != 0xffffffffull, slope, s);
        }
        good = coming;
      }
    } else {
      run(std::false_type{});
    }
    if (__syncthreads_or(w.doubtful())) {  // (all of them: the tiles are shared)
      w.reset();
      run(std::true_type{});
    }
  }
  if (col.row < 0) return;
  const float l = other_half_sum(w.l), mb = w.m == -INFINITY ? -INFINITY : w.m * w.c;
  const int h = lane >> 5;
  if (live == 1) {
    const float f = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        store_out<BF16>(a, col.row, col.head, 32 * d + 2 * i + 4 * h, w.o[d][i] * f, w.o[d][i + 1] * f, w.o[d][i + 2] * f,
                        w.o[d][i + 3] * f);
  } else {
    const int at = blockIdx.x * kWideCols + wave * 32 + (lane & 31);
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *(float4*)(part.o + (size_t)at * DHP + 32 * d + 2 * i + 4 * h) = float4{w.o[d][i], w.o[d][i + 1], w.o[d][i + 2], w.o[d][i + 3]};
    if (h == 0) *(float2*)(part.ml + (size_t)at * 2) = float2{mb, l};
  }
}

// Few columns: the waves of a workgroup hold the same 32 columns and take the
// tiles of 32 keys by turns, each with tiles of its own in LDS and no barrier;
// their results are joined through LDS at the end.  Bound by memory: a token each
// of 64 sequences of 8192 keys 370 us, 5.8 TB/s; of 32 of 1024 to 8192 keys 143 us,
// 4.9 TB/s.
constexpr int kFewCols = 32;
template <int DHP>
constexpr int few_waves() { return DHP == 256 ? 2 : 4; }
template <int DHP>
constexpr int few_lds() { return few_waves<DHP>() * 2 * 2 * 32 * DHP * 2; }

template <int DHP, bool BF16, bool TURN>
__global__ __launch_bounds__(64 * few_waves<DHP>(), DHP == 256 ? 1 : 2) void attend_few(AttendArgs a, Cut cut, int blocks) {
  extern __shared__ __align__(1024) unsigned char tiles[];  // (addresses in them are made by XOR)
  unsigned char* const smem = tiles;
  constexpr int NW = few_waves<DHP>();
  __shared__ float stat[NW][32][2];
  using G = Geo<DHP>;
  constexpr int TILE = 32 * G::ROW;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int idx = blockIdx.x / a.H, kvh = blockIdx.x - idx * a.H;
  Item it;
  if (!find_item(a, cut, idx, it)) return;
  const Column col = column_of(a, it, it.tile * kFewCols + (lane & 31), kvh * (a.Hq / a.H));
  const Span sp = span_of(a, col);
  const Part part = part_of(a, blocks, kFewCols, DHP);
  int k0, k1, live;
  if (!cut_keys(it, sp.lo, sp.hi, k0, k1, live)) return;
  if (tid < 32) tell_where(a, part, it, col, blockIdx.x * kFewCols + lane, live);
  Wave<DHP, BF16, 1, TURN> w;
  w.init(a, col, lane >> 5);
  const float slope = a.slopes && col.row >= 0 ? a.slopes[col.head] * kLog2e : 0.f;
  unsigned char* my = smem + wave * 4 * TILE;
  if (a.D < DHP) {
    for (int i = lane; i < 4 * TILE / 16; i += 64) ((uint4*)my)[i] = uint4{0, 0, 0, 0};
    __syncthreads();
  }
  const int32_t* table = a.b.pages + (it.s < a.b.S ? it.s : 0) * a.b.pages_stride;
  const int end = min(sp.hi, it.len);
  constexpr int N = 32 / G::KPI, STEP = 32 * NW;
  // lane l holds the page of half l & 1 of this wave's tile l / 2
  const auto pages_from = [&](int key) { return pages_of(a, table, kvh, key + (lane >> 1) * STEP + (lane & 1) * 16, end); };
  const int first = k0 + wave * 32;
  Copies<DHP, N, DHP <= 128> copies;
  copies.init(a, 0);
  const auto run = [&](auto careful) __attribute__((always_inline)) {
    Pages pg = pages_from(first);
    uint64_t good = good_keys<32>(pg.has, 0, first, end), next_good = 0;
    copies.issue(a, 0, pg, 0, good, my, 0, TILE);
    for (int key = first, t = 0; key < k1; key += STEP, ++t) {
      const uint32_t now = (t & 1) * 2 * TILE, next = ((t + 1) & 1) * 2 * TILE;
      bool all = false;
      if (key + STEP < k1) {
        const int g = (t + 1) * 2 & 63;
        if (g == 0) pg = pages_from(key + STEP);
        next_good = good_keys<32>(pg.has, g, key + STEP, end);
        all = copies.issue(a, 0, pg, g, next_good, my, next, next + TILE);
      }
      if (all) vm_wait<2 * N>();
      else vm_wait<0>();
      asm volatile("" ::: "memory");
      w.template step<decltype(careful)::value>(a, col, my + now, my + now + TILE, key, good,
                                                key < sp.all_lo || key + 32 > sp.all_hi || good != 0xffffffffull, slope);
      good = next_good;
    }
  };
  if (first < k1) {
    run(std::false_type{});
    if (w.doubtful()) {
      w.reset();
      run(std::true_type{});
    }
  }
  // join the waves
  const float l = other_half_sum(w.l), mb = w.m == -INFINITY ? -INFINITY : w.m * w.c;
  if (lane < 32) {
    stat[wave][lane][0] = mb;
    stat[wave][lane][1] = l;
  }
  __syncthreads();  // (every wave has read its last tile)
  float* so = (float*)smem;  // [NW][32][DHP], pieces of 4 swizzled by column
  {
    const int r = lane & 31, h = lane >> 5;
#pragma unroll
    for (int d = 0; d < DHP / 32; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        const int piece = 8 * d + (i >> 1) + h;
        *(float4*)(so + (wave * 32 + r) * DHP + (piece ^ (r & 15)) * 4) =
            float4{w.o[d][i], w.o[d][i + 1], w.o[d][i + 2], w.o[d][i + 3]};
      }
  }
  __syncthreads();
  const int G_ = a.Hq / a.H;
  const int cols = (int)min((int64_t)kFewCols, (int64_t)it.n * G_ - (int64_t)it.tile * kFewCols);
  for (int u = tid; u < cols * (DHP / 4); u += 64 * NW) {
    const int r = u / (DHP / 4), piece = u - r * (DHP / 4);
    float top = -INFINITY;
#pragma unroll
    for (int v = 0; v < NW; ++v) top = fmaxf(top, stat[v][r][0]);
    float sum = 0.f, x = 0.f, y = 0.f, z = 0.f, q = 0.f;
#pragma unroll
    for (int v = 0; v < NW; ++v) {
      const float f = stat[v][r][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stat[v][r][0] - top);
      const float4 t = *(const float4*)(so + (v * 32 + r) * DHP + (piece ^ (r & 15)) * 4);
      if (stat[v][r][0] > -INFINITY || !(stat[v][r][1] == 0.f)) {
        sum += f * stat[v][r][1];
        x += f * t.x;
        y += f * t.y;
        z += f * t.z;
        q += f * t.w;
      }
    }
    if (live == 1) {
      const float f = sum == 0.f ? 0.f : 1.f / sum;
      const int mm = it.tile * kFewCols + r, i = mm / G_;
      store_out<BF16>(a, it.row0 + i, kvh * G_ + (mm - i * G_), piece * 4, x * f, y * f, z * f, q * f);
    } else {
      const size_t at = (size_t)blockIdx.x * kFewCols + r;
      *(float4*)(part.o + at * DHP + piece * 4) = float4{x, y, z, q};
      if (piece == 0) *(float2*)(part.ml + at * 2) = float2{top, sum};
    }
  }
}

// Joins the splits of each row and head: NW waves each, which take them by turns,
// their lanes over the dimensions.
template <int DHP, bool BF16, int NW>
__global__ __launch_bounds__(NW == 1 ? 256 : 64 * NW) void attend_join(AttendArgs a, int cols, int blocks) {
  constexpr int VL = DHP / 64;  // dimensions per lane
  typedef float vec __attribute__((ext_vector_type(VL)));
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t rh = NW == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  const int first = NW == 1 ? 0 : wave;
  if (rh >= (int64_t)a.b.T * a.Hq) return;
  const Part part = part_of(a, blocks, cols, DHP);
  const int2 where = part.where[rh];
  const int live = where.y;
  const int64_t step = (int64_t)a.H * cols;  // places from one split to the next
  // (nor if it is no place: a row that no sequence has, where starts does not begin at 0)
  if (live <= 1 || where.x < 0 || where.x + (live - 1) * step >= (int64_t)blocks * cols) return;
  float top = -INFINITY, sum = 0.f;
  float x[VL] = {};
  for (int s0 = first; s0 < live; s0 += 64 * NW) {
    const int mine = s0 + lane * NW, n = min(64, (live - s0 + NW - 1) / NW);
    float2 ml = float2{-INFINITY, 0.f};
    if (mine < live) ml = *(const float2*)(part.ml + (where.x + mine * step) * 2);
    float t = ml.x;
    for (int o = 32; o > 0; o >>= 1) t = fmaxf(t, __shfl_xor(t, o));
    t = fmaxf(t, top);
    const float old = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - t);
    // (nothing seen: no weight; but a NaN is handed on)
    const float f = ml.x > -INFINITY ? __builtin_amdgcn_exp2f(ml.x - t) : ml.y == 0.f ? 0.f : 1.f;
    sum = sum * old + wave_sum(f * ml.y);
    top = t;
#pragma unroll
    for (int j = 0; j < VL; ++j) x[j] *= old;
    const float* o = part.o + (where.x + s0 * step) * DHP + lane * VL;
    constexpr int U = 4;  // on their way at once (the last one again past the end, without weight)
    for (int i = 0; i < n; i += U) {
      vec v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = *(const vec*)(o + min(i + u, n - 1) * NW * step * DHP);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const float fi = i + u < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), i + u)) : 0.f;
#pragma unroll
        for (int j = 0; j < VL; ++j) x[j] += fi == 0.f ? 0.f : fi * v[u][j];
      }
    }
  }
  if constexpr (NW > 1) {
    __shared__ float so[NW][DHP], st[NW][2];
#pragma unroll
    for (int j = 0; j < VL; ++j) so[wave][lane * VL + j] = x[j];
    if (lane == 0) {
      st[wave][0] = top;
      st[wave][1] = sum;
    }
    __syncthreads();
    if (wave != 0) return;
    const int waves = min(NW, live);
    for (int w = 0; w < waves; ++w) top = fmaxf(top, st[w][0]);
    sum = 0.f;
#pragma unroll
    for (int j = 0; j < VL; ++j) x[j] = 0.f;
    for (int w = 0; w < waves; ++w) {
      const float f = st[w][0] > -INFINITY ? __builtin_amdgcn_exp2f(st[w][0] - top) : st[w][1] == 0.f ? 0.f : 1.f;
      if (f == 0.f) continue;
      sum += f * st[w][1];
#pragma unroll
      for (int j = 0; j < VL; ++j) x[j] += f * so[w][lane * VL + j];
    }
  }
  const int row = (int)(rh / a.Hq), head = (int)(rh - (int64_t)row * a.Hq);
  const float f = sum == 0.f ? 0.f : 1.f / sum;
  uint16_t* out = (uint16_t*)a.out + (int64_t)row * a.out_row + head * a.out_head;
#pragma unroll
  for (int j = 0; j < VL; ++j)
    if (lane * VL + j < a.D) out[lane * VL + j] = Half<BF16>::bits(x[j] * f);
}

// ------------------------------------------------------------------- launches

struct Plan {
  Cut cut;
  int blocks;
  bool few;
};
int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

Plan plan_of(const AttendArgs& a) {
  Plan p{};
  const int64_t cols = (int64_t)a.b.T * (a.Hq / a.H);
  const int seqs = std::min(a.b.S, a.b.T);
  // One form for the whole call, by the mean: what the sequences' rows are the host does
  // not know.  (127 tokens and a prompt's 512 rows in one call 662 us, apart 412 + 164.)
  p.few = cols <= (int64_t)32 * std::max(1, seqs);
  p.cut.cols = p.few ? kFewCols : kWideCols;
  const int64_t most = cols / p.cut.cols + std::min(a.b.S + 1, a.b.T);  // tiles there can be
  const int64_t likely = std::max<int64_t>(seqs, (cols + p.cut.cols - 1) / p.cut.cols);
  // workgroups at once, by a kernel's registers and the LDS of its tiles
  const int dim = padded_dim(a.D), at_once = p.few ? (dim == 64 ? 2 : 1) : dim == 64 ? 3 : dim == 128 ? 2 : 1, slots = 256 * at_once;
  p.cut.min_chunk = 128;
  // Three rounds of whole tiles or more are not split, nor looked at by the join.  (By counts
  // alone: one sequence of 131072 keys among 94 of 1024 takes 182 us, among 127 1200.)
  p.cut.slots = likely * a.H < 3 * slots ? slots : 0;
  int64_t items = most;
  if (p.cut.slots) {  // (nor more than splits of the longest sequence that the table holds)
    const int64_t splits = (((int64_t)a.b.P << a.page_shift) + 63 + p.cut.min_chunk - 1) / p.cut.min_chunk;
    items = std::min(most + most / 2 + 2 * slots / a.H + 9, most * splits);
  }
  p.cut.items = (int)items;
  // An item takes about 3 us before its first key; a split's sums are written and read
  // again, which takes as long as this many keys do (35 ns a key of a wide tile's at
  // its matrix products' rate, a narrow one's keys at the memory's).  Half or twice as much
  // for an item, or twice for a split, changed no case timed by more than 1%; half for a
  // split took 4 prompts from 148 to 200 us.
  p.cut.item = 80.f;
  p.cut.split = p.few ? 64.f : dim == 256 ? 250.f : 400.f;
  p.blocks = (int)(items * a.H);
  return p;
}

template <class F>
hipError_t allow_lds(F kernel, int bytes, std::atomic<uint64_t>& done) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess || (done.load(std::memory_order_acquire) >> (dev & 63) & 1)) return e;
  e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e == hipSuccess) done.fetch_or(1ull << (dev & 63), std::memory_order_release);
  return e;
}

template <int DHP, bool BF16, bool TURN>
hipError_t launch_kernel(const AttendArgs& a, const Plan& p, hipStream_t s) {
  static std::atomic<uint64_t> few_done{0}, wide_done{0};
  if (p.few) {
    hipError_t e = allow_lds(attend_few<DHP, BF16, TURN>, few_lds<DHP>(), few_done);
    if (e != hipSuccess) return e;
    hvd_launch((attend_few<DHP, BF16, TURN>), dim3(p.blocks), dim3(64 * few_waves<DHP>()), few_lds<DHP>(), s, a, p.cut, p.blocks);
  } else {
    hipError_t e = allow_lds(attend_wide<DHP, BF16, TURN>, wide_lds<DHP>(), wide_done);
    if (e != hipSuccess) return e;
    hvd_launch((attend_wide<DHP, BF16, TURN>), dim3(p.blocks), dim3(256), wide_lds<DHP>(), s, a, p.cut, p.blocks);
  }
  return hipGetLastError();
}

template <int DHP, bool BF16>
hipError_t launch_dh(const AttendArgs& a, const Plan& p, hipStream_t s) {
  const bool turn = a.cap > 0.f || a.slopes || !(a.scale > 0.f);
  hipError_t e = turn ? launch_kernel<DHP, BF16, true>(a, p, s) : launch_kernel<DHP, BF16, false>(a, p, s);
  if (e == hipSuccess && p.cut.slots) {
    const int64_t n = (int64_t)a.b.T * a.Hq;
    if (n >= 1024) hvd_launch((attend_join<DHP, BF16, 1>), dim3((unsigned)((n + 3) / 4)), dim3(256), 0, s, a, p.cut.cols, p.blocks);
    else hvd_launch((attend_join<DHP, BF16, 8>), dim3((unsigned)n), dim3(512), 0, s, a, p.cut.cols, p.blocks);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

size_t attend_workspace(const AttendArgs& a) {
  const Plan p = plan_of(a);
  if (!p.cut.slots) return 0;
  return (size_t)p.blocks * p.cut.cols * (padded_dim(a.D) + 2) * sizeof(float) + (size_t)a.b.T * a.Hq * sizeof(int2);
}

hipError_t launch_attend(const AttendArgs& a, hipStream_t s) {
  const Plan p = plan_of(a);
  const bool bf = a.type == ET_BF16;
  switch (padded_dim(a.D)) {
    case 64: return bf ? launch_dh<64, true>(a, p, s) : launch_dh<64, false>(a, p, s);
    case 128: return bf ? launch_dh<128, true>(a, p, s) : launch_dh<128, false>(a, p, s);
    default: return bf ? launch_dh<256, true>(a, p, s) : launch_dh<256, false>(a, p, s);
  }
}

}  // namespace hvd
