// Kernels of the paged key/value cache: append with position rotation, attention over all tokens of a sequence, attention
// over listed tokens.
//
// Pages are [n_pages][Hkv][P][D] of bf16, or of e4m3 with one float scale per (page, head): a row's value is code * scale.
// bf16 holds every e4m3 value exactly, so 8-bit rows enter the matrix cores as bf16 (one conversion instruction per two
// values) and the scale of keys multiplies the logits, that of values the softmax weights.
#pragma once
#include "pqc_device.h"

namespace pqc {
namespace paged {

constexpr int kRows = 16;          // query rows of a tile: (query token, query head of the group) pairs
constexpr int kBlockRows = 128;    // of a tile of the kernel for many queries
constexpr int kBlockTokens = 64;   // tokens that it stages at a time
constexpr int kStep = 32;          // tokens that a wave takes at a time
constexpr int kWaves = 4;
constexpr int kGrain = kWaves * kStep;  // tokens of a split are a multiple of this
constexpr int kStaged = 512;       // pages (or listed tokens) whose place and scales lie in LDS at a time
constexpr float kLowest = -3.402823466e38f;  // maximum of the logits of a row that has seen nothing: no finite logit is below it
constexpr float kFp8Max = 448.0f;  // largest e4m3 value, 0.875 * 2^9

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;

struct Geometry {
  int B, Hq, Hkv, G;
  int P, shift;           // tokens per page, and its logarithm
  int n_pages, max_pages;
  int n_q;                // query (or new) tokens of all sequences
  int R;                  // query tokens per tile
  int per_head, least;    // items per head that the split length aims at, and the shortest split
  int items, slots;       // bounds of the numbers of items and of partial results per head
  int workers, grain;     // kernel of 16 rows: workgroups per head, tokens of a unit of their work
  bool out_bf16;
  float scale_log2e;
};
struct Cache {
  unsigned char *k, *v;
  float *ks, *vs;
  const int *table, *lengths;
  unsigned* counters;  // of the parts of tiles, zero between calls; nullptr: parts are folded by a kernel of their own
};

// A partial result: O[rows][D], then maximum and sum of every row; 16-byte aligned.
__host__ __device__ constexpr size_t partial_floats(int rows, int dim) { return (size_t)rows * dim + (2 * rows + 3) / 4 * 4; }

// ------------------------------------------------------------------ sequences and items
struct Seq {
  int first, nq, len;  // first query token and their number, tokens in the cache
};
// Of whatever the arrays hold: inside [0, n_q] and the page table's room.
__device__ __forceinline__ Seq seq_of(const Geometry& g, const int* lengths, const int* offsets, int b) {
  Seq s;
  s.len = min(max(lengths[b], 0), g.max_pages << g.shift);
  s.first = b;
  s.nq = 1;
  if (offsets) {
    s.first = min(max(offsets[b], 0), g.n_q);
    s.nq = min(max(offsets[b + 1], s.first), g.n_q) - s.first;
  }
  return s;
}

// Work of the attention of one head: every sequence has ceil(nq / R) tiles, each over its tokens cut into splits of `tokens`.
// The length of a split is that which gives about per_head items in all, whatever the lengths are, so that one long sequence
// among short ones is spread over the card.  A wave works it out by itself from the lengths (64 sequences per load).
struct Item {
  int b, tile, split, n_split, tokens;
  int slot;  // of the tile's first partial result; -1: the tile is one split
  Seq s;
};
__device__ __forceinline__ int split_tokens(const Geometry& g, const int* lengths, const int* offsets) {
  float work = 0.0f;
  for (int b0 = 0; b0 < g.B; b0 += 64) {
    const int b = b0 + (threadIdx.x & 63);
    if (b < g.B) {
      const Seq s = seq_of(g, lengths, offsets, b);
      work += (float)((s.nq + g.R - 1) / g.R) * (float)s.len;
    }
  }
  // a little more than the quotient, so that rounding keeps the number of items within its bound
  const float tokens = ceilf(wave_sum(work) * 1.001f / (float)(g.per_head * kGrain));
  return max(g.least, max(1, (int)fminf(tokens, 1e7f)) * kGrain);
}
// The j-th item, or the j-th tile of more than one split (whole_tiles); b < 0: there are fewer.
__device__ __forceinline__ Item find_item(const Geometry& g, const int* lengths, const int* offsets, int j, bool whole_tiles) {
  Item it;
  it.b = -1;
  it.tokens = split_tokens(g, lengths, offsets);
  int before = 0, slots = 0;
  for (int b0 = 0; b0 < g.B; b0 += 64) {
    const int b = b0 + (threadIdx.x & 63);
    Seq s{0, 0, 0};
    int n = 0, tiles = 0;
    if (b < g.B) {
      s = seq_of(g, lengths, offsets, b);
      tiles = (s.nq + g.R - 1) / g.R;
      n = max(1, (s.len + it.tokens - 1) / it.tokens);
    }
    const int mine = n > 1 ? tiles * n : 0;
    const int slot_end = wave_inclusive_scan(mine);
    if (n > 1 && slots + slot_end > g.slots) n = 1;  // (the bound of split_tokens keeps this from happening with offsets that ascend)
    const int count = whole_tiles ? (n > 1 ? tiles : 0) : tiles * n;
    const int end = wave_inclusive_scan(count);
    const unsigned long long has = __ballot(before + end > j);
    if (has) {
      const int l = __ffsll((long long)has) - 1;
      const int at = j - before - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(count, l));
      it.b = b0 + l;
      it.n_split = __builtin_amdgcn_readlane(n, l);
      const int nth = whole_tiles ? at : at / it.n_split;
      it.tile = __builtin_amdgcn_readlane(tiles, l) - 1 - nth;  // the last one, which sees most, first
      it.split = whole_tiles ? 0 : at - nth * it.n_split;
      if (it.n_split > 1) it.tokens = ((__builtin_amdgcn_readlane(s.len, l) + it.n_split - 1) / it.n_split + kGrain - 1) / kGrain * kGrain;  // equal splits
      it.slot = it.n_split > 1 ? slots + __builtin_amdgcn_readlane(slot_end - mine, l) + nth * it.n_split : -1;
      it.s.first = __builtin_amdgcn_readlane(s.first, l);
      it.s.nq = __builtin_amdgcn_readlane(s.nq, l);
      it.s.len = __builtin_amdgcn_readlane(s.len, l);
      return it;
    }
    before += wave_last(end);
    slots += wave_last(slot_end);
  }
  return it;
}

// The kernel of 16 rows, which waits for bytes: all tiles of a head laid end to end, one per query tile of every sequence, a tile
// being its sequence's tokens in units of `grain` and kTileCost units in front of them for what a tile costs by itself.  Every
// worker of the head takes the same share of units, wherever that begins and ends (the quotient rounded up, so that of few units the last workers
// have none), so that the workgroups, which are all resident at once, end about together: 48 ragged sequences of 8 heads as whole splits over 512 workgroups took 80 us.  A border inside a
// tile's first kTileCost units counts as its beginning.
constexpr int kTileCost = 2;
struct Border {
  int b, tile, unit;  // unit 0: the tile's beginning
  int tiles, units;   // of the sequence, of each of its tiles
  int at;             // of the border's tile in the sum of all units
  Seq s;
};
// listed >= 0: every sequence has one tile of that many tokens.
__device__ __forceinline__ int tile_units(const Geometry& g, const Seq& s, int listed, int& tiles) {
  tiles = listed >= 0 ? 1 : (s.nq + g.R - 1) / g.R;
  return max(1, ((listed >= 0 ? listed : s.len) + g.grain - 1) / g.grain) + kTileCost;
}
// Units of a share, and the border at `nth` shares (b = B: there is none).  Up to 64 sequences take one load, one lane each.
__device__ __forceinline__ Border border_of(const Geometry& g, const int* lengths, const int* offsets, int listed, int nth, int& total, int& share) {
  Border r;
  r.b = g.B;
  if (listed >= 0) {
    r.s = Seq{0, 1, 0};
    r.units = tile_units(g, r.s, listed, r.tiles);
    total = r.units * g.B;
    share = (total + g.workers - 1) / g.workers;
    const int x = nth * share;
    if (x >= total) return r;
    r.b = r.s.first = x / r.units;
    r.s.len = seq_of(g, lengths, nullptr, r.b).len;
    r.tile = 0;
    r.at = r.b * r.units;
    r.unit = max(x - r.at - kTileCost, 0);
    return r;
  }
  const int lane = threadIdx.x & 63;
  Seq s{0, 0, 0};
  int tiles = 0, units = 1, end = 0;
  auto look = [&](int b0) {
    s = Seq{0, 0, 0};
    tiles = 0;
    units = 1;
    if (b0 + lane < g.B) {
      s = seq_of(g, lengths, offsets, b0 + lane);
      units = tile_units(g, s, listed, tiles);
    }
    end = wave_inclusive_scan(tiles * units);
  };
  total = 0;
  for (int b0 = 0; b0 < g.B; b0 += 64) {
    look(b0);
    total += wave_last(end);
  }
  share = (total + g.workers - 1) / g.workers;
  const int x = nth * share;
  if (x >= total) return r;
  int before = 0;
  for (int b0 = 0; b0 < g.B; b0 += 64) {
    if (g.B > 64) look(b0);
    const unsigned long long has = __ballot(before + end > x);
    if (has) {
      const int l = __ffsll((long long)has) - 1;
      r.b = b0 + l;
      r.tiles = __builtin_amdgcn_readlane(tiles, l);
      r.units = __builtin_amdgcn_readlane(units, l);
      const int first = before + __builtin_amdgcn_readlane(end, l) - r.tiles * r.units;
      r.tile = (x - first) / r.units;
      r.at = first + r.tile * r.units;
      r.unit = max(x - r.at - kTileCost, 0);
      r.s.first = __builtin_amdgcn_readlane(s.first, l);
      r.s.nq = __builtin_amdgcn_readlane(s.nq, l);
      r.s.len = __builtin_amdgcn_readlane(s.len, l);
      return r;
    }
    before += wave_last(end);
  }
  return r;
}

// Maximum and sum over the four lanes l, l^16, l^32, l^48.
__device__ __forceinline__ float quad_max(float x) {
  u32x2_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  u32x2_t r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ unsigned pack_bf16(float a, float b) {  // nearest even
  const bf16x2_t p = {(__bf16)a, (__bf16)b};
  unsigned u;
  __builtin_memcpy(&u, &p, 4);
  return u;
}

// ------------------------------------------------------------------ how rows are held
// A wave's tile is 16 tokens.  Keys are the first operand of S^T[token][query] = K Q^T, 16x16x32 matrix instructions: lane
// (col = l % 16, quad = l / 16) holds eight dimensions of token `col` per instruction, which ones is free as long as the
// query has the same: `dim` names the first.  Values are the first operand of O^T[dim][query] += V^T P^T: the lane holds
// dimension slot `col` of eight tokens, those whose weights the logits' layout left in the same lane (4 quad .. + 3 of either
// tile), so no weight moves between lanes.  A lane loads D / 16 adjacent dimensions of each of its eight tokens and
// turns them into such columns with byte permutations: no pass through LDS.
struct Fp8 {
  static constexpr int kBytes = 1;
  static constexpr int kFoldAhead = 8;  // parts of a tile that are requested at a time: as many as the registers hold
  template <int D> static constexpr int kLoads = D / 64;  // 16-byte loads of a key row per lane
  __device__ static __forceinline__ int dim(int f, int quad) { return 64 * (f >> 1) + 16 * quad + 8 * (f & 1); }
  __device__ static __forceinline__ int load_dim(int j, int quad) { return 64 * j + 16 * quad; }
  // two values times a power of two: the conversion adds exponents
  static __device__ __forceinline__ unsigned two(unsigned x, bool high, float scale = 1.0f) {
    const bf16x2_t p = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, scale, false);
    unsigned u;
    __builtin_memcpy(&u, &p, 4);
    return u;
  }
  template <int N>
  __device__ static __forceinline__ bf16x8_t fragment(const u32x4_t (&k)[N], int f) {
    const unsigned a = k[f >> 1][2 * (f & 1)], b = k[f >> 1][2 * (f & 1) + 1];
    const u32x4_t w = {two(a, false), two(a, true), two(b, false), two(b, true)};
    bf16x8_t r;
    __builtin_memcpy(&r, &w, 16);
    return r;
  }
  // dimensions 2j, 2j + 1 of the lane's chunk as a pair of bf16
  template <int N>
  __device__ static __forceinline__ unsigned pair(const unsigned (&v)[N], int j) { return two(v[j >> 1], (j & 1) != 0); }
  // the bits of a word's values that are not finite
  __device__ static __forceinline__ unsigned odd(unsigned w) {
    const unsigned t = ~w & 0x7f7f7f7fu;  // zero where the value is
    return ((~(t + 0x7f7f7f7fu) & 0x80808080u) >> 7) * 0xffu;
  }
  // value `dim` of a row if it is not finite, else zero
  __device__ static __forceinline__ float odd_value(const unsigned char* row, int dim) { return (row[dim] & 0x7f) == 0x7f ? __builtin_nanf("") : 0.0f; }
};
struct Bf16 {
  static constexpr int kBytes = 2;
  static constexpr int kFoldAhead = 4;
  template <int D> static constexpr int kLoads = D / 32;
  __device__ static __forceinline__ int dim(int f, int quad) { return 32 * f + 8 * quad; }
  __device__ static __forceinline__ int load_dim(int j, int quad) { return 32 * j + 8 * quad; }
  template <int N>
  __device__ static __forceinline__ bf16x8_t fragment(const u32x4_t (&k)[N], int f) {
    bf16x8_t r;
    __builtin_memcpy(&r, &k[f], 16);
    return r;
  }
  template <int N>
  __device__ static __forceinline__ unsigned pair(const unsigned (&v)[N], int j) { return v[j]; }
  __device__ static __forceinline__ unsigned odd(unsigned w) {
    const unsigned t = ~w & 0x7f807f80u;
    return ((~(t + 0x7fff7fffu) & 0x80008000u) >> 15) * 0xffffu;
  }
  __device__ static __forceinline__ float odd_value(const unsigned char* row, int dim) {
    const unsigned x = reinterpret_cast<const uint16_t*>(row)[dim];
    return (x & 0x7f80u) == 0x7f80u ? __uint_as_float(x << 16) : 0.0f;
  }
};
// Tokens that some queries of a tile see and others do not have a weight of zero for the others, which an infinity or NaN among their values would
// turn into NaN.  Such values are taken out of the product (`odd`) and added to the queries that see them by themselves (`odd_value`).

template <class C, int D>
struct Stage {
  static constexpr int kWords = D / 16 * C::kBytes / 4;  // of a lane's part of a value row
  u32x4_t k[2][C::template kLoads<D>];
  unsigned v[8][kWords];
};
template <int N>
__device__ __forceinline__ void load_words(const unsigned char* p, unsigned (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const unsigned*>(p);
  } else if constexpr (N == 2) {
    const u32x2_t x = *reinterpret_cast<const u32x2_t*>(p);
    w[0] = x[0];
    w[1] = x[1];
  } else {
    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  }
}

// Query fragments (second operand): eight values as one bf16 term, or of single precision as three, whose sum is the value.
template <typename T, class C, int D>
struct Query {
  static constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
  bf16x8_t f[kTerms][D / 32];
  __device__ __forceinline__ void load(const T* row /* nullptr: zero */, int quad) {
#pragma unroll
    for (int i = 0; i < D / 32; ++i) {
      if constexpr (sizeof(T) == 2) {
        u32x4_t x = {0u, 0u, 0u, 0u};
        if (row) x = *reinterpret_cast<const u32x4_t*>(row + C::dim(i, quad));
        __builtin_memcpy(&f[0][i], &x, 16);
      } else {
        f32x4_t a = {0.f, 0.f, 0.f, 0.f}, b = a;
        if (row) {
          a = *reinterpret_cast<const f32x4_t*>(row + C::dim(i, quad));
          b = *reinterpret_cast<const f32x4_t*>(row + C::dim(i, quad) + 4);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float x = e < 4 ? a[e & 3] : b[e & 3];
#pragma unroll
          for (int t = 0; t < 3; ++t) {
            const __bf16 h = (__bf16)x;
            f[t][i][e] = h;
            x -= (float)h;
          }
        }
      }
    }
  }
};

// Running softmax of the lane's query (col) over the tokens so far: O^T[dim][query], maximum (base 2), and the sum over
// this lane's tokens.
template <int D>
struct State {
  f32x4_t o[D / 16];  // o[n][i]: dimension (D / 16) * (4 quad + i) + n
  float m, l;
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int n = 0; n < D / 16; ++n) o[n] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    m = kLowest;
    l = 0.0f;
  }
};

// One step: logits of 32 tokens, one rescaling if a maximum grew, weights, values.  `see(tile, i)` says whether the lane's query
// sees its i-th token of the tile, `live(tile, i)` whether any query of the tile does (else its value row may hold anything, NaN
// among it, and is taken as zero); both only matter if `masked` (wave-uniform).  The weights enter as three bf16 terms,
// whose sum is the fp32 weight: two leave out up to 2^-17 of it, which was the largest error of all over a few tokens (1.1e-6 of
// the result against 1e-7), and the third is free where the bytes of the rows are what the step waits for.
constexpr int kTerms = 3;
// `next_k` and `next_v` request the rows of the wave's next step as soon as this step's are no longer needed.  `partly` (wave-uniform, and masked
// then): some queries may not see what others see; `add_odd` adds the tokens' values that are not finite.
template <typename T, class C, int D, class SeeFn, class LiveFn, class KsFn, class VsFn, class NextK, class NextV, class AddOdd>
__device__ __forceinline__ void attend(Stage<C, D>& st, const Query<T, C, D>& q, State<D>& a, bool masked, bool partly, SeeFn see, LiveFn live, KsFn ks,
                                       VsFn vs, NextK next_k, NextV next_v, AddOdd add_odd) {
  float s[2][4];
  float mx = kLowest;
#pragma unroll
  for (int tl = 0; tl < 2; ++tl) {
    f32x4_t acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int f = 0; f < D / 32; ++f) {
      const bf16x8_t k = C::fragment(st.k[tl], f);
#pragma unroll
      for (int t = 0; t < Query<T, C, D>::kTerms; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q.f[t][f], acc, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[tl][i] = acc[i] * ks(tl, i);
  }
  next_k();
  PQC_LOADS_ISSUED();
  if (masked) {
#pragma unroll
    for (int tl = 0; tl < 2; ++tl)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!see(tl, i)) s[tl][i] = -INFINITY;
        if (!live(tl, i)) {
#pragma unroll
          for (int w = 0; w < Stage<C, D>::kWords; ++w) st.v[4 * tl + i][w] = 0u;
        }
      }
  }
  bool found = false;
  if (partly) {
    unsigned any = 0u;
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int w = 0; w < Stage<C, D>::kWords; ++w) {
        const unsigned odd = C::odd(st.v[e][w]);
        st.v[e][w] &= ~odd;
        any |= odd;
      }
    found = __any(any != 0u);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) mx = fmaxf(mx, fmaxf(s[0][i], s[1][i]));
  const float mnew = fmaxf(a.m, quad_max(mx));
  if (__any(mnew > a.m)) {
    const float corr = __builtin_amdgcn_exp2f(a.m - mnew);
    a.m = mnew;
    a.l *= corr;
#pragma unroll
    for (int n = 0; n < D / 16; ++n) a.o[n] *= corr;
  }
  u32x4_t term[kTerms];
#pragma unroll
  for (int tl = 0; tl < 2; ++tl)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      float p0 = __builtin_amdgcn_exp2f(s[tl][i] - a.m), p1 = __builtin_amdgcn_exp2f(s[tl][i + 1] - a.m);
      a.l += p0 + p1;
      p0 *= vs(tl, i);
      p1 *= vs(tl, i + 1);
#pragma unroll
      for (int t = 0; t < kTerms; ++t) {
        const unsigned h = pack_bf16(p0, p1);
        term[t][2 * tl + i / 2] = h;
        p0 -= __uint_as_float(h << 16);
        p1 -= __uint_as_float(h & 0xffff0000u);
      }
    }
  bf16x8_t p[kTerms];
#pragma unroll
  for (int t = 0; t < kTerms; ++t) __builtin_memcpy(&p[t], &term[t], 16);
#pragma unroll
  for (int j = 0; j < D / 32; ++j) {
    unsigned w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = C::pair(st.v[e], j);
    u32x4_t even, odd;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      even[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x05040100u);
      odd[e] = __builtin_amdgcn_perm(w[2 * e + 1], w[2 * e], 0x07060302u);
    }
    bf16x8_t v0, v1;
    __builtin_memcpy(&v0, &even, 16);
    __builtin_memcpy(&v1, &odd, 16);
#pragma unroll
    for (int t = 0; t < kTerms; ++t) {
      a.o[2 * j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v0, p[t], a.o[2 * j], 0, 0, 0);
      a.o[2 * j + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v1, p[t], a.o[2 * j + 1], 0, 0, 0);
    }
  }
  next_v();
  PQC_LOADS_ISSUED();
  if (found) add_odd();
}

__device__ __forceinline__ void store_out(const Geometry& g, void* out, size_t at, float x) {
  if (g.out_bf16)
    static_cast<__bf16*>(out)[at] = (__bf16)x;
  else
    static_cast<float*>(out)[at] = x;
}

// Of a row's softmax weights.  0 for a row that saw nothing; a sum that is not a number stays one (a NaN in the query or in a key that it sees,
// a logit of +inf), whichever kernel comes to it.
__device__ __forceinline__ float reciprocal_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }

// A barrier for LDS alone: loads from memory stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

constexpr size_t rows_static_lds(int dim) { return 4 * kStaged * 4 + (size_t)kWaves * kRows * (dim + 2) * 4 + 12; }

// Parts of a tile travel between workgroups of one kernel that may run on different dies, whose L2 caches don't see each other: they are
// written and read as relaxed atomics of device scope, which go through to memory.  (Plain stores with a release fence, which
// writes back the whole L2, and an acquire fence cost 9 us on a call of 12 and 18 on one of 60.)
__device__ __forceinline__ void store_part(float* p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float2 load_part2(const float* p) {  // 8-byte aligned
  const unsigned long long u = __hip_atomic_load(reinterpret_cast<const unsigned long long*>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)u), __uint_as_float((unsigned)(u >> 32)));
}

// Folds `n` parts of rows row0 .. row1 - 1 of a tile, in one pass over them with a running maximum: D / 4 lanes per row, and as many lanes groups per row (`side`)
// as the workgroup has, whose results meet in LDS.  part(i): where the i-th
// lies.  AHEAD of them are requested at a time. 
template <int D, int AHEAD, class PartFn>
__device__ __forceinline__ void fold_parts(const Geometry& g, const Seq& s, int tile, int h, int row0, int row1, int n, PartFn part, void* out, f32x4_t* red_o /* [256] */,
                                           float2* red_ml /* [256 * 4 / D] */) {
  constexpr int kLanes = D / 4, kGroups = 256 / kLanes, kAhead = AHEAD;
  const int rows = g.R * g.G;
  int sides = kGroups;  // a power of two with sides * rows <= kGroups, if there is one
  while (sides > 1 && sides * (row1 - row0) > kGroups) sides >>= 1;
  const int at = threadIdx.x % kLanes, group = threadIdx.x / kLanes, side = group & (sides - 1), at_once = kGroups / sides;
  for (int r0 = row0; r0 < row1; r0 += at_once) {
    const int r = r0 + group / sides, qr = tile * g.R + r / g.G;
    const bool live = r < row1 && qr < s.nq;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    float m = kLowest, l = 0.0f;
    if (live) {
      for (int i = side; i < n; i += kAhead * sides) {
        float2 ml[kAhead];
        f32x4_t x[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {  // past the end the last part is read again and left out
          const float* p = part(min(i + e * sides, n - 1));
          ml[e] = load_part2(p + rows * D + 2 * r);
          const float2 x0 = load_part2(p + r * D + 4 * at), x1 = load_part2(p + r * D + 4 * at + 2);
          x[e] = f32x4_t{x0.x, x0.y, x1.x, x1.y};
          if (i + e * sides >= n) ml[e] = make_float2(-INFINITY, 0.0f);
        }
        float mnew = m;
#pragma unroll
        for (int e = 0; e < kAhead; ++e) mnew = fmaxf(mnew, ml[e].x);
        const float corr = __builtin_amdgcn_exp2f(m - mnew);
        m = mnew;
        l *= corr;
        o *= corr;
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const float f = __builtin_amdgcn_exp2f(ml[e].x - m);
          l += f * ml[e].y;
          o += f * x[e];
        }
      }
    }
    if (sides > 1) {
      __syncthreads();  // the rows before have been read
      red_o[threadIdx.x] = o;
      if (at == 0) red_ml[group] = make_float2(m, l);
      __syncthreads();
      if (side == 0) {
        for (int e = 1; e < sides; ++e) m = fmaxf(m, red_ml[group + e].x);
        l = 0.0f;
        o = f32x4_t{0.f, 0.f, 0.f, 0.f};
        for (int e = 0; e < sides; ++e) {
          const float f = __builtin_amdgcn_exp2f(red_ml[group + e].x - m);
          l += f * red_ml[group + e].y;
          o += f * red_o[threadIdx.x + e * kLanes];
        }
      }
    }
    if (side == 0 && live) {
      const size_t a = ((size_t)(s.first + qr) * g.Hq + (size_t)h * g.G + r % g.G) * D + 4 * at;
      o *= reciprocal_sum(l);
      if (g.out_bf16)
        *reinterpret_cast<u32x2_t*>(static_cast<bf16_t*>(out) + a) = u32x2_t{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
      else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(out) + a) = o;
    }
  }
}

// A stretch of a tile: as much of a worker's part of it as has its pages in LDS at a time.
struct Stretch {
  Border t;
  bool begins, ends;  // the worker begins the tile, ends it
  int most;           // tokens that some query of the tile sees
  int from, to, stop; // tokens of the stretch, end of the worker's part
};

// Attention of tiles of up to 16 query rows.  Each workgroup goes through its share of the head's tiles; four waves take 32 tokens
// of a tile each in turn, with a softmax state of their own, folded at the tile's end.  What a workgroup has of a tile that it does not
// finish, or not begin, goes to `partials` as (O, m, l): place 2 w + 1 of worker w for a tile that it begins, 2 w for one that it goes on with.
// Loads never stop at a stretch's end: the next one's pages are looked up while this one is computed, and its first rows are
// requested before this one's waves are folded.
// LISTED: one query token per sequence, over the tokens that idx names; entries outside the sequence are left out.
template <typename T, class C, int D, bool LISTED>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(Geometry g, Cache c, const T* __restrict__ q, const int* __restrict__ offsets,
                                                           const int* __restrict__ idx, int n_idx, void* __restrict__ out, float* __restrict__ partials) {
  __shared__ int place[2][kStaged];  // page, or row of the listed token; negative: none
  __shared__ float kscale[kStaged], vscale[kStaged];
  __shared__ float red_o[kWaves][kRows][D];
  __shared__ float red_m[kWaves][kRows], red_l[kWaves][kRows];
  __shared__ int missing[2];  // a page of the stretch is not there
  __shared__ int last_part;
  constexpr int kPer = kStaged / 256;
  constexpr bool kScaled = C::kBytes == 1;
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);  // scalar, and so are the addresses of the wave's pages
  const int worker = blockIdx.x / g.Hkv, h = blockIdx.x - worker * g.Hkv;
  const int rows = g.R * g.G;
  const size_t row_bytes = (size_t)D * C::kBytes;
  const int my_token = col / g.G, my_head = col - my_token * g.G;
  int total, share;
  Stretch now;
  now.t = border_of(g, c.lengths, offsets, LISTED ? n_idx : -1, worker, total, share);
  if (now.t.b >= g.B) return;
  const int x_end = min((worker + 1) * share, total);
  // (an even number of pages: a stretch is a multiple of 32 tokens)
  const int most_staged = LISTED ? kStaged : ((kStaged - 2) << g.shift);
  // the worker's part of tile y.t; false: it has none
  auto enter = [&](Stretch& y) {
    y.begins = y.t.unit == 0;
    y.ends = x_end >= y.t.at + y.t.units;
    const int last = y.ends ? 0 : max(x_end - y.t.at - kTileCost, 0);
    if (!y.ends && y.begins && last == 0) return false;
    const int hidden = y.t.s.len - y.t.s.nq;
    y.most = LISTED ? n_idx : max(hidden + min((y.t.tile + 1) * g.R, y.t.s.nq), 0);
    y.from = y.t.unit * g.grain;
    y.stop = y.ends ? y.most : min(last * g.grain, y.most);
    y.to = min(y.from + most_staged, y.stop);
    return true;
  };
  auto advance = [&](Stretch& y) {
    if (y.to < y.stop) {
      y.from = y.to;
      y.to = min(y.from + most_staged, y.stop);
      return true;
    }
    y.t.at += y.t.units;
    if (y.t.at >= x_end) return false;
    if (y.t.tile + 1 < y.t.tiles) {
      ++y.t.tile;
    } else {
      do {  // the next sequence that has a query
        if (++y.t.b >= g.B) return false;
        y.t.s = seq_of(g, c.lengths, LISTED ? nullptr : offsets, y.t.b);
        y.t.units = tile_units(g, y.t.s, LISTED ? n_idx : -1, y.t.tiles);
      } while (y.t.tiles == 0);
      y.t.tile = 0;
    }
    y.t.unit = 0;
    return enter(y);
  };
  int raw[kPer];  // entries of the page table or of the list
  auto look_up = [&](const Stretch& y) {
    const int p0 = y.from >> g.shift, n = LISTED ? y.to - y.from : ((y.to - 1) >> g.shift) - p0 + 1;
    const int* at = LISTED ? idx + ((size_t)y.t.b * g.Hkv + h) * n_idx + y.from : c.table + (size_t)y.t.b * g.max_pages + p0;
    if constexpr (LISTED) {
      if (y.from >= n_idx) at = idx;  // (an empty stretch reads some entry)
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) raw[e] = at[max(min((int)threadIdx.x + 256 * e, n - 1), 0)];
  };
  float ks[kPer], vs[kPer];
  auto put_places = [&](const Stretch& y, int buf) {
    int row[kPer];
    if constexpr (LISTED) {
      const int* table = c.table + (size_t)y.t.b * g.max_pages;
#pragma unroll
      for (int e = 0; e < kPer; ++e) {
        const int t = raw[e];
        row[e] = t & (g.P - 1);
        raw[e] = t >= 0 && t < y.t.s.len ? table[t >> g.shift] : -1;
      }
    }
    bool bad = false;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const bool ok = raw[e] >= 0 && raw[e] < g.n_pages;
      bad |= !ok;
      const size_t p = (size_t)(ok ? raw[e] : 0) * g.Hkv + h;
      ks[e] = kScaled ? c.ks[p] : 1.0f;
      vs[e] = kScaled ? c.vs[p] : 1.0f;
      place[buf][threadIdx.x + 256 * e] = !ok ? -1 : LISTED ? (int)(p << g.shift) + row[e] : raw[e];
      if (!ok) ks[e] = vs[e] = 0.0f;
    }
    if (bad) missing[buf] = 1;
  };
  auto at = [&](const Stretch& y, int t) { return LISTED ? t - y.from : (t >> g.shift) - (y.from >> g.shift); };
  Stage<C, D> st;
  auto issue_k = [&](const Stretch& y, int buf, int t) {
#pragma unroll
    for (int tl = 0; tl < 2; ++tl) {
      const int tt = t + 16 * tl;
      if constexpr (LISTED) {
        const unsigned char* kp = c.k + (size_t)max(place[buf][at(y, tt + col)], 0) * row_bytes;
#pragma unroll
        for (int j = 0; j < C::template kLoads<D>; ++j) st.k[tl][j] = *reinterpret_cast<const u32x4_t*>(kp + C::load_dim(j, quad) * C::kBytes);
      } else {
        const int pg = __builtin_amdgcn_readfirstlane(max(place[buf][at(y, tt)], 0));
        const unsigned char* kp = c.k + ((((size_t)pg * g.Hkv + h) << g.shift) + (tt & (g.P - 1))) * row_bytes;
#pragma unroll
        for (int j = 0; j < C::template kLoads<D>; ++j)
          st.k[tl][j] = *reinterpret_cast<const u32x4_t*>(kp + (unsigned)((col * D + C::load_dim(j, quad)) * C::kBytes));
      }
    }
  };
  auto issue_v = [&](const Stretch& y, int buf, int t) {
#pragma unroll
    for (int tl = 0; tl < 2; ++tl) {
      const int tt = t + 16 * tl;
      if constexpr (LISTED) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          load_words(c.v + (size_t)max(place[buf][at(y, tt + 4 * quad + i)], 0) * row_bytes + col * (D / 16) * C::kBytes, st.v[4 * tl + i]);
      } else {
        const int pg = __builtin_amdgcn_readfirstlane(max(place[buf][at(y, tt)], 0));
        const unsigned char* vp = c.v + ((((size_t)pg * g.Hkv + h) << g.shift) + (tt & (g.P - 1))) * row_bytes;
#pragma unroll
        for (int i = 0; i < 4; ++i) load_words(vp + (unsigned)(((4 * quad + i) * D + col * (D / 16)) * C::kBytes), st.v[4 * tl + i]);
      }
    }
  };
  auto first_rows = [&](const Stretch& y, int buf) {
    const int t = y.from + wave * kStep;
    if (t < y.to) {
      issue_k(y, buf, t);
      issue_v(y, buf, t);
    }
    PQC_LOADS_ISSUED();
  };
  if (!enter(now)) return;
  Query<T, C, D> qf;
  State<D> a;
  int lim = 0, least = 0;
  auto add_odd = [&](int t, int buf) {
    for (int tt = t; tt < min(t + kStep, now.most); ++tt) {
      const int page = place[buf][at(now, tt)];
      if (page < 0 || tt >= lim) continue;
      const unsigned char* row = c.v + ((((size_t)page * g.Hkv + h) << g.shift) + (tt & (g.P - 1))) * row_bytes;
#pragma unroll
      for (int n = 0; n < D / 16; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) a.o[n][i] += C::odd_value(row, D / 16 * (4 * quad + i) + n);
    }
  };
  look_up(now);
  if (threadIdx.x < 2) missing[threadIdx.x] = 0;
  __syncthreads();
  put_places(now, 0);
  lds_barrier();
  first_rows(now, 0);
  bool fresh = true;  // a tile begins
  for (int buf = 0;; buf ^= 1) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      kscale[threadIdx.x + 256 * e] = ks[e] * g.scale_log2e;
      vscale[threadIdx.x + 256 * e] = vs[e];
    }
    if (threadIdx.x == 0) missing[buf ^ 1] = 0;
    Stretch next = now;
    const bool more = advance(next);
    if (more) look_up(next);
    if (fresh) {
      const Seq& s = now.t.s;
      const int qi = now.t.tile * g.R + my_token;  // the lane's query token
      const bool row_ok = col < rows && qi < s.nq;
      // tokens that the lane's query and the tile's first one see
      lim = row_ok ? max(LISTED ? n_idx : s.len - s.nq + qi + 1, 0) : 0;
      least = LISTED ? n_idx : max(s.len - s.nq + now.t.tile * g.R + 1, 0);
      qf.load(row_ok ? q + ((size_t)(s.first + qi) * g.Hq + (size_t)h * g.G + my_head) * D : nullptr, quad);
      a.init();
    }
    lds_barrier();
    const bool any_missing = missing[buf] != 0;
    const int most = now.most;
    for (int t = now.from + wave * kStep; t < now.to; t += kGrain) {
      const bool again = t + kGrain < now.to;
      auto token = [&](int tl, int i) { return t + 16 * tl + 4 * quad + i; };
      auto slot = [&](int tl, int i) { return at(now, LISTED ? token(tl, i) : t + 16 * tl); };
      attend<T, C, D>(
          st, qf, a, any_missing || t + kStep > least, !LISTED && g.R > 1 && t + kStep > least, [&](int tl, int i) { return token(tl, i) < lim && place[buf][slot(tl, i)] >= 0; },
          [&](int tl, int i) { return token(tl, i) < most && place[buf][slot(tl, i)] >= 0; }, [&](int tl, int i) { return kscale[slot(tl, i)]; },
          [&](int tl, int i) { return vscale[slot(tl, i)]; },
          [&]() {
            if (again) issue_k(now, buf, t + kGrain);
          },
          [&]() {
            if (again) issue_v(now, buf, t + kGrain);
          },
          [&]() { add_odd(t, buf); });
    }
    if (more) put_places(next, buf ^ 1);
    lds_barrier();
    if (more) first_rows(next, buf ^ 1);
    fresh = now.to >= now.stop;
    if (fresh) {  // fold the waves
      const float l = quad_sum(a.l);
      if (quad == 0) {
        red_m[wave][col] = a.m;
        red_l[wave][col] = l;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int n = 0; n < D / 16; ++n) red_o[wave][col][D / 16 * (4 * quad + i) + n] = a.o[n][i];
      lds_barrier();
      const bool whole = now.begins && now.ends;
      const size_t one = partial_floats(rows, D);
      float* po = partials + ((size_t)(2 * worker + (now.begins ? 1 : 0)) * g.Hkv + h) * one;
      for (int i = threadIdx.x; i < rows * D; i += 256) {
        const int r = i / D, d = i % D;
        float m = red_m[0][r], sum = 0.0f, o = 0.0f;
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, red_m[w][r]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          const float f = __builtin_amdgcn_exp2f(red_m[w][r] - m);
          sum += f * red_l[w][r];
          o += f * red_o[w][r][d];
        }
        if (!whole) {
          store_part(po + i, o);
          if (d == 0) {
            store_part(po + rows * D + 2 * r, m);
            store_part(po + rows * D + 2 * r + 1, sum);
          }
        } else {
          const int qr = now.t.tile * g.R + r / g.G;
          if (qr < now.t.s.nq) store_out(g, out, ((size_t)(now.t.s.first + qr) * g.Hq + (size_t)h * g.G + r % g.G) * D + d, sum == 0.0f ? 0.0f : o / sum);  // as reciprocal_sum
        }
      }
      if (!whole && c.counters) {
        // The last of the tile's workgroups to come here folds all parts: every wave's stores have reached memory before it meets the
        // barrier in front of the count, and what is read behind the count is read from there.
        const int w1 = (now.t.at + kTileCost) / share + 1;  // the first border inside the tile
        const int parts = (now.t.at + now.t.units - 1) / share - w1 + 2;
        if (w1 >= g.workers) return;  // (offsets that do not ascend)
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0) {
          unsigned* count = c.counters + (size_t)w1 * g.Hkv + h;
          last_part = __hip_atomic_fetch_add(count, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (unsigned)(parts - 1);
          if (last_part) __hip_atomic_store(count, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        __syncthreads();
        if (last_part) {
          fold_parts<D, C::kFoldAhead>(g, now.t.s, now.t.tile, h, 0, rows, parts,
                        [&](int i) { return partials + ((size_t)(2 * (w1 - 1 + i) + (i == 0 ? 1 : 0)) * g.Hkv + h) * one; }, out,
                        reinterpret_cast<f32x4_t*>(&red_o[0][0][0]), reinterpret_cast<float2*>(&red_m[0][0]));
          __syncthreads();
        }
      }
    }
    if (!more) return;
    now = next;
  }
}

// The parts of tiles of the kernel of 16 rows where that does not fold them itself: one workgroup per (border between workers, head, row).  The first
// border inside a tile stands for it.
template <class C, int D>
__global__ __launch_bounds__(256) void attn_fold_kernel(Geometry g, const int* __restrict__ lengths, const int* __restrict__ offsets, int listed,
                                                        const float* __restrict__ partials, void* __restrict__ out) {
  __shared__ f32x4_t red_o[256];
  __shared__ float2 red_ml[256 * 4 / D];
  const int w = blockIdx.x + 1, h = blockIdx.y;
  int total, share;
  const Border e = border_of(g, lengths, offsets, listed, w, total, share);
  if (e.b >= g.B || e.unit == 0 || (w - 1) * share > e.at + kTileCost) return;
  const size_t one = partial_floats(g.R * g.G, D);
  fold_parts<D, C::kFoldAhead>(g, e.s, e.tile, h, blockIdx.z, blockIdx.z + 1, (e.at + e.units - 1) / share - w + 2,
                [&](int i) { return partials + ((size_t)(2 * (w - 1 + i) + (i == 0 ? 1 : 0)) * g.Hkv + h) * one; }, out, red_o, red_ml);
}

// ------------------------------------------------------------------ many queries
// Attention of tiles of 128 query rows: bound by the matrix cores and by the vector ALU's exponentials, not by bytes, so that
// keys and values are brought into the form of the matrix instructions once per workgroup (LDS) and not once per 16 rows.
// Four waves hold 32 rows each.  Per 64 tokens: S^T[64][32] = K Q^T and O^T[D][32] += V^T P^T, 32x32x16 instructions, whose first
// operands are 16-byte LDS reads.  A wave's logits leave the first product in the lanes that need the weights as second operand
// of the other one (lane col = query, half = l / 32: tokens 8 j + 4 half + 0..3), which the token order of V^T in LDS follows.
//   K   [64 tokens][D]: 16-byte chunk c of token t lies at c ^ (t & 7)
//   V^T [D][64 tokens]: chunk 2 k + half of dimension d, tokens 16 k + 4 half + {0..3, 8..11}, lies at c ^ (d ^ (d >> 2)) & 7
// so that neither the staging stores nor the operands' reads meet in a bank.  The next 64 tokens' rows are loaded while these are
// computed, the page of those behind them one round earlier.
typedef __attribute__((ext_vector_type(16))) float f32x16_t;

// Keys of 64 tokens and values of 64 others on their way from the pages to LDS.  A wave brings 16 of either, which lie in one page, so
// that pages, scales and addresses are scalar.
template <class C, int D>
struct BlockStage {
  static constexpr int kK = D / 64 * C::kBytes;   // 16-byte loads of keys per thread: token tid / 4
  static constexpr int kV = C::kBytes;            // words of each of eight tokens' values: four dimensions
  static constexpr int kVLanes = D / 2;           // lanes of a wave that bring values
  u32x4_t k[kK];
  unsigned v[8][kV];
  float ks, vs;
  bool k_ok, v_ok;
  int vzero;  // 0 in a vector register: pages and scales come by vector loads, which keep their order.  A scalar load that misses is
              // what every wait for LDS behind it waits for too.

  // `t`: the wave's first token, `page`: its page, negative if there is none
  __device__ __forceinline__ void load_k(const Geometry& g, const Cache& c, int h, int t, int page) {
    const int lane = threadIdx.x & 63, q = lane & 3;
    k_ok = page >= 0;
    const size_t p = (size_t)max(page, 0) * g.Hkv + h;
    ks = C::kBytes == 1 ? c.ks[p + vzero] : 1.0f;
    const unsigned char* kr = c.k + ((p << g.shift) + (t & (g.P - 1))) * (size_t)(D * C::kBytes);
#pragma unroll
    for (int j = 0; j < kK; ++j) {
      const int dim = C::kBytes == 1 ? 64 * j + 16 * q : 64 * (j >> 1) + 16 * q + 8 * (j & 1);
      k[j] = *reinterpret_cast<const u32x4_t*>(kr + (unsigned)((lane / 4 * D + dim) * C::kBytes));
    }
  }
  __device__ __forceinline__ void load_v(const Geometry& g, const Cache& c, int h, int t, int page) {
    const int lane = threadIdx.x & 63;
    v_ok = page >= 0;
    const size_t p = (size_t)max(page, 0) * g.Hkv + h;
    vs = C::kBytes == 1 ? c.vs[p + vzero] : 1.0f;
    if (lane < kVLanes) {
      const unsigned char* vr = c.v + ((p << g.shift) + (t & (g.P - 1))) * (size_t)(D * C::kBytes);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        load_words(vr + (unsigned)(((4 * (lane / (D / 4)) + (e < 4 ? e : e + 4)) * D + lane % (D / 4) * 4) * C::kBytes), v[e]);
    }
  }
  // Tokens from `most` on are zero, and those of pages that are not there: their rows may hold anything.
  __device__ __forceinline__ void clear_k(int t, int most) {
    if (!k_ok || t + (int)(threadIdx.x & 63) / 4 >= most) {
#pragma unroll
      for (int j = 0; j < kK; ++j) k[j] = u32x4_t{0u, 0u, 0u, 0u};
    }
    if (!k_ok) ks = 1.0f;
  }
  __device__ __forceinline__ void clear_v(int t, int most) {
    const int first = t + 4 * ((threadIdx.x & 63) / (D / 4));
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!v_ok || first + (e < 4 ? e : e + 4) >= most) {
#pragma unroll
        for (int i = 0; i < kV; ++i) v[e][i] = 0u;
      }
    if (!v_ok) vs = 1.0f;
  }
  // Takes values that are not finite out; true where a lane had some.
  __device__ __forceinline__ bool clear_odd() {
    unsigned any = 0u;
    if ((threadIdx.x & 63) < kVLanes) {
#pragma unroll
      for (int e = 0; e < 8; ++e)
#pragma unroll
        for (int i = 0; i < kV; ++i) {
          const unsigned odd = C::odd(v[e][i]);
          v[e][i] &= ~odd;
          any |= odd;
        }
    }
    return any != 0u;
  }
  __device__ __forceinline__ void store_k(unsigned char* lk) const {
    const int tid = threadIdx.x, row = tid / 4, q = tid & 3;
    unsigned char* kr = lk + row * (D * 2);
#pragma unroll
    for (int j = 0; j < D / 64; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        u32x4_t w;
        if constexpr (C::kBytes == 1)
          w = u32x4_t{C::two(k[j][2 * e], false, ks), C::two(k[j][2 * e], true, ks), C::two(k[j][2 * e + 1], false, ks), C::two(k[j][2 * e + 1], true, ks)};
        else
          w = k[2 * j + e];
        *reinterpret_cast<u32x4_t*>(kr + (((8 * j + 2 * q + e) ^ (row & 7)) << 4)) = w;
      }
  }
  __device__ __forceinline__ void store_v(unsigned char* lv, int wave) const {
    const int lane = threadIdx.x & 63;
    if (lane >= kVLanes) return;
    const int chunk = 2 * wave + lane / (D / 4), dg = lane % (D / 4);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      u32x4_t even, odd;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        unsigned a, b;
        if constexpr (C::kBytes == 1) {
          a = C::two(v[2 * e][0], j == 1, vs);
          b = C::two(v[2 * e + 1][0], j == 1, vs);
        } else {
          a = v[2 * e][j];
          b = v[2 * e + 1][j];
        }
        even[e] = __builtin_amdgcn_perm(b, a, 0x05040100u);
        odd[e] = __builtin_amdgcn_perm(b, a, 0x07060302u);
      }
      const int d = 4 * dg + 2 * j;
      *reinterpret_cast<u32x4_t*>(lv + d * 128 + ((chunk ^ ((d ^ (d >> 2)) & 7)) << 4)) = even;
      *reinterpret_cast<u32x4_t*>(lv + (d + 1) * 128 + ((chunk ^ (((d + 1) ^ ((d + 1) >> 2)) & 7)) << 4)) = odd;
    }
  }
};

// The conversion of codes takes a scale's power of two alone.  Of its bits: what there is beside (a sign or a significand), and that as a factor.
__device__ __forceinline__ unsigned beside_power(unsigned scale) { return scale & 0x807fffffu; }
__device__ __forceinline__ float rest_of_scale(unsigned scale) {
  return __uint_as_float((scale & 0x7f800000u) == 0x7f800000u ? 0x7fc00000u : beside_power(scale) | 0x3f800000u);
}

// Folds the splits of the tiles of the kernel below: many rows, few splits.
template <int D>
__global__ __launch_bounds__(256) void attn_block_fold_kernel(Geometry g, const int* __restrict__ lengths, const int* __restrict__ offsets,
                                                              const float* __restrict__ partials, void* __restrict__ out) {
  constexpr int kLanes = D / 4, kAtOnce = 256 / kLanes;
  const int h = blockIdx.y, rows = g.R * g.G, at = threadIdx.x % kLanes;
  const Item it = find_item(g, lengths, offsets, blockIdx.x, true);
  if (it.b < 0) return;
  const size_t one = partial_floats(rows, D), stride = (size_t)g.Hkv * one;
  const float* base = partials + (size_t)it.slot * stride + h * one;
  for (int r = blockIdx.z * kAtOnce + threadIdx.x / kLanes; r < rows; r += gridDim.z * kAtOnce) {
    const int qr = it.tile * g.R + r / g.G;
    if (qr >= it.s.nq) return;
    float m = kLowest, l = 0.0f;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
    for (int i = 0; i < it.n_split; ++i) {
      const float* p = base + i * stride;
      const float2 ml = *reinterpret_cast<const float2*>(p + rows * D + 2 * r);
      const f32x4_t x = *reinterpret_cast<const f32x4_t*>(p + r * D + 4 * at);
      const float mnew = fmaxf(m, ml.x), corr = __builtin_amdgcn_exp2f(m - mnew), f = __builtin_amdgcn_exp2f(ml.x - mnew);
      m = mnew;
      l = l * corr + f * ml.y;
      o = o * corr + f * x;
    }
    const size_t a = ((size_t)(it.s.first + qr) * g.Hq + (size_t)h * g.G + r % g.G) * D + 4 * at;
    o *= reciprocal_sum(l);
    if (g.out_bf16)
      *reinterpret_cast<u32x2_t*>(static_cast<bf16_t*>(out) + a) = u32x2_t{pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3])};
    else
      *reinterpret_cast<f32x4_t*>(static_cast<float*>(out) + a) = o;
  }
}

// TERMS: bf16 terms of a weight: three, which is all of it, for an fp32 output, two for a bf16 output (2^-17 of a weight, of the output's own
// rounding a 512th).  One, 2^-8, moves a bf16 output by as much again as its rounding does: prompts of 8192 tokens 2.1e-3 off 64 bits,
// with two 1.63e-3, which is the rounding alone, for 1.3 times the time.
// The vector ALU has as much to do as the matrix cores (64 tokens, one wave: 32 exponentials and some 300 other instructions against 48
// matrix instructions of 32 cycles; busy 57 % and 49 % of the time), so the two run side by side within a wave: the weights of a round's tokens
// are computed while the values of the round before are multiplied, keys being a round ahead of values.  Two workgroups share a compute
// unit (one alone takes 1.4 times as long).  Prompts of 8192 tokens, 32 query heads, 8 KV heads: 757 to 799 us over several runs, 688 to 726
// TFLOP/s; for an fp32 output 900 to 976.  (Measured with one term, 581 us: round after round without the overlap 634; operands read one
// instruction ahead instead of four 604.)  Splitting weights into terms as they are computed instead of in front of their product took 766
// against 757.  64 rows per wave, which would halve the reads of LDS, need more registers than the vector ALU reaches and spend the gain on copies.
// Of that time 1.5 % are for scales that may be no powers of two.
template <typename T, class C, int D, int TERMS>
__global__ __launch_bounds__(256, sizeof(T) == 4 && D == 128 ? 1 : 2) void attn_block_kernel(Geometry g, Cache c, const T* __restrict__ q,
                                                                                            const int* __restrict__ offsets,
                                                            void* __restrict__ out, float* __restrict__ partials) {
  __shared__ __align__(16) unsigned char lds_k[2][kBlockTokens * D * 2], lds_v[2][kBlockTokens * D * 2];
  // A byte per 16 tokens of keys: their page is there (1), its scale is no power of two (2), nor that of the values one round earlier (4); and
  // what those scales are beside their powers of two.
  __shared__ unsigned present[2];
  __shared__ float k_rest[2][4], v_rest[2][4];
  __shared__ int odd_values;       // of tokens that not all rows see some were not finite, and were taken out
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // the heads of a KV head's tokens follow each other, so that with eight of them an XCD's L2 holds the rows of one
  const int item = blockIdx.x / g.Hkv, h = blockIdx.x - item * g.Hkv;
  const Item it = find_item(g, c.lengths, offsets, item, false);
  if (it.b < 0) return;
  const int r = 32 * wave + col, qi = it.tile * g.R + r / g.G;
  const bool row_ok = r < g.R * g.G && qi < it.s.nq;
  const int hidden = it.s.len - it.s.nq;
  const int lim = row_ok ? max(hidden + qi + 1, 0) : 0;
  const int most = max(hidden + min((it.tile + 1) * g.R, it.s.nq), 0);
  // what the wave's first and last rows see
  const int row0 = 32 * wave, row1 = min(row0 + 31, g.R * g.G - 1);
  const int least = row0 < g.R * g.G ? hidden + it.tile * g.R + row0 / g.G + 1 : 0;
  const int wave_most = row0 < g.R * g.G ? min(most, hidden + it.tile * g.R + row1 / g.G + 1) : 0;
  constexpr int kQ = sizeof(T) == 4 ? 3 : 1;  // bf16 terms of a query's value
  bf16x8_t qf[kQ][D / 16];
  {
    const T* row = q + ((size_t)(it.s.first + qi) * g.Hq + (size_t)h * g.G + r % g.G) * D + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      if constexpr (kQ == 1) {
        u32x4_t x = {0u, 0u, 0u, 0u};
        if (row_ok) x = *reinterpret_cast<const u32x4_t*>(row + 16 * i);
        __builtin_memcpy(&qf[0][i], &x, 16);
      } else {
        f32x4_t x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if (row_ok) {
          x[0] = *reinterpret_cast<const f32x4_t*>(row + 16 * i);
          x[1] = *reinterpret_cast<const f32x4_t*>(row + 16 * i + 4);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float y = x[e >> 2][e & 3];
#pragma unroll
          for (int t = 0; t < kQ; ++t) {
            const __bf16 b = (__bf16)y;
            qf[t][i][e] = b;
            y -= (float)b;
          }
        }
      }
    }
  }
  f32x16_t o[D / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.0f;
  float m = kLowest, l = 0.0f;

  const int all_see = hidden + it.tile * g.R + 1;  // tokens that every row sees
  if (tid == 0) odd_values = 0;
  const int t0 = it.split * it.tokens, t1 = it.n_split == 1 ? most : min(t0 + it.tokens, most);
  const int rounds = t0 < t1 ? (t1 - t0 + kBlockTokens - 1) / kBlockTokens : 0;
  const int mine = min(rounds, max(0, (wave_most - t0 + kBlockTokens - 1) / kBlockTokens));  // that the wave's rows see anything of
  if (rounds > 0) {
    const int* table = c.table + (size_t)it.b * g.max_pages;
    BlockStage<C, D> st;
    asm("v_mov_b32 %0, 0" : "=v"(st.vzero));
    auto page_of = [&](int i) {  // of the wave's tokens of round i
      const int t = t0 + i * kBlockTokens + 16 * wave;
      return t < t1 ? table[(t >> g.shift) + st.vzero] : -1;
    };
    auto valid = [&](int loaded) {
      const int p = __builtin_amdgcn_readfirstlane(loaded);
      return p < g.n_pages ? p : -1;
    };
    auto wave_token = [&](int i) { return t0 + i * kBlockTokens + 16 * wave; };
    auto put_v = [&](int i) {
      if (!st.v_ok || wave_token(i) + 16 > most) st.clear_v(wave_token(i), most);
      if (wave_token(i) + 16 > all_see && st.clear_odd()) odd_values = 1;
      st.store_v(lds_v[i & 1], wave);
    };
    // keys of round i and values of round i - 1
    auto put = [&](int i, bool values) {
      if (!st.k_ok || wave_token(i) + 16 > most) st.clear_k(wave_token(i), most);
      st.store_k(lds_k[i & 1]);
      if (values) put_v(i - 1);
      unsigned flags = st.k_ok ? 1u : 0u;
      if constexpr (C::kBytes == 1) {
        const unsigned ks = __float_as_uint(st.ks), vs = __float_as_uint(st.vs);
        if (__builtin_amdgcn_readfirstlane(beside_power(ks | vs))) {
          flags |= (beside_power(ks) ? 2u : 0u) | (beside_power(vs) ? 4u : 0u);
          if (lane == 0) {
            k_rest[i & 1][wave] = rest_of_scale(ks);
            v_rest[(i & 1) ^ 1][wave] = rest_of_scale(vs);
          }
        }
      }
      if (lane == 0) reinterpret_cast<unsigned char*>(&present[i & 1])[wave] = (unsigned char)flags;
    };
    constexpr int kAhead = 4;
    f32x16_t s[2];
    float w[32];  // weights of a round, fp32 until they are multiplied
    // Where the lane reads its operands; the chunk of an instruction is an exclusive or with its number (worked out anew in each
    // round: sixteen addresses kept in registers leave too few for operands read ahead).
    unsigned k_at = col * (D * 2) + ((half ^ (col & 7)) << 4), v_at = col * 128 + ((half ^ ((col ^ (col >> 2)) & 7)) << 4);
    float reference = 0.0f;
    auto logits = [&](int i) {
      asm("" : "+v"(k_at));
      const unsigned char* at = lds_k[i & 1];
      bf16x8_t k[2 * (D / 16)];
#pragma unroll
      for (int e = 0; e < D / 16; ++e)
#pragma unroll
        for (int b = 0; b < 2; ++b) __builtin_memcpy(&k[2 * e + b], at + 32 * b * (D * 2) + (k_at ^ (e << 5)), 16);
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int e = 0; e < 16; ++e) s[b][e] = 0.0f;
#pragma unroll
      for (int e = 0; e < D / 16; ++e)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int t = 0; t < kQ; ++t) s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[2 * e + b], qf[t][e], s[b], 0, 0, 0);
      // operands are read kAhead instructions ahead
#pragma unroll
      for (int e = 0; e < kAhead; ++e) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
      for (int e = 0; e < 2 * (D / 16) - kAhead; ++e) {
        __builtin_amdgcn_sched_group_barrier(0x008, kQ, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, kQ * kAhead, 0);
    };
    auto flags_of = [&](int i) { return (unsigned)__builtin_amdgcn_readfirstlane(present[i & 1]); };
    // weights of round i by what the scales of its values are beside their powers of two
    auto scale_weights = [&](int i, unsigned there) {
      if (C::kBytes == 1 && (there & 0x04040404u)) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
          if ((there >> (8 * (e >> 3))) & 4u) w[e] *= v_rest[i & 1][e >> 3];
      }
    };
    // logits of round i, and weights of the round before: all that is not the same for most rounds, behind one branch
    auto mask = [&](int i) {
      const int t = t0 + i * kBlockTokens;
      const unsigned there = flags_of(i);
      if (t + kBlockTokens > least || there != 0x01010101u) {
        if (C::kBytes == 1 && (there & 0x02020202u)) {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if ((there >> (8 * (e >> 3))) & 2u) s[e >> 4][e & 15] *= k_rest[i & 1][e >> 3];
        }
        if (i > 0) scale_weights(i - 1, there);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int at = 32 * b + 8 * (e >> 2) + 4 * half + (e & 3);
            if (t + at >= lim || !((there >> (8 * (at >> 4))) & 1u)) s[b][e] = -INFINITY;
          }
      }
    };
    // Exponents of the weights, relative to m (to 0 as long as the row has seen nothing).  Weights may reach 2^8 before a larger
    // maximum is taken: O and l are relative to the same.  Product and difference are one rounding, but for maxima beyond 2^24 (`far`), whose own
    // rounding would then count as a weight, of up to infinity: there the product is rounded as the maximum was.
    bool far = false;
    auto raise = [&](float& corr) {
      float factor = g.scale_log2e;
      if (far) {
#pragma clang fp contract(off)
        factor = 1.0f;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[0][e] *= g.scale_log2e;
          s[1][e] *= g.scale_log2e;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[0][e] = fmaf(s[0][e], factor, -reference);
        s[1][e] = fmaf(s[1][e], factor, -reference);
        mx = fmaxf(mx, fmaxf(s[0][e], s[1][e]));
      }
      const u32x2_t both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) + reference;
      const bool up = __any(mx > m + 8.0f);
      if (up) {
        const float mnew = fmaxf(m, mx), before = reference;
        corr = __builtin_amdgcn_exp2f(m - mnew);
        m = mnew;
        l *= corr;
        reference = m > kLowest ? m : 0.0f;
        far = __any(fabsf(reference) > 0x1p24f);
        const float back = far ? before : 0.0f, by = far ? reference : reference - before;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          s[0][e] = (s[0][e] + back) - by;
          s[1][e] = (s[1][e] + back) - by;
        }
      }
      return up;
    };
    auto weigh = [&](int b, int k) {  // 16 tokens
#pragma unroll
      for (int e = 8 * k; e < 8 * k + 8; ++e) l += w[16 * b + e] = __builtin_amdgcn_exp2f(s[b][e]);
    };
    auto multiply = [&](int i, int b, int k) {
      bf16x8_t p[TERMS];
      u32x4_t x[TERMS];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float p0 = w[16 * b + 8 * k + 2 * e], p1 = w[16 * b + 8 * k + 2 * e + 1];
#pragma unroll
        for (int y = 0; y < TERMS; ++y) {
          x[y][e] = pack_bf16(p0, p1);
          p0 -= __uint_as_float(x[y][e] << 16);
          p1 -= __uint_as_float(x[y][e] & 0xffff0000u);
        }
      }
#pragma unroll
      for (int y = 0; y < TERMS; ++y) __builtin_memcpy(&p[y], &x[y], 16);
#pragma unroll
      for (int n = 0; n < D / 32; ++n) {
        bf16x8_t v;
        __builtin_memcpy(&v, lds_v[i & 1] + 4096 * n + (v_at ^ ((2 * b + k) << 5)), 16);
#pragma unroll
        for (int y = 0; y < TERMS; ++y) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[y], o[n], 0, 0, 0);
      }
    };

    // in front of round i LDS holds keys i + 1 and values i, the registers keys i + 2 and values i + 1
    const int page1 = valid(page_of(1));
    int page2 = valid(page_of(2)), page3 = page_of(3);
    {
      const int page0 = valid(page_of(0));
      st.load_k(g, c, h, wave_token(0), page0);
      st.load_v(g, c, h, wave_token(0), page0);
    }
    put(0, false);
    st.load_k(g, c, h, wave_token(1), page1);
    __syncthreads();
    if (mine > 0) {
      float corr;
      logits(0);
      mask(0);
      raise(corr);
#pragma unroll
      for (int b = 0; b < 4; ++b) weigh(b >> 1, b & 1);
    }
    put(1, true);
    st.load_k(g, c, h, wave_token(2), page2);
    st.load_v(g, c, h, wave_token(1), page1);
    auto stage = [&](int i) {
      put(i + 2, true);
      const int next = valid(page3);
      st.load_k(g, c, h, wave_token(i + 3), next);
      st.load_v(g, c, h, wave_token(i + 2), page2);
      page2 = next;
      page3 = page_of(i + 4);
    };
    // a larger maximum reaches O one round late, behind the values whose weights were relative to the old one
    float late = 1.0f;
    bool up = false;
    auto rescale = [&]() {
      if (up) {
#pragma unroll
        for (int n = 0; n < D / 32; ++n) o[n] *= late;
      }
    };
    int i = 0;
    for (; i + 1 < mine; ++i) {
      __syncthreads();
      logits(i + 1);
      stage(i);
      mask(i + 1);
      rescale();
      up = raise(late);
      asm("" : "+v"(v_at));
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        multiply(i, b >> 1, b & 1);
        weigh(b >> 1, b & 1);
      }
    }
    for (; i < rounds; ++i) {  // the wave's last, and those of other waves
      __syncthreads();
      if (i + 1 < rounds) stage(i);
      if (i < mine) {
        scale_weights(i, flags_of(i + 1));
        rescale();
#pragma unroll
        for (int b = 0; b < 4; ++b) multiply(i, b >> 1, b & 1);
      }
    }
    if (odd_values) {  // (set in front of the last barrier, if at all)
      for (int t = t0 + max(all_see - t0, 0) / 16 * 16; t < min(t1, lim); ++t) {
        const int page = table[t >> g.shift];
        if (page < 0 || page >= g.n_pages) continue;
        const unsigned char* row = c.v + ((((size_t)page * g.Hkv + h) << g.shift) + (t & (g.P - 1))) * (size_t)(D * C::kBytes);
#pragma unroll
        for (int n = 0; n < D / 32; ++n)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[n][e] += C::odd_value(row, 32 * n + 8 * (e >> 2) + 4 * half + (e & 3));
      }
    }
  }
  const u32x2_t both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (!row_ok) return;
  if (it.slot >= 0) {
    const int rows = g.R * g.G;
    float* po = partials + ((size_t)(it.slot + it.split) * g.Hkv + h) * partial_floats(rows, D);
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) *reinterpret_cast<f32x4_t*>(po + r * D + 32 * n + 8 * j + 4 * half) = f32x4_t{o[n][4 * j], o[n][4 * j + 1], o[n][4 * j + 2], o[n][4 * j + 3]};
    if (half == 0) {
      po[rows * D + 2 * r] = m;
      po[rows * D + 2 * r + 1] = l;
    }
    return;
  }
  const float inv = reciprocal_sum(l);
  const size_t at = ((size_t)(it.s.first + qi) * g.Hq + (size_t)h * g.G + r % g.G) * D + 4 * half;
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t a = at + 32 * n + 8 * j;
      if (g.out_bf16)
        *reinterpret_cast<u32x2_t*>(static_cast<bf16_t*>(out) + a) = u32x2_t{pack_bf16(o[n][4 * j] * inv, o[n][4 * j + 1] * inv), pack_bf16(o[n][4 * j + 2] * inv, o[n][4 * j + 3] * inv)};
      else
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(out) + a) = f32x4_t{o[n][4 * j] * inv, o[n][4 * j + 1] * inv, o[n][4 * j + 2] * inv, o[n][4 * j + 3] * inv};
    }
}

// ------------------------------------------------------------------ append
struct AppendArgs {
  const void *q, *k, *v;      // [T][heads][D], a token's heads adjacent, tokens `*_stride` values apart
  long long q_stride, k_stride, v_stride;
  const int* positions;       // nullptr: a token's place in its sequence
  const float* table;         // [rot_positions][rot]: cosines, then sines
  int rot, rot_positions;
  bool pairs;                 // (2j, 2j + 1) are rotated together, else (j, j + rot / 2)
  void *q_out, *k_out;        // [T][heads][D]
  int kv_items;               // bound of the number of (sequence, page) pairs
  int together;          // pages of which the workgroups of one head lie side by side; divides kv_items
  int q_tokens;               // query tokens per workgroup
};

__device__ __forceinline__ int token_count(int length) { return min(max(length, 0), 1 << 30); }
template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4_t w = *reinterpret_cast<const u32x4_t*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  } else {
    const f32x4_t a = *reinterpret_cast<const f32x4_t*>(p), b = *reinterpret_cast<const f32x4_t*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
}
// Past the caches: a prompt's rotated rows are larger than those (with eight query tokens per workgroup 32768 tokens 175 us with plain stores,
// 168 so, 4096 tokens 25.8, 21.6).
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4_t w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_t*>(p));
  } else {
    __builtin_nontemporal_store(f32x4_t{x[0], x[1], x[2], x[3]}, reinterpret_cast<f32x4_t*>(p));
    __builtin_nontemporal_store(f32x4_t{x[4], x[5], x[6], x[7]}, reinterpret_cast<f32x4_t*>(p + 4));
  }
}
// What a scale is chosen by: an infinity would leave the other values of its page no codes but zero, so that it becomes the type's NaN like a
// NaN itself, and the scale is that of the finite values.
__device__ __forceinline__ float finite_size(float x) { return fabsf(x) < INFINITY ? fabsf(x) : 0.0f; }
// Eight e4m3 codes of x * inv, |x * inv| <= 448 (nearest even), or NaN of what is not finite.
__device__ __forceinline__ u32x2_t encode8(const float (&x)[8], float inv) {
  u32x2_t w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int c = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i] * inv, x[4 * i + 1] * inv, 0, false);
    w[i] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2] * inv, x[4 * i + 3] * inv, c, true);
  }
  return w;
}
__device__ __forceinline__ void decode8(u32x2_t w, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i], true);
    x[4 * i] = a[0];
    x[4 * i + 1] = a[1];
    x[4 * i + 2] = b[0];
    x[4 * i + 3] = b[1];
  }
}
// Smallest power of two s with amax <= 448 s, within 2^-100 .. 2^120; powers of two keep the re-encoding of a page whose scale
// grows exact (but for codes that fall below the normal range), however often it grows.
__device__ __forceinline__ float power_scale(float amax) {
  const unsigned u = __float_as_uint(amax);
  int e = (int)(u >> 23) - 126;                  // amax = m 2^e, 0.5 <= m < 1
  e = e - 9 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);  // m > 0.875
  e = min(max(e, -100), 120);
  return __uint_as_float((unsigned)(e + 127) << 23);
}

// A thread has sixteen dimensions of a head: part j of D / 16.  Rotated ones are eight pairs, 8 j .. 8 j + 7, in halves
// (dimensions 8 j.. and rot / 2 + 8 j..) or next to each other (16 j..); behind the rotated parts come sixteen adjacent ones.
struct Dims {
  int lo, hi;    // the two groups of eight
  bool rotated;
};
__device__ __forceinline__ Dims dims_of(const AppendArgs& a, int j) {
  const bool rotated = 16 * j < a.rot;
  const bool halves = rotated && !a.pairs;
  return Dims{halves ? 8 * j : 16 * j, halves ? 8 * j + (a.rot >> 1) : 16 * j + 8, rotated};
}
struct Angles {
  float co[8], si[8];
  __device__ __forceinline__ void load(const AppendArgs& a, int j, int pos) {
    const float* row = a.table + (size_t)min(max(pos, 0), a.rot_positions - 1) * a.rot + 8 * j;
    load8(row, co);
    load8(row + (a.rot >> 1), si);
  }
};
// Every product and sum is rounded by itself.
__device__ __forceinline__ void rotate(const AppendArgs& a, const Angles& w, float (&lo)[8], float (&hi)[8]) {
#pragma clang fp contract(off)
  if (a.pairs) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x = lo[2 * i], y = lo[2 * i + 1];
      lo[2 * i] = x * w.co[i] - y * w.si[i];
      lo[2 * i + 1] = y * w.co[i] + x * w.si[i];
      x = hi[2 * i];
      y = hi[2 * i + 1];
      hi[2 * i] = x * w.co[4 + i] - y * w.si[4 + i];
      hi[2 * i + 1] = y * w.co[4 + i] + x * w.si[4 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = lo[i], y = hi[i];
      lo[i] = x * w.co[i] - y * w.si[i];
      hi[i] = y * w.co[i] + x * w.si[i];
    }
  }
}

// Queries of a.q_tokens tokens: a thread goes through the heads of one token with the same angles, which are read once.
template <typename T, int D>
__device__ __forceinline__ void append_queries(const Geometry& g, const Cache& c, const AppendArgs& a, const int* __restrict__ offsets, int group) {
  constexpr int kParts = D / 16, kSlots = 256 / kParts;
  const int j = threadIdx.x % kParts, slot = threadIdx.x / kParts;
  const int heads_at_once = kSlots / a.q_tokens;
  const int t = group * a.q_tokens + slot / heads_at_once;
  if (t >= g.n_q) return;
  int b = t, begin = t, end = t + 1;
  if (offsets) {  // the sequence of token t: the offsets ascend
    int lo = 0, hi = g.B;  // the first b whose end is beyond t
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (offsets[mid + 1] <= t)
        lo = mid + 1;
      else
        hi = mid;
    }
    b = lo;
    if (b >= g.B) return;  // behind the last sequence: left as it is
    begin = offsets[b];
    end = offsets[b + 1];
    if (t < begin) return;
  }
  const Dims d = dims_of(a, j);
  Angles w;
  if (d.rotated) w.load(a, j, a.positions ? a.positions[t] : token_count(c.lengths[b]) - (end - t));
  const T* src = static_cast<const T*>(a.q) + (size_t)t * a.q_stride;
  T* dst = static_cast<T*>(a.q_out) + (size_t)t * g.Hq * D;
#pragma unroll 4
  for (int h = slot % heads_at_once; h < g.Hq; h += heads_at_once) {
    float lo[8], hi[8];
    load8(src + (size_t)h * D + d.lo, lo);
    load8(src + (size_t)h * D + d.hi, hi);
    if (d.rotated) rotate(a, w, lo, hi);
    store8(dst + (size_t)h * D + d.lo, lo);
    store8(dst + (size_t)h * D + d.hi, hi);
  }
}

// One workgroup per (sequence, page that the call touches, head, key or value), and behind them workgroups that rotate queries.
// Of the page's new tokens a thread keeps up to kHeld parts between the pass that finds the largest value and the one that writes the
// codes; where there are more the inputs are read again.
template <typename T, bool FP8, int D>
__global__ __launch_bounds__(256) void append_kernel(Geometry g, Cache c, AppendArgs a, const int* __restrict__ offsets) {
  constexpr int kParts = D / 16, kSlots = 256 / kParts, kHeld = 2;
  const int tid = threadIdx.x, lane = tid & 63;
  const int kv_groups = a.kv_items * 2 * g.Hkv;
  if ((int)blockIdx.x >= kv_groups) {
    append_queries<T, D>(g, c, a, offsets, (int)blockIdx.x - kv_groups);
    return;
  }
  const int chunk = blockIdx.x / (2 * g.Hkv * a.together), in_chunk = blockIdx.x - chunk * 2 * g.Hkv * a.together;
  const int which = in_chunk / a.together, j = chunk * a.together + in_chunk % a.together;
  const bool is_key = which < g.Hkv;
  const int h = is_key ? which : which - g.Hkv;
  // the j-th touched page
  int b = -1, page_at = 0, first = 0, start = 0, stop = 0;
  for (int b0 = 0, before = 0; b0 < g.B; b0 += 64) {
    const int bl = b0 + lane;
    int n = 0, lo = 0, hi = 0, o0 = 0, at0 = 0;
    if (bl < g.B) {
      const Seq s = seq_of(g, c.lengths, offsets, bl);
      const int len = token_count(c.lengths[bl]);
      o0 = s.first;
      at0 = len - s.nq;                         // place of its first new token
      lo = max(at0, 0);
      hi = min(len, g.max_pages << g.shift);
      n = hi > lo ? ((hi - 1) >> g.shift) - (lo >> g.shift) + 1 : 0;
    }
    const int end = wave_inclusive_scan(n);
    const unsigned long long has = __ballot(before + end > j);
    if (has) {
      const int l = __ffsll((long long)has) - 1;
      b = b0 + l;
      const int nth = j - before - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(n, l));
      const int blo = __builtin_amdgcn_readlane(lo, l), bhi = __builtin_amdgcn_readlane(hi, l);
      page_at = (blo >> g.shift) + nth;
      start = max(blo, page_at << g.shift);
      stop = min(bhi, (page_at + 1) << g.shift);
      first = __builtin_amdgcn_readlane(o0, l) - __builtin_amdgcn_readlane(at0, l);  // token of place p: first + p
      break;
    }
    before += wave_last(end);
  }
  if (b < 0) return;
  const int page = c.table[(size_t)b * g.max_pages + page_at];
  const bool stored = page >= 0 && page < g.n_pages;
  const int n = stop - start, held = start & (g.P - 1);
  const T* src = static_cast<const T*>(is_key ? a.k : a.v);
  const long long stride = is_key ? a.k_stride : a.v_stride;
  const int part = tid % kParts, slot = tid / kParts;
  Dims d = dims_of(a, part);
  if (!is_key && d.rotated) d = Dims{16 * part, 16 * part + 8, false};
  auto value = [&](int i, float (&lo)[8], float (&hi)[8]) {  // new token start + i
    const int t = first + start + i;
    const T* p = src + (size_t)t * stride + (size_t)h * D;
    load8(p + d.lo, lo);
    load8(p + d.hi, hi);
    if (d.rotated) {
      Angles w;
      w.load(a, part, a.positions ? a.positions[t] : start + i);
      rotate(a, w, lo, hi);
    }
  };
  auto key_out = [&](int i, const float (&lo)[8], const float (&hi)[8]) {
    if (!is_key || !a.k_out) return;
    T* p = static_cast<T*>(a.k_out) + ((size_t)(first + start + i) * g.Hkv + h) * D;
    store8(p + d.lo, lo);
    store8(p + d.hi, hi);
  };
  const size_t block = (((size_t)(stored ? page : 0) * g.Hkv + h) << g.shift) * D;
  if constexpr (FP8) {
    __shared__ float wave_max_of[4];
    float* scale = (is_key ? c.ks : c.vs) + (size_t)(stored ? page : 0) * g.Hkv + h;
    const float old = stored && held > 0 ? *scale : 0.0f;
    float lo[kHeld][8], hi[kHeld][8], amax = 0.0f;
    auto largest = [&](const float (&x)[8], const float (&y)[8]) {
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fmaxf(finite_size(x[e]), finite_size(y[e])));
    };
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
      if (slot + e * kSlots < n) {
        value(slot + e * kSlots, lo[e], hi[e]);
        largest(lo[e], hi[e]);
      }
    for (int i = slot + kHeld * kSlots; i < n; i += kSlots) {
      float x[8], y[8];
      value(i, x, y);
      largest(x, y);
    }
    amax = wave_max(amax);
    if (lane == 0) wave_max_of[tid >> 6] = amax;
    __syncthreads();  // (every wave has read the old scale)
    amax = fmaxf(fmaxf(wave_max_of[0], wave_max_of[1]), fmaxf(wave_max_of[2], wave_max_of[3]));
    const float want = power_scale(amax), s = fmaxf(old, want);
    unsigned char* codes = (is_key ? c.k : c.v) + block;
    if (stored && held > 0 && s > old) {
      for (int i = tid; i < held * (D / 8); i += 256) {
        float y[8];
        u32x2_t* w = reinterpret_cast<u32x2_t*>(codes + (size_t)i * 8);
        decode8(*w, y);
        *w = encode8(y, old / s);
      }
    }
    const float inv = 1.0f / s;
    auto write = [&](int i, const float (&x)[8], const float (&y)[8]) {
      key_out(i, x, y);
      if (stored) {
        unsigned char* row = codes + (size_t)(held + i) * D;
        *reinterpret_cast<u32x2_t*>(row + d.lo) = encode8(x, inv);
        *reinterpret_cast<u32x2_t*>(row + d.hi) = encode8(y, inv);
      }
    };
#pragma unroll
    for (int e = 0; e < kHeld; ++e)
      if (slot + e * kSlots < n) write(slot + e * kSlots, lo[e], hi[e]);
    for (int i = slot + kHeld * kSlots; i < n; i += kSlots) {
      float x[8], y[8];
      value(i, x, y);
      write(i, x, y);
    }
    if (stored && tid == 0) *scale = s;
  } else {
    bf16_t* rows = reinterpret_cast<bf16_t*>(is_key ? c.k : c.v) + block + (size_t)held * D;
    for (int i = slot; i < n; i += kSlots) {
      float x[8], y[8];
      value(i, x, y);
      key_out(i, x, y);
      if (stored) {
        store8(rows + (size_t)i * D + d.lo, x);
        store8(rows + (size_t)i * D + d.hi, y);
      }
    }
  }
}

}  // namespace paged
}  // namespace pqc
