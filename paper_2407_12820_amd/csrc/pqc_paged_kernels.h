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
constexpr float kFp8Max = 448.0f;  // largest e4m3 value, 0.875 * 2^9

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) unsigned u32x2_t;

struct Geometry {
  int B, Hq, Hkv, G;
  int P, shift;           // tokens per page, and its logarithm
  int n_pages, max_pages;
  int n_q;                // query (or new) tokens of all sequences
  int R;                  // query tokens per tile
  int per_head;           // items per head that the split length aims at
  int items, slots;       // bounds of the numbers of items and of partial results per head
  int split, n_split;     // listed tokens: tokens per split and splits (the same for every head)
  bool out_bf16;
  float scale_log2e;
};
struct Cache {
  unsigned char *k, *v;
  float *ks, *vs;
  const int *table, *lengths;
};

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
  return max(1, (int)fminf(tokens, 1e7f)) * kGrain;
}
// The j-th item (MERGE: the j-th tile of more than one split); b < 0: there are fewer.
template <bool MERGE>
__device__ __forceinline__ Item find_item(const Geometry& g, const int* lengths, const int* offsets, int j) {
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
    const int count = MERGE ? (n > 1 ? tiles : 0) : tiles * n;
    const int end = wave_inclusive_scan(count);
    const unsigned long long has = __ballot(before + end > j);
    if (has) {
      const int l = __ffsll((long long)has) - 1;
      const int at = j - before - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(count, l));
      it.b = b0 + l;
      it.n_split = __builtin_amdgcn_readlane(n, l);
      const int nth = MERGE ? at : at / it.n_split;
      it.tile = __builtin_amdgcn_readlane(tiles, l) - 1 - nth;  // the last one, which sees most, first
      it.split = MERGE ? 0 : at - nth * it.n_split;
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
};
struct Bf16 {
  static constexpr int kBytes = 2;
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
};

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
    m = kNegBig;
    l = 0.0f;
  }
};

// One step: logits of 32 tokens, one rescaling if a maximum grew, weights, values.  `see(tile, i)` says whether the lane's query
// sees its i-th token of the tile, `live(tile, i)` whether any query of the tile does (else its value row may hold anything, NaN
// among it, and is taken as zero); both only matter if `masked` (wave-uniform).  The weights enter as three bf16 terms,
// whose sum is the fp32 weight: two leave out up to 2^-18 of it, which was the largest error of all over a few tokens (1.1e-6 of
// the result against 1e-7), and the third is free where the bytes of the rows are what the step waits for.
constexpr int kTerms = 3;
template <typename T, class C, int D, class SeeFn, class LiveFn, class KsFn, class VsFn>
__device__ __forceinline__ void attend(Stage<C, D>& st, const Query<T, C, D>& q, State<D>& a, bool masked, SeeFn see, LiveFn live, KsFn ks, VsFn vs) {
  float s[2][4];
  float mx = kNegBig;
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
}

__device__ __forceinline__ void store_out(const Geometry& g, void* out, size_t at, float x) {
  if (g.out_bf16)
    static_cast<__bf16*>(out)[at] = (__bf16)x;
  else
    static_cast<float*>(out)[at] = x;
}

// Attention of one tile of up to 16 query rows over one split of its tokens.  Four waves take 32 tokens each in turn, with a
// softmax state of their own, folded at the end.  A tile of more than one split leaves (m, l, O) in `partials`, per (slot, head)
// O[R G][D], then m and l of every row.
// LISTED: one query token per sequence, over the tokens that idx names; entries outside the sequence are left out.
template <typename T, class C, int D, bool LISTED>
__global__ __launch_bounds__(256, 2) void attn_rows_kernel(Geometry g, Cache c, const T* __restrict__ q, const int* __restrict__ offsets,
                                                           const int* __restrict__ idx, int n_idx, void* __restrict__ out, float* __restrict__ partials) {
  __shared__ int place[kStaged];  // page of the split, or row of the listed token; negative: none
  __shared__ float kscale[kStaged], vscale[kStaged];
  __shared__ float red_o[kWaves][kRows][D];
  __shared__ float red_m[kWaves][kRows], red_l[kWaves][kRows];
  const int lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4, wave = threadIdx.x >> 6;
  const int h = blockIdx.y;
  Item it;
  if constexpr (LISTED) {
    it.b = blockIdx.x / g.n_split;
    it.split = blockIdx.x - it.b * g.n_split;
    it.n_split = g.n_split;
    it.tokens = g.split;
    it.tile = 0;
    it.slot = g.n_split > 1 ? it.b * g.n_split : -1;
    it.s = seq_of(g, c.lengths, nullptr, it.b);
  } else {
    it = find_item<false>(g, c.lengths, offsets, blockIdx.x);
    if (it.b < 0) return;
  }
  const int qi = it.tile * g.R + col / g.G;  // the lane's query token
  const bool row_ok = col < g.R * g.G && qi < it.s.nq;
  const int hidden = it.s.len - it.s.nq;     // tokens in front of the first query's own
  // tokens that the lane's query, the tile's first and its last query see
  const int lim = row_ok ? max(LISTED ? n_idx : hidden + qi + 1, 0) : 0;
  const int most = LISTED ? n_idx : max(hidden + min((it.tile + 1) * g.R, it.s.nq), 0);
  const int least = LISTED ? n_idx : max(hidden + it.tile * g.R + 1, 0);
  Query<T, C, D> qf;
  qf.load(row_ok ? q + ((size_t)(it.s.first + qi) * g.Hq + (size_t)h * g.G + col % g.G) * D : nullptr, quad);
  State<D> a;
  a.init();
  const int t0 = it.split * it.tokens, t1 = it.n_split == 1 ? most : min(t0 + it.tokens, most);
  const int* table = c.table + (size_t)it.b * g.max_pages;
  const size_t row_bytes = (size_t)D * C::kBytes;
  constexpr bool kScaled = C::kBytes == 1;
  // (an even number of pages: a segment is a multiple of 32 tokens)
  const int seg_tokens = LISTED ? kStaged : ((kStaged - 2) << g.shift);
  for (int seg = t0; seg < t1; seg += seg_tokens) {
    const int seg_end = min(seg + seg_tokens, t1);
    const int p0 = seg >> g.shift, staged = LISTED ? seg_end - seg : ((seg_end - 1) >> g.shift) - p0 + 1;
    __syncthreads();
    bool bad = false;
    for (int i = threadIdx.x; i < staged; i += 256) {
      int page = -1, row = 0;
      if constexpr (LISTED) {
        const int t = idx[((size_t)it.b * g.Hkv + h) * n_idx + seg + i];
        if (t >= 0 && t < it.s.len) page = table[t >> g.shift];
        row = t & (g.P - 1);
      } else {
        page = table[p0 + i];
      }
      const bool ok = page >= 0 && page < g.n_pages;
      bad |= !ok;
      place[i] = !ok ? -1 : LISTED ? ((page * g.Hkv + h) << g.shift) + row : page;
      kscale[i] = ok ? g.scale_log2e * (kScaled ? c.ks[(size_t)page * g.Hkv + h] : 1.0f) : 0.0f;
      vscale[i] = ok ? (kScaled ? c.vs[(size_t)page * g.Hkv + h] : 1.0f) : 0.0f;
    }
    const bool any_bad = __syncthreads_or(bad);
    auto at = [&](int t) { return LISTED ? min(t - seg, staged - 1) : min((t >> g.shift) - p0, staged - 1); };
    auto issue = [&](Stage<C, D>& st, int t) {
#pragma unroll
      for (int tl = 0; tl < 2; ++tl) {
        const int tt = t + 16 * tl;
        if constexpr (LISTED) {
          const unsigned char* kp = c.k + (size_t)max(place[at(tt + col)], 0) * row_bytes;
#pragma unroll
          for (int j = 0; j < C::template kLoads<D>; ++j) st.k[tl][j] = *reinterpret_cast<const u32x4_t*>(kp + C::load_dim(j, quad) * C::kBytes);
#pragma unroll
          for (int i = 0; i < 4; ++i)
            load_words(c.v + (size_t)max(place[at(tt + 4 * quad + i)], 0) * row_bytes + col * (D / 16) * C::kBytes, st.v[4 * tl + i]);
        } else {
          const int page = __builtin_amdgcn_readfirstlane(max(place[at(tt)], 0));
          const size_t base = ((((size_t)page * g.Hkv + h) << g.shift) + (tt & (g.P - 1))) * row_bytes;
          const unsigned char *kp = c.k + base, *vp = c.v + base;
#pragma unroll
          for (int j = 0; j < C::template kLoads<D>; ++j)
            st.k[tl][j] = *reinterpret_cast<const u32x4_t*>(kp + (col * D + C::load_dim(j, quad)) * C::kBytes);
#pragma unroll
          for (int i = 0; i < 4; ++i) load_words(vp + ((4 * quad + i) * D + col * (D / 16)) * C::kBytes, st.v[4 * tl + i]);
        }
      }
    };
    auto consume = [&](Stage<C, D>& st, int t) {
      auto token = [&](int tl, int i) { return t + 16 * tl + 4 * quad + i; };
      auto slot = [&](int tl, int i) { return at(LISTED ? token(tl, i) : t + 16 * tl); };
      attend<T, C, D>(
          st, qf, a, any_bad || t + kStep > least, [&](int tl, int i) { return token(tl, i) < lim && place[slot(tl, i)] >= 0; },
          [&](int tl, int i) { return token(tl, i) < most && place[slot(tl, i)] >= 0; }, [&](int tl, int i) { return kscale[slot(tl, i)]; },
          [&](int tl, int i) { return vscale[slot(tl, i)]; });
    };
    Stage<C, D> sa, sb;
    int t = seg + wave * kStep;
    if (t < seg_end) {
      issue(sa, t);
      for (;;) {  // the next step's loads travel while this one is computed; past the end the last rows are read again
        const int n1 = min(t + kGrain, (seg_end - 1) & ~(kStep - 1));
        issue(sb, n1);
        PQC_LOADS_ISSUED();
        consume(sa, t);
        t += kGrain;
        if (t >= seg_end) break;
        issue(sa, min(t + kGrain, (seg_end - 1) & ~(kStep - 1)));
        PQC_LOADS_ISSUED();
        consume(sb, t);
        t += kGrain;
        if (t >= seg_end) break;
      }
    }
  }
  // fold the waves
  const float l = quad_sum(a.l);
  if (quad == 0) {
    red_m[wave][col] = a.m;
    red_l[wave][col] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int n = 0; n < D / 16; ++n) red_o[wave][col][D / 16 * (4 * quad + i) + n] = a.o[n][i];
  __syncthreads();
  const int rows = g.R * g.G;
  float* po = partials + ((size_t)(it.slot + it.split) * g.Hkv + h) * (size_t)(rows * (D + 2));
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
    if (it.slot >= 0) {
      po[i] = o;
      if (d == 0) {
        po[rows * D + 2 * r] = m;
        po[rows * D + 2 * r + 1] = sum;
      }
    } else {
      const int qr = it.tile * g.R + r / g.G;
      if (qr < it.s.nq) store_out(g, out, ((size_t)(it.s.first + qr) * g.Hq + (size_t)h * g.G + r % g.G) * D + d, sum > 0.0f ? o / sum : 0.0f);
    }
  }
}

// Folds the splits of a tile: one workgroup per (tile, head, row).
template <int D, bool LISTED>
__global__ __launch_bounds__(256) void attn_merge_kernel(Geometry g, const int* __restrict__ lengths, const int* __restrict__ offsets,
                                                         const float* __restrict__ partials, void* __restrict__ out) {
  constexpr int kGroups = 256 / D;
  __shared__ float wave_m[4], red_o[kGroups][D], red_l[kGroups];
  const int h = blockIdx.y;
  Item it;
  if constexpr (LISTED) {
    it.b = blockIdx.x;
    it.n_split = g.n_split;
    it.tile = 0;
    it.slot = it.b * g.n_split;
    it.s = Seq{it.b, 1, 0};
  } else {
    it = find_item<true>(g, lengths, offsets, blockIdx.x);
    if (it.b < 0) return;
  }
  const int rows = g.R * g.G;
  const size_t stride = (size_t)g.Hkv * rows * (D + 2);
  const float* base = partials + ((size_t)it.slot * g.Hkv + h) * (size_t)(rows * (D + 2));
  const int d = threadIdx.x % D, part = threadIdx.x / D;
  for (int r = blockIdx.z; r < rows; r += gridDim.z) {
    const int qr = it.tile * g.R + r / g.G;
    if (qr >= it.s.nq) return;
    float m = kNegBig;
    for (int i = threadIdx.x; i < it.n_split; i += 256) m = fmaxf(m, base[i * stride + rows * D + 2 * r]);
    m = wave_max(m);
    __syncthreads();  // the row before has been read
    if ((threadIdx.x & 63) == 0) wave_m[threadIdx.x >> 6] = m;
    __syncthreads();
    m = fmaxf(fmaxf(wave_m[0], wave_m[1]), fmaxf(wave_m[2], wave_m[3]));
    float o = 0.0f, l = 0.0f;
#pragma unroll 4
    for (int i = part; i < it.n_split; i += kGroups) {
      const float* p = base + i * stride;
      const float f = __builtin_amdgcn_exp2f(p[rows * D + 2 * r] - m);
      l += f * p[rows * D + 2 * r + 1];
      o += f * p[r * D + d];
    }
    red_o[part][d] = o;
    if (d == 0) red_l[part] = l;
    __syncthreads();
    if (part == 0) {
#pragma unroll
      for (int i = 1; i < kGroups; ++i) {
        o += red_o[i][d];
        l += red_l[i];
      }
      store_out(g, out, ((size_t)(it.s.first + qr) * g.Hq + (size_t)h * g.G + r % g.G) * D + d, l > 0.0f ? o / l : 0.0f);
    }
  }
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

template <class C, int D>
struct BlockStage {
  static constexpr int kK = D / 64 * C::kBytes;           // 16-byte loads of keys per thread: token tid / 4
  static constexpr int kV = C::kBytes;                    // words of each of eight tokens' values: four dimensions
  static constexpr bool kHalfV = D == 64;                 // half of the threads stage values
  u32x4_t k[kK];
  unsigned v[8][kV];
  float ks, vs;
  bool k_ok, v_ok;
  int token;  // the first of the 64

  // pages of the thread's key token and of its eight value tokens
  __device__ __forceinline__ void load(const Geometry& g, const Cache& c, int h, int t, int k_page, int v_page) {
    const int tid = threadIdx.x;
    token = t;
    k_ok = k_page >= 0;
    v_ok = v_page >= 0;
    const size_t kp = (size_t)max(k_page, 0) * g.Hkv + h, vp = (size_t)max(v_page, 0) * g.Hkv + h;
    ks = vs = 1.0f;
    if constexpr (C::kBytes == 1) {
      if (k_ok) ks = c.ks[kp];
      if (v_ok) vs = c.vs[vp];
    }
    const unsigned char* kr = c.k + ((kp << g.shift) + ((t + tid / 4) & (g.P - 1))) * (size_t)(D * C::kBytes);
    const int q = tid & 3;
#pragma unroll
    for (int j = 0; j < kK; ++j) {
      const int dim = C::kBytes == 1 ? 64 * j + 16 * q : 64 * (j >> 1) + 16 * q + 8 * (j & 1);
      k[j] = *reinterpret_cast<const u32x4_t*>(kr + dim * C::kBytes);
    }
    if (!kHalfV || tid < 128) {
      const int chunk = tid / (D / 4), dg = tid % (D / 4);
      const unsigned char* vr = c.v + ((vp << g.shift) + ((t + 16 * (chunk >> 1) + 4 * (chunk & 1)) & (g.P - 1))) * (size_t)(D * C::kBytes) + dg * 4 * C::kBytes;
#pragma unroll
      for (int e = 0; e < 8; ++e) load_words(vr + (e < 4 ? e : e + 4) * (D * C::kBytes), v[e]);
    }
  }
  // tokens from `most` on are zero, and those of pages that are not there
  __device__ __forceinline__ void store(unsigned char* lk, unsigned char* lv, int most) {
    const int tid = threadIdx.x, row = tid / 4, q = tid & 3;
    if (!k_ok || token + row >= most) {
#pragma unroll
      for (int j = 0; j < kK; ++j) k[j] = u32x4_t{0u, 0u, 0u, 0u};
      ks = 1.0f;
    }
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
    if (!kHalfV || tid < 128) {
      const int chunk = tid / (D / 4), dg = tid % (D / 4);
      const int first = token + 16 * (chunk >> 1) + 4 * (chunk & 1);
      if (!v_ok || first + 12 > most) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (!v_ok || first + (e < 4 ? e : e + 4) >= most) {
#pragma unroll
            for (int i = 0; i < kV; ++i) v[e][i] = 0u;
          }
        if (!v_ok) vs = 1.0f;
      }
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
  }
};

// TERMS: bf16 terms of a weight: one where the output is bf16 (2^-9 of a weight, no more than the output's own rounding), three
// for an fp32 output.
template <class C, int D, int TERMS>
__global__ __launch_bounds__(256, 2) void attn_block_kernel(Geometry g, Cache c, const bf16_t* __restrict__ q, const int* __restrict__ offsets,
                                                            void* __restrict__ out, float* __restrict__ partials) {
  __shared__ __align__(16) unsigned char lds_k[2][kBlockTokens * D * 2], lds_v[2][kBlockTokens * D * 2];
  __shared__ unsigned present[2];  // a byte per 16 tokens: their page is there
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, half = lane >> 5, wave = tid >> 6;
  // the heads of a KV head's tokens follow each other, so that with eight of them an XCD's L2 holds the rows of one
  const int item = blockIdx.x / g.Hkv, h = blockIdx.x - item * g.Hkv;
  const Item it = find_item<false>(g, c.lengths, offsets, item);
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
  bf16x8_t qf[D / 16];
  {
    const bf16_t* row = q + ((size_t)(it.s.first + qi) * g.Hq + (size_t)h * g.G + r % g.G) * D + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      u32x4_t x = {0u, 0u, 0u, 0u};
      if (row_ok) x = *reinterpret_cast<const u32x4_t*>(row + 16 * i);
      __builtin_memcpy(&qf[i], &x, 16);
    }
  }
  f32x16_t o[D / 32];
#pragma unroll
  for (int n = 0; n < D / 32; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[n][i] = 0.0f;
  float m = kNegBig, l = 0.0f;

  const int t0 = it.split * it.tokens, t1 = it.n_split == 1 ? most : min(t0 + it.tokens, most);
  if (t0 < t1) {
    const int* table = c.table + (size_t)it.b * g.max_pages;
    const int v_at = 16 * ((tid / (D / 4)) >> 1);  // the thread's value tokens' page (threads without any: some page of the row)
    auto page_of = [&](int t) {
      const int p = t < t1 ? table[t >> g.shift] : -1;
      return p < g.n_pages ? p : -1;
    };
    BlockStage<C, D> st;
    auto put = [&](int buf) {
      st.store(lds_k[buf], lds_v[buf], most);
      if ((tid & 63) == 0) reinterpret_cast<unsigned char*>(&present[buf])[wave] = (unsigned char)st.k_ok;  // wave: tokens 16 wave .. + 15
    };
    st.load(g, c, h, t0, page_of(t0 + tid / 4), page_of(t0 + (v_at & 63)));
    int k_page = page_of(t0 + kBlockTokens + tid / 4), v_page = page_of(t0 + kBlockTokens + (v_at & 63));
    put(0);
    __syncthreads();
    for (int t = t0, buf = 0; t < t1; t += kBlockTokens, buf ^= 1) {
      const bool more = t + kBlockTokens < t1;
      if (more) {
        st.load(g, c, h, t + kBlockTokens, k_page, v_page);
        k_page = page_of(t + 2 * kBlockTokens + tid / 4);
        v_page = page_of(t + 2 * kBlockTokens + (v_at & 63));
      }
      if (t < wave_most) {
        f32x16_t s[2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
          for (int i = 0; i < 16; ++i) s[b][i] = 0.0f;
          const int row = 32 * b + col;
#pragma unroll
          for (int i = 0; i < D / 16; ++i) {
            bf16x8_t k;
            __builtin_memcpy(&k, lds_k[buf] + row * (D * 2) + (((2 * i + half) ^ (row & 7)) << 4), 16);
            s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, qf[i], s[b], 0, 0, 0);
          }
        }
        const unsigned there = __builtin_amdgcn_readfirstlane(present[buf]);
        if (t + kBlockTokens > least || there != 0x01010101u) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int at = 32 * b + 8 * (i >> 2) + 4 * half + (i & 3);
              if (t + at >= lim || !((there >> (8 * (at >> 4))) & 1u)) s[b][i] = -INFINITY;
            }
        }
        float mx = kNegBig;
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, fmaxf(s[0][i], s[1][i]));
        const u32x2_t both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * g.scale_log2e;
        // weights may reach 2^8 before a larger maximum is taken: they are relative to it in O and l alike
        if (__any(mx > m + 8.0f)) {
          const float mnew = fmaxf(m, mx), corr = __builtin_amdgcn_exp2f(m - mnew);
          m = mnew;
          l *= corr;
#pragma unroll
          for (int n = 0; n < D / 32; ++n) o[n] *= corr;
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          unsigned w[TERMS][8];
#pragma unroll
          for (int i = 0; i < 16; i += 2) {
            float p0 = __builtin_amdgcn_exp2f(fmaf(s[b][i], g.scale_log2e, -m)), p1 = __builtin_amdgcn_exp2f(fmaf(s[b][i + 1], g.scale_log2e, -m));
            l += p0 + p1;
#pragma unroll
            for (int e = 0; e < TERMS; ++e) {
              w[e][i / 2] = pack_bf16(p0, p1);
              p0 -= __uint_as_float(w[e][i / 2] << 16);
              p1 -= __uint_as_float(w[e][i / 2] & 0xffff0000u);
            }
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            bf16x8_t p[TERMS];
#pragma unroll
            for (int e = 0; e < TERMS; ++e) __builtin_memcpy(&p[e], &w[e][4 * k], 16);
#pragma unroll
            for (int n = 0; n < D / 32; ++n) {
              const int d = 32 * n + col;
              bf16x8_t v;
              __builtin_memcpy(&v, lds_v[buf] + d * 128 + (((2 * (2 * b + k) + half) ^ ((d ^ (d >> 2)) & 7)) << 4), 16);
#pragma unroll
              for (int e = 0; e < TERMS; ++e) o[n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, p[e], o[n], 0, 0, 0);
            }
          }
        }
      }
      if (more) put(buf ^ 1);
      __syncthreads();
    }
  }
  const u32x2_t both = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  l = __uint_as_float(both[0]) + __uint_as_float(both[1]);
  if (r >= g.R * g.G) return;
  if (it.slot >= 0) {
    const int rows = g.R * g.G;
    float* po = partials + ((size_t)(it.slot + it.split) * g.Hkv + h) * (size_t)(rows * (D + 2));
#pragma unroll
    for (int n = 0; n < D / 32; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) po[r * D + 32 * n + 8 * j + 4 * half + i] = o[n][4 * j + i];
    if (half == 0) {
      po[rows * D + 2 * r] = m;
      po[rows * D + 2 * r + 1] = l;
    }
    return;
  }
  if (!row_ok) return;
  const float inv = l > 0.0f ? 1.0f / l : 0.0f;
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
template <typename T>
__device__ __forceinline__ void store8(T* p, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const u32x4_t w = {pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
    *reinterpret_cast<u32x4_t*>(p) = w;
  } else {
    *reinterpret_cast<f32x4_t*>(p) = f32x4_t{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4_t*>(p + 4) = f32x4_t{x[4], x[5], x[6], x[7]};
  }
}
// Eight e4m3 codes of x * inv, |x * inv| <= 448 (nearest even).
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

// Rotated values of dimensions 8 c .. 8 c + 7 of a head at `p`.  Every product and sum is rounded by itself.
template <typename T>
__device__ __forceinline__ void rotate8(const AppendArgs& a, const T* p, int c, int pos, float (&y)[8]) {
#pragma clang fp contract(off)
  float x[8];
  load8(p + 8 * c, x);
  const int half = a.rot >> 1;
  if (8 * c >= a.rot) {
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i];
    return;
  }
  const float* row = a.table + (size_t)min(max(pos, 0), a.rot_positions - 1) * a.rot;
  if (a.pairs) {
    const f32x4_t co = *reinterpret_cast<const f32x4_t*>(row + 4 * c), si = *reinterpret_cast<const f32x4_t*>(row + half + 4 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      y[2 * i] = x[2 * i] * co[i] - x[2 * i + 1] * si[i];
      y[2 * i + 1] = x[2 * i + 1] * co[i] + x[2 * i] * si[i];
    }
  } else {
    const bool low = 8 * c < half;
    const int j = 8 * c - (low ? 0 : half);
    float z[8], co[8], si[8];
    load8(p + (low ? 8 * c + half : j), z);
    load8(row + j, co);
    load8(row + half + j, si);
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = low ? x[i] * co[i] - z[i] * si[i] : x[i] * co[i] + z[i] * si[i];
  }
}

// One workgroup per (sequence, page that the call touches, head, key or value), and behind them workgroups that rotate queries.
template <typename T, bool FP8, int D>
__global__ __launch_bounds__(256) void append_kernel(Geometry g, Cache c, AppendArgs a, const int* __restrict__ offsets) {
  constexpr int kChunks = D / 8;
  const int tid = threadIdx.x, lane = tid & 63;
  const int kv_groups = a.kv_items * 2 * g.Hkv;
  if ((int)blockIdx.x >= kv_groups) {  // queries
    const int first = ((int)blockIdx.x - kv_groups) * a.q_tokens;
    for (int t = first; t < min(first + a.q_tokens, g.n_q); ++t) {
      int b = t;
      if (offsets) {  // the sequence of token t: how many end at or before it
        b = 0;
        for (int b0 = 0; b0 < g.B; b0 += 64) b += __popcll(__ballot(b0 + lane < g.B && offsets[b0 + lane + 1] <= t));
      }
      if (b >= g.B) return;  // behind the last sequence: left as it is
      const int begin = offsets ? offsets[b] : b, end = offsets ? offsets[b + 1] : b + 1;
      if (t < begin) continue;
      const int pos = a.positions ? a.positions[t] : token_count(c.lengths[b]) - (end - t);
      const T* src = static_cast<const T*>(a.q) + (size_t)t * a.q_stride;
      T* dst = static_cast<T*>(a.q_out) + (size_t)t * g.Hq * D;
      for (int i = tid; i < g.Hq * kChunks; i += 256) {
        float y[8];
        rotate8(a, src + (size_t)(i / kChunks) * D, i % kChunks, pos, y);
        store8(dst + (size_t)i * 8, y);
      }
    }
    return;
  }
  const int j = blockIdx.x / (2 * g.Hkv), which = blockIdx.x - j * 2 * g.Hkv;
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
  auto value = [&](int i, int chunk, float (&y)[8]) {  // new token start + i
    const int t = first + start + i;
    const T* p = src + (size_t)t * stride + (size_t)h * D;
    if (is_key && a.rot > 0)
      rotate8(a, p, chunk, a.positions ? a.positions[t] : start + i, y);
    else
      load8(p + 8 * chunk, y);
  };
  auto key_out = [&](int i, int chunk, const float (&y)[8]) {
    if (is_key && a.k_out) store8(static_cast<T*>(a.k_out) + ((size_t)(first + start + i) * g.Hkv + h) * D + 8 * chunk, y);
  };
  const size_t block = (((size_t)(stored ? page : 0) * g.Hkv + h) << g.shift) * D;
  if constexpr (FP8) {
    __shared__ float wave_max_of[4];
    float amax = 0.0f;
    for (int i = tid; i < n * kChunks; i += 256) {
      float y[8];
      value(i / kChunks, i % kChunks, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) amax = fmaxf(amax, fabsf(y[e]));
    }
    amax = wave_max(amax);
    if (lane == 0) wave_max_of[tid >> 6] = amax;
    __syncthreads();
    amax = fmaxf(fmaxf(wave_max_of[0], wave_max_of[1]), fmaxf(wave_max_of[2], wave_max_of[3]));
    float* scale = (is_key ? c.ks : c.vs) + (size_t)(stored ? page : 0) * g.Hkv + h;
    const float old = stored && held > 0 ? *scale : 0.0f, want = power_scale(amax), s = fmaxf(old, want);
    unsigned char* codes = (is_key ? c.k : c.v) + block;
    if (stored && held > 0 && s > old) {
      for (int i = tid; i < held * kChunks; i += 256) {
        float y[8];
        u32x2_t* w = reinterpret_cast<u32x2_t*>(codes + (size_t)i * 8);
        decode8(*w, y);
        *w = encode8(y, old / s);
      }
    }
    const float inv = 1.0f / s;
    for (int i = tid; i < n * kChunks; i += 256) {
      float y[8];
      value(i / kChunks, i % kChunks, y);
      key_out(i / kChunks, i % kChunks, y);
      if (stored) *reinterpret_cast<u32x2_t*>(codes + (size_t)held * D + (size_t)i * 8) = encode8(y, inv);
    }
    __syncthreads();  // every wave has read the old scale
    if (stored && tid == 0) *scale = s;
  } else {
    bf16_t* rows = reinterpret_cast<bf16_t*>(is_key ? c.k : c.v) + block + (size_t)held * D;
    for (int i = tid; i < n * kChunks; i += 256) {
      float y[8];
      value(i / kChunks, i % kChunks, y);
      key_out(i / kChunks, i % kChunks, y);
      if (stored) store8(rows + (size_t)i * 8, y);
    }
  }
}

}  // namespace paged
}  // namespace pqc
