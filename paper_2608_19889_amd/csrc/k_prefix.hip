// Attention of new tokens over a shared prefix and their own keys in a paged cache:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - max),
// j over the group's prefix and the sequence's own keys up to the token itself.
//
// A *segment* is a list of keys and the tokens that read it: a group's prefix with the
// tokens of all of its sequences, or a sequence's own keys with its own tokens.  The
// rows of a segment and kv head are its tokens' query heads of that kv head, so a
// prefix is multiplied with everything that shares it.  Rows go in tiles: a *wide* one
// of 128 (32 to a wavefront, every wavefront over all keys), or, when a segment has at
// most 16 rows, a *narrow* one (all rows in every wavefront, the keys shared out).
//
// Work is cut into units of 64 keys of a tile, in the order (segment, kv head, tile,
// keys), and every workgroup takes an equal run of consecutive units, whatever the
// lengths are, which only the device knows.  Where a run covers part of a tile's keys it
// leaves (max, sum, product) of them; a second kernel joins a row's parts of both
// segments.  Both are deterministic: what is added to what depends on the lengths alone.
#include <algorithm>

#include "common.h"
#include "kernels.h"

namespace axon {

constexpr float LOG2E_F = 1.4426950408889634f;
constexpr int PA_THREADS = 256;
constexpr int PA_KEYS = 64;   // keys of a unit, 16 staged by each wavefront
constexpr int PA_WIDE = 128;  // rows of a wide tile
constexpr int PA_NARROW = 16;
constexpr int PA_BLOCKS = PA_WIDE / 16;  // 16-row blocks of a wide tile's part
constexpr int PA_BATCH = PA_THREADS / 4;  // units whose pages are looked up at a time

// ---------------------------------------------------------------- plan

struct Segment {
  int tok0, tokens;  // rows: query heads of the group of tokens tok0 ..
  int64_t len;       // keys of every token (prefix), or before token 0 (own)
  int room;          // keys that the table row can list
  const int32_t* table;
  bool own;
};

template <typename T>
AXON_DEV Segment segment_of(const PrefixAttnArgs<T>& a, int s) {
  Segment g;
  const int groups = a.shared.groups;
  if (s < groups) {
    const int lo = a.shared.cu[s], hi = a.shared.cu[s + 1];
    g.tok0 = a.seqs.cu ? a.seqs.cu[lo] : lo;
    g.tokens = (a.seqs.cu ? a.seqs.cu[hi] : hi) - g.tok0;
    g.len = a.shared.lens[s];
    g.table = a.shared.table + (int64_t)s * a.shared.stride;
    g.room = a.shared.stride * a.kv.ps;
    g.own = false;
  } else {
    const int b = s - groups;
    g.tok0 = a.seqs.cu ? a.seqs.cu[b] : b;
    g.tokens = a.seqs.cu ? a.seqs.cu[b + 1] - g.tok0 : 1;
    g.len = a.seqs.lens[b];
    g.table = a.seqs.table + (int64_t)b * a.seqs.stride;
    g.room = a.seqs.stride * a.kv.ps;
    g.own = true;
  }
  return g;
}
AXON_DEV int tile_rows(int rows) { return rows <= PA_NARROW ? PA_NARROW : PA_WIDE; }
AXON_DEV int tiles_of(int rows) { return (rows + tile_rows(rows) - 1) / tile_rows(rows); }
// keys that some row of tile rt reads (G query heads a token)
AXON_DEV int tile_keys(const Segment& g, int G, int rt) {
  if (g.len < 0 || g.tokens <= 0) return 0;
  int64_t n = g.len;
  if (g.own) n += min(g.tokens - 1, (rt * PA_WIDE + PA_WIDE - 1) / G) + 1;
  return (int)min(n, (int64_t)g.room);
}
AXON_DEV int units_of(int keys) { return (keys + PA_KEYS - 1) / PA_KEYS; }

// the place of a part: blocks of 16 rows, [16][hd] products, 16 maxima, 16 sums
constexpr int part_floats(int hd) { return 16 * hd + 32; }

// where the parts of the tile that starts at row ``row`` of (kind, kv head) are
struct TileParts {
  int32_t first;  // block of the first one, the others PA_BLOCKS apart
  int32_t count;
};

// ---------------------------------------------------------------- tiles in LDS

// A unit's keys and values: [64][HD] each, 16-byte chunks of a row at chunk ^ swizzle,
// so that the lanes that read together meet different banks.
template <typename T, int HD>
struct Lds {
  static constexpr int CH = HD * sizeof(T) / 16;  // chunks of a row
  static constexpr int EL = 16 / sizeof(T);       // elements of a chunk
  static constexpr int TILE = PA_KEYS * HD;       // elements of K or V
  static AXON_DEV int swz_k(int key) { return (CH >= 16 ? key & 15 : (key >> 1) & 7); }
  static AXON_DEV int swz_v(int key) {
    if (sizeof(T) == 4) return ((key >> 2) & 1) << 3 | ((key >> 3) & 1) << 2;
    return CH >= 16 ? (key & 3) << 2 | ((key >> 2) & 1) << 1 : ((key >> 1) & 1) << 2 | ((key >> 2) & 1) << 1;
  }
  static AXON_DEV int k_at(int key, int d) { return key * HD + ((d / EL) ^ swz_k(key)) * EL + d % EL; }
  static AXON_DEV int v_at(int key, int d) { return key * HD + ((d / EL) ^ swz_v(key)) * EL + d % EL; }
};

// copies the 16 keys of this wavefront (rows 16 wave .. of the unit) that start at
// element ``src`` of both caches into a stage
template <typename T, int HD>
AXON_DEV void stage_keys(const T* kc, const T* vc, int64_t src, T* stage, int wave, int lane) {
  using L = Lds<T, HD>;
  constexpr int RPI = 64 / L::CH;  // rows of an instruction
#pragma unroll
  for (int i = 0; i < 16 / RPI; ++i) {
    const int r = i * RPI + lane / L::CH, c = lane % L::CH;
    const int64_t at = src + r * HD;
    T* dst = stage + (16 * wave + i * RPI) * HD;
    load_lds16((const bf16*)(kc + at + (c ^ L::swz_k(r)) * L::EL), (bf16x8*)dst);
    load_lds16((const bf16*)(vc + at + (c ^ L::swz_v(r)) * L::EL), (bf16x8*)(dst + L::TILE));
  }
}

// ---------------------------------------------------------------- arithmetic

typedef __attribute__((__vector_size__(8 * sizeof(float)))) float f32x8;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;
template <typename T>
struct Vec8;
template <>
struct Vec8<bf16> {
  typedef bf16x8 t;
};
template <>
struct Vec8<float> {
  typedef f32x8 t;
};

// 8 elements of a query row, negated for a negative scale (any element alignment)
template <typename T>
AXON_DEV typename Vec8<T>::t load_q8(const T* p, bool negate) {
  typename Vec8<T>::t v;
  Run8<T> r;
  r.load(p);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = from_f32<T>(negate ? -r[j] : r[j]);
  return v;
}
AXON_DEV bf16x8 read8(const bf16* p, const bf16*) { return *(const bf16x8*)p; }
AXON_DEV f32x8 read8(const float* p, const float* p2) {
  const f32x4 a = *(const f32x4*)p, b = *(const f32x4*)p2;
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
// 32 (16) keys x 32 (16) rows, 8 dimensions of each lane group
AXON_DEV f32x16 mul_wide(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
AXON_DEV f32x16 mul_wide(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
  return c;
}
AXON_DEV f32x4 mul_narrow(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
AXON_DEV f32x4 mul_narrow(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}
AXON_DEV f32x4 mul_narrow4(bf16x4 a, bf16x4 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}
AXON_DEV f32x4 mul_narrow4(f32x4 a, f32x4 b, f32x4 c) {
#pragma unroll
  for (int j = 0; j < 4; ++j) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[j], b[j], c, 0, 0, 0);
  return c;
}

AXON_DEV bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
AXON_DEV bool finite(bf16 v) { return finite((float)v); }

// ---------------------------------------------------------------- the kernel

template <typename T, int HD>
struct Ctx {
  const PrefixAttnArgs<T>& a;
  T* tiles;       // two stages of K and V
  int32_t* pids;  // pages of a batch of units, 4 to a unit, -1: none
  int32_t* odd;   // [2][4]: keys of each stage's wavefront whose values were not all finite
  float* parts;
  int G, lane, wave;
  float sc;  // |scale| log2 e
};

// A masked key has p = 0, but 0 times what stands there is NaN when that is infinite or
// NaN.  So the values of a unit with masked keys are made finite where they are staged;
// returns which of the wavefront's 16 keys had others (those that are not masked get
// them added by add_odd).
template <typename T, int HD>
AXON_DEV int make_finite(T* v, int lane) {
  constexpr int EL = Lds<T, HD>::EL, CH = Lds<T, HD>::CH;
  typedef typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type Chunk;
  int keys = 0;
#pragma unroll
  for (int i = 0; i < 16 * CH / 64; ++i) {
    Chunk* p = (Chunk*)v + i * 64 + lane;
    Chunk c = *p;
    bool ok = true;
#pragma unroll
    for (int j = 0; j < EL; ++j) ok = ok && finite(c[j]);
    const uint64_t odd = __ballot(!ok);
    if (!odd) continue;
    if (!ok) {
#pragma unroll
      for (int j = 0; j < EL; ++j) c[j] = finite(c[j]) ? c[j] : (T)0.f;
      *p = c;
    }
#pragma unroll
    for (int r = 0; r < 64 / CH; ++r)
      if (odd >> (r * CH) & ((1ull << (CH - 1) << 1) - 1)) keys |= 1 << (i * (64 / CH) + r);
  }
  return keys;
}

// Runs f(u, stage, pages, odd) over units first .. last - 1 of a segment (64 keys each,
// from key 64 u): the stage that holds them, which of its 16-key blocks have a page, and
// which of its keys make_finite changed.  Keys from ``least`` on are masked for some row.
// barrier: f reads all of a unit's keys, not only the 16 that the wavefront staged.
template <typename T, int HD, typename F>
AXON_DEV void for_units(const Ctx<T, HD>& x, const Segment& g, int kvh, int first, int last, int least, bool barrier,
                        F&& f) {
  constexpr int TILE = Lds<T, HD>::TILE;
  const auto& kv = x.a.kv;
  for (int u0 = first; u0 < last; u0 += PA_BATCH) {
    const int n = min(last - u0, PA_BATCH);
    __syncthreads();  // the stages and pages of what came before are read
    {
      const int key = (u0 * 4 + (int)threadIdx.x) * 16;
      int page = -1;
      if ((int)threadIdx.x < 4 * n && key < g.room) page = g.table[key / kv.ps];
      x.pids[threadIdx.x] = page >= 0 && page < kv.num_pages ? page : -1;
    }
    __syncthreads();
    auto stage = [&](int i) {
      const int key = (u0 + i) * PA_KEYS + 16 * x.wave;
      const int page = max(__builtin_amdgcn_readfirstlane(x.pids[4 * i + x.wave]), 0);  // (none: masked, but read)
      const int64_t src = (((int64_t)page * kv.kv_heads + kvh) * kv.ps + key % kv.ps) * HD;
      stage_keys<T, HD>((const T*)kv.k, (const T*)kv.v, src, x.tiles + (i & 1) * 2 * TILE, x.wave, x.lane);
    };
    stage(0);
    for (int i = 0; i < n; ++i) {
      T* st = x.tiles + (i & 1) * 2 * TILE;
      int pages = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) pages |= (x.pids[4 * i + j] >= 0) << j;
      pages = __builtin_amdgcn_readfirstlane(pages);
      const bool masked = (u0 + i) * PA_KEYS + PA_KEYS > least || pages != 15;
      // (the unit is here; what was read of the stage that is filled next as well)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      if (masked) {
        const int odd = make_finite<T, HD>(st + TILE + 16 * x.wave * HD, x.lane);
        if (x.lane == 0) x.odd[4 * (i & 1) + x.wave] = odd;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      }
      if (barrier) phase_barrier();
      if (i + 1 < n) stage(i + 1);
      f(u0 + i, st, pages, masked ? x.odd + 4 * (i & 1) : nullptr);
    }
  }
}

// Adds the infinite and NaN values that make_finite took out of block ``blk`` of unit u
// where the lane's row sees their keys: o[i], i < N, is dimension dim(i).
template <typename T, int HD, int N, typename D>
AXON_DEV void add_odd(const Ctx<T, HD>& x, const Segment& g, int kvh, int u, int blk, int odd, int limit, float (&o)[N],
                      D&& dim) {
  const auto& kv = x.a.kv;
  for (; odd; odd &= odd - 1) {
    const int key = u * PA_KEYS + 16 * blk + __ffs(odd) - 1;
    if (key >= limit) continue;
    const int page = g.table[key / kv.ps];
    if (page < 0 || page >= kv.num_pages) continue;
    const T* v = (const T*)kv.v + (((int64_t)page * kv.kv_heads + kvh) * kv.ps + key % kv.ps) * HD;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = to_f32(v[dim(i)]);
      if (!finite(e)) o[i] += e;
    }
  }
}

// Row r of a tile's segment as an element of q: its token and head
template <typename T, int HD>
AXON_DEV const T* q_row(const Ctx<T, HD>& x, const Segment& g, int kvh, int r) {
  return x.a.q + (int64_t)(g.tok0 + r / x.G) * x.a.ldq + (int64_t)(kvh * x.G + r % x.G) * HD;
}
// keys that row r sees
template <typename T, int HD>
AXON_DEV int row_limit(const Ctx<T, HD>& x, const Segment& g, int r) {
  return (int)min(g.own ? g.len + r / x.G + 1 : g.len, (int64_t)g.room);
}

template <typename T, int HD>
AXON_DEV void wide_tile(const Ctx<T, HD>& x, const Segment& g, int kvh, int rt, int first, int last, int block) {
  using L = Lds<T, HD>;
  using V8 = typename Vec8<T>::t;
  constexpr int DT = HD / 32, QS = HD / 16;
  const int hl = x.lane >> 5, c = x.lane & 31;
  const int rows = g.tokens * x.G, r0 = rt * PA_WIDE + 32 * x.wave, r = min(r0 + c, rows - 1);
  V8 q[QS];
  {
    const T* p = q_row(x, g, kvh, r) + 8 * hl;
#pragma unroll
    for (int k = 0; k < QS; ++k) q[k] = load_q8<T>(p + 16 * k, x.a.scale < 0.f);
  }
  const int limit = row_limit(x, g, r);
  const int least = row_limit(x, g, min(r0, rows - 1)), most = row_limit(x, g, min(r0 + 31, rows - 1));
  f32x16 o[DT] = {};
  float m = -INFINITY, l = 0.f;  // m: the largest score times sc
  for_units(x, g, kvh, first, last, row_limit(x, g, rt * PA_WIDE), true, [&](int u, const T* st, int pages, const int* odd) {
    const int key0 = u * PA_KEYS;
    if (r0 >= rows || key0 >= most) return;
    f32x16 s[2] = {};
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int k = 0; k < QS; ++k) {
        const int d = 16 * k + 8 * hl;
        s[kb] = mul_wide(read8(st + L::k_at(32 * kb + c, d), st + L::k_at(32 * kb + c, d + 4)), q[k], s[kb]);
      }
    // s[kb][i]: key key0 + 32 kb + 8 (i / 4) + 4 hl + i % 4, row c
    const bool masked = key0 + PA_KEYS > least || pages != 15;
    if (masked) {
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 32 * kb + 8 * (i >> 2) + 4 * hl + (i & 3);
          if (key0 + key >= limit || !(pages >> (key >> 4) & 1)) s[kb][i] = -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[kb][i]);
    top = fmaxf(top, lane_xor32(top)) * x.sc;
    const float m_new = fmaxf(m, top);
    const float base = m_new == -INFINITY ? 0.f : m_new;
    const float fall = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    l *= fall;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] *= fall;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 p;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[kb][i], x.sc, -base));
        l += p[i];
      }
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // keys 16 e .. of the block
          bf16x8 pb;
#pragma unroll
          for (int j = 0; j < 8; ++j) pb[j] = (bf16)p[8 * e + j];
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            const int key = 32 * kb + 16 * e + 4 * hl + ((x.lane & 15) >> 2);
            const int dim = 32 * d + 16 * ((x.lane >> 4) & 1) + 4 * (x.lane & 3);
            o[d] = mul_wide(read_tr8(st + L::TILE + L::v_at(key, dim), st + L::TILE + L::v_at(key + 8, dim)), pb, o[d]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = 32 * kb + 8 * (i >> 2) + 4 * hl + (i & 3);
#pragma unroll
          for (int d = 0; d < DT; ++d)
            o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(st[L::TILE + L::v_at(key, 32 * d + c)], p[i], o[d], 0, 0, 0);
        }
      }
    }
    if (odd)
      for (int blk = 0; blk < 4; ++blk)
        if (const int keys = __builtin_amdgcn_readfirstlane(odd[blk])) {
          float e[16 * DT];
#pragma unroll
          for (int i = 0; i < 16 * DT; ++i) e[i] = o[i / 16][i % 16];
          add_odd(x, g, kvh, u, blk, keys, limit, e, [&](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * hl + i % 4; });
#pragma unroll
          for (int i = 0; i < 16 * DT; ++i) o[i / 16][i % 16] = e[i];
        }
  });
  if (r0 + c >= rows) return;
  l += lane_xor32(l);
  float* part = x.parts + (int64_t)(block + 2 * x.wave + (c >> 4)) * part_floats(HD);
  const int row = c & 15;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(f32x4*)(part + row * HD + 32 * d + 8 * j + 4 * hl) = f32x4{o[d][4 * j], o[d][4 * j + 1], o[d][4 * j + 2], o[d][4 * j + 3]};
  if (hl == 0) {
    part[16 * HD + row] = m;
    part[16 * HD + 16 + row] = l;
  }
}

template <typename T, int HD>
AXON_DEV void narrow_tile(const Ctx<T, HD>& x, const Segment& g, int kvh, int first, int last, int block) {
  using L = Lds<T, HD>;
  using V8 = typename Vec8<T>::t;
  constexpr int DT = HD / 16, QS = HD / 32;
  const int gq = x.lane >> 4, c = x.lane & 15;
  const int rows = g.tokens * x.G, r = min(c, rows - 1);
  V8 q[QS];
  {
    const T* p = q_row(x, g, kvh, r) + 8 * gq;
#pragma unroll
    for (int k = 0; k < QS; ++k) q[k] = load_q8<T>(p + 32 * k, x.a.scale < 0.f);
  }
  const int limit = row_limit(x, g, r), least = row_limit(x, g, 0);
  f32x4 o[DT] = {};
  float m = -INFINITY, l = 0.f;
  for_units(x, g, kvh, first, last, least, false, [&](int u, const T* st, int pages, const int* odd) {
    const int mine = 16 * x.wave, key0 = u * PA_KEYS + mine;
    f32x4 s = {};
#pragma unroll
    for (int k = 0; k < QS; ++k) {
      const int d = 32 * k + 8 * gq;
      s = mul_narrow(read8(st + L::k_at(mine + c, d), st + L::k_at(mine + c, d + 4)), q[k], s);
    }
    // s[i]: key key0 + 4 gq + i, row c
    const bool there = pages >> x.wave & 1, masked = key0 + 16 > least || !there;
    if (masked) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (key0 + 4 * gq + i >= limit || !there) s[i] = -INFINITY;
    }
    float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    top = fmaxf(top, lane_xor16(top));
    top = fmaxf(top, lane_xor32(top)) * x.sc;
    const float m_new = fmaxf(m, top);
    const float base = m_new == -INFINITY ? 0.f : m_new;
    const float fall = __builtin_amdgcn_exp2f(m - base);
    m = m_new;
    l *= fall;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] *= fall;
    typename std::conditional<sizeof(T) == 2, bf16x4, f32x4>::type p;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float e = __builtin_amdgcn_exp2f(fmaf(s[i], x.sc, -base));
      l += e;
      p[i] = from_f32<T>(e);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      decltype(p) v;
      if constexpr (sizeof(T) == 2) {
        typedef __attribute__((address_space(3))) bf16x4 lds4;
        v = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
            (lds4*)(st + L::TILE + L::v_at(mine + 4 * gq + (c >> 2), 16 * d + 4 * (c & 3))));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = st[L::TILE + L::v_at(mine + 4 * gq + i, 16 * d + c)];
      }
      o[d] = mul_narrow4(v, p, o[d]);
    }
    if (odd)
      if (const int keys = __builtin_amdgcn_readfirstlane(odd[x.wave])) {
        float e[4 * DT];
#pragma unroll
        for (int i = 0; i < 4 * DT; ++i) e[i] = o[i / 4][i % 4];
        add_odd(x, g, kvh, u, x.wave, keys, limit, e, [&](int i) { return 16 * (i / 4) + 4 * gq + i % 4; });
#pragma unroll
        for (int i = 0; i < 4 * DT; ++i) o[i / 4][i % 4] = e[i];
      }
  });
  l += lane_xor16(l);
  l += lane_xor32(l);
  // the four wavefronts' keys
  float* so = (float*)x.tiles;  // [4][16][HD]
  float* sm = so + 4 * 16 * HD;  // [4][16] maxima, then sums
  __syncthreads();
#pragma unroll
  for (int d = 0; d < DT; ++d) *(f32x4*)(so + (x.wave * 16 + c) * HD + 16 * d + 4 * gq) = o[d];
  if (gq == 0) {
    sm[x.wave * 16 + c] = m;
    sm[64 + x.wave * 16 + c] = l;
  }
  __syncthreads();
  float* part = x.parts + (int64_t)block * part_floats(HD);
  for (int i = threadIdx.x; i < rows * HD / 4; i += PA_THREADS) {
    const int row = i / (HD / 4), d = i % (HD / 4) * 4;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, sm[w * 16 + row]);
    f32x4 sum = {};
    float ls = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sm[w * 16 + row] - top);
      ls += f * sm[64 + w * 16 + row];
      if (f > 0.f) sum += f * *(const f32x4*)(so + (w * 16 + row) * HD + d);
    }
    *(f32x4*)(part + row * HD + d) = sum;
    if (d == 0) {
      part[16 * HD + row] = top;
      part[16 * HD + 16 + row] = ls;
    }
  }
}

template <typename T, int HD>
constexpr int stage_bytes() {
  // two stages; a narrow tile's join needs [4][16][HD] + 128 floats
  const int tiles = 2 * 2 * PA_KEYS * HD * (int)sizeof(T), join = (64 * HD + 128) * 4;
  return tiles > join ? tiles : join;
}

template <typename T, int HD>
__global__ void __launch_bounds__(PA_THREADS, 2) prefix_attn_kernel(PrefixAttnArgs<T> a, float sc, TileParts* info,
                                                                 float* parts) {
  __shared__ __align__(16) char lds[stage_bytes<T, HD>()];
  __shared__ int32_t pids[PA_THREADS], odd[8];
  __shared__ int64_t scan[2][PA_THREADS / 64];
  __shared__ int start[4];
  const int KV = a.kv.kv_heads, G = a.heads / KV, segs = a.shared.groups + a.seqs.seqs;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // units and part blocks of each thread's segments, and before them
  const int each = (segs + PA_THREADS - 1) / PA_THREADS, s0 = min(segs, (int)threadIdx.x * each), s1 = min(segs, s0 + each);
  auto sizes = [&](const Segment& g, int& units, int& blocks) {  // of one kv head
    const int rows = g.tokens * G, tiles = tiles_of(rows);
    units = 0;
    if (g.own && tiles > 1)
      for (int rt = 0; rt < tiles; ++rt) units += units_of(tile_keys(g, G, rt));
    else
      units = tiles * units_of(tile_keys(g, G, tiles - 1));
    blocks = tiles * (tile_rows(rows) / 16);
  };
  int64_t mine[2] = {};
  for (int s = s0; s < s1; ++s) {
    int u, b;
    sizes(segment_of(a, s), u, b);
    mine[0] += (int64_t)u * KV;
    mine[1] += (int64_t)b * KV;
  }
  int64_t upto[2] = {mine[0], mine[1]};
#pragma unroll
  for (int d = 1; d < 64; d <<= 1)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int64_t v = __shfl_up(upto[j], d);
      if (lane >= d) upto[j] += v;
    }
  if (lane == 63) {
    scan[0][wave] = upto[0];
    scan[1][wave] = upto[1];
  }
  __syncthreads();
  int64_t total = 0, before[2] = {upto[0] - mine[0], upto[1] - mine[1]};
#pragma unroll
  for (int w = 0; w < PA_THREADS / 64; ++w) {
    if (w < wave) {
      before[0] += scan[0][w];
      before[1] += scan[1][w];
    }
    total += scan[0][w];
  }
  // Consecutive runs on one XCD, whose L2 holds what they share; fewer units than
  // workgroups: one each, over all XCDs.
  const int n = (int)min((int64_t)gridDim.x, total);
  const int wg = n < (int)gridDim.x || n % 8 ? blockIdx.x : blockIdx.x % 8 * (n / 8) + blockIdx.x / 8;
  if (wg >= n) return;
  int64_t at = total * wg / n;
  const int64_t end = total * (wg + 1) / n;
  if (before[0] <= at && at < before[0] + mine[0]) {  // one thread
    int64_t u0 = before[0], b0 = before[1];
    for (int s = s0; s < s1; ++s) {
      int u, b;
      sizes(segment_of(a, s), u, b);
      if (at < u0 + (int64_t)u * KV) {
        start[0] = s;
        start[1] = (int)(at - u0);
        start[2] = (int)b0;
        start[3] = u;
        break;
      }
      u0 += (int64_t)u * KV;
      b0 += (int64_t)b * KV;
    }
  }
  __syncthreads();
  // the first segment from s on that has units, where sequences take no part: the
  // workgroup looks at as many at a time as it has threads
  auto next_segment = [&](int s, int& block) {
    for (;; s += PA_THREADS) {
      int u = 0, b = 0;
      if (s + (int)threadIdx.x < segs) sizes(segment_of(a, s + threadIdx.x), u, b);
      __syncthreads();
      if (threadIdx.x == 0) {
        start[0] = PA_THREADS;
        start[1] = 0;
      }
      __syncthreads();
      if (u) atomicMin(&start[0], (int)threadIdx.x);
      __syncthreads();
      const int first = start[0];
      if ((int)threadIdx.x < first) atomicAdd(&start[1], b * KV);
      __syncthreads();
      block += __builtin_amdgcn_readfirstlane(start[1]);
      if (first < PA_THREADS || s + PA_THREADS >= segs) return s + __builtin_amdgcn_readfirstlane(first);
    }
  };
  int s = __builtin_amdgcn_readfirstlane(start[0]), block = __builtin_amdgcn_readfirstlane(start[2]);
  const int off = __builtin_amdgcn_readfirstlane(start[1]), per_head = __builtin_amdgcn_readfirstlane(start[3]);
  const Ctx<T, HD> x{a, (T*)lds, pids, odd, parts, G, lane, wave, sc};
  Segment g = segment_of(a, s);
  int kvh = off / per_head, u = off % per_head, rt = 0;
  {
    const int rows = g.tokens * G;
    block += kvh * tiles_of(rows) * (tile_rows(rows) / 16);
    for (;;) {  // the tile
      const int nu = units_of(tile_keys(g, G, rt));
      if (u < nu) break;
      u -= nu;
      ++rt;
      block += tile_rows(rows) / 16;
    }
  }
  while (at < end) {
    const int rows = g.tokens * G, nu = units_of(tile_keys(g, G, rt));
    if (nu > 0) {
      const int take = (int)min((int64_t)(nu - u), end - at);
      const int64_t tile0 = at - u;  // the tile's first unit
      if (u == 0 && threadIdx.x == 0) {
        const int w1 = (int)(((tile0 + nu) * n - 1) / total);  // who has its last unit
        const int64_t row0 = (int64_t)g.tok0 * G + rt * PA_WIDE;
        info[((g.own ? KV : 0) + kvh) * (int64_t)a.tokens * G + row0] = TileParts{block + PA_BLOCKS * wg, w1 - wg + 1};
      }
      if (rows <= PA_NARROW) narrow_tile(x, g, kvh, u, u + take, block + PA_BLOCKS * wg);
      else wide_tile(x, g, kvh, rt, u, u + take, block + PA_BLOCKS * wg);
      at += take;
    }
    u = 0;
    block += tile_rows(rows) / 16;
    if (++rt >= tiles_of(rows)) {
      rt = 0;
      if (++kvh == KV) {
        kvh = 0;
        if (at >= end) break;
        g = segment_of(a, ++s);  // (units are left, so a segment that has some follows)
        if (!units_of(tile_keys(g, G, tiles_of(g.tokens * G) - 1))) {
          s = next_segment(s, block);
          g = segment_of(a, s);
        }
      }
    }
  }
}

// A row's parts of both segments: out = sum f o / sum f l, f = 2^(m - max).  A workgroup
// per (token, kv head), HD / 4 lanes a row.
template <typename T, int HD>
__global__ void __launch_bounds__(PA_THREADS) prefix_join_kernel(PrefixAttnArgs<T> a, const TileParts* info,
                                                                 const float* parts) {
  constexpr int LANES = HD / 4;
  constexpr int64_t NEXT = PA_BLOCKS * part_floats(HD);  // from a tile's part to its next
  const int t = blockIdx.x, kvh = blockIdx.y, KV = a.kv.kv_heads, G = a.heads / KV;
  const int lane = threadIdx.x & 63;
  auto among = [&](const int32_t* cu, int n, int v) {  // how many of cu[1 .. n] are <= v
    int c = 0;
    for (int i = lane; i - lane < n; i += 64) c += __popcll(__ballot(i < n && cu[i + 1] <= v));
    return c;
  };
  const int b = a.seqs.cu ? among(a.seqs.cu, a.seqs.seqs, t) : t;
  if (b >= a.seqs.seqs) return;  // behind the last sequence
  const bool active = a.seqs.lens[b] >= 0;
  const int grp = a.shared.groups ? among(a.shared.cu, a.shared.groups, b) : 0;
  const bool has[2] = {grp < a.shared.groups, true};
  for (int j = threadIdx.x / LANES; j < G; j += PA_THREADS / LANES) {
    const int d = threadIdx.x % LANES * 4;
    const float *at[2], *ml[2];  // the first part's row; its maximum (and, 16 on, sum)
    int count[2] = {0, 0};
    float top = -INFINITY;
    for (int k = 0; k < 2; ++k) {
      if (!has[k] || !active) continue;
      const Segment g = segment_of(a, k ? a.shared.groups + b : grp);
      const int r = (t - g.tok0) * G + j, rt = r / tile_rows(g.tokens * G), row = r - rt * PA_WIDE;
      if (tile_keys(g, G, rt) <= 0) continue;
      const TileParts p = info[(k * KV + kvh) * (int64_t)a.tokens * G + (int64_t)g.tok0 * G + rt * PA_WIDE];
      const float* first = parts + (int64_t)(p.first + row / 16) * part_floats(HD);
      at[k] = first + row % 16 * HD + d;
      ml[k] = first + 16 * HD + row % 16;
      count[k] = p.count;
      for (int i = 0; i < count[k]; ++i) top = fmaxf(top, ml[k][i * NEXT]);
    }
    f32x4 o = {};
    float l = 0.f;
    if (top > -INFINITY)
      for (int k = 0; k < 2; ++k)
        for (int i = 0; i < count[k]; ++i) {
          const float f = __builtin_amdgcn_exp2f(ml[k][i * NEXT] - top);
          l += f * ml[k][i * NEXT + 16];
          if (f > 0.f) o += f * *(const f32x4*)(at[k] + i * NEXT);
        }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;
    T* out = a.out + (int64_t)t * a.ldo + (int64_t)(kvh * G + j) * HD + d;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = from_f32<T>(l == 0.f ? 0.f : o[i] * inv);
    if (a.lse && d == 0)
      a.lse[(int64_t)t * a.heads + kvh * G + j] = l == 0.f ? -INFINITY : (top + __log2f(l)) / LOG2E_F;
  }
}

// ---------------------------------------------------------------- host

namespace {

int wgs_of(bool f32, int hd) { return f32 && hd == 128 ? 256 : 512; }
// (upper bounds of) the part blocks and rows of a call
int64_t blocks_of(int64_t tokens, int seqs, int groups, int heads, int kv_heads, int wgs) {
  const int64_t G = heads / kv_heads, rows = tokens * G;
  // a segment of r rows: one block, or 8 ceil(r / 128) <= r / 16 + 8 and less than r
  // (r > 16), so at most min(r, r / 16 + 8) of them
  auto bound = [&](int64_t segs) { return std::min(rows / 16 + PA_BLOCKS * segs, rows + segs); };
  return (bound(seqs) + (groups ? bound(groups) : 0)) * kv_heads + (int64_t)PA_BLOCKS * wgs;
}

}  // namespace

int64_t prefix_attn_workspace(int64_t tokens, int seqs, int groups, int heads, const PagedKV& kv, bool f32) {
  const int64_t rows = 2 * tokens * heads;
  return (rows * (int64_t)sizeof(TileParts) + 15) / 16 * 16 +
         blocks_of(tokens, seqs, groups, heads, kv.kv_heads, wgs_of(f32, kv.hd)) * part_floats(kv.hd) * 4;
}

int64_t prefix_attn_units(int64_t tokens, int seqs, int groups, int heads, const PagedKV& kv, int64_t pages) {
  const int64_t rows = tokens * (heads / kv.kv_heads), tiles = seqs + groups + 2 * (rows / PA_WIDE);
  return tiles * kv.kv_heads * ((pages * kv.ps + PA_KEYS - 1) / PA_KEYS);
}

template <typename T, int HD>
static void launch(const PrefixAttnArgs<T>& a, void* workspace, hipStream_t s) {
  TileParts* info = (TileParts*)workspace;
  float* parts = (float*)((char*)workspace + (2 * (int64_t)a.tokens * a.heads * sizeof(TileParts) + 15) / 16 * 16);
  // a scale of 0 leaves every score, masked ones apart, the same
  const float sc = a.scale == 0.f ? 1e-37f : fabsf(a.scale) * LOG2E_F;
  prefix_attn_kernel<T, HD><<<wgs_of(sizeof(T) == 4, HD), PA_THREADS, 0, s>>>(a, sc, info, parts);
  prefix_join_kernel<T, HD><<<dim3(a.tokens, a.kv.kv_heads), PA_THREADS, 0, s>>>(a, info, parts);
}

template <typename T>
void launch_prefix_attn(const PrefixAttnArgs<T>& a, void* workspace, hipStream_t s) {
  if (!a.tokens) return;
  if (a.kv.hd == 64) launch<T, 64>(a, workspace, s);
  else launch<T, 128>(a, workspace, s);
}
template void launch_prefix_attn<float>(const PrefixAttnArgs<float>&, void*, hipStream_t);
template void launch_prefix_attn<bf16>(const PrefixAttnArgs<bf16>&, void*, hipStream_t);

}  // namespace axon
