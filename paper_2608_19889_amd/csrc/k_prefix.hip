// Attention of new tokens over a shared prefix and their own keys in a paged cache:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - max),
// j over the group's prefix and the sequence's own keys up to the token itself.
//
// A *segment* is a list of keys and the tokens that read it: a group's prefix with the
// tokens of all of its sequences, or a sequence's own keys with its own tokens.  The
// rows of a segment and kv head are its tokens' query heads of that kv head, so a
// prefix is multiplied with everything that shares it.  Rows go in tiles: a segment of
// at most 16 rows is one *narrow* tile (a single token's own keys), any other is cut
// into *wide* ones of 256 rows.  Each kind has its kernel:
//   prefix_wide_kernel    a workgroup of 8 wavefronts, 32 rows each, over keys that all
//                         of them read from LDS (with few rows the keys are halved
//                         between wavefronts): matrix instructions' work
//   prefix_narrow_kernel  every wavefront by itself over 16 keys at a time, many of them
//                         on a CU: memory's work
//   prefix_join_kernel    joins the parts that they leave
//
// Work is cut into units of keys of a tile, in the order (segment, kv head, tile, keys),
// and every worker takes an equal run of consecutive units, whatever the lengths are,
// which only the device knows.  Of the keys of a tile in its run it leaves (max, sum,
// product).  What is added to what depends on the lengths alone: the same bits every
// time.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace axon {

constexpr float LOG2E_F = 1.4426950408889634f;
constexpr int WIDE_THREADS = 512, WIDE_WAVES = 8, WIDE_KEYS = 64, WIDE_ROWS = 256;
constexpr int NARROW_THREADS = 256, NARROW_WAVES = 4, NARROW_KEYS = 16, NARROW_ROWS = 16;
constexpr int WIDE_LEAST = 4, NARROW_LEAST = 2;        // steps of a worker
constexpr int SLOT_BLOCKS = WIDE_ROWS / 16;           // 16-row blocks of a wide part

// ---------------------------------------------------------------- plan

struct Segment {
  int tok0, tokens;  // rows: query heads of tokens tok0 ..
  int64_t len;       // keys of every token (prefix), or before token 0 (own)
  int room;          // keys that the table row can list
  const int32_t* table;
  bool own;
};

template <typename T>
AXON_DEV Segment segment_of(const PrefixAttnArgs<T>& a, int s) {
  Segment g;
  const int groups = a.shared.groups;
  int end;
  auto among = [](int v, int n) { return min(max(v, 0), n); };
  if (s < groups) {
    const int lo = among(a.shared.cu[s], a.seqs.seqs), hi = among(a.shared.cu[s + 1], a.seqs.seqs);
    g.tok0 = a.seqs.cu ? a.seqs.cu[lo] : lo;
    end = a.seqs.cu ? a.seqs.cu[hi] : hi;
    g.len = a.shared.lens[s];
    g.table = a.shared.table + (int64_t)s * a.shared.stride;
    g.room = a.shared.stride * a.kv.ps;
    g.own = false;
  } else {
    const int b = s - groups;
    g.tok0 = a.seqs.cu ? a.seqs.cu[b] : b;
    end = a.seqs.cu ? a.seqs.cu[b + 1] : b + 1;
    g.len = a.seqs.lens[b];
    g.table = a.seqs.table + (int64_t)b * a.seqs.stride;
    g.room = a.seqs.stride * a.kv.ps;
    g.own = true;
  }
  g.tok0 = among(g.tok0, a.tokens);
  g.tokens = among(end, a.tokens) - g.tok0;
  return g;
}
// keys that some of rows ``row0`` .. row0 + n - 1 reads (G query heads a token)
AXON_DEV int tile_keys(const Segment& g, int G, int row0, int n) {
  if (g.len < 0 || g.tokens <= 0) return 0;
  const int64_t k = g.own ? g.len + min(g.tokens - 1, (row0 + n - 1) / G) + 1 : g.len;
  return (int)min(k, (int64_t)g.room);
}
// keys that row r reads
AXON_DEV int row_keys(const Segment& g, int G, int r) {
  return (int)min(g.own ? g.len + r / G + 1 : g.len, (int64_t)g.room);
}

// The tiles of one kind, their units, and their steps: as many as units, and START more
// at its beginning that stand for what a tile costs by itself (looking up pages, loading
// queries, filling the pipeline).  Workers share the steps.
template <bool WIDE>
struct Tiles {
  static constexpr int ROWS = WIDE ? WIDE_ROWS : NARROW_ROWS, KEYS = WIDE ? WIDE_KEYS : NARROW_KEYS;
  static constexpr int START = 4;
  static AXON_DEV int of(const Segment& g, int G) {  // of a kv head
    const int rows = g.tokens * G;
    return rows > NARROW_ROWS ? (WIDE ? (rows + ROWS - 1) / ROWS : 0) : (WIDE || rows <= 0 ? 0 : 1);
  }
  static AXON_DEV int units(const Segment& g, int G, int rt) {
    return (tile_keys(g, G, rt * ROWS, ROWS) + KEYS - 1) / KEYS;
  }
  static AXON_DEV int steps(const Segment& g, int G, int rt) {
    const int u = units(g, G, rt);
    return u ? u + START : 0;
  }
  // (steps, tiles) of a kv head
  static AXON_DEV int2 sizes(const Segment& g, int G) {
    const int n = of(g, G);
    int u = 0;
    if (g.own)
      for (int rt = 0; rt < n; ++rt) u += steps(g, G, rt);
    else if (n)
      u = n * steps(g, G, 0);
    return int2{u, n};
  }
};

// where the parts of a tile are: slots first .. first + count - 1
struct TileParts {
  int32_t first, count;
};
// [prefix, own][kv head][first row of the tile among all tokens' rows]
AXON_DEV int64_t info_at(bool own, int kvh, int KV, int64_t rows, int tok0, int G, int row0) {
  return ((own ? KV : 0) + kvh) * rows + (int64_t)tok0 * G + row0;
}
// a block of 16 rows of a part: [16][hd] products, 16 maxima, 16 sums
constexpr int part_floats(int hd) { return 16 * hd + 32; }

// A place in the order of steps
struct Place {
  int s, kvh, rt, step, tile;  // tile: number among all tiles of the kind
};
template <int WAVES>
struct PlanShared {
  int64_t sum[2][WAVES];
  int place[WAVES][4];
  int next[2];
};

// Steps of all segments (total), and what the threads before this one (segments s0 ..
// s1 - 1 are its own) have; every thread of the workgroup calls it.
template <typename T, bool WIDE, int THREADS>
struct Plan {
  const PrefixAttnArgs<T>& a;
  PlanShared<THREADS / 64>& sh;
  int G, KV, segs, s0, s1;
  int64_t total, before[2], mine[2];  // steps, tiles
  AXON_DEV Plan(const PrefixAttnArgs<T>& args, PlanShared<THREADS / 64>& shared) : a(args), sh(shared) {
    KV = a.kv.kv_heads;
    G = a.heads / KV;
    segs = a.shared.groups + a.seqs.seqs;
    const int each = (segs + THREADS - 1) / THREADS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    s0 = min(segs, (int)threadIdx.x * each);
    s1 = min(segs, s0 + each);
    mine[0] = mine[1] = 0;
    for (int s = s0; s < s1; ++s) {
      const int2 n = Tiles<WIDE>::sizes(segment_of(a, s), G);
      mine[0] += (int64_t)n.x * KV;
      mine[1] += (int64_t)n.y * KV;
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
      sh.sum[0][wave] = upto[0];
      sh.sum[1][wave] = upto[1];
    }
    __syncthreads();
    total = 0;
    before[0] = upto[0] - mine[0];
    before[1] = upto[1] - mine[1];
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
      if (w < wave) {
        before[0] += sh.sum[0][w];
        before[1] += sh.sum[1][w];
      }
      total += sh.sum[0][w];
    }
  }
  // step ``at`` (< total) of worker ``w`` of the workgroup, for get(w) after a barrier
  AXON_DEV void find(int w, int64_t at) {
    if (at < before[0] || at >= before[0] + mine[0]) return;  // one thread goes on
    int64_t u0 = before[0], t0 = before[1];
    for (int s = s0; s < s1; ++s) {
      const int2 n = Tiles<WIDE>::sizes(segment_of(a, s), G);
      if (at < u0 + (int64_t)n.x * KV) {
        sh.place[w][0] = s;
        sh.place[w][1] = (int)(at - u0);
        sh.place[w][2] = (int)t0;
        sh.place[w][3] = n.x;
        return;
      }
      u0 += (int64_t)n.x * KV;
      t0 += (int64_t)n.y * KV;
    }
  }
  AXON_DEV Place get(int w, Segment& g) const {
    Place p;
    p.s = __builtin_amdgcn_readfirstlane(sh.place[w][0]);
    const int off = __builtin_amdgcn_readfirstlane(sh.place[w][1]), per = __builtin_amdgcn_readfirstlane(sh.place[w][3]);
    p.tile = __builtin_amdgcn_readfirstlane(sh.place[w][2]);
    g = segment_of(a, p.s);
    p.kvh = off / per;
    p.step = off % per;
    p.rt = 0;
    p.tile += p.kvh * Tiles<WIDE>::of(g, G);
    for (;;) {
      const int n = Tiles<WIDE>::steps(g, G, p.rt);
      if (p.step < n) return p;
      p.step -= n;
      ++p.rt;
      ++p.tile;
    }
  }
  // the next tile that has units (there is one); lane-parallel over segments without any
  AXON_DEV void advance(Place& p, Segment& g) const {
    const int lane = threadIdx.x & 63;
    p.step = 0;
    for (;;) {
      ++p.tile;
      if (++p.rt < Tiles<WIDE>::of(g, G)) {
        if (Tiles<WIDE>::units(g, G, p.rt)) return;
        continue;
      }
      p.rt = 0;
      if (++p.kvh < KV) return;  // (the first tile of a segment has units if any has)
      p.kvh = 0;
      ++p.s;
      for (;;) {
        int2 n = {0, 0};
        if (p.s + lane < segs) n = Tiles<WIDE>::sizes(segment_of(a, p.s + lane), G);
        const uint64_t has = __ballot(n.x > 0);
        const int skip = has ? __ffsll((long long)has) - 1 : 64;
        int tiles = lane < skip ? n.y : 0;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) tiles += __shfl_xor(tiles, d);
        p.tile += __builtin_amdgcn_readfirstlane(tiles) * KV;
        p.s += skip;
        if (has || p.s >= segs) break;
      }
      p.s = __builtin_amdgcn_readfirstlane(p.s);
      g = segment_of(a, min(p.s, segs - 1));
      return;
    }
  }
};

// ---------------------------------------------------------------- tiles in LDS

AXON_DEV uint32_t lds_address(const void* p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p; }
// 16 bytes of each lane from global memory to LDS (lane L's to lds + 16 L), in flight
// until a wait for vmcnt.  As assembly where the waits are all written out: of the builtin
// the compiler knows that it writes LDS, and before a transposing read it then waits for
// every copy in flight, those of the later stages too (a third of the kernel's time).
AXON_DEV void copy_lds16(const void* src, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
               :
               : "v"(src), "s"(__builtin_amdgcn_readfirstlane(lds))
               : "memory", "m0");
}

// Keys and values of a unit: rows of HD, the 16-byte chunks of a row at chunk ^ swizzle,
// so that the lanes that read together meet different banks.
template <typename T, int HD>
struct Lds {
  static constexpr int CH = HD * sizeof(T) / 16;  // chunks of a row
  static constexpr int EL = 16 / sizeof(T);       // elements of a chunk
  static constexpr int RPI = 64 / CH;             // rows of a wavefront's 16-byte copy
  static AXON_DEV int swz_k(int key) { return (CH >= 16 ? key & 15 : (key >> 1) & 7); }
  static AXON_DEV int swz_v(int key) {
    if (sizeof(T) == 4) return ((key >> 2) & 1) << 3 | ((key >> 3) & 1) << 2;
    return CH >= 16 ? (key & 3) << 2 | ((key >> 2) & 1) << 1 : ((key >> 1) & 1) << 2 | ((key >> 2) & 1) << 1;
  }
  static AXON_DEV int k_at(int key, int d) { return key * HD + ((d / EL) ^ swz_k(key)) * EL + d % EL; }
  static AXON_DEV int v_at(int key, int d) { return key * HD + ((d / EL) ^ swz_v(key)) * EL + d % EL; }
  // Rows key0 .. key0 + n - 1 of a unit, which lie one after another at ``src``, to
  // row 0 .. of ``dst`` (a wavefront's copy).
  template <bool K, bool ASM>
  static AXON_DEV void stage(const T* src, T* dst, int key0, int n, int lane) {
#pragma unroll
    for (int i = 0; i < n / RPI; ++i) {
      const int r = i * RPI + lane / CH, c = lane % CH;
      const int sw = K ? swz_k(key0 + r) : swz_v(key0 + r);
      const T* from = src + r * HD + (c ^ sw) * EL;
      if constexpr (ASM) copy_lds16(from, lds_address(dst + i * RPI * HD));
      else load_lds16((const bf16*)from, (bf16x8*)(dst + i * RPI * HD));
    }
  }
};

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

// Transposing LDS reads of 4 or 8 places, as assembly with their wait: before the builtin
// the compiler waits for every copy to LDS in flight, the next unit's too.
AXON_DEV void read_tr(const uint32_t (&at)[4], bf16x4 (&r)[4]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %5\n\tds_read_b64_tr_b16 %2, %6\n\t"
      "ds_read_b64_tr_b16 %3, %7\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3])
      : "memory");
}
AXON_DEV void read_tr(const uint32_t (&at)[8], bf16x4 (&r)[8]) {
  asm volatile(
      "ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %9\n\tds_read_b64_tr_b16 %2, %10\n\t"
      "ds_read_b64_tr_b16 %3, %11\n\tds_read_b64_tr_b16 %4, %12\n\tds_read_b64_tr_b16 %5, %13\n\t"
      "ds_read_b64_tr_b16 %6, %14\n\tds_read_b64_tr_b16 %7, %15\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
      : "v"(at[0]), "v"(at[1]), "v"(at[2]), "v"(at[3]), "v"(at[4]), "v"(at[5]), "v"(at[6]), "v"(at[7])
      : "memory");
}

AXON_DEV bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
AXON_DEV bool finite(bf16 v) { return finite((float)v); }

// A masked key has p = 0, but 0 times what stands there is NaN when that is infinite or
// NaN.  So the values of a unit with masked keys are made finite where they are staged
// (n rows of a wavefront); returns which rows had others.  Where a row of the tile sees
// those keys, they are added by add_odd.
template <typename T, int HD>
AXON_DEV int make_finite(T* v, int n, int lane) {
  using L = Lds<T, HD>;
  typedef typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type Chunk;
  int keys = 0;
#pragma unroll
  for (int i = 0; i < n / L::RPI; ++i) {
    Chunk* p = (Chunk*)v + i * 64 + lane;
    Chunk c = *p;
    bool ok = true;
#pragma unroll
    for (int j = 0; j < L::EL; ++j) ok = ok && finite(c[j]);
    const uint64_t odd = __ballot(!ok);
    if (!odd) continue;
    if (!ok) {
#pragma unroll
      for (int j = 0; j < L::EL; ++j) c[j] = finite(c[j]) ? c[j] : (T)0.f;
      *p = c;
    }
#pragma unroll
    for (int r = 0; r < L::RPI; ++r)
      if (odd >> (r * L::CH) & ((1ull << (L::CH - 1) << 1) - 1)) keys |= 1 << (i * L::RPI + r);
  }
  return keys;
}

template <typename T, int HD>
struct Cache {
  const PrefixAttnArgs<T>& a;
  const Segment& g;
  int kvh;
  // page of a key, -1: none
  AXON_DEV int page(int key) const {
    const int p = key < g.room ? g.table[key / a.kv.ps] : -1;
    return p >= 0 && p < a.kv.num_pages ? p : -1;
  }
  // the 16-key block of a key, as a number of such blocks from the cache's start
  AXON_DEV int block(int key) const {
    const int p = page(key);
    return p < 0 ? -1 : (p * a.kv.kv_heads + kvh) * (a.kv.ps / 16) + key % a.kv.ps / 16;
  }
  AXON_DEV int64_t at(int page, int key) const {
    return (((int64_t)page * a.kv.kv_heads + kvh) * a.kv.ps + key % a.kv.ps) * HD;
  }
};

// Adds the infinite and NaN values of keys key0 + (bits of odd) where the lane's row sees
// them: o[i], i < N, is dimension dim(i).
template <typename T, int HD, int N, typename D>
AXON_DEV void add_odd(const Cache<T, HD>& c, int key0, int odd, int limit, float (&o)[N], D&& dim) {
  for (; odd; odd &= odd - 1) {
    const int key = key0 + __ffs(odd) - 1;
    if (key >= limit) continue;
    const int page = c.page(key);
    if (page < 0) continue;
    const T* v = (const T*)c.a.kv.v + c.at(page, key);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float e = to_f32(v[dim(i)]);
      if (!finite(e)) o[i] += e;
    }
  }
}

// Row r of a segment as it lies in q
template <typename T, int HD>
AXON_DEV const T* q_row(const PrefixAttnArgs<T>& a, const Segment& g, int G, int kvh, int r) {
  return a.q + (int64_t)(g.tok0 + r / G) * a.ldq + (int64_t)(kvh * G + r % G) * HD;
}

// The reference m of a row's weights 2^(score - m): the running maximum (in base 2, times
// the scale), or up to 8 less, so that the sum and the products are hardly rescaled after
// the first keys (a weight is 256 at most).
template <int N, typename V>
AXON_DEV void raise(float& m, float top, float& l, V (&o)[N]) {
  if (!__any(top > m + 8.f)) return;
  const float m_new = fmaxf(m, top);
  const float fall = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - m_new);
  m = m_new;
  l *= fall;
#pragma unroll
  for (int d = 0; d < N; ++d) o[d] *= fall;
}

// ---------------------------------------------------------------- wide tiles

template <typename T, int HD>
struct Wide {
  using L = Lds<T, HD>;
  // bf16: 4 stages of 64 keys; float32 (keys and values twice as wide): 2 or 4
  static constexpr int TILE = WIDE_KEYS * HD, STAGES = sizeof(T) == 4 && HD == 128 ? 2 : 4;
  static constexpr int MY_KEYS = WIDE_KEYS / WIDE_WAVES;  // staged by a wavefront
  static constexpr int LOADS = 2 * (MY_KEYS / L::RPI);    // its copies
  static constexpr int BATCH = WIDE_THREADS / 4;          // units whose pages are looked up at a time
  struct Shared {
    alignas(16) T tiles[STAGES][2][TILE];
    int32_t blocks[WIDE_THREADS];     // where a batch's 16-key blocks are in the cache, 4 a unit, -1: none
    int32_t odd[STAGES][WIDE_WAVES];  // make_finite's rows
    PlanShared<WIDE_WAVES> plan;
  };
};

// A wavefront's 32 rows of a wide tile over blocks of 32 keys in LDS
template <typename T, int HD>
struct WideRows {
  using W = Wide<T, HD>;
  using L = Lds<T, HD>;
  using V8 = typename Vec8<T>::t;
  static constexpr int DT = HD / 32, QS = HD / 16;
  const PrefixAttnArgs<T>& a;
  const Segment& g;
  const Cache<T, HD> cache;
  float sc;
  int G, row0, lane, wave, hl, c, rows, kgroup, r0, limit, least, most, tile_least;
  bool halves, works;
  V8 q[QS];
  f32x16 o[DT] = {};
  float m = -INFINITY, l = 0.f;

  AXON_DEV WideRows(const PrefixAttnArgs<T>& args, float scale, const Segment& seg, int group, int kvh, int first_row)
      : a(args), g(seg), cache{args, seg, kvh}, sc(scale), G(group), row0(first_row) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    hl = lane >> 5;
    c = lane & 31;
    rows = g.tokens * G;
    // up to 128 rows: two groups of 4 wavefronts, each half of a unit's keys
    halves = min(rows - row0, WIDE_ROWS) <= WIDE_ROWS / 2;
    kgroup = halves ? wave >> 2 : 0;
    r0 = row0 + 32 * (halves ? wave & 3 : wave);
    works = r0 < rows;
    const int r = min(r0 + c, rows - 1);
    const T* p = q_row<T, HD>(a, g, G, kvh, r) + 8 * hl;
#pragma unroll
    for (int k = 0; k < QS; ++k) q[k] = load_q8<T>(p + 16 * k, a.scale < 0.f);
    limit = row_keys(g, G, r);
    least = row_keys(g, G, min(r0, rows - 1));
    most = row_keys(g, G, min(r0 + 31, rows - 1));
    tile_least = row_keys(g, G, row0);
  }

  // s = the scores of block kb: s[i] of key 32 kb + 8 (i / 4) + 4 hl + i % 4 and row c
  AXON_DEV void read_k(const T* ks, int kb, V8 (&kf)[QS]) const {
#pragma unroll
    for (int k = 0; k < QS; ++k) {
      const int d = 16 * k + 8 * hl;
      kf[k] = read8(ks + L::k_at(32 * kb + c, d), ks + L::k_at(32 * kb + c, d + 4));
    }
  }
  AXON_DEV void scores(const V8 (&kf)[QS], f32x16& s) const {
    s = f32x16{};
#pragma unroll
    for (int k = 0; k < QS; ++k) s = mul_wide(kf[k], q[k], s);
  }
  // s = the weights of block kb of the unit at key0
  AXON_DEV void weights(f32x16& s, int key0, int kb, int pages, const int32_t* odd) {
    if (key0 + WIDE_KEYS > least || pages != 15) {
      const int seen = limit - key0 - 32 * kb - 4 * hl;
      const int seen0 = pages >> (2 * kb) & 1 ? seen : 0, seen1 = pages >> (2 * kb + 1) & 1 ? seen : 0;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = 8 * (i >> 2) + (i & 3) < (i < 8 ? seen0 : seen1) ? s[i] : -INFINITY;
    }
    float top = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
    raise(m, fmaxf(top, lane_xor32(top)) * sc, l, o);
    const float base = m == -INFINITY ? 0.f : m;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], sc, -base));
      sum += s[i];
    }
    l += sum;
    if (odd)
      for (int w = 32 / W::MY_KEYS * kb; w < 32 / W::MY_KEYS * (kb + 1); ++w)
        if (const int keys = __builtin_amdgcn_readfirstlane(odd[w])) {
          float e[16 * DT];
#pragma unroll
          for (int i = 0; i < 16 * DT; ++i) e[i] = o[i / 16][i % 16];
          add_odd(cache, key0 + W::MY_KEYS * w, keys, limit, e,
                  [&](int i) { return 32 * (i / 16) + 8 * (i % 16 / 4) + 4 * hl + i % 4; });
#pragma unroll
          for (int i = 0; i < 16 * DT; ++i) o[i / 16][i % 16] = e[i];
        }
  }
  AXON_DEV void store(float* part) {
    if (r0 + c >= rows) return;
    l += lane_xor32(l);
    const int block = (halves ? 8 * kgroup + 2 * (wave & 3) : 2 * wave) + (c >> 4), row = c & 15;
    part += (int64_t)block * part_floats(HD);
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
};

// Staging of a batch of units: pages looked up, each wavefront copies 8 keys of a unit.
template <typename T, int HD>
struct WideStages {
  using W = Wide<T, HD>;
  using L = Lds<T, HD>;
  typename W::Shared& sh;
  const WideRows<T, HD>& x;
  int u0 = 0, n = 0, next = 0;  // the batch
  bool all_there = true;

  AXON_DEV void look_up(int first, int count) {
    u0 = first;
    n = count;
    __syncthreads();  // the stages and pages of what came before are read
    const int key = (4 * u0 + (int)threadIdx.x) * 16;
    const bool mine = (int)threadIdx.x < 4 * n;
    const int b = mine ? x.cache.block(key) : 0;
    if (mine) sh.blocks[threadIdx.x] = b;
    all_there = __syncthreads_and(b >= 0);
    fetch(0);
  }
  // (the block of the next copy is read a unit ahead)
  AXON_DEV void fetch(int i) { next = sh.blocks[4 * min(i, n - 1) + W::MY_KEYS * x.wave / 16]; }
  AXON_DEV void copy(int i) {
    const int in_unit = W::MY_KEYS * x.wave;
    const int b = max(__builtin_amdgcn_readfirstlane(next), 0);  // (none: masked, but read)
    fetch(i + 1);
    const int64_t src = ((int64_t)b * 16 + in_unit % 16) * HD;
    T* dst = sh.tiles[i % W::STAGES][0] + in_unit * HD;
    L::template stage<true, true>((const T*)x.a.kv.k + src, dst, in_unit, W::MY_KEYS, x.lane);
    L::template stage<false, true>((const T*)x.a.kv.v + src, dst + W::TILE, in_unit, W::MY_KEYS, x.lane);
  }
  // which of a unit's 16-key blocks have a page
  AXON_DEV int pages(int i) const {
    if (all_there) return 15;
    int p = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) p |= (sh.blocks[4 * i + j] >= 0) << j;
    return __builtin_amdgcn_readfirstlane(p);
  }
  // whether some key of the unit is masked for some row of the tile
  AXON_DEV bool masked(int i) const { return (u0 + i + 1) * WIDE_KEYS > x.tile_least || pages(i) != 15; }
  // this wavefront's keys of unit i are in LDS when at most ``later`` units' copies are in
  // flight; they are made finite where some key is masked
  template <int MOST>
  AXON_DEV void arrive(int i, int later) {
    wait_loads<W::LOADS, MOST>(later);
    if (masked(i)) {
      const int at = i % W::STAGES;
      const int odd = make_finite<T, HD>(sh.tiles[at][1] + W::MY_KEYS * x.wave * HD, W::MY_KEYS, x.lane);
      if (x.lane == 0) sh.odd[at][x.wave] = odd;
    }
  }
  // ends a phase: what was read of LDS is here, what was written there is to be seen
  AXON_DEV void barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    phase_barrier();
  }
};

// Units first .. last - 1 of the tile of row0.  A wavefront alternates between phases of
// matrix instructions (a unit's scores, the product with the values of the unit before)
// and of everything else (the weights); wavefronts 4 .. 7 are a phase behind 0 .. 3, with
// which they share the SIMDs, so that one's matrix instructions run beside the other's
// exponentials.  HALVES: a wavefront takes 32 of a unit's keys, else all 64.
template <bool HALVES, int HD>
AXON_DEV void wide_phases(WideRows<bf16, HD>& x, WideStages<bf16, HD>& st, int first, int last) {
  using W = Wide<bf16, HD>;
  using L = Lds<bf16, HD>;
  using X = WideRows<bf16, HD>;
  constexpr int DT = X::DT, S = W::STAGES, NB = HALVES ? 1 : 2;
  static_assert(S == 4, "what the phases of copies and waits count on");
  const int late = x.wave >> 2, kb0 = HALVES ? x.kgroup : 0;
  for (int u0 = first; u0 < last; u0 += W::BATCH) {
    st.look_up(u0, min(last - u0, W::BATCH));
    const int n = st.n;
    // Phase p of all wavefronts: unit u is multiplied from phase 2 u (scores) to 2 u + 3
    // (the late ones' product), so unit u + 4 is copied over it in phase 2 u + 4, and
    // waited for before phase 2 u + 8.
    int p = 0;
    auto begin = [&] {
      if (!(p & 1) && (p >> 1) + 2 < n) st.copy((p >> 1) + 2);
    };
    auto end = [&] {
      ++p;
      const int u = p >> 1;
      if (!(p & 1) && u < n) st.template arrive<1>(u, min(n - 1 - u, 1));
      st.barrier();
    };
    st.copy(0);
    if (n > 1) st.copy(1);
    st.template arrive<1>(0, min(n - 1, 1));
    st.barrier();
    if (late) {
      begin();
      end();
    }
    bf16x8 w[NB][2];  // the weights of the unit before, and its values' place
    const bf16* wv = nullptr;
    // The operands of DT matrix instructions are read from LDS before the DT before them
    // are issued (one at a time, each instruction would wait for its own): f[0], f[1] in
    // turn.  First K, 16 dimensions an operand; then V, keys 16 e .., two times 4 a lane.
    bf16x8 f[2][DT];
    f32x16 s[NB];
    auto read_k = [&](const bf16* tile, int b, int half) {
#pragma unroll
      for (int k = 0; k < DT; ++k)
        f[half][k] = *(const bf16x8*)(tile + L::k_at(32 * (kb0 + b) + x.c, 16 * (half * DT + k) + 8 * x.hl));
      __builtin_amdgcn_sched_barrier(0);
    };
    auto scores = [&](int b, int half) {
      if (half == 0) s[b] = f32x16{};
#pragma unroll
      for (int k = 0; k < DT; ++k) s[b] = mul_wide(f[half][k], x.q[half * DT + k], s[b]);
      __builtin_amdgcn_sched_barrier(0);
    };
    auto read_v = [&](int b, int e) {
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        const int key = 32 * b + 16 * e + 4 * x.hl + ((x.lane & 15) >> 2);
        const int dim = 32 * d + 16 * ((x.lane >> 4) & 1) + 4 * (x.lane & 3);
        f[e][d] = read_tr8(wv + L::v_at(key, dim), wv + L::v_at(key + 8, dim));
      }
      __builtin_amdgcn_sched_barrier(0);
    };
    auto product = [&](int b, int e) {
#pragma unroll
      for (int d = 0; d < DT; ++d) x.o[d] = mul_wide(f[e][d], w[b][e], x.o[d]);
      __builtin_amdgcn_sched_barrier(0);
    };
    // (f[1] is free when the first values are read into f[0])
    auto products = [&] {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        read_v(b, 1);
        product(b, 0);
        if (b + 1 < NB) read_v(b + 1, 0);
        product(b, 1);
      }
    };
    static_assert(X::QS == 2 * DT, "as many operands of K as of V");
    for (int i = 0; i < n; ++i) {
      const bf16* tile = st.sh.tiles[i % S][0];
      begin();
      if (x.works) {
        read_k(tile, 0, 0);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          read_k(tile, b, 1);
          scores(b, 0);
          if (b + 1 < NB) read_k(tile, b + 1, 0);
          else if (wv) read_v(0, 0);
          scores(b, 1);
        }
        if (wv) products();
      }
      end();
      begin();
      if (x.works) {
        const int pages = st.pages(i);
        const int32_t* odd = st.masked(i) ? st.sh.odd[i % S] : nullptr;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          x.weights(s[b], (u0 + i) * WIDE_KEYS, kb0 + b, pages, odd);
#pragma unroll
          for (int j = 0; j < 16; ++j) w[b][j / 8][j % 8] = (bf16)s[b][j];
        }
        wv = tile + W::TILE + 32 * kb0 * HD;
      }
      end();
    }
    begin();
    if (x.works) {
      read_v(0, 0);
      products();
    }
    end();
    if (!late) {
      begin();
      end();
    }
  }
}

template <int HD>
AXON_DEV void wide_tile(const PrefixAttnArgs<bf16>& a, float sc, typename Wide<bf16, HD>::Shared& sh, const Segment& g,
                        int G, int kvh, int row0, int first, int last, float* part) {
  WideRows<bf16, HD> x(a, sc, g, G, kvh, row0);
  WideStages<bf16, HD> st{sh, x};
  if (x.halves) wide_phases<true>(x, st, first, last);
  else wide_phases<false>(x, st, first, last);
  x.store(part);
}

// In float32 the matrix instructions take 16 times as long: all wavefronts in step.
template <int HD>
AXON_DEV void wide_tile(const PrefixAttnArgs<float>& a, float sc, typename Wide<float, HD>::Shared& sh, const Segment& g,
                        int G, int kvh, int row0, int first, int last, float* part) {
  using W = Wide<float, HD>;
  using L = Lds<float, HD>;
  using X = WideRows<float, HD>;
  constexpr int S = W::STAGES;
  X x(a, sc, g, G, kvh, row0);
  WideStages<float, HD> st{sh, x};
  for (int u0 = first; u0 < last; u0 += W::BATCH) {
    st.look_up(u0, min(last - u0, W::BATCH));
    const int n = st.n;
    for (int i = 0; i < S - 1 && i < n; ++i) st.copy(i);
    for (int i = 0; i < n; ++i) {
      st.template arrive<S - 2>(i, min(n - 1 - i, S - 2));
      st.barrier();
      if (i + S - 1 < n) st.copy(i + S - 1);
      const int key0 = (u0 + i) * WIDE_KEYS;
      if (!x.works || key0 >= x.most) continue;
      const float* tile = sh.tiles[i % S][0];
#pragma unroll 1
      for (int kb = x.kgroup; kb < (x.halves ? x.kgroup + 1 : 2); ++kb) {
        f32x8 kf[X::QS];
        x.read_k(tile, kb, kf);
        f32x16 s;
        x.scores(kf, s);
        x.weights(s, key0, kb, st.pages(i), st.masked(i) ? sh.odd[i % S] : nullptr);
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
          for (int d = 0; d < X::DT; ++d)
            x.o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                tile[W::TILE + L::v_at(32 * kb + 8 * (j >> 2) + 4 * x.hl + (j & 3), 32 * d + x.c)], s[j], x.o[d], 0, 0, 0);
      }
    }
  }
  x.store(part);
}

// Worker w of n takes steps total w / n .. total (w + 1) / n - 1: as many as there are,
// unless that leaves one too little to be worth the part it writes.
AXON_DEV int workers(int most, int64_t total, int least) {
  return (int)max(min((int64_t)most, total / least), min(total, (int64_t)1));
}
AXON_DEV int worker_of(int64_t step, int64_t total, int n) { return (int)(((step + 1) * n - 1) / total); }

// What worker ``me`` does of the tile at p (its steps at .. at + take - 1): units first ..
// last - 1; the one with the tile's first unit notes where the parts are.
struct Work {
  int take, first, last;
};
template <bool WIDE, int HD, typename T>
AXON_DEV Work work_of(const PrefixAttnArgs<T>& a, const Segment& g, const Place& p, int G, int KV, int64_t at, int64_t end,
                      int64_t total, int me, int n, TileParts* info, bool leader) {
  constexpr int START = Tiles<WIDE>::START;
  const int steps = Tiles<WIDE>::steps(g, G, p.rt);
  Work w;
  w.take = (int)min((int64_t)(steps - p.step), end - at);
  w.first = max(p.step - START, 0);
  w.last = max(p.step + w.take - START, 0);
  if (leader && p.step <= START && w.last > 0)
    info[info_at(g.own, p.kvh, KV, (int64_t)a.tokens * G, g.tok0, G, p.rt * Tiles<WIDE>::ROWS)] =
        TileParts{p.tile + me, worker_of(at - p.step + steps - 1, total, n) - me + 1};
  return w;
}

template <typename T, int HD>
__global__ void __launch_bounds__(WIDE_THREADS, 2) prefix_wide_kernel(PrefixAttnArgs<T> a, float sc, TileParts* info,
                                                                      float* parts, int slots) {
  __shared__ typename Wide<T, HD>::Shared sh;
  Plan<T, true, WIDE_THREADS> plan(a, sh.plan);
  const int G = plan.G, KV = plan.KV;
  // Consecutive runs on one XCD, whose L2 holds what they share; fewer workers than
  // workgroups: over all XCDs.
  const int n = workers(gridDim.x, plan.total, WIDE_LEAST);
  const int me = n < (int)gridDim.x || n % 8 ? blockIdx.x : blockIdx.x % 8 * (n / 8) + blockIdx.x / 8;
  if (me >= n) return;
  int64_t at = plan.total * me / n;
  const int64_t end = plan.total * (me + 1) / n;
  plan.find(0, at);
  __syncthreads();
  Segment g;
  Place p = plan.get(0, g);
  for (;;) {
    const int slot = p.tile + me;
    if (slot >= slots) return;  // (cu_seqlens are not those of the host)
    const Work w = work_of<true, HD>(a, g, p, G, KV, at, end, plan.total, me, n, info, threadIdx.x == 0);
    if (w.last > w.first)
      wide_tile<HD>(a, sc, sh, g, G, p.kvh, p.rt * WIDE_ROWS, w.first, w.last,
                       parts + (int64_t)slot * SLOT_BLOCKS * part_floats(HD));
    at += w.take;
    if (at >= end) return;
    plan.advance(p, g);
  }
}

// ---------------------------------------------------------------- narrow tiles

template <typename T, int HD>
struct Narrow {
  using L = Lds<T, HD>;
  static constexpr int TILE = NARROW_KEYS * HD, QS = HD / 32;
  static constexpr int LOADS = NARROW_KEYS / L::RPI + QS * (int)sizeof(T) / 2;  // of a unit
  struct Shared {
    alignas(16) T v[NARROW_WAVES][2][TILE];
    PlanShared<NARROW_WAVES> plan;
  };
};

// Units first .. last - 1 of a tile, by one wavefront: keys to registers, where a lane
// has those of one key that multiply its dimensions, values through LDS, a unit ahead.
template <typename T, int HD>
AXON_DEV void narrow_tile(const PrefixAttnArgs<T>& a, float sc, T (&lds)[2][Narrow<T, HD>::TILE], const Segment& g, int G,
                          int kvh, int first, int last, float* part) {
  using N = Narrow<T, HD>;
  using L = Lds<T, HD>;
  using V8 = typename Vec8<T>::t;
  constexpr int DT = HD / 16, QS = N::QS;
  const int lane = threadIdx.x & 63, gq = lane >> 4, c = lane & 15;
  const int rows = g.tokens * G, r = min(c, rows - 1);
  const Cache<T, HD> cache{a, g, kvh};
  int pages = 0;  // of units u & ~63 .., one a lane
  V8 q[QS], k[2][QS];
  auto look_up = [&](int u0) { pages = u0 + lane < last ? cache.page((u0 + lane) * NARROW_KEYS) : -1; };
  auto page_of = [&](int u) { return __builtin_amdgcn_readlane(pages, (u - first) & 63); };
  auto fetch = [&](int u, int b) {
    const int64_t src = cache.at(max(page_of(u), 0), u * NARROW_KEYS);  // (none: masked, but read)
    L::template stage<false, false>((const T*)a.kv.v + src, lds[b], 0, NARROW_KEYS, lane);
    const T* kp = (const T*)a.kv.k + src + c * HD + 8 * gq;
#pragma unroll
    for (int j = 0; j < QS; ++j) k[b][j] = read8(kp + 32 * j, kp + 32 * j + 4);
  };
  look_up(first);
  {
    const T* p = q_row<T, HD>(a, g, G, kvh, r) + 8 * gq;
#pragma unroll
    for (int j = 0; j < QS; ++j) q[j] = load_q8<T>(p + 32 * j, a.scale < 0.f);
  }
  const int limit = row_keys(g, G, r), least = row_keys(g, G, 0);
  f32x4 o[DT] = {};
  float m = -INFINITY, l = 0.f;
  fetch(first, 0);
  auto unit = [&](int u, const int b) {
    const int key0 = u * NARROW_KEYS;
    const bool there = page_of(u) >= 0, masked = key0 + NARROW_KEYS > least || !there;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the stage that is filled next is read)
    if (u + 1 < last) {
      if (((u + 1 - first) & 63) == 0) look_up(u + 1);
      fetch(u + 1, b ^ 1);
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N::LOADS) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
    T* vs = lds[b];
    const int odd = masked ? make_finite<T, HD>(vs, NARROW_KEYS, lane) : 0;
    f32x4 s = {};
#pragma unroll
    for (int j = 0; j < QS; ++j) s = mul_narrow(k[b][j], q[j], s);
    typename std::conditional<sizeof(T) == 2, bf16x4, f32x4>::type p, v[DT];
    if constexpr (sizeof(T) == 2) {
      uint32_t at[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d) at[d] = lds_address(vs + L::v_at(4 * gq + (c >> 2), 16 * d + 4 * (c & 3)));
      __builtin_amdgcn_sched_barrier(0);
      read_tr(at, v);
    } else {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[d][i] = vs[L::v_at(4 * gq + i, 16 * d + c)];
    }
    // s[i]: key key0 + 4 gq + i, row c
    if (masked) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (key0 + 4 * gq + i >= limit || !there) s[i] = -INFINITY;
    }
    float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    top = fmaxf(top, lane_xor16(top));
    raise(m, fmaxf(top, lane_xor32(top)) * sc, l, o);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float e = __builtin_amdgcn_exp2f(fmaf(s[i], sc, -base));
      l += e;
      p[i] = from_f32<T>(e);
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] = mul_narrow4(v[d], p, o[d]);
    if (odd) {
      float e[4 * DT];
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i) e[i] = o[i / 4][i % 4];
      add_odd(cache, key0, there ? odd : 0, limit, e, [&](int i) { return 16 * (i / 4) + 4 * gq + i % 4; });
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i) o[i / 4][i % 4] = e[i];
    }
  };
  for (int u = first; u < last; u += 2) {
    unit(u, 0);
    if (u + 1 < last) unit(u + 1, 1);
  }
  l += lane_xor16(l);
  l += lane_xor32(l);
  if (c >= rows) return;
#pragma unroll
  for (int d = 0; d < DT; ++d) *(f32x4*)(part + c * HD + 16 * d + 4 * gq) = o[d];
  if (gq == 0) {
    part[16 * HD + c] = m;
    part[16 * HD + 16 + c] = l;
  }
}

template <typename T, int HD>
__global__ void __launch_bounds__(NARROW_THREADS, 3) prefix_narrow_kernel(PrefixAttnArgs<T> a, float sc, TileParts* info,
                                                                          float* parts, int slots) {
  __shared__ typename Narrow<T, HD>::Shared sh;
  Plan<T, false, NARROW_THREADS> plan(a, sh.plan);
  const int G = plan.G, KV = plan.KV, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // a wavefront is a worker; as the wide kernel's otherwise
  const int grid = gridDim.x * NARROW_WAVES, n = workers(grid, plan.total, NARROW_LEAST);
  const int wg = n < grid || gridDim.x % 8 ? blockIdx.x : blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8;
  // (fewer workers than wavefronts: spread over the workgroups)
  auto worker = [&](int w) { return n < grid ? w * (int)gridDim.x + wg : wg * NARROW_WAVES + w; };
  for (int w = 0; w < NARROW_WAVES; ++w)
    if (worker(w) < n) plan.find(w, plan.total * worker(w) / n);
  __syncthreads();
  const int me = worker(wave);
  if (me >= n) return;
  int64_t at = plan.total * me / n;
  const int64_t end = plan.total * (me + 1) / n;
  Segment g;
  Place p = plan.get(wave, g);
  for (;;) {
    const int slot = p.tile + me;
    if (slot >= slots) return;
    const Work w = work_of<false, HD>(a, g, p, G, KV, at, end, plan.total, me, n, info, (threadIdx.x & 63) == 0);
    if (w.last > w.first)
      narrow_tile<T, HD>(a, sc, sh.v[wave], g, G, p.kvh, w.first, w.last, parts + (int64_t)slot * part_floats(HD));
    at += w.take;
    if (at >= end) return;
    plan.advance(p, g);
  }
}

// ---------------------------------------------------------------- the join

// A row's parts of both segments: out = sum f o / sum f l, f = 2^(m - max).  A workgroup
// per (token, kv head): HD / 4 lanes for a part of a row, the parts shared out over as
// many groups of them as it has for the R rows at a time, whose sums are joined in LDS.
constexpr int JOIN_MAX = 1024;
template <typename T, int HD>
__global__ void __launch_bounds__(JOIN_MAX) prefix_join_kernel(PrefixAttnArgs<T> a, const TileParts* info, const float* wide,
                                                               const float* narrow, int wide_slots, int narrow_slots,
                                                               int R) {
  constexpr int LANES = HD / 4, AHEAD = 4;
  __shared__ f32x4 sum_o[JOIN_MAX];
  __shared__ float sum_m[JOIN_MAX / LANES], sum_l[JOIN_MAX / LANES];
  const int t = blockIdx.x, kvh = blockIdx.y, KV = a.kv.kv_heads, G = a.heads / KV;
  const int lane = threadIdx.x & 63, d = threadIdx.x % LANES, team = threadIdx.x / LANES;
  const int groups = (int)blockDim.x / (LANES * R), group = team / R;  // of parts
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
  for (int j0 = 0; j0 < G; j0 += R) {
    const int j = j0 + team % R;
    f32x4 o = {};
    float top = -INFINITY, l = 0.f;
    for (int k = 0; k < 2; ++k) {
      if (!has[k] || !active || j >= G) continue;
      const Segment g = segment_of(a, k ? a.shared.groups + b : grp);
      const int r = (t - g.tok0) * G + j, rows = g.tokens * G;
      const bool is_wide = rows > NARROW_ROWS;
      const int row0 = is_wide ? r / WIDE_ROWS * WIDE_ROWS : 0, row = r - row0;
      if (tile_keys(g, G, row0, is_wide ? WIDE_ROWS : NARROW_ROWS) <= 0) continue;
      const TileParts p = info[info_at(k, kvh, KV, (int64_t)a.tokens * G, g.tok0, G, row0)];
      if (p.first < 0 || p.count < 0 || p.count > (is_wide ? wide_slots : narrow_slots) - p.first) continue;
      // a tile of up to 128 rows has two parts in a slot
      const bool halves = is_wide && rows - row0 <= WIDE_ROWS / 2;
      const int64_t step = (int64_t)(is_wide ? (halves ? SLOT_BLOCKS / 2 : SLOT_BLOCKS) : 1) * part_floats(HD);
      const int count = halves ? 2 * p.count : p.count;
      const float* part = (is_wide ? wide : narrow) + ((int64_t)p.first * (is_wide ? SLOT_BLOCKS : 1) + row / 16) * part_floats(HD);
      const float *po = part + row % 16 * HD + 4 * d, *pm = part + 16 * HD + row % 16;
      for (int i0 = group; i0 < count; i0 += AHEAD * groups) {
        f32x4 v[AHEAD];
        float m[AHEAD], s[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {  // (loads without a condition stay in flight together)
          const int64_t at = min(i0 + i * groups, count - 1) * step;
          m[i] = pm[at];
          s[i] = pm[at + 16];
          v[i] = *(const f32x4*)(po + at);
        }
        float next = top;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) next = fmaxf(next, m[i]);
        const float fall = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - next);
        top = next;
        l = fall > 0.f ? l * fall : l != l ? l : 0.f;
        o = fall > 0.f ? o * fall : f32x4{};
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
          if (i0 + i * groups >= count) continue;
          const float f = m[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[i] - top);
          l += f > 0.f || s[i] != s[i] ? f * s[i] : 0.f;  // (scores that are all NaN: no maximum)
          o += f > 0.f ? f * v[i] : f32x4{};
        }
      }
    }
    if (groups > 1) {
      sum_o[threadIdx.x] = o;
      if (d == 0) {
        sum_m[team] = top;
        sum_l[team] = l;
      }
      __syncthreads();
      if (group == 0) {
        for (int i = 1; i < groups; ++i) top = fmaxf(top, sum_m[team + i * R]);
        o = f32x4{};
        l = 0.f;
        for (int i = 0; i < groups; ++i) {
          const float m = sum_m[team + i * R], s = sum_l[team + i * R];
          const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
          l += f > 0.f || s != s ? f * s : 0.f;
          o += f > 0.f ? f * sum_o[threadIdx.x + i * R * LANES] : f32x4{};
        }
      }
      __syncthreads();
    }
    if (group > 0 || j >= G) continue;
    T* out = a.out + (int64_t)t * a.ldo + (int64_t)(kvh * G + j) * HD + 4 * d;
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = from_f32<T>(l == 0.f ? 0.f : o[i] * inv);
    if (a.lse && d == 0)
      a.lse[(int64_t)t * a.heads + kvh * G + j] = l == 0.f ? -INFINITY : (top + __log2f(l)) / LOG2E_F;
  }
}

// ---------------------------------------------------------------- host

namespace {

constexpr int WIDE_WGS = 256, NARROW_WGS = 768;

struct Sizes {
  int64_t wide, narrow;       // slots of each kind (0: no such tile)
  int64_t wide_at, narrow_at, bytes;
};
Sizes sizes_of(const PrefixAttnShape& x) {
  const int64_t G = x.heads / x.kv_heads;
  auto token = [&](int b) -> int64_t { return x.h_cu ? x.h_cu[b] : b; };
  int64_t wide = 0, narrow = 0;
  auto add = [&](int64_t tokens) {
    const int64_t rows = tokens * G;
    if (rows > NARROW_ROWS) wide += (rows + WIDE_ROWS - 1) / WIDE_ROWS;
    else if (rows > 0) ++narrow;
  };
  for (int g = 0; g < x.groups; ++g) add(token(x.h_groups[g + 1]) - token(x.h_groups[g]));
  for (int b = 0; b < x.seqs; ++b) add(x.h_cu ? x.h_cu[b + 1] - x.h_cu[b] : 1);
  Sizes s;
  s.wide = wide ? wide * x.kv_heads + WIDE_WGS : 0;
  s.narrow = narrow ? narrow * x.kv_heads + NARROW_WGS * NARROW_WAVES : 0;
  s.wide_at = (2 * x.tokens * x.heads * (int64_t)sizeof(TileParts) + 15) / 16 * 16;
  s.narrow_at = s.wide_at + s.wide * SLOT_BLOCKS * part_floats(x.hd) * 4;
  s.bytes = s.narrow_at + s.narrow * part_floats(x.hd) * 4;
  return s;
}

}  // namespace

int64_t prefix_attn_workspace(const PrefixAttnShape& x) { return sizes_of(x).bytes; }

int64_t prefix_attn_units(const PrefixAttnShape& x, int64_t keys) {
  const Sizes s = sizes_of(x);
  return std::max(s.wide * ((keys + WIDE_KEYS - 1) / WIDE_KEYS), s.narrow * ((keys + NARROW_KEYS - 1) / NARROW_KEYS));
}

template <typename T, int HD>
static void launch(const PrefixAttnArgs<T>& a, const PrefixAttnShape& x, void* workspace, hipStream_t s) {
  const Sizes n = sizes_of(x);
  TileParts* info = (TileParts*)workspace;
  float *wide = (float*)((char*)workspace + n.wide_at), *narrow = (float*)((char*)workspace + n.narrow_at);
  // a scale of 0 leaves every score, masked ones apart, the same
  const float sc = a.scale == 0.f ? 1e-37f : fabsf(a.scale) * LOG2E_F;
  if (n.wide) prefix_wide_kernel<T, HD><<<WIDE_WGS, WIDE_THREADS, 0, s>>>(a, sc, info, wide, (int)n.wide);
  if (n.narrow) prefix_narrow_kernel<T, HD><<<NARROW_WGS, NARROW_THREADS, 0, s>>>(a, sc, info, narrow, (int)n.narrow);
  // few tokens: many threads each, whose parts are many
  const int G = a.heads / a.kv.kv_heads, threads = (int64_t)a.tokens * a.kv.kv_heads <= 1024 ? JOIN_MAX : 256;
  int R = 1;
  while (R < G && R < threads / (HD / 4)) R *= 2;
  prefix_join_kernel<T, HD><<<dim3(a.tokens, a.kv.kv_heads), threads, 0, s>>>(a, info, wide, narrow, (int)n.wide,
                                                                             (int)n.narrow, R);
}

template <typename T>
void launch_prefix_attn(const PrefixAttnArgs<T>& a, const PrefixAttnShape& x, void* workspace, hipStream_t s) {
  if (!a.tokens) return;
  if (a.kv.hd == 64) launch<T, 64>(a, x, workspace, s);
  else launch<T, 128>(a, x, workspace, s);
}
template void launch_prefix_attn<float>(const PrefixAttnArgs<float>&, const PrefixAttnShape&, void*, hipStream_t);
template void launch_prefix_attn<bf16>(const PrefixAttnArgs<bf16>&, const PrefixAttnShape&, void*, hipStream_t);

}  // namespace axon
