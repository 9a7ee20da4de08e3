// Attention of new tokens over a shared prefix and their own keys in a paged cache:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale q k_j - max),
// j over the group's prefix and the sequence's own keys up to the token itself.
//
// A *segment* is a list of keys and the tokens that read it: a group's prefix with the
// tokens of all of its sequences, or a sequence's own keys with its own tokens.  The
// rows of a segment and kv head are its tokens' query heads of that kv head, so a
// prefix is read once for 256 rows of what shares it.  Rows go in tiles: a segment of
// at most 16 rows is one *narrow* tile (a single token's own keys), any other is cut
// into *wide* ones of 256 rows.  A workgroup works on tiles of one kind:
//   wide    its 8 wavefronts take 32 rows each, over keys that all of them read from LDS
//           (with few rows the keys are halved between wavefronts): matrix instructions'
//           work
//   narrow  every wavefront by itself, over 16 keys at a time: memory's work
// and a second kernel joins a row's parts.
//
// Work is cut into units of keys of a tile, in the order (segment, kv head, tile, keys),
// and every worker (a workgroup, or a narrow one's wavefront) takes an equal run of
// consecutive units, whatever the lengths are, which only the device knows.  Of the keys
// of a tile in its run it leaves (max, sum, product).  What is added to what depends on
// the lengths alone: the same bits every time.
//
// Measured (bf16 but for the first; us a call, back to back, with the join): 4 answers to
// 300 keys 16, of which the two launches' chains of dependent loads are 14; 64 of 28 heads
// over 4 to 4096 keys and 600 of their own 36 (83 MB); 256 of 32 over 8 to 16 prompts of
// 1100 66 (195 MB, 3.0 TB/s); 48 of 40 over 8 to 50011 keys 107 (376 MB and 50 GFLOP: 3.5
// TB/s, 470 TFLOP/s); 20 questions of 150 tokens of 28 over 4 behind 2500 keys 201 (110
// GFLOP; a unit of 256 rows and 64 keys 2.2 against 0.9 of matrix instructions alone, and 130
// MB of parts written and read again; under the profiler the two kernels add up to 228).
// In float32 a wide unit's matrix instructions take 16 times as long, and WEIGHT below is
// bf16's: 64 answers of 9 over 3 to 4096 keys 49, of 28 over 4 of 128 dimensions 192.
#include <algorithm>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace axon {

constexpr float LOG2E_F = 1.4426950408889634f;
constexpr int PA_WGS = 256, PA_THREADS = 512, PA_WAVES = 8;
constexpr int WIDE_KEYS = 64, WIDE_ROWS = 256, NARROW_KEYS = 16, NARROW_ROWS = 16;
constexpr int WIDE_START = 6, NARROW_START = 4;  // steps of a tile's beginning
constexpr int SLOT_BLOCKS = WIDE_ROWS / 16;  // 16-row blocks of a wide part

// ---------------------------------------------------------------- plan

struct Segment {
  int tok0, tokens;  // rows: query heads of tokens tok0 ..
  int64_t len;       // keys of every token (prefix), or before token 0 (own)
  int room;          // keys that the table row can list
  const int32_t* table;
  bool own;
};

// segment s, whose tokens and length are known
template <typename T>
AXON_DEV Segment segment_with(const PrefixAttnArgs<T>& a, int s, int tok0, int tokens, int64_t len) {
  const int groups = a.shared.groups;
  Segment g{tok0, tokens, len, 0, nullptr, s >= groups};
  const int stride = g.own ? a.seqs.stride : a.shared.stride;
  g.table = g.own ? a.seqs.table + (int64_t)(s - groups) * stride : a.shared.table + (int64_t)s * stride;
  g.room = stride * a.kv.ps;
  return g;
}
template <typename T>
AXON_DEV Segment segment_of(const PrefixAttnArgs<T>& a, int s) {
  const int groups = a.shared.groups;
  auto among = [](int v, int n) { return min(max(v, 0), n); };
  int tok0, end;
  int64_t len;
  if (s < groups) {
    const int lo = among(a.shared.cu[s], a.seqs.seqs), hi = among(a.shared.cu[s + 1], a.seqs.seqs);
    len = a.shared.lens[s];
    tok0 = a.seqs.cu ? a.seqs.cu[lo] : lo;
    end = a.seqs.cu ? a.seqs.cu[hi] : hi;
  } else {
    const int b = s - groups;
    len = a.seqs.lens[b];
    tok0 = a.seqs.cu ? a.seqs.cu[b] : b;
    end = a.seqs.cu ? a.seqs.cu[b + 1] : b + 1;
  }
  tok0 = among(tok0, a.tokens);
  return segment_with(a, s, tok0, among(end, a.tokens) - tok0, len);
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

// The tiles of one kind, their units, and their steps: one for each unit, and START more
// at its beginning that stand for what a tile costs by itself (looking up pages, loading
// queries, filling the pipeline).  Workers share the steps of a kind, workgroups are shared
// out over the kinds by WEIGHT: a wide unit takes a workgroup as long as 9 (128 dimensions)
// or 14 (64) narrow ones take its 8 wavefronts.  Measured (us, attention of 64 answers to
// 4096 tokens, 256 to 16 prompts of 64 dimensions, 48 to 50011): WEIGHT 4 and START 3 44,
// 115, 135; 8 and 6 36, 77, 114; 12 and 6 35, 68, 123.
template <bool WIDE, int HD>
struct Tiles {
  static constexpr int ROWS = WIDE ? WIDE_ROWS : NARROW_ROWS, KEYS = WIDE ? WIDE_KEYS : NARROW_KEYS;
  static constexpr int WEIGHT = !WIDE ? 1 : HD == 128 ? 9 : 14, START = WIDE ? WIDE_START : NARROW_START;
  static constexpr int LEAST = WIDE ? 4 : 2;  // steps that are worth a worker
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

// Where a row's parts are: in 16-row blocks ``block``, block + step, ... of the parts
struct RowParts {
  int32_t block;
  int32_t count;  // 512 times the number, 16 times the step (1 .. 16), the row in its block
};
AXON_DEV RowParts row_parts(int block, int count, int step, int row) {
  return RowParts{block, count << 9 | step << 4 | row};
}
// [prefix, own][kv head][row among all tokens' rows]
AXON_DEV int64_t info_at(bool own, int kvh, int KV, int64_t rows, int64_t row) {
  return ((own ? KV : 0) + kvh) * rows + row;
}
// a block of 16 rows of a part: [16][hd] products, 16 maxima, 16 sums
constexpr int part_floats(int hd) { return 16 * hd + 32; }

// a worker's steps: equal shares, the first ones a step more
struct Shares {
  int n, each, more;  // workers
  AXON_DEV Shares(int workers, int total) : n(workers), each(total / max(workers, 1)), more(total - workers * each) {}
  AXON_DEV int start(int w) const { return each * w + min(w, more); }
  AXON_DEV int of(int step) const {
    const int longer = (each + 1) * more;
    return step < longer ? step / (each + 1) : more + (step - longer) / max(each, 1);
  }
};

// A place in the order of a kind's steps
struct Place {
  int s, kvh, rt, step, tile;  // tile: number among all tiles of the kind
};
struct PlanShared {
  int sum[4][PA_WAVES];
  int place[PA_WAVES][8];
};

// inclusive sum over the lanes before, by row and half moves of registers
template <int CTRL, int ROWS>
AXON_DEV int add_moved(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true);
}
AXON_DEV int wave_scan(int v) {
  v = add_moved<0x111, 0xf>(v);  // from 1, 2, 4, 8 lanes before in a row of 16
  v = add_moved<0x112, 0xf>(v);
  v = add_moved<0x114, 0xf>(v);
  v = add_moved<0x118, 0xf>(v);
  v = add_moved<0x142, 0xa>(v);  // a row's last lane to the next row
  return add_moved<0x143, 0xc>(v);  // and the first half's to the second
}

// Steps and tiles of all segments, of each kind, and of those before a thread's own
// (s0 .. s1 - 1); every thread of the workgroup calls it.
template <typename T, int HD>
struct Plan {
  const PrefixAttnArgs<T>& a;
  PlanShared& sh;
  int G, KV, segs, s0, s1;
  int total[2], before[4], mine[4];  // narrow and wide: steps (0, 1), tiles (2, 3)
  AXON_DEV Plan(const PrefixAttnArgs<T>& args, PlanShared& shared) : a(args), sh(shared) {
    KV = a.kv.kv_heads;
    G = a.heads / KV;
    segs = a.shared.groups + a.seqs.seqs;
    const int each = (segs + PA_THREADS - 1) / PA_THREADS, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    s0 = min(segs, (int)threadIdx.x * each);
    s1 = min(segs, s0 + each);
#pragma unroll
    for (int j = 0; j < 4; ++j) mine[j] = 0;
    for (int s = s0; s < s1; ++s) {
      const Segment g = segment_of(a, s);
      const int2 n = Tiles<false, HD>::sizes(g, G), w = Tiles<true, HD>::sizes(g, G);
      mine[0] += n.x * KV;
      mine[1] += w.x * KV;
      mine[2] += n.y * KV;
      mine[3] += w.y * KV;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int upto = wave_scan(mine[j]);
      before[j] = upto - mine[j];
      if (lane == 63) sh.sum[j][wave] = upto;
    }
    __syncthreads();
    total[0] = total[1] = 0;
#pragma unroll
    for (int w = 0; w < PA_WAVES; ++w)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int v = sh.sum[j][w];
        before[j] += w < wave ? v : 0;
        if (j < 2) total[j] += v;
      }
  }
  // notes step ``at`` of worker ``w`` of the workgroup, for get(w) after a barrier
  template <bool WIDE>
  AXON_DEV void find(int w, int at) {
    if (at < before[WIDE] || at >= before[WIDE] + mine[WIDE]) return;  // one thread goes on
    int u0 = before[WIDE], t0 = before[2 + WIDE];
    for (int s = s0; s < s1; ++s) {
      const Segment g = segment_of(a, s);
      const int2 n = Tiles<WIDE, HD>::sizes(g, G);
      if (at < u0 + n.x * KV) {
        const int kvh = (at - u0) / n.x;
        int* p = sh.place[w];
        p[0] = s;
        p[1] = kvh;
        p[2] = at - u0 - kvh * n.x;
        p[3] = t0 + kvh * n.y;
        p[4] = g.tok0;
        p[5] = g.tokens;
        p[6] = (int)g.len;  // (a length is 32 bits)
        return;
      }
      u0 += n.x * KV;
      t0 += n.y * KV;
    }
  }
  template <bool WIDE>
  AXON_DEV Place get(int w, Segment& g) const {
    int v[7];
#pragma unroll
    for (int j = 0; j < 7; ++j) v[j] = __builtin_amdgcn_readfirstlane(sh.place[w][j]);
    g = segment_with(a, v[0], v[4], v[5], (int64_t)v[6]);
    Place p{v[0], v[1], 0, v[2], v[3]};
    for (;;) {
      const int n = Tiles<WIDE, HD>::steps(g, G, p.rt);
      if (p.step < n) return p;
      p.step -= n;
      ++p.rt;
      ++p.tile;
    }
  }
  // the next tile that has units (there is one); lane-parallel over segments without any
  template <bool WIDE>
  AXON_DEV void advance(Place& p, Segment& g) const {
    const int lane = threadIdx.x & 63;
    p.step = 0;
    ++p.tile;
    if (++p.rt < Tiles<WIDE, HD>::of(g, G)) return;  // (a tile of a segment has units if any has)
    p.rt = 0;
    if (++p.kvh < KV) return;
    p.kvh = 0;
    ++p.s;
    for (;;) {
      int2 n = {0, 0};
      if (p.s + lane < segs) n = Tiles<WIDE, HD>::sizes(segment_of(a, p.s + lane), G);
      const uint64_t has = __ballot(n.x > 0);
      const int skip = has ? __ffsll((long long)has) - 1 : 64;
      if (skip > 0) p.tile += __builtin_amdgcn_readlane(wave_scan(lane < skip ? n.y : 0), 63) * KV;
      p.s = __builtin_amdgcn_readfirstlane(p.s + skip);
      if (has || p.s >= segs) break;
    }
    g = segment_of(a, min(p.s, segs - 1));
  }
};

// What worker ``me`` does of the tile at p (its steps at .. at + take - 1): units first ..
// last - 1.
struct Work {
  int take, first, last;
  bool leads;  // has the tile's first unit
  int parts;   // that the tile will have, if so
};
template <bool WIDE, int HD>
AXON_DEV Work work_of(const Segment& g, const Place& p, int G, int at, int end, const Shares& shares, int me) {
  using X = Tiles<WIDE, HD>;
  const int steps = X::steps(g, G, p.rt);
  auto unit_at = [](int step) { return max(step - X::START, 0); };
  Work w;
  w.take = min(steps - p.step, end - at);
  w.first = unit_at(p.step);
  w.last = unit_at(p.step + w.take);
  w.leads = w.first == 0 && w.last > 0;
  w.parts = w.leads ? shares.of(at - p.step + steps - 1) - me + 1 : 0;
  return w;
}

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

// 8 elements of a query row (any element alignment)
AXON_DEV bf16x8 load_q8_as(const bf16* p, bf16x8) { return *(const bf16x8_any*)p; }
AXON_DEV f32x8 load_q8_as(const float* p, f32x8) {
  const f32x4 a = *(const f32x4_any*)p, b = *(const f32x4_any*)(p + 4);
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <typename T>
AXON_DEV typename Vec8<T>::t load_q8(const T* p) {
  return load_q8_as(p, typename Vec8<T>::t{});
}
// for a negative scale
template <typename V, int N>
AXON_DEV void negate(V (&q)[N]) {
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int j = 0; j < 8; ++j) q[k][j] = -q[k][j];
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

// The reference m of a row's weights 2^(score - m): where the maximum (in base 2, times the
// scale) passes it, it goes 8 above it, so that the sum and the products are hardly rescaled
// after the first keys.  A weight is 1 at most: what is summed leaves float32's range no
// earlier than with the maximum itself for a reference.
template <int N, typename V>
AXON_DEV void raise(float& m, float top, float& l, V (&o)[N]) {
  if (!__any(top > m)) return;
  const float m_new = top > m ? top + 8.f : m;
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
  static constexpr int MY_KEYS = WIDE_KEYS / PA_WAVES;  // staged by a wavefront
  static constexpr int LOADS = 2 * (MY_KEYS / L::RPI);    // its copies
  static constexpr int BATCH = PA_THREADS / 4;          // units whose pages are looked up at a time
  struct Shared {
    alignas(16) T tiles[STAGES][2][TILE];
    int32_t blocks[PA_THREADS];     // where a batch's 16-key blocks are in the cache, 4 a unit, -1: none
    int32_t odd[STAGES][PA_WAVES];  // make_finite's rows
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
    for (int k = 0; k < QS; ++k) q[k] = load_q8<T>(p + 16 * k);
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
  // s[b] = the weights of blocks kb0 + b of the unit at key0, all to one reference: raising
  // it rescales the products that are there, and no weights wait for theirs then
  template <int NB>
  AXON_DEV void weights(f32x16 (&s)[NB], int key0, int kb0, int pages, const int32_t* odd) {
    if (key0 + WIDE_KEYS > least || pages != 15) {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const int kb = kb0 + b, seen = limit - key0 - 32 * kb - 4 * hl;
        const int seen0 = pages >> (2 * kb) & 1 ? seen : 0, seen1 = pages >> (2 * kb + 1) & 1 ? seen : 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[b][i] = 8 * (i >> 2) + (i & 3) < (i < 8 ? seen0 : seen1) ? s[b][i] : -INFINITY;
      }
    }
    float top = s[0][0];
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
    raise(m, fmaxf(top, lane_xor32(top)) * sc, l, o);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], sc, -base));
        sum += s[b][i];
      }
      l += sum;
    }
    if (odd)
      for (int w = 32 / W::MY_KEYS * kb0; w < 32 / W::MY_KEYS * (kb0 + NB); ++w)
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
        x.weights(s, (u0 + i) * WIDE_KEYS, kb0, pages, odd);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int j = 0; j < 16; ++j) w[b][j / 8][j % 8] = (bf16)s[b][j];
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
  if (a.scale < 0.f) negate(x.q);
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
  if (a.scale < 0.f) negate(x.q);
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
        f32x16 s[1];
        x.scores(kf, s[0]);
        x.weights(s, key0, kb, st.pages(i), st.masked(i) ? sh.odd[i % S] : nullptr);
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
          for (int d = 0; d < X::DT; ++d)
            x.o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(
                tile[W::TILE + L::v_at(32 * kb + 8 * (j >> 2) + 4 * x.hl + (j & 3), 32 * d + x.c)], s[0][j], x.o[d], 0, 0, 0);
      }
    }
  }
  x.store(part);
}

// ---------------------------------------------------------------- narrow tiles

template <typename T, int HD>
struct Narrow {
  using L = Lds<T, HD>;
  static constexpr int TILE = NARROW_KEYS * HD, QS = HD / 32;
  static constexpr int LOADS = NARROW_KEYS / L::RPI + QS * (int)sizeof(T) / 2;  // of a unit
  static constexpr int DEPTH = sizeof(T) == 4 && HD == 128 ? 2 : 3;             // units in flight or in use
  struct Shared {
    alignas(16) T v[PA_WAVES][DEPTH][TILE];
  };
};

// Units first .. last - 1 of a tile, by one wavefront: keys to registers, where a lane
// has those of one key that multiply its dimensions, values through LDS.
template <typename T, int HD>
AXON_DEV void narrow_tile(const PrefixAttnArgs<T>& a, float sc, T (&lds)[Narrow<T, HD>::DEPTH][Narrow<T, HD>::TILE],
                          const Segment& g, int G, int kvh, int first, int last, float* part) {
  using N = Narrow<T, HD>;
  using L = Lds<T, HD>;
  using V8 = typename Vec8<T>::t;
  constexpr int DT = HD / 16, QS = N::QS, D = N::DEPTH;
  const int lane = threadIdx.x & 63, gq = lane >> 4, c = lane & 15;
  const int rows = g.tokens * G, r = min(c, rows - 1);
  const Cache<T, HD> cache{a, g, kvh};
  int blocks = 0;  // of 64 units, one a lane; -1: no page
  bool there[D];
  V8 q[QS], k[D][QS];
  {
    const T* p = q_row<T, HD>(a, g, G, kvh, r) + 8 * gq;
#pragma unroll
    for (int j = 0; j < QS; ++j) q[j] = load_q8<T>(p + 32 * j);
  }
  auto fetch = [&](int u, const int b) {
    if (((u - first) & 63) == 0) blocks = u + lane < last ? cache.block((u + lane) * NARROW_KEYS) : -1;
    const int at = __builtin_amdgcn_readlane(blocks, (u - first) & 63);
    there[b] = at >= 0;
    const int64_t src = (int64_t)max(at, 0) * NARROW_KEYS * HD;  // (none: masked, but read)
    L::template stage<false, false>((const T*)a.kv.v + src, lds[b], 0, NARROW_KEYS, lane);
    const T* kp = (const T*)a.kv.k + src + c * HD + 8 * gq;
#pragma unroll
    for (int j = 0; j < QS; ++j) k[b][j] = read8(kp + 32 * j, kp + 32 * j + 4);
  };
  const int limit = row_keys(g, G, r), least = row_keys(g, G, 0);
  f32x4 o[DT] = {};
  float m = -INFINITY, l = 0.f;
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the tile before is read)
#pragma unroll
  for (int b = 0; b < D - 1; ++b)
    if (first + b < last) fetch(first + b, b);
  if (a.scale < 0.f) negate(q);
  auto unit = [&](int u, const int b) {
    const int key0 = u * NARROW_KEYS;
    const bool masked = key0 + NARROW_KEYS > least || !there[b];
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (the stage that is filled next is read)
    if (u + D - 1 < last) fetch(u + D - 1, (b + D - 1) % D);
    wait_loads<N::LOADS, D - 1>(min(last - 1 - u, D - 1));
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
        if (key0 + 4 * gq + i >= limit || !there[b]) s[i] = -INFINITY;
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
      add_odd(cache, key0, there[b] ? odd : 0, limit, e, [&](int i) { return 16 * (i / 4) + 4 * gq + i % 4; });
#pragma unroll
      for (int i = 0; i < 4 * DT; ++i) o[i / 4][i % 4] = e[i];
    }
  };
  for (int u = first; u < last; u += D)
#pragma unroll
    for (int b = 0; b < D; ++b)
      if (u + b < last) unit(u + b, b);
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

// ---------------------------------------------------------------- the kernel

// Where the parts of the kinds lie, in blocks
struct PartsAt {
  int wide_slots, narrow_slots;  // a wide one has SLOT_BLOCKS blocks, the narrow ones follow
  AXON_DEV int narrow() const { return wide_slots * SLOT_BLOCKS; }
};

template <typename T, int HD>
__global__ void __launch_bounds__(PA_THREADS, 2) prefix_attn_kernel(PrefixAttnArgs<T> a, float sc, RowParts* info,
                                                                    float* parts, PartsAt at_) {
  union Stages {
    typename Wide<T, HD>::Shared wide;
    typename Narrow<T, HD>::Shared narrow;
  };
  __shared__ Stages sh;
  __shared__ PlanShared plan_sh;
  Plan<T, HD> plan(a, plan_sh);
  const int G = plan.G, KV = plan.KV, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t all_rows = (int64_t)a.tokens * G;
  // The workgroups of an XCD (blockIdx % 8) are shared out over the kinds as the steps and
  // their weight are; consecutive runs go to one XCD, whose L2 holds what they share.
  constexpr int PER = PA_WGS / 8;
  const int total_n = __builtin_amdgcn_readfirstlane(plan.total[0]), total_w = __builtin_amdgcn_readfirstlane(plan.total[1]);
  const float cost_w = (float)Tiles<true, HD>::WEIGHT * total_w;
  const int wide_wgs = !total_w ? 0 : !total_n ? PER : min(max((int)(PER * cost_w / (cost_w + total_n) + 0.5f), 1), PER - 1);
  const int xcd = blockIdx.x % 8, nth = blockIdx.x / 8;
  if (nth < wide_wgs) {
    const Shares shares(min(8 * wide_wgs, max(total_w / Tiles<true, HD>::LEAST, 1)), total_w);
    // (fewer workers than workgroups: over all XCDs)
    const int me = shares.n < 8 * wide_wgs ? (int)blockIdx.x : xcd * wide_wgs + nth;
    if (me >= shares.n) return;
    int at = shares.start(me);
    const int end = shares.start(me + 1);
    plan.template find<true>(0, at);
    __syncthreads();
    Segment g;
    Place p = plan.template get<true>(0, g);
    for (;;) {
      const int slot = p.tile + me;
      if (slot >= at_.wide_slots) return;  // (cu_seqlens are not those of the host)
      const Work w = work_of<true, HD>(g, p, G, at, end, shares, me);
      const int row0 = p.rt * WIDE_ROWS, here = min(g.tokens * G - row0, WIDE_ROWS);
      if (w.leads && (int)threadIdx.x < here) {
        // a tile of up to 128 rows has two parts in a slot
        const bool halves = here <= WIDE_ROWS / 2;
        info[info_at(g.own, p.kvh, KV, all_rows, (int64_t)g.tok0 * G + row0 + threadIdx.x)] =
            row_parts(slot * SLOT_BLOCKS + ((int)threadIdx.x >> 4), halves ? 2 * w.parts : w.parts,
                      halves ? SLOT_BLOCKS / 2 : SLOT_BLOCKS, threadIdx.x & 15);
      }
      if (w.last > w.first)
        wide_tile<HD>(a, sc, sh.wide, g, G, p.kvh, row0, w.first, w.last, parts + (int64_t)slot * SLOT_BLOCKS * part_floats(HD));
      at += w.take;
      if (at >= end) return;
      plan.template advance<true>(p, g);
    }
  } else {
    // a wavefront is a worker
    const int wgs = PER - wide_wgs, waves = 8 * wgs * PA_WAVES;
    const Shares shares(min(waves, max(total_n / Tiles<false, HD>::LEAST, min(total_n, 1))), total_n);
    // (fewer workers than wavefronts: over all workgroups)
    auto worker = [&](int w) {
      const int wg = nth - wide_wgs;
      return shares.n < waves ? w * 8 * wgs + wg * 8 + xcd : (xcd * wgs + wg) * PA_WAVES + w;
    };
    for (int w = 0; w < PA_WAVES; ++w)
      if (worker(w) < shares.n) plan.template find<false>(w, shares.start(worker(w)));
    __syncthreads();
    const int me = worker(wave);
    if (me >= shares.n) return;
    int at = shares.start(me);
    const int end = shares.start(me + 1);
    Segment g;
    Place p = plan.template get<false>(wave, g);
    for (;;) {
      const int slot = p.tile + me, lane = threadIdx.x & 63;
      if (slot >= at_.narrow_slots) return;
      const Work w = work_of<false, HD>(g, p, G, at, end, shares, me);
      if (w.leads && lane < g.tokens * G)
        info[info_at(g.own, p.kvh, KV, all_rows, (int64_t)g.tok0 * G + lane)] = row_parts(at_.narrow() + slot, w.parts, 1, lane);
      if (w.last > w.first)
        narrow_tile<T, HD>(a, sc, sh.narrow.v[wave], g, G, p.kvh, w.first, w.last,
                           parts + (int64_t)(at_.narrow() + slot) * part_floats(HD));
      at += w.take;
      if (at >= end) return;
      plan.template advance<false>(p, g);
    }
  }
}

// ---------------------------------------------------------------- the join

// A row's parts of both segments: out = sum f o / sum f l, f = 2^(m - max).  A workgroup
// per (token, kv head): HD / 4 lanes for a part of a row, the parts shared out over as
// many groups of them as it has for the R rows at a time, whose sums are joined in LDS.
// Few tokens' rows have many parts: a large workgroup each, several loads ahead (48
// answers, 384 workgroups with 26 parts a row: 10.6 us; of 1024 threads 14.0).  Many
// tokens' have one or two of either segment: small ones, in few enough registers that 8
// fit a CU's SIMDs (20 questions of 150 tokens: 150 MB, 37 us; 5 at a time 44).
constexpr int JOIN_MAX = 512;
template <typename T, int HD, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == JOIN_MAX ? 4 : 8)
    prefix_join_kernel(PrefixAttnArgs<T> a, const RowParts* info, const float* parts, int blocks, int R) {
  constexpr int LANES = HD / 4, FIRST = THREADS == JOIN_MAX ? 2 : 1, AHEAD = THREADS == JOIN_MAX ? 4 : 1;
  __shared__ f32x4 sum_o[THREADS];
  __shared__ float sum_m[THREADS / LANES], sum_l[THREADS / LANES];
  const int t = blockIdx.y * GRID_TOKENS + blockIdx.x, kvh = blockIdx.z, KV = a.kv.kv_heads, G = a.heads / KV;
  const int lane = threadIdx.x & 63, d = threadIdx.x % LANES, team = threadIdx.x / LANES, row = team % R;
  const int groups = THREADS / (LANES * R), group = team / R;  // of parts
  if (t >= a.tokens) return;
  // (read before it is known whether they are there, beside what says it)
  RowParts where[2];
#pragma unroll
  for (int k = 0; k < 2; ++k) where[k] = info[info_at(k, kvh, KV, (int64_t)a.tokens * G, (int64_t)t * G + min(row, G - 1))];
  auto among = [&](const int32_t* cu, int n, int v) {  // how many of cu[1 .. n] are <= v
    int c = 0;
    for (int i = lane; i - lane < n; i += 64) c += __popcll(__ballot(i < n && cu[i + 1] <= v));
    return c;
  };
  const int b = a.seqs.cu ? among(a.seqs.cu, a.seqs.seqs, t) : t;
  if (b >= a.seqs.seqs) return;  // behind the last sequence
  const int grp = a.shared.groups ? among(a.shared.cu, a.shared.groups, b) : 0;
  const int own_len = a.seqs.lens[b], prefix_len = grp < a.shared.groups ? a.shared.lens[grp] : 0;
  for (int j0 = 0; j0 < G; j0 += R) {
    const int j = j0 + row;
    f32x4 o = {};
    float top = -INFINITY, l = 0.f;
    // parts i0, i0 + groups, ... from ``part`` on (the last one where there are fewer)
    auto read = [&](const float* part, int64_t step, int in, int count, int i0, auto& v, auto& m, auto& s) {
#pragma unroll
      for (int i = 0; i < (int)(sizeof(m) / sizeof(float)); ++i) {  // (loads without a condition stay in flight together)
        const float* at = part + max(min(i0 + i * groups, count - 1), 0) * step;
        m[i] = at[16 * HD + in];
        s[i] = at[16 * HD + 16 + in];
        v[i] = *(const f32x4*)(at + in * HD + 4 * d);
      }
    };
    auto add = [&](int count, int i0, const auto& v, const auto& m, const auto& s) {
      constexpr int N = sizeof(m) / sizeof(float);
      float next = top;
#pragma unroll
      for (int i = 0; i < N; ++i) next = fmaxf(next, m[i]);
      const float fall = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - next);
      top = next;
      l = fall > 0.f ? l * fall : l != l ? l : 0.f;
      o = fall > 0.f ? o * fall : f32x4{};
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if (i0 + i * groups >= count) continue;
        const float f = m[i] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[i] - top);
        l += f > 0.f || s[i] != s[i] ? f * s[i] : 0.f;  // (scores that are all NaN: no maximum)
        o += f > 0.f ? f * v[i] : f32x4{};
      }
    };
    // The first parts of either segment are read before the lengths have come that say
    // whether there are any (where not: some other place of the parts).
    const float* part[2];
    int64_t step[2];
    int count[2], in[2];
    f32x4 v[2][FIRST];
    float m[2][FIRST], s[2][FIRST];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const RowParts p = j0 ? info[info_at(k, kvh, KV, (int64_t)a.tokens * G, (int64_t)t * G + min(j, G - 1))] : where[k];
      const int apart = p.count >> 4 & 31;
      count[k] = p.count >> 9;
      const bool inside = p.block >= 0 && count[k] > 0 && (int64_t)p.block + (int64_t)(count[k] - 1) * apart < blocks;
      count[k] = inside ? count[k] : 0;
      in[k] = p.count & 15;
      step[k] = (int64_t)apart * part_floats(HD);
      part[k] = parts + (inside ? (int64_t)p.block : 0) * part_floats(HD);
      read(part[k], step[k], in[k], count[k], group, v[k], m[k], s[k]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      if (own_len < 0 || (k == 0 && prefix_len <= 0) || j >= G || group >= count[k]) continue;
      add(count[k], group, v[k], m[k], s[k]);
      for (int i0 = group + FIRST * groups; i0 < count[k]; i0 += AHEAD * groups) {
        f32x4 w[AHEAD];
        float wm[AHEAD], ws[AHEAD];
        read(part[k], step[k], in[k], count[k], i0, w, wm, ws);
        add(count[k], i0, w, wm, ws);
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

struct Tally {  // tiles of a kind: of own keys, of prefixes
  int64_t own = 0, shared = 0;
  int64_t all() const { return own + shared; }
};
struct Sizes {
  Tally wide_tiles, narrow_tiles;
  int64_t wide, narrow;  // slots of each kind (0: no such tile)
  int64_t parts_at, bytes;
  int64_t blocks() const { return wide * SLOT_BLOCKS + narrow; }
};
Sizes sizes_of(const PrefixAttnShape& x) {
  const int64_t G = x.heads / x.kv_heads;
  auto token = [&](int b) -> int64_t { return x.h_cu ? x.h_cu[b] : b; };
  Sizes s;
  auto add = [&](int64_t Tally::*of, int64_t tokens) {
    const int64_t rows = tokens * G;
    if (rows > NARROW_ROWS) s.wide_tiles.*of += (rows + WIDE_ROWS - 1) / WIDE_ROWS * x.kv_heads;
    else if (rows > 0) s.narrow_tiles.*of += x.kv_heads;
  };
  for (int g = 0; g < x.groups; ++g) add(&Tally::shared, token(x.h_groups[g + 1]) - token(x.h_groups[g]));
  for (int b = 0; b < x.seqs; ++b) add(&Tally::own, x.h_cu ? x.h_cu[b + 1] - x.h_cu[b] : 1);
  s.wide = s.wide_tiles.all() ? s.wide_tiles.all() + PA_WGS : 0;
  s.narrow = s.narrow_tiles.all() ? s.narrow_tiles.all() + PA_WGS * PA_WAVES : 0;
  s.parts_at = (2 * x.tokens * x.heads * (int64_t)sizeof(RowParts) + 15) / 16 * 16;
  s.bytes = s.parts_at + s.blocks() * part_floats(x.hd) * 4;
  return s;
}

}  // namespace

int64_t prefix_attn_workspace(const PrefixAttnShape& x) { return sizes_of(x).bytes; }

bool prefix_attn_fits(const PrefixAttnShape& x, int64_t own_keys, int64_t prefix_keys) {
  const Sizes s = sizes_of(x);
  // A tile's steps are those of the longest row of its table.  The slots past the tiles',
  // one a worker, count as tiles of the longest: of tables up to some 2^24 keys that is
  // little, and longer ones it leaves to few calls.
  auto steps = [&](const Tally& n, int64_t slots, int64_t keys, int64_t start) {
    auto of = [&](int64_t k) { return (k + keys - 1) / keys + start; };
    return n.own * of(own_keys) + n.shared * of(prefix_keys) + (slots - n.all()) * of(std::max(own_keys, prefix_keys));
  };
  constexpr int64_t MOST = ((int64_t)1 << 31) - 1;
  return steps(s.wide_tiles, s.wide, WIDE_KEYS, WIDE_START) <= MOST &&
         steps(s.narrow_tiles, s.narrow, NARROW_KEYS, NARROW_START) <= MOST && s.blocks() <= MOST &&
         s.bytes < (int64_t)1 << 39;  // (no card has that; 264 bytes a row and more leave rows 32 bits)
}

template <typename T, int HD>
static void launch(const PrefixAttnArgs<T>& a, const PrefixAttnShape& x, void* workspace, hipStream_t s) {
  const Sizes n = sizes_of(x);
  RowParts* info = (RowParts*)workspace;
  float* parts = (float*)((char*)workspace + n.parts_at);
  // a scale of 0 leaves every score, masked ones apart, the same (-inf times 0 is NaN)
  const float sc = std::max(fabsf(a.scale) * LOG2E_F, 1e-37f);
  prefix_attn_kernel<T, HD><<<PA_WGS, PA_THREADS, 0, s>>>(a, sc, info, parts, PartsAt{(int)n.wide, (int)n.narrow});
  // few tokens: many threads each, whose parts are many
  auto join = [&](auto threads) {
    constexpr int N = decltype(threads)::value;
    const int G = a.heads / a.kv.kv_heads;
    int R = 1;
    while (R < G && R < N / (HD / 4)) R *= 2;
    dim3 grid = token_grid(a.tokens);
    grid.z = a.kv.kv_heads;
    prefix_join_kernel<T, HD, N><<<grid, N, 0, s>>>(a, info, parts, (int)n.blocks(), R);
  };
  // (512 large workgroups run at once; 384 of them 10.6 us, small ones 15, 2048 of them 19.3 and 8.6)
  if ((int64_t)a.tokens * a.kv.kv_heads <= 512) join(std::integral_constant<int, JOIN_MAX>{});
  else join(std::integral_constant<int, 256>{});
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
