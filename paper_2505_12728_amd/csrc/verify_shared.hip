// Attention of drafted blocks whose sequences share long prefixes: the B
// sequences lie in groups, every row of a group sees the group's prefix in
// full and, causal inside the block, its own sequence's cache behind it.
//
// Mathematics.  With s_t = scale q . K_t over the prefix's and the visible
// own keys, out = sum_t exp(s_t) V_t / sum_t exp(s_t).  Softmax statistics
// (m, l, O) over disjoint key sets combine exactly, so that a prefix is
// attended once by all rows of its group (S k g rows of a KV head: S
// sequences, k block positions, g query heads) and its keys and values are
// read from HBM once, not once per sequence.
//
// Bound: 4 D operations per (row, key) against 4 D bytes per key and KV head
// (bf16), so HBM up to about 300 rows per KV head and the matrix cores beyond.
//
// Kernel 1 (stream).  Units are the groups' prefixes, then the sequences' own
//   caches; a unit's rows in tiles of ROWS and its KV heads give pairs; the
//   32-key tiles of all pairs form one list, of which each work-group of a
//   fixed grid takes an equal contiguous range.  Ragged lengths and groups are
//   balanced to a tile, and lengths and groups are read on the device alone.
//   Tiles come HBM -> LDS through a ring of global_load_lds copies; a wave
//   holds RB blocks of 16 rows, so that a fragment read from LDS feeds RB
//   matrix-core operations:  S^T = K Q^T, online softmax in fp32 (base 2),
//   O^T += V^T P^T.  Where its range leaves a pair, a work-group writes the
//   segment's normalised partial (o, lse).
// Kernel 2 (merge).  One wave per output row finds the partials of its prefix
//   pair and of its own pair from the same arithmetic and combines them.
//
// P is rounded to bf16 for the second product.  fp32 outputs take it as a pair
// hi + lo (2^-17 of p kept), two products per step; bf16 outputs, rounded to
// 2^-9 themselves, take hi alone.  The row sums add the fp32 values.
#include <math.h>

#include <algorithm>

#include "device_common.hpp"
#include "launch.hpp"

namespace sd {
namespace {

constexpr int kTile = 32;   // keys per tile

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void gbl_cvoid;
typedef const __attribute__((address_space(4))) int32_t cint32;   // scalar loads

// One unit of the list: a group's prefix (u < G) or a sequence's own cache
// (sequence u - G).  first: its first sequence; end: the sequence behind its last.
struct Unit {
  int L, rows, first, end;
};

// Start of group g before monotony is imposed
__device__ __forceinline__ int group_bound(const SharedArgs& a, int g) {
  if (a.group_start == nullptr) return g * (a.B / a.G);
  return min(max(((cint32*)a.group_start)[g], 0), a.B);
}

__device__ __forceinline__ int tiles_of(int L) { return (L + kTile - 1) / kTile; }
__device__ __forceinline__ int row_tiles(int rows, int per) { return (rows + per - 1) / per; }

// Place of a pair in the list
struct Cursor {
  int u;             // unit
  int hk, rt, t;     // KV head, row tile, key tile
  int nt, RT;        // key tiles and row tiles of the unit
  int L, rows, first, end;
  int pair;          // pairs of the same kind (prefix or own) before this one
};

// What a scan over the units finds: lane l holds unit u0 + l.
struct Span {
  Unit un;
  int tiles, pairs;      // of this unit
  int t_before, p_before;   // before it, in the whole list / among its kind
};

// Units u0 .. u0 + 63 with their exclusive sums, given the sums and the group
// bound carried from the units before.  Group bounds are made monotone by a
// running maximum, so that no sequence is in two groups.
struct Carry {
  int tiles = 0, pairs = 0, bound = 0;
};
template <int ROWS>
__device__ __forceinline__ Span scan_units(const SharedArgs& a, int u0, Carry& c) {
  const int lane = threadIdx.x & 63;
  const int u = u0 + lane;
  Span s;
  s.un = Unit{0, 0, 0, 0};
  int bound = 0;
  if (u < a.G) {
    bound = a.group_start != nullptr ? min(max(a.group_start[u], 0), a.B) : u * (a.B / a.G);
    s.un.L = min(max(a.prefix_len[u], 0), a.prefix_cap);
    s.un.end = a.group_start != nullptr ? min(max(a.group_start[u + 1], 0), a.B) : (u + 1) * (a.B / a.G);
  } else if (u < a.G + a.B) {
    s.un.L = min(max(a.kv_len[u - a.G], 0), a.cap);
  }
  if (u0 < a.G) {
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int x = __shfl_up(bound, off, 64);   // (on every lane)
      if (lane >= off) bound = max(bound, x);
    }
    bound = max(bound, c.bound);
  }
  const int R = a.k * (a.Hq / a.Hkv);
  if (u < a.G) {
    s.un.first = bound;
    s.un.end = max(s.un.end, bound);
    s.un.rows = (s.un.end - bound) * R;
  } else if (u < a.G + a.B) {
    s.un.first = u - a.G;
    s.un.end = s.un.first + 1;
    s.un.rows = R;
  }
  c.bound = max(c.bound, __shfl(bound, 63, 64));
  s.pairs = a.Hkv * row_tiles(s.un.rows, ROWS);
  s.tiles = s.pairs * tiles_of(s.un.L);
  int ti = s.tiles, pi = s.pairs;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int x = __shfl_up(ti, off, 64), y = __shfl_up(pi, off, 64);
    if (lane >= off) {
      ti += x;
      pi += y;
    }
  }
  s.t_before = c.tiles + ti - s.tiles;
  s.p_before = c.pairs + pi - s.pairs;
  c.tiles += __shfl(ti, 63, 64);
  c.pairs += __shfl(pi, 63, 64);
  return s;
}

// length T of the list
template <int ROWS>
__device__ __forceinline__ int total_tiles(const SharedArgs& a) {
  Carry c;
  for (int u0 = 0; u0 < a.G + a.B; u0 += 64) scan_units<ROWS>(a, u0, c);
  return c.tiles;
}

// cursor of tile n of the list (0 <= n < T); wave-uniform, in scalar registers.
// The pair counts its kind only: own pairs start at 0 again (R rows each).
template <int ROWS>
__device__ __forceinline__ Cursor locate(const SharedArgs& a, int n) {
  Carry c;
  for (int u0 = 0; u0 < a.G + a.B; u0 += 64) {
    const Span s = scan_units<ROWS>(a, u0, c);
    if (n >= c.tiles) continue;
    const int f = __builtin_ctzll(__ballot(s.t_before + s.tiles > n));
    auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
    Cursor cu;
    cu.u = u0 + f;
    cu.L = of(s.un.L);
    cu.rows = of(s.un.rows);
    cu.first = of(s.un.first);
    cu.end = of(s.un.end);
    cu.nt = tiles_of(cu.L);
    cu.RT = row_tiles(cu.rows, ROWS);
    const int rem = n - of(s.t_before);
    const int x = rem / cu.nt;
    cu.t = rem - x * cu.nt;
    cu.hk = x / cu.RT;
    cu.rt = x - cu.hk * cu.RT;
    cu.pair = cu.u < a.G ? of(s.p_before) + x : (cu.u - a.G) * a.Hkv * cu.RT + x;
    return cu;
  }
  return Cursor{};   // n >= T: not reached
}

// next tile of the list; the caller never steps past the last one
template <int ROWS>
__device__ __forceinline__ void advance(const SharedArgs& a, Cursor& cu) {
  if (++cu.t < cu.nt) return;
  cu.t = 0;
  ++cu.pair;
  if (++cu.rt < cu.RT) return;
  cu.rt = 0;
  if (++cu.hk < a.Hkv) return;
  cu.hk = 0;
  do {
    ++cu.u;
    if (cu.u < a.G) {
      cu.first = cu.end;
      cu.end = max(cu.end, group_bound(a, cu.u + 1));
      cu.rows = (cu.end - cu.first) * a.k * (a.Hq / a.Hkv);
      cu.L = min(max(((cint32*)a.prefix_len)[cu.u], 0), a.prefix_cap);
    } else {
      if (cu.u == a.G) cu.pair = 0;
      cu.first = cu.u - a.G;
      cu.end = cu.first + 1;
      cu.rows = a.k * (a.Hq / a.Hkv);
      cu.L = cu.first < a.B ? min(max(((cint32*)a.kv_len)[cu.first], 0), a.cap) : 0;
    }
    cu.nt = tiles_of(cu.L);
    cu.RT = row_tiles(cu.rows, ROWS);
    if (cu.nt == 0 || cu.RT == 0) cu.pair += a.Hkv * cu.RT;
  } while ((cu.nt == 0 || cu.RT == 0) && cu.u < a.G + a.B);
}

// First row of the partial that work-group w writes for the pair of cursor cu:
// along the list both the pair and w only grow, so that pair + w is distinct
// for every segment.  Own pairs have an area of their own, rows_own each.
template <int ROWS>
__device__ __forceinline__ size_t part_row(const SharedArgs& a, bool own, int pair, int w) {
  return own ? (size_t)a.own_base + (size_t)(pair + w) * a.rows_own : (size_t)(pair + w) * ROWS;
}

// output row (flat over [B, k, Hq]) of row r of a unit that starts at sequence `first`
__device__ __forceinline__ int out_row(const SharedArgs& a, int first, int hk, int r) {
  const int g = a.Hq / a.Hkv;
  const int q = r / g;
  return (first * a.k + q) * a.Hq + hk * g + (r - q * g);
}

// ------------------------------------------------------------ bf16 stream
template <int D, int NW, int RB, int NBUF, bool HILO>
__global__ __launch_bounds__(NW * 64, 2) void shared_stream_bf16(SharedArgs a, int G) {
  constexpr int TK = kTile;
  constexpr int DC = D / 32;                   // 32-channel slices (S^T = K Q^T)
  constexpr int DB = D / 16;                   // 16-channel blocks (O^T)
  constexpr int PK = D / 8;                    // 16-byte pieces per key row
  constexpr int ROW_BYTES = D * 2;
  constexpr int HALF_BYTES = TK * ROW_BYTES;   // K (or V) part of a slot
  constexpr int BUF_BYTES = 2 * HALF_BYTES;
  constexpr int DMA_PER_HALF = TK * PK / 64;
  constexpr int DMA_PER_WAVE = 2 * DMA_PER_HALF / NW;
  constexpr int ROWS = NW * RB * 16;
  static_assert((2 * DMA_PER_HALF) % NW == 0, "tile copy must split evenly");
  static_assert(NBUF >= 3 && (NBUF - 2) * DMA_PER_WAVE < 64, "ring depth and vmcnt range");
  constexpr float kRescale = 8.f;              // log2 headroom before rescaling
  __shared__ __align__(16) unsigned char ring[NBUF][BUF_BYTES];

  const int lane = threadIdx.x & 63, G4 = lane >> 4, c = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = blockIdx.x;
  const int T = __builtin_amdgcn_readfirstlane(total_tiles<ROWS>(a));
  const int n0 = (int)((long long)T * wg / G), n1 = (int)((long long)T * (wg + 1) / G);
  if (n0 >= n1) return;
  const int last = n1 - 1;

  // copies: copy i of this wave covers pieces P of K or V: key P / PK, LDS slot
  // P % PK holding global piece slot ^ lds_swizzle(key)
  int ckey[DMA_PER_WAVE], cpiece[DMA_PER_WAVE];
#pragma unroll
  for (int i = 0; i < DMA_PER_WAVE; ++i) {
    const int P = ((w * DMA_PER_WAVE + i) % DMA_PER_HALF) * 64 + lane;
    ckey[i] = P / PK;
    cpiece[i] = ((P % PK) ^ lds_swizzle<PK>(P / PK)) * 8;
  }
  // copies of the tile under cursor cu; keys past the unit's length re-read its
  // last key (masked)
  auto issue = [&](const Cursor& cu, unsigned char* slot) {
    const bool own = cu.u >= a.G;
    const int row = own ? cu.first : cu.u;     // row of the tables and contiguous caches
    const uint16_t* kb = static_cast<const uint16_t*>(own ? a.k_cache : a.k_prefix);
    const uint16_t* vb = static_cast<const uint16_t*>(own ? a.v_cache : a.v_prefix);
    const int32_t* table = own ? a.page_table : a.prefix_table;
    const int t0 = cu.t * TK;
    const int lim = cu.L - 1 - t0;             // last key of the tile that is there
    if (table != nullptr) {
      const int pages = own ? a.num_pages : a.prefix_num_pages;
      cint32* pt = (cint32*)(table + (size_t)row * (own ? a.max_pages : a.prefix_pages));
      const int lastp = (cu.L - 1) >> 4;
      const int pg0 = min(max((int)pt[min(t0 >> 4, lastp)], 0), pages - 1);
      const int pg1 = min(max((int)pt[min((t0 >> 4) + 1, lastp)], 0), pages - 1);
      const size_t b0 = ((size_t)pg0 * a.Hkv + cu.hk) * 16 * D, b1 = ((size_t)pg1 * a.Hkv + cu.hk) * 16 * D;
#pragma unroll
      for (int i = 0; i < DMA_PER_WAVE; ++i) {
        const int ii = w * DMA_PER_WAVE + i;
        const int key = min(ckey[i], lim);
        const size_t off = (key >> 4 ? b1 : b0) + (uint32_t)((key & 15) * D + cpiece[i]);
        __builtin_amdgcn_global_load_lds((gbl_cvoid*)((ii / DMA_PER_HALF ? vb : kb) + off),
                                         (lds_void*)(slot + (ii / DMA_PER_HALF) * HALF_BYTES + (ii % DMA_PER_HALF) * 1024),
                                         16, 0, 0);
      }
    } else {
      const size_t base = (((size_t)row * (own ? a.Lmax : a.prefix_cap) + t0) * a.Hkv + cu.hk) * D;
#pragma unroll
      for (int i = 0; i < DMA_PER_WAVE; ++i) {
        const int ii = w * DMA_PER_WAVE + i;
        const size_t off = base + (uint32_t)(min(ckey[i], lim) * a.Hkv * D + cpiece[i]);
        __builtin_amdgcn_global_load_lds((gbl_cvoid*)((ii / DMA_PER_HALF ? vb : kb) + off),
                                         (lds_void*)(slot + (ii / DMA_PER_HALF) * HALF_BYTES + (ii % DMA_PER_HALF) * 1024),
                                         16, 0, 0);
      }
    }
  };

  // fragment offsets inside a slot for the first 16 keys; the swizzle depends on
  // key % 16 only, so the second block is an immediate offset
  uint32_t koff[DC], voff[DB];
#pragma unroll
  for (int dc = 0; dc < DC; ++dc) koff[dc] = c * ROW_BYTES + (((dc * 4 + G4) ^ lds_swizzle<PK>(c)) * 16);
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int key = 4 * G4 + (c >> 2), ch = db * 16 + 4 * (c & 3);
    voff[db] = HALF_BYTES + key * ROW_BYTES + (((ch >> 3) ^ lds_swizzle<PK>(key)) * 16) + (ch & 7) * 2;
  }

  // segment state of this wave: its rows' queries (B operand of S^T = K Q^T),
  // last visible keys and running (max, sum, O^T).  Scores stay raw, the scale
  // enters the exponent as exp2(S sl2 - m); a negative one is folded into the
  // queries.
  int cur_pair = 0, cur_rt = 0, seg_rows = 0, unmasked = 0;
  bool cur_own = false, busy = false;          // busy: this wave has rows (uniform)
  int lim[RB];
  bf16x8 qf[RB][DC];
  float m[RB], l[RB];
  floatx4 o[RB][DB];
  const bool neg = a.scale_log2 < 0.f;
  const float sl2 = fabsf(a.scale_log2);
  const int kg = a.k * (a.Hq / a.Hkv);

  auto start_segment = [&](const Cursor& cu) {
    cur_pair = cu.pair;
    cur_own = cu.u >= a.G;
    cur_rt = cu.rt;
    seg_rows = cu.rows;
    busy = cu.rt * ROWS + w * RB * 16 < cu.rows;
    unmasked = cur_own ? cu.L - a.k : cu.L - 1;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = cu.rt * ROWS + (w * RB + rb) * 16 + c;
      Pack8 pk;
      pk.u = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) qf[rb][dc] = pk.b;
      lim[rb] = -1;
      if (r < cu.rows) {
        const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) +
                                                          (size_t)out_row(a, cu.first, cu.hk, r) * D);
#pragma unroll
        for (int dc = 0; dc < DC; ++dc) {
          pk.u = src[dc * 4 + G4];
          if (neg) pk.u ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
          qf[rb][dc] = pk.b;
        }
        lim[rb] = cur_own ? cu.L - a.k + (r % kg) / (kg / a.k) : cu.L - 1;
      }
      m[rb] = -INFINITY;
      l[rb] = 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[rb][db] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
  };
  auto flush = [&]() {
    if (!busy) return;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float lsum = wave_sum_across_groups(l[rb]);
      const int lr = (w * RB + rb) * 16 + c;
      if (cur_rt * ROWS + lr >= seg_rows) continue;
      const size_t prow = part_row<ROWS>(a, cur_own, cur_pair, wg) + lr;
      const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<floatx4*>(a.part_o + prow * D + db * 16 + 4 * G4) = o[rb][db] * inv;
      if (G4 == 0) a.part_lse[prow] = lsum > 0.f ? m[rb] + log2f(lsum) : -INFINITY;
    }
  };

  auto compute = [&](int t0, const unsigned char* slot) {
    const uint32_t sb = lds_addr(slot);
    u32x4 kr[2][DC];
#pragma unroll
    for (int dc = 0; dc < DC; ++dc) {
      kr[0][dc] = lds_read_b128_off<0>(sb + koff[dc]);
      kr[1][dc] = lds_read_b128_off<16 * ROW_BYTES>(sb + koff[dc]);
    }
    lds_wait();
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) tie(kr[kb][dc]);
    u32x2 vr[2][DB];
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      vr[0][db] = lds_read_tr16_b64_off<0>(sb + voff[db]);
      vr[1][db] = lds_read_tr16_b64_off<16 * ROW_BYTES>(sb + voff[db]);
    }
    // S^T = K Q^T: lane holds S[row c][key t0 + kb * 16 + 4 G4 + i]
    float x[RB][8];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      floatx4 acc[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) acc[rb] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) {
        Pack8 pk;
        pk.u = kr[kb][dc];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) acc[rb] = mfma_bf16(pk.b, qf[rb][dc], acc[rb]);
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < 4; ++i) x[rb][kb * 4 + i] = acc[rb][i];
    }
    bf16x8 ph[RB], pl[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      // Exponents before the mask: their largest bounds the masked ones, so
      // that m, raised only when a lane passes 2^8, may exceed the true maximum;
      // it cancels in o = O / l and lse = m + log2 l.
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) y[e] = fmaf(x[rb][e], sl2, -m[rb]);
      const float ly = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
      if (__ballot(ly > kRescale) != 0ull) {
        const float lm = fmaxf(fmaxf(fmaxf(x[rb][0], x[rb][1]), fmaxf(x[rb][2], x[rb][3])),
                               fmaxf(fmaxf(x[rb][4], x[rb][5]), fmaxf(x[rb][6], x[rb][7])));
        const float mnew = fmaxf(m[rb], wave_max_across_groups(lm) * sl2);
        const float alpha = m[rb] == -INFINITY ? 0.f : fast_exp2(m[rb] - mnew);
        l[rb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] *= alpha;
        m[rb] = mnew;
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = fmaf(x[rb][e], sl2, -m[rb]);
      }
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) p[e] = fast_exp2(y[e]);
      if (t0 + TK - 1 > unmasked) {            // tail tiles
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (t0 + (e >> 2) * 16 + 4 * G4 + (e & 3) > lim[rb]) p[e] = 0.f;
      }
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        sum += p[e];
        ph[rb][e] = float_to_bf16(p[e]);
        if constexpr (HILO) pl[rb][e] = float_to_bf16(p[e] - bf16_to_float(ph[rb][e]));
      }
      l[rb] += sum;
    }
    // O^T += V^T P^T over keys {4 G4 .. + 3, 16 + 4 G4 .. + 3}, the order in
    // which the score accumulator handed this lane its values
    lds_wait();
#pragma unroll
    for (int hh = 0; hh < 2; ++hh)
#pragma unroll
      for (int db = 0; db < DB; ++db) tie(vr[hh][db]);
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      Pack8 vv;
      vv.u = u32x4{vr[0][db][0], vr[0][db][1], vr[1][db][0], vr[1][db][1]};
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        o[rb][db] = mfma_bf16(vv.b, ph[rb], o[rb][db]);
        if constexpr (HILO) o[rb][db] = mfma_bf16(vv.b, pl[rb], o[rb][db]);
      }
    }
  };

  // Every step issues one tile (past the range it re-reads the last one), so
  // that at each wait exactly NBUF - 2 tiles' copies are newer than the step's
  // own; the barrier also frees the previous step's slot.  A new segment drains
  // this wave's memory counter, so that the counted waits only see copies.
  Cursor cc = locate<ROWS>(a, n0);
  Cursor ic = cc;
  int in = n0;
#pragma unroll 1
  for (int i = 0; i < NBUF - 1; ++i) {
    issue(ic, ring[i]);
    if (in < last) {
      advance<ROWS>(a, ic);
      ++in;
    }
  }
  bool fresh = true;
#pragma unroll 1
  for (int n = n0; n < n1; ++n) {
    const int s = n - n0;
    wait_vm_then_barrier<(NBUF - 2) * DMA_PER_WAVE>();
    issue(ic, ring[(s + NBUF - 1) % NBUF]);
    if (in < last) {
      advance<ROWS>(a, ic);
      ++in;
    }
    if (fresh) {
      if (n != n0) flush();
      start_segment(cc);
      __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // vmcnt(0)
    }
    if (busy) compute(cc.t * TK, ring[s % NBUF]);
    fresh = cc.t + 1 == cc.nt;
    if (n < last) advance<ROWS>(a, cc);
  }
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // no copy may still write this LDS
  flush();
}

// ------------------------------------------------------------- fp32 stream
// fp32 inputs: scores, softmax and P V in float64, as everywhere for fp32.
// The same list with 16 rows per work-group; a tile's keys and values and the
// segment's queries are staged in LDS (rows padded by one float), thread i
// forms two of the 16 x 32 scores, and O of the 16 x D elements.
constexpr int kRowsF32 = 16;
template <int D>
__global__ __launch_bounds__(256) void shared_stream_f32(SharedArgs a, int G) {
  constexpr int TK = kTile, R = kRowsF32, DS = D + 1;
  constexpr int PER = R * D / 256;             // elements of O per thread
  __shared__ float qs[R * DS], ks[TK * DS], vs[TK * DS];
  __shared__ double ps[R][TK + 1], st[R][3];   // scores / weights; max, sum, factor
  const int tid = threadIdx.x;
  const int wg = blockIdx.x;
  const int T = total_tiles<R>(a);
  const int n0 = (int)((long long)T * wg / G), n1 = (int)((long long)T * (wg + 1) / G);
  if (n0 >= n1) return;
  Cursor cu = locate<R>(a, n0);
  const int kg = a.k * (a.Hq / a.Hkv);
  double o[PER];
  bool fresh = true;
  for (int n = n0; n < n1; ++n) {
    const bool own = cu.u >= a.G;
    const int t0 = cu.t * TK, here = min(TK, cu.L - t0);
    __syncthreads();
    if (fresh) {
      for (int i = tid; i < R * D; i += 256) {
        const int r = cu.rt * R + i / D;
        qs[(i / D) * DS + i % D] =
            r < cu.rows ? static_cast<const float*>(a.q)[(size_t)out_row(a, cu.first, cu.hk, r) * D + i % D] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] = 0.0;
      if (tid < R) {
        st[tid][0] = -INFINITY;
        st[tid][1] = 0.0;
      }
    }
    const int row = own ? cu.first : cu.u;
    const float* kb = static_cast<const float*>(own ? a.k_cache : a.k_prefix);
    const float* vb = static_cast<const float*>(own ? a.v_cache : a.v_prefix);
    const int32_t* table = own ? a.page_table : a.prefix_table;
    for (int i = tid; i < here * D; i += 256) {
      const int t = t0 + i / D;
      size_t off;
      if (table != nullptr) {
        const int pages = own ? a.num_pages : a.prefix_num_pages;
        const int page = min(max(table[(size_t)row * (own ? a.max_pages : a.prefix_pages) + (t >> 4)], 0), pages - 1);
        off = (((size_t)page * a.Hkv + cu.hk) * 16 + (t & 15)) * D;
      } else {
        off = (((size_t)row * (own ? a.Lmax : a.prefix_cap) + t) * a.Hkv + cu.hk) * D;
      }
      ks[(i / D) * DS + i % D] = kb[off + i % D];
      vs[(i / D) * DS + i % D] = vb[off + i % D];
    }
    __syncthreads();
    for (int i = tid; i < R * TK; i += 256) {
      const int r = i / TK, t = i % TK, gr = cu.rt * R + r;
      const int lim = own ? cu.L - a.k + (gr % kg) / (kg / a.k) : cu.L - 1;
      double s = -INFINITY;
      if (gr < cu.rows && t < here && t0 + t <= lim) {
        double acc = 0.0;
        for (int e = 0; e < D; ++e) acc = fma((double)qs[r * DS + e], (double)ks[t * DS + e], acc);
        s = acc * (double)a.scale;
      }
      ps[r][t] = s;
    }
    __syncthreads();
    if (tid < R) {
      double mx = st[tid][0];
      for (int t = 0; t < TK; ++t) mx = fmax(mx, ps[tid][t]);
      const double f = st[tid][0] == -INFINITY ? 0.0 : exp(st[tid][0] - mx);
      double sum = st[tid][1] * f;
      for (int t = 0; t < TK; ++t) {
        const double p = mx == -INFINITY ? 0.0 : exp(ps[tid][t] - mx);
        ps[tid][t] = p;
        sum += p;
      }
      st[tid][0] = mx;
      st[tid][1] = sum;
      st[tid][2] = f;
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) {
      const int i = tid + e * 256, r = i / D, ch = i % D;
      double acc = o[e] * st[r][2];
      for (int t = 0; t < here; ++t) {
        const double p = ps[r][t];
        acc = fma(p, p != 0.0 ? (double)vs[t * DS + ch] : 0.0, acc);   // a zero weight adds nothing
      }
      o[e] = acc;
    }
    fresh = cu.t + 1 == cu.nt;
    if (fresh || n + 1 == n1) {
      const size_t base = part_row<R>(a, own, cu.pair, wg);
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const int i = tid + e * 256, r = i / D;
        if (cu.rt * R + r < cu.rows) a.part_o[(base + r) * D + i % D] = st[r][1] > 0.0 ? (float)(o[e] / st[r][1]) : 0.f;
      }
      if (tid < R && cu.rt * R + tid < cu.rows)
        a.part_lse[base + tid] =
            st[tid][1] > 0.0 ? (float)((st[tid][0] + log(st[tid][1])) * 1.4426950408889634) : -INFINITY;
    }
    if (n + 1 < n1) advance<R>(a, cu);
  }
}

// ------------------------------------------------------------------ merge
// One wave per output row.  The tiles [U, U + nt) of a pair lie with work-groups
// owner(U) .. owner(U + nt - 1), owner(n) = floor(((n + 1) G - 1) / T), each of
// which wrote one partial (with fewer tiles than work-groups, each owner did).  Candidates of the prefix pair, then of the own pair,
// are taken 32 at a time: lanes 0..31 load their lse while each half-wave loads
// the outputs of 16 of them (4 channels per lane), and the chunk's weights
// 2^(lse - max) rescale a running sum.  Every shuffle runs on all lanes.
template <int ROWS>
__global__ __launch_bounds__(256) void shared_merge(SharedArgs a, int G) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const long long orow = (long long)blockIdx.x * 4 + w;
  if (orow >= (long long)a.B * a.k * a.Hq) return;
  const int D = a.D, g = a.Hq / a.Hkv;
  const int h = (int)(orow % a.Hq), bj = (int)(orow / a.Hq);
  const int b = bj / a.k;
  const int hk = h / g;
  const int r_own = (bj - b * a.k) * g + (h - hk * g);

  // tiles before, key tiles, pair and row of the prefix pair and of the own pair
  int U[2] = {0, 0}, nt[2] = {0, 0}, pair[2] = {0, 0}, lr[2] = {0, 0};
  Carry c;
  for (int u0 = 0; u0 < a.G + a.B; u0 += 64) {
    const Span s = scan_units<ROWS>(a, u0, c);
    const int u = u0 + lane;
    const bool is_group = u < a.G && s.un.first <= b && b < s.un.end;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const unsigned long long hit = __ballot(kind == 0 ? is_group : u == a.G + b);
      if (hit == 0ull) continue;
      const int f = __builtin_ctzll(hit);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
      const int rows = of(s.un.rows), RT = row_tiles(rows, ROWS);
      const int r = kind == 0 ? (b - of(s.un.first)) * a.k * g + r_own : r_own;
      const int x = hk * RT + r / ROWS;
      nt[kind] = tiles_of(of(s.un.L));
      U[kind] = of(s.t_before) + x * nt[kind];
      pair[kind] = kind == 0 ? of(s.p_before) + x : b * a.Hkv * RT + x;
      lr[kind] = r - r / ROWS * ROWS;
    }
  }
  const int T = c.tiles;
  auto owner = [&](int n) { return (int)((((long long)n + 1) * G - 1) / T); };
  const bool sparse = T < G;   // then a work-group has one tile or none: a candidate per tile
  int wf[2] = {0, 0}, nc[2] = {0, 0};
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    if (nt[kind] == 0) continue;
    wf[kind] = owner(U[kind]);
    nc[kind] = sparse ? nt[kind] : owner(U[kind] + nt[kind] - 1) - wf[kind] + 1;
  }
  auto writer = [&](int kind, int i) { return sparse ? owner(U[kind] + i) : wf[kind] + i; };
  const int half = lane >> 5, d4 = lane & 31;
  const bool active = d4 < D / 4;
  floatx4 acc = {0.f, 0.f, 0.f, 0.f};
  float mx = -INFINITY, wsum = 0.f;
  const int ncand = nc[0] + nc[1];
  for (int c0 = 0; c0 < ncand; c0 += 32) {
    const int n = min(32, ncand - c0);
    // partial row of candidate c0 + i
    auto prow = [&](int i) {
      const int cand = c0 + i;
      const bool own = cand >= nc[0];
      return own ? part_row<ROWS>(a, true, pair[1], writer(1, cand - nc[0])) + lr[1]
                 : part_row<ROWS>(a, false, pair[0], writer(0, cand)) + lr[0];
    };
    const float ls = lane < n ? a.part_lse[prow(lane)] : -INFINITY;
    floatx4 po[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int j = 2 * i + half;
      po[i] = floatx4{0.f, 0.f, 0.f, 0.f};
      if (j < n && active) po[i] = *reinterpret_cast<const floatx4*>(a.part_o + prow(j) * D + d4 * 4);
    }
    float cm = ls;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) cm = fmaxf(cm, __shfl_xor(cm, off, 64));
    const float nm = fmaxf(mx, __shfl(cm, 0, 64));
    if (nm == -INFINITY) continue;             // no key in any partial so far (uniform)
    const float keep = mx == -INFINITY ? 0.f : exp2f(mx - nm);
    const float wl = ls == -INFINITY ? 0.f : exp2f(ls - nm);
    float ws = wl;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) ws += __shfl_xor(ws, off, 64);
    wsum = wsum * keep + __shfl(ws, 0, 64);
    acc = acc * keep;
#pragma unroll
    for (int i = 0; i < 16; ++i) acc += __shfl(wl, 2 * i + half, 64) * po[i];
    mx = nm;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], 32, 64);
  const float inv = wsum > 0.f ? 1.f / wsum : 0.f;
  if (half == 0 && active) {
    const floatx4 v = acc * inv;
    if (a.out_bf16) {
      Pack8 pk;
#pragma unroll
      for (int e = 0; e < 4; ++e) pk.b[e] = float_to_bf16(v[e]);
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + (size_t)orow * D + d4 * 4) = u32x2{pk.u[0], pk.u[1]};
    } else {
      *reinterpret_cast<floatx4*>(static_cast<float*>(a.out) + (size_t)orow * D + d4 * 4) = v;
    }
  }
  if (a.lse != nullptr && lane == 0) a.lse[orow] = wsum > 0.f ? (mx + log2f(wsum)) * kLn2 : -INFINITY;
}

template <int D, int NW, int RB, int NBUF>
hipError_t launch_bf16(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  if (a.out_bf16)
    hipLaunchKernelGGL((shared_stream_bf16<D, NW, RB, NBUF, false>), dim3(p.wgs), dim3(NW * 64), 0, st, a, p.wgs);
  else
    hipLaunchKernelGGL((shared_stream_bf16<D, NW, RB, NBUF, true>), dim3(p.wgs), dim3(NW * 64), 0, st, a, p.wgs);
  return hipGetLastError();
}

template <int ROWS>
hipError_t launch_merge(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  const long long rows = (long long)a.B * a.k * a.Hq;
  hipLaunchKernelGGL(shared_merge<ROWS>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st, a, p.wgs);
  return hipGetLastError();
}

}  // namespace

SharedPlan plan_shared(int B, int k, int Hq, int Hkv, int D, int G, int prefix_cap, int cap, int dtype, int cus) {
  SharedPlan p{};
  const int kg = k * (Hq / Hkv);
  const long long rows = (long long)B * kg;     // of a KV head
  cus = std::max(1, cus);
  int per_cu;
  if (dtype == 0) {
    p.rows_wg = kRowsF32;
    per_cu = 4;
  } else {
    // rows of an average group; a wave of two 16-row blocks halves the LDS reads
    // per product, eight such waves halve the HBM reads per row again
    const long long avg = (rows + G - 1) / G;
    p.rows_wg = avg <= 64 ? 64 : avg <= 128 ? 128 : 256;
    per_cu = p.rows_wg == 256 ? 1 : 2;
  }
  p.rows_own = std::min((kg + 15) / 16 * 16, p.rows_wg);
  const int own_tiles = (kg + p.rows_wg - 1) / p.rows_wg;
  const long long prefix_pairs = Hkv * (rows / p.rows_wg + G);
  const long long own_pairs = (long long)B * Hkv * own_tiles;
  const long long tiles = prefix_pairs * ((prefix_cap + kTile - 1) / kTile) +
                          own_pairs * ((cap + kTile - 1) / kTile);
  p.ok = tiles < (1LL << 30);
  p.wgs = (int)std::max(1LL, std::min((long long)cus * per_cu, tiles / 4));
  p.own_base = (prefix_pairs + p.wgs) * p.rows_wg;
  p.part_rows = (size_t)p.own_base + (size_t)(own_pairs + p.wgs) * p.rows_own;
  p.workspace_bytes = p.part_rows * ((size_t)D + 1) * sizeof(float);
  return p;
}

hipError_t launch_shared(const SharedArgs& a, const SharedPlan& p, int dtype, hipStream_t st) {
  hipError_t e;
  if (dtype == 0) {
    if (a.D == 128)
      hipLaunchKernelGGL(shared_stream_f32<128>, dim3(p.wgs), dim3(256), 0, st, a, p.wgs);
    else
      hipLaunchKernelGGL(shared_stream_f32<64>, dim3(p.wgs), dim3(256), 0, st, a, p.wgs);
    e = hipGetLastError();
    return e != hipSuccess ? e : launch_merge<kRowsF32>(a, p, st);
  }
  if (p.rows_wg == 64) {
    e = a.D == 128 ? launch_bf16<128, 4, 1, 4>(a, p, st) : launch_bf16<64, 4, 1, 8>(a, p, st);
    return e != hipSuccess ? e : launch_merge<64>(a, p, st);
  }
  if (p.rows_wg == 128) {
    e = a.D == 128 ? launch_bf16<128, 4, 2, 4>(a, p, st) : launch_bf16<64, 4, 2, 8>(a, p, st);
    return e != hipSuccess ? e : launch_merge<128>(a, p, st);
  }
  e = a.D == 128 ? launch_bf16<128, 8, 2, 8>(a, p, st) : launch_bf16<64, 8, 2, 8>(a, p, st);
  return e != hipSuccess ? e : launch_merge<256>(a, p, st);
}

}  // namespace sd
