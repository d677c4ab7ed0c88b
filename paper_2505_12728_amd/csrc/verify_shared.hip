// Attention of drafted blocks whose sequences share long prefixes: the B
// sequences lie in groups, every row of a group sees the group's prefix in
// full and, causal inside the block, its own sequence's cache behind it.
//
// Mathematics.  With s_t = scale q . K_t over the prefix's and the visible
// own keys, out = sum_t exp(s_t) V_t / sum_t exp(s_t).  Softmax statistics
// (m, l, O) over disjoint key sets combine exactly, so that a prefix is
// attended once by all rows of its group (S k g rows of a KV head: S
// sequences, k block positions, g query heads) and its keys and values are
// read once for each tile of those rows (128 or 256 of them, 16 for fp32), not
// once per sequence.  Tiles of one prefix run at different times on different
// XCDs: what they read again comes from the memory-side cache at best.
//
// Bound: 4 D operations per (row, key) against 4 D bytes per key and KV head
// (bf16), so HBM up to about 300 rows per KV head and the matrix cores beyond.
//
// Kernel 1 (stream).  Units are the groups' prefixes, then the sequences' own
//   caches; a unit's rows in tiles of ROWS and its KV heads give pairs; the key
//   tiles of all pairs form one list, of which each work-group of a fixed grid
//   takes an equal contiguous range.  Ragged lengths and groups are balanced to a
//   tile, and lengths and groups are read on the device alone.  A tile's keys and
//   values pass through LDS once for all ROWS rows:  S^T = K Q^T, online softmax
//   in fp32 (base 2), O^T += V^T P^T.  Where its range leaves a pair, a work-group
//   writes the segment's partial: its normalised output, its maximum and its sum.
// Kernel 2 (merge).  Finds the partials of a row's prefix pair and of its own pair
//   from the same arithmetic and combines them.  Maximum and sum come apart: a
//   log-sum-exp in one float would be off by half a step of its own size, 5e-6 of
//   a partial's weight at scores of 100, 1e-3 at 30000.
//
// P goes into the second product as a sum of bf16 terms.  fp32 outputs take three
// (all 24 bits of p, eight each, three products): two would leave 2e-6 of the
// output, where fp32 products leave 4e-7, and cost 14% less where the matrix cores
// bound (16 blocks of 6 x 4 rows, 16001 keys: 61 us in two terms, 70 in three).
// bf16 outputs take two (16 bits): the output's own rounding is then all that is
// lost, 1.7e-3 of rms, where a single term left 2.3e-3 and 2^-9 of |V| in outputs
// that cancel, and took 278 us for 369 (1024 rows over 65500 keys).  The row sums
// add the fp32 values.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "launch.hpp"

namespace sd {
namespace {

constexpr int kTileF32 = 32, kTile = 64;   // keys per tile (fp32, bf16)
constexpr int kRowsF32 = 16;               // rows per work-group (fp32)
// Places that the list gives to a tile and to the start of a pair (its queries'
// latency, the partial of the one before), so that equal ranges take equal times.
// On the matrix cores, in thirds of a tile whose rows are all there (measured with P
// in one term for bf16 outputs, when such a tile took about 2.2 us): a tile with
// half of them or fewer takes two (1.4 us with fp32 outputs, 1.3 in tiles of 256
// rows), a start six, which one-tile pairs need, whose latencies nothing hides (3.9
// us; pairs of 11 tiles 2.2).  Whole tiles for all and two for a start: own caches of
// 24 rows and 700 keys took 39 us where the prefixes' work-groups took 60 (the call
// 73.5 us, 70.5 so); three thirds for a start: 1024 rows with 64 own keys 378 us
// against 330.
constexpr int kWhole = 3, kStartPlaces = 6;
constexpr int start_places(int rows_wg) { return rows_wg == kRowsF32 ? 0 : kStartPlaces; }
constexpr int most_places(int rows_wg) { return rows_wg == kRowsF32 ? 1 : kWhole; }
__host__ __device__ constexpr int tile_places(int rows_wg, int rows) {   // of a unit of `rows` rows
  return rows_wg == kRowsF32 ? 1 : 2 * rows <= rows_wg ? 2 : kWhole;
}
// Rows in all up to which four merge waves share a row (224 rows: 23.0 us for the
// call with one wave a row, 17.9 so; 512: 58.6 and 55.8; 1792: 33.2 and 34.6), and
// waves beyond which each takes several rows.
constexpr int kSplitRows = 1024, kMergeWaves = 8192;
constexpr float kHeadroom = 24.f;   // log2 of the largest weight before the maximum is raised

typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(1))) const void gbl_cvoid;
typedef const __attribute__((address_space(4))) int32_t cint32;   // scalar loads

// Inclusive scan over the wave's 64 lanes by DPP moves (four shifts inside the
// rows of 16 lanes, then the rows' last lanes to the rows behind), a tenth of
// the latency of shuffles through LDS.  op(0, x) = x.
template <typename Op>
__device__ __forceinline__ int wave_scan(int v, Op op) {
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));   // row_shr:1
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));   // row_shr:2
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));   // row_shr:4
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));   // row_shr:8
  v = op(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false));   // row_bcast:15
  return op(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false));   // row_bcast:31
}
__device__ __forceinline__ int last_lane(int v) { return __builtin_amdgcn_readlane(v, 63); }

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

template <int TK>
__device__ __forceinline__ int tiles_of(int L) {
  return (L + TK - 1) / TK;
}
__device__ __forceinline__ int row_tiles(int rows, int per) { return (rows + per - 1) / per; }

// A tile of the list
struct Cursor {
  int n;             // its place
  int u;             // unit
  int hk, rt, t;     // KV head, row tile, key tile
  int nt, RT;        // key tiles and row tiles of the unit
  int wt;            // places of one of its tiles
  int L, rows, first, end;
  int pair;          // pairs of the same kind (prefix or own) before this one
};

// What a scan over the units finds: lane l holds unit u0 + l.
struct Span {
  Unit un;
  int places, pairs;        // of this unit
  int n_before, p_before;   // before it
};

// Units u0 .. u0 + 63 with their exclusive sums, given the sums and the group
// bound carried from the units before.  Group bounds are made monotone by a
// running maximum, so that no sequence is in two groups.
struct Carry {
  int places = 0, pairs = 0, bound = 0;
};
template <int ROWS, int TK>
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
  if (u0 < a.G) bound = max(wave_scan(bound, [](int x, int y) { return max(x, y); }), c.bound);
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
  c.bound = max(c.bound, last_lane(bound));
  s.pairs = a.Hkv * row_tiles(s.un.rows, ROWS);
  s.places = s.un.L > 0 ? s.pairs * (tiles_of<TK>(s.un.L) * tile_places(ROWS, s.un.rows) + start_places(ROWS)) : 0;
  auto add = [](int x, int y) { return x + y; };
  const int ti = wave_scan(s.places, add), pi = wave_scan(s.pairs, add);
  s.n_before = c.places + ti - s.places;
  s.p_before = c.pairs + pi - s.pairs;
  c.places += last_lane(ti);
  c.pairs += last_lane(pi);
  return s;
}

// place of the tile behind cu
template <int ROWS>
__device__ __forceinline__ int place_behind(const Cursor& cu) {
  return cu.n + cu.wt + (cu.t + 1 == cu.nt ? start_places(ROWS) : 0);
}

// next tile of the list; behind the last one a place past the list
template <int ROWS, int TK>
__device__ __forceinline__ void advance(const SharedArgs& a, Cursor& cu) {
  cu.n += cu.wt;
  if (++cu.t < cu.nt) return;
  cu.t = 0;
  cu.n += start_places(ROWS);
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
    cu.nt = tiles_of<TK>(cu.L);
    cu.RT = row_tiles(cu.rows, ROWS);
    cu.wt = tile_places(ROWS, cu.rows);
    if (cu.nt == 0 || cu.RT == 0) cu.pair += a.Hkv * cu.RT;
  } while ((cu.nt == 0 || cu.RT == 0) && cu.u < a.G + a.B);
}

// Cursor of the first tile at place n or behind it (a tile's place is its first),
// from the span that holds place n; behind the list's last tile that is a place
// past the list.  The pair counts its kind only: own pairs start at 0 again.
template <int ROWS, int TK>
__device__ __forceinline__ Cursor tile_in(const SharedArgs& a, const Span& s, int u0, int n) {
  constexpr int kStart = start_places(ROWS);
  const int f = __builtin_ctzll(__ballot(s.n_before + s.places > n));
  auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
  Cursor cu;
  cu.u = u0 + f;
  cu.L = of(s.un.L);
  cu.rows = of(s.un.rows);
  cu.first = of(s.un.first);
  cu.end = of(s.un.end);
  cu.nt = tiles_of<TK>(cu.L);
  cu.RT = row_tiles(cu.rows, ROWS);
  cu.wt = tile_places(ROWS, cu.rows);
  const int rem = n - of(s.n_before), len = cu.nt * cu.wt + kStart;
  const int x = rem / len;
  const int t = (max(rem - x * len - kStart, 0) + cu.wt - 1) / cu.wt;
  cu.t = min(t, cu.nt - 1);
  cu.n = of(s.n_before) + x * len + kStart + cu.t * cu.wt;
  cu.hk = x / cu.RT;
  cu.rt = x - cu.hk * cu.RT;
  cu.pair = cu.u < a.G ? of(s.p_before) + x : (cu.u - a.G) * a.Hkv * cu.RT + x;
  if (t == cu.nt) advance<ROWS, TK>(a, cu);    // n lies inside the pair's last tile
  return cu;
}

// The range of work-group w of G: its first tile and the place behind its last;
// false: no tile.  In scalar registers (the compiler cannot see that the scan
// ends alike on every lane), so that its bookkeeping stays off the vector unit.
template <int ROWS, int TK>
__device__ __forceinline__ bool first_tile(const SharedArgs& a, int w, int G, Cursor* first, int* behind) {
  const int units = a.G + a.B;
  Carry c;
  const Span s0 = scan_units<ROWS, TK>(a, 0, c);
  for (int u0 = 64; u0 < units; u0 += 64) scan_units<ROWS, TK>(a, u0, c);
  const int T = __builtin_amdgcn_readfirstlane(c.places);
  const int n0 = (int)((long long)T * w / G), n1 = (int)((long long)T * (w + 1) / G);
  if (n0 >= n1) return false;
  Cursor cu{};
  if (units <= 64) {
    cu = tile_in<ROWS, TK>(a, s0, 0, n0);
  } else {
    Carry d;
    for (int u0 = 0; u0 < units; u0 += 64) {
      const Span s = scan_units<ROWS, TK>(a, u0, d);
      if (n0 >= d.places) continue;
      cu = tile_in<ROWS, TK>(a, s, u0, n0);
      break;
    }
  }
  int* f[] = {&cu.n, &cu.u, &cu.hk, &cu.rt, &cu.t, &cu.nt, &cu.RT, &cu.wt, &cu.L, &cu.rows, &cu.first, &cu.end, &cu.pair};
#pragma unroll
  for (int* x : f) *x = __builtin_amdgcn_readfirstlane(*x);
  *first = cu;
  *behind = n1;
  return cu.n < n1;
}

// First row of the partial that work-group w writes for the pair of cursor cu:
// along the list both the pair and w only grow, so that pair + w is distinct
// for every segment.  Own pairs have an area of their own, rows_own each.
template <int ROWS>
__device__ __forceinline__ size_t part_row(const SharedArgs& a, bool own, int pair, int w) {
  return own ? (size_t)a.own_base + (size_t)(pair + w) * a.rows_own : (size_t)(pair + w) * ROWS;
}

// Partials and their merge: float32, maxima in log2 units; float64 for fp32
// inputs, maxima of the scores themselves.
template <typename T, int N>
using Vec = T __attribute__((ext_vector_type(N)));
template <int ROWS>
using PartT = std::conditional_t<ROWS == kRowsF32, double, float>;
__device__ __forceinline__ float weight_of(float x) { return exp2f(x); }
__device__ __forceinline__ double weight_of(double x) { return exp(x); }
__device__ __forceinline__ float lse_of(float m, float l) { return (m + log2f(l)) * kLn2; }
__device__ __forceinline__ float lse_of(double m, double l) { return (float)(m + log(l)); }

// output row (flat over [B, k, Hq]) of row r of a unit that starts at sequence `first`
__device__ __forceinline__ int out_row(const SharedArgs& a, int first, int hk, int r) {
  const int g = a.Hq / a.Hkv;
  const int q = r / g;
  return (first * a.k + q) * a.Hq + hk * g + (r - q * g);
}

// ------------------------------------------------------------ bf16 stream
// Eight waves of RB 16-row blocks on 64-key tiles.  A step computes the scores
// of tile x + 1 under the exponentials of tile x, then P V of tile x under the
// lane maxima of tile x + 1; the running maxima are raised (rarely) after it.  It
// runs in groups of four LDS fragments: a group's reads are issued one group
// ahead and waited for by count.  K and V have rings of four slots: a tile's copy
// has two steps to land.
//   64 rows over 65500 keys of 8 heads of 128 (268 MB): 47 us, 5.7 TB/s, HBM.
//   1024 rows there, bf16 out (275 GFLOP in the formula, 413 in two terms): 350
// us, 1180 TFLOP/s of products, where one of 8192^3 reaches 1346.  Matrix cores
// busy 54%, no LDS conflicts.  A step's 96 matrix instructions take 1536 cycles of
// a wave, its 230 vector ones (32 of them exponentials) about 1300; the two waves
// of a SIMD overlap them little.
template <int V>
struct Const {
  static constexpr int value = V;
};
template <int I, int N, typename F>
__device__ __forceinline__ void unrolled(F&& f) {
  if constexpr (I < N) {
    f(Const<I>{});
    unrolled<I + 1, N>(f);
  }
}

template <int D, int RB, int TERMS>
__global__ __launch_bounds__(512, 2) void shared_stream_bf16(SharedArgs a, int G) {
  constexpr int NW = 8, TK = kTile, NBUF = 4;
  constexpr int DC = D / 32;                   // 32-channel slices (S^T = K Q^T)
  constexpr int DB = D / 16;                   // 16-channel blocks (O^T)
  constexpr int PK = D / 8;                    // 16-byte pieces per key row
  constexpr int ROW = D * 2;
  constexpr int HALF = TK * ROW;               // a tile's K (or V)
  constexpr int KEYS = 64 / PK;                // keys of one 64-lane copy
  constexpr int COPIES = TK / KEYS / NW;       // per wave and half: 8 keys a wave
  constexpr int TILE_COPIES = 2 * COPIES;
  constexpr int ROWS = NW * RB * 16;
  constexpr int KPG = 4 / DC;                  // 16-key blocks of a score group
  constexpr int NQK = 4 / KPG, NPVH = DB / 4, NG = NQK + 2 * NPVH;
  static_assert(NBUF * HALF <= 65536, "ring slots within the LDS instructions' offsets");
  static_assert(COPIES * KEYS == 8, "a wave copies 8 keys, which lie in one page");
  __shared__ __align__(16) unsigned char ring[2][NBUF * HALF];   // K, V

  const int lane = threadIdx.x & 63, G4 = lane >> 4, c = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = blockIdx.x;
  Cursor cc;
  int n1;
  if (!first_tile<ROWS, TK>(a, wg, G, &cc, &n1)) return;

  // Copies.  This wave takes keys 8 w .. 8 w + 7 of a tile's K and V; a lane's
  // 16-byte piece goes to LDS slot piece ^ lds_swizzle(key).  Keys past the
  // unit's length re-read its last key (masked).  cur: the tile copied next.
  // (The swizzle of key + 4 differs in bit 3 where a wave takes two copies.)
  const int ckey = lane / PK;
  const uint32_t cpiece = ((lane % PK) ^ lds_swizzle<PK>(w * 8 + ckey)) * 16;
  static_assert(COPIES == 1 || lds_swizzle<PK>(4) == 8, "second copy's piece");
  Cursor ic = cc;
  const unsigned char *ck = nullptr, *cv = nullptr;   // of the pair: its keys and values
  cint32* cpages = nullptr;                    // its row of the page table
  int cpool = 0, cstep = 0, clim = 0;          // pages of the pool, bytes between keys, last key of the 8
  size_t cbase = 0;                            // offset of the wave's keys
  auto enter_pair = [&]() {
    const bool own = ic.u >= a.G;
    const int row = own ? ic.first : ic.u;
    const int32_t* table = own ? a.page_table : a.prefix_table;
    size_t at;
    if (table != nullptr) {
      cpages = (cint32*)(table + (size_t)row * (own ? a.max_pages : a.prefix_pages));
      cpool = own ? a.num_pages : a.prefix_num_pages;
      cstep = ROW;
      at = (size_t)ic.hk * (16 * ROW);
    } else {
      cpages = nullptr;
      cstep = a.Hkv * ROW;
      at = ((size_t)row * (own ? a.Lmax : a.prefix_cap) * a.Hkv + ic.hk) * ROW;
    }
    ck = static_cast<const unsigned char*>(own ? a.k_cache : a.k_prefix) + at;
    cv = static_cast<const unsigned char*>(own ? a.v_cache : a.v_prefix) + at;
  };
  auto enter_tile = [&]() {
    const int key0 = min(ic.t * TK + w * 8, (ic.L - 1) & ~7);
    clim = ic.L - 1 - key0;
    if (cpages != nullptr) {
      const int page = min(max((int)cpages[key0 >> 4], 0), cpool - 1);
      cbase = (size_t)page * (size_t)(a.Hkv * 16 * ROW) + (key0 & 15) * ROW;
    } else {
      cbase = (size_t)key0 * (size_t)cstep;
    }
  };
  // the copy of one tile, and the step to the next; past the range the last one
  // is copied again
  auto copy_next = [&](int slot) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const size_t off = cbase + ((uint32_t)min(ckey + i * KEYS, clim) * (uint32_t)cstep + (cpiece ^ (i * 128)));
      const int at = slot * HALF + (w * COPIES + i) * 1024;
      __builtin_amdgcn_global_load_lds((gbl_cvoid*)(ck + off), (lds_void*)(ring[0] + at), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gbl_cvoid*)(cv + off), (lds_void*)(ring[1] + at), 16, 0, 0);
    }
    if (place_behind<ROWS>(ic) < n1) {
      advance<ROWS, TK>(a, ic);
      if (ic.t == 0) enter_pair();
      enter_tile();
    }
  };

  // fragment addresses for the first 16 keys of slot 0 (the swizzle depends on
  // key % 16 only, so further blocks and slots are offsets).  K: 16 keys x one
  // piece; V, transposed: lane j of group G4 addresses key 4 G4 + j / 4 at
  // channels db * 16 + 4 (j % 4) and receives 4 keys at channel db * 16 + c.
  // Blocks db and db + 4 differ in bit 7 of the address (128 bytes of a row).
  uint32_t kaddr[DC], vaddr[4];
#pragma unroll
  for (int dc = 0; dc < DC; ++dc)
    kaddr[dc] = lds_addr(ring[0]) + c * ROW + (((dc * 4 + G4) ^ lds_swizzle<PK>(c)) * 16);
#pragma unroll
  for (int db = 0; db < 4; ++db) {
    const int key = 4 * G4 + (c >> 2), ch = db * 16 + 4 * (c & 3);
    vaddr[db] = lds_addr(ring[1]) + key * ROW + (((ch >> 3) ^ lds_swizzle<PK>(key)) * 16) + (ch & 7) * 2;
  }

  // Segment state: queries (B operand of S^T = K Q^T), last visible keys, running
  // (max, sum, O^T) and the raw scores of the tile whose turn it is.  The scale
  // enters the exponents as exp2(S sl2 - m); a negative one is folded into the
  // queries.
  bf16x8 qf[RB][DC];
  int lim[RB];
  float m[RB], l[RB];
  floatx4 o[RB][DB], ex[4][RB];
  const bool neg = a.scale_log2 < 0.f;
  const float sl2 = fabsf(a.scale_log2);
  const int g = a.Hq / a.Hkv, kg = a.k * g;
  // queries of the pair under cursor cu; true if this wave has rows of it
  auto load_rows = [&](const Cursor& cu) {
    const int r0 = cu.rt * ROWS + w * RB * 16;
    if (r0 >= cu.rows) return false;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int r = r0 + rb * 16 + c;
      const bool here = r < cu.rows;
      const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) +
                                                        (size_t)out_row(a, cu.first, cu.hk, here ? r : r0) * D);
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) {
        Pack8 pk;
        pk.u = src[dc * 4 + G4];
        qf[rb][dc] = pk.b;
      }
    }
    return true;
  };

  u32x4 xr[2][4];
  u32x2 vr[2][4][2];
  // LDS reads of group gr, or the ties that make their values usable
  auto reads = [&](auto gtag, auto ph_next, auto ph_here, uint32_t dn, uint32_t dh, auto tie_only) {
    constexpr int gr = decltype(gtag)::value, PN = decltype(ph_next)::value, PH = decltype(ph_here)::value;
    if constexpr (gr < NQK) {
      unrolled<0, 4>([&](auto jt) {
        constexpr int j = decltype(jt)::value, kb = gr * KPG + j / DC;
        if constexpr (decltype(tie_only)::value)
          tie(xr[gr & 1][j]);
        else
          xr[gr & 1][j] = lds_read_b128_off<PN * HALF + kb * 16 * ROW>(kaddr[j % DC] + dn);
      });
    } else if constexpr (gr < NG) {
      constexpr int q = gr - NQK, hf = q / NPVH, pb = q % NPVH;
      unrolled<0, 4>([&](auto dt) {
        constexpr int d = decltype(dt)::value;
        if constexpr (decltype(tie_only)::value) {
          tie(vr[gr & 1][d][0]);
          tie(vr[gr & 1][d][1]);
        } else {
          const uint32_t at = (vaddr[d] ^ (pb * 128)) + dh;
          vr[gr & 1][d][0] = lds_read_tr16_b64_off<PH * HALF + hf * 32 * ROW>(at);
          vr[gr & 1][d][1] = lds_read_tr16_b64_off<PH * HALF + hf * 32 * ROW + 16 * ROW>(at);
        }
      });
    }
  };
  // scores of score group gr from its fragments
  auto scores = [&](auto gtag, floatx4 (&s)[4][RB]) {
    constexpr int gr = decltype(gtag)::value;
#pragma unroll
    for (int kk = 0; kk < KPG; ++kk) {
      const int kb = gr * KPG + kk;
#pragma unroll
      for (int dc = 0; dc < DC; ++dc) {
        Pack8 pk;
        pk.u = xr[gr & 1][kk * DC + dc];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          s[kb][rb] = mfma_bf16(pk.b, qf[rb][dc], dc == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : s[kb][rb]);
      }
    }
  };
  auto lane_max = [&](const floatx4& s, float top) {
    return fmaxf(fmaxf(fmaxf(fmaxf(top, s[0]), s[1]), s[2]), s[3]);   // two instructions
  };
  // (max, sum) of the softmax stand apart from S by exponents S sl2 - m.  Maxima are
  // taken over them, not over S: the compiler knows a fused product's result for
  // quiet and needs no instruction to make it so
  auto exponents = [&](floatx4& s, int rb) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = fmaf(s[i], sl2, -m[rb]);
  };
  // the same over the keys that row block rb may see, s those from key t on: a
  // masked score that exceeds all visible ones by 2^126 would leave them no weight
  auto seen_max = [&](floatx4 s, int t, int rb, float top) {
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = t + i > lim[rb] ? -FLT_MAX : s[i];
    return lane_max(s, top);
  };

  // One step, tile t0 / TK of the segment at ring step x.  NEXT: there is a tile
  // behind it in the segment.  MASK: a row's last visible key may lie in the tile.
  // PH: x % NBUF where known (the slots then sit in the instructions' offsets),
  // else -1.
  auto step = [&](int x, int t0, auto ph_tag, auto next_tag, auto mask_tag) {
    constexpr int PH = decltype(ph_tag)::value;
    constexpr bool NEXT = decltype(next_tag)::value, MASK = decltype(mask_tag)::value;
    constexpr int PN = PH >= 0 ? (PH + 1) % NBUF : 0, P0 = PH >= 0 ? PH : 0;
    const uint32_t dh = PH >= 0 ? 0u : (uint32_t)(x % NBUF) * HALF;
    const uint32_t dn = PH >= 0 ? 0u : (uint32_t)((x + 1) % NBUF) * HALF;
    constexpr int G0 = NEXT ? 0 : NQK;         // the last tile has no scores to form
    Pack8 p16[TERMS][2][RB];                   // weights as sums of bf16 terms
    floatx4 sn[4][RB];
    float lm[RB];
    auto weights = [&](int kb) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = fast_exp2(ex[kb][rb][i]);
          if constexpr (MASK) {
            if (t0 + kb * 16 + 4 * G4 + i > lim[rb]) p[i] = 0.f;
          }
        }
        // the upper halves of p and of what they leave, exactly; the last of two
        // terms rounded
        float rest[4] = {p[0], p[1], p[2], p[3]};
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
          if (TERMS == 2 && t == 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) p16[t][kb >> 1][rb].b[(kb & 1) * 4 + i] = float_to_bf16(rest[i]);
            continue;
          }
#pragma unroll
          for (int i = 0; i < 4; i += 2)
            p16[t][kb >> 1][rb].u[(kb & 1) * 2 + i / 2] =
                __builtin_amdgcn_perm(__float_as_uint(rest[i + 1]), __float_as_uint(rest[i]), 0x07060302u);
#pragma unroll
          for (int i = 0; i < 4; ++i) rest[i] -= __uint_as_float(__float_as_uint(rest[i]) & 0xffff0000u);
        }
        l[rb] += (p[0] + p[1]) + (p[2] + p[3]);
      }
    };
    // tile x + 1 has landed (its wait leaves tile x + 2's copy under way), tile
    // x - 1's slot is free
    wait_vm_then_barrier<TILE_COPIES>();
    copy_next(PH >= 0 ? (PH + 3) % NBUF : (x + 3) % NBUF);
    reads(Const<G0>{}, Const<PN>{}, Const<P0>{}, dn, dh, Const<0>{});
    if constexpr (!NEXT) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) weights(kb);
    }
    unrolled<G0, NG>([&](auto gtag) {
      constexpr int gr = decltype(gtag)::value;
      reads(Const<gr + 1>{}, Const<PN>{}, Const<P0>{}, dn, dh, Const<0>{});
      lds_wait_n<(gr + 1 < NQK ? 4 : gr + 1 < NG ? 8 : 0)>();
      reads(gtag, Const<PN>{}, Const<P0>{}, dn, dh, Const<1>{});
      if constexpr (gr < NQK) {
        scores(gtag, sn);
#pragma unroll
        for (int kk = 0; kk < KPG; ++kk) weights(gr * KPG + kk);
      } else {
        constexpr int q = gr - NQK, hf = q / NPVH, pb = q % NPVH, per = 4 / (2 * NPVH);
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          Pack8 vv;
          vv.u = u32x4{vr[gr & 1][d][0][0], vr[gr & 1][d][0][1], vr[gr & 1][d][1][0], vr[gr & 1][d][1][1]};
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
#pragma unroll
            for (int t = TERMS - 1; t >= 0; --t)
              o[rb][4 * pb + d] = mfma_bf16(vv.b, p16[t][hf][rb].b, o[rb][4 * pb + d]);
          }
        }
        if constexpr (NEXT) {
#pragma unroll
          for (int kb = q * per; kb < (q + 1) * per; ++kb)
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
              exponents(sn[kb][rb], rb);
              if constexpr (MASK)
                lm[rb] = seen_max(sn[kb][rb], t0 + TK + kb * 16 + 4 * G4, rb, kb == 0 ? -FLT_MAX : lm[rb]);
              else
                lm[rb] = lane_max(sn[kb][rb], kb == 0 ? sn[0][rb][0] : lm[rb]);
            }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (NEXT) {
      // m, raised only where an exponent passes 2^24, cancels in o = O / l and
      // lse = m + log2 l (in log2 units).  The exponents, rounded after the difference, have lost
      // what an m far below the scores dwarfs: the scores are formed again from the
      // tile's fragments, which lie in LDS until step x + 2, and the exponents from
      // the new maximum
      bool over = false;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) over = over || lm[rb] > kHeadroom;
      if (__ballot(over) != 0ull) {
        const uint32_t d1 = (uint32_t)((x + 1) % NBUF) * HALF;
        unrolled<0, NQK>([&](auto gtag) {
          reads(gtag, Const<0>{}, Const<0>{}, d1, 0u, Const<0>{});
          lds_wait();
          reads(gtag, Const<0>{}, Const<0>{}, d1, 0u, Const<1>{});
          scores(gtag, sn);
        });
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
          float top = -FLT_MAX;
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) {
            if constexpr (MASK)
              top = seen_max(sn[kb][rb], t0 + TK + kb * 16 + 4 * G4, rb, top);
            else
              top = lane_max(sn[kb][rb], top);
          }
          top = fmaxf(wave_max_across_groups(top) * sl2, m[rb]);
          const float f = fast_exp2(m[rb] - top);
          l[rb] *= f;
#pragma unroll
          for (int db = 0; db < DB; ++db) o[rb][db] *= f;
          m[rb] = top;
#pragma unroll
          for (int kb = 0; kb < 4; ++kb) exponents(sn[kb][rb], rb);
        }
      }
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) ex[kb][rb] = sn[kb][rb];
    }
  };

  enter_pair();
  enter_tile();
  bool busy = load_rows(cc);
#pragma unroll 1
  for (int i = 0; i < NBUF - 1; ++i) copy_next(i);
  int x = 0;                                   // ring step
  while (true) {
    const int steps = min(cc.nt - cc.t, (n1 - cc.n + cc.wt - 1) / cc.wt);
    const int t_first = cc.t * TK;
    const Cursor seg = cc;
    cc.t += steps - 1;
    cc.n += (steps - 1) * cc.wt;
    const bool more = place_behind<ROWS>(cc) < n1;
    if (more) advance<ROWS, TK>(a, cc);        // the next segment
    if (x == 0) wait_vm_then_barrier<2 * TILE_COPIES>();   // the first tile has landed
    if (busy) {
      if (neg) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
#pragma unroll
          for (int dc = 0; dc < DC; ++dc) {
            Pack8 pk;
            pk.b = qf[rb][dc];
            pk.u ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
            qf[rb][dc] = pk.b;
          }
      }
      // scores of the first tile, and their maxima
      const uint32_t d0 = (uint32_t)(x % NBUF) * HALF;
      unrolled<0, NQK>([&](auto gtag) {
        reads(gtag, Const<0>{}, Const<0>{}, d0, 0u, Const<0>{});
        lds_wait();
        reads(gtag, Const<0>{}, Const<0>{}, d0, 0u, Const<1>{});
        scores(gtag, ex);
      });
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int r = seg.rt * ROWS + (w * RB + rb) * 16 + c;
        lim[rb] = seg.u >= a.G ? seg.L - a.k + r % kg / g : seg.L - 1;
        float top = -FLT_MAX;
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) top = seen_max(ex[kb][rb], t_first + kb * 16 + 4 * G4, rb, top);
        top = wave_max_across_groups(top);
        // no finite score here (none that the row sees, -inf alone, or below the
        // range once scaled): l stays 0, and the first that is one raises m
        m[rb] = fmaxf(top * sl2, -FLT_MAX);
#pragma unroll
        for (int kb = 0; kb < 4; ++kb) exponents(ex[kb][rb], rb);
        l[rb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
    }
    if (!busy) {
      for (int i = 0; i < steps; ++i, ++x) {   // no rows: its copies only
        wait_vm_then_barrier<TILE_COPIES>();
        copy_next((x + 3) % NBUF);
      }
      busy = more && load_rows(cc);
      if (!more) break;
      continue;
    }
    int i = 0;                                 // step of the segment
    // the steps before `open` neither weigh a tile with masked keys nor form the
    // scores of one
    const int seen = seg.u >= a.G ? max(seg.L - a.k + 1, 0) : seg.L;   // keys that all rows see
    const int open = min(seen / TK - 1 - t_first / TK, steps - 1);
    for (; i < open && x % NBUF != 0; ++i, ++x) step(x, 0, Const<-1>{}, Const<1>{}, Const<0>{});
    for (; i + NBUF <= open; i += NBUF, x += NBUF) {
      step(x, 0, Const<0>{}, Const<1>{}, Const<0>{});
      step(x, 0, Const<1>{}, Const<1>{}, Const<0>{});
      step(x, 0, Const<2>{}, Const<1>{}, Const<0>{});
      step(x, 0, Const<3>{}, Const<1>{}, Const<0>{});
    }
    for (; i < open; ++i, ++x) step(x, 0, Const<-1>{}, Const<1>{}, Const<0>{});
#pragma unroll 1
    for (; i < steps - 1; ++i, ++x) step(x, t_first + i * TK, Const<-1>{}, Const<1>{}, Const<1>{});
    step(x, t_first + i * TK, Const<-1>{}, Const<0>{}, Const<1>{});
    ++x;
    int row = c, ch = 4 * G4;                  // (formed here: no registers for them through the steps)
    asm volatile("" : "+v"(row), "+v"(ch));
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float lsum = wave_sum_across_groups(l[rb]);
      const int lr = (w * RB + rb) * 16 + row;
      if (seg.rt * ROWS + lr >= seg.rows) continue;
      const size_t prow = part_row<ROWS>(a, seg.u >= a.G, seg.pair, wg) + lr;
      const float inv = lsum != 0.f ? 1.f / lsum : 0.f;   // (a NaN stays one)
#pragma unroll
      for (int db = 0; db < DB; ++db)
        *reinterpret_cast<floatx4*>(static_cast<float*>(a.part_o) + prow * D + db * 16 + ch) = o[rb][db] * inv;
      if (ch == 0) static_cast<Vec<float, 2>*>(a.part_ml)[prow] = {lsum != 0.f ? m[rb] : -INFINITY, lsum};
    }
    if (!more) break;
    busy = load_rows(cc);
  }
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // no copy may still write this LDS
}

// ------------------------------------------------------------- fp32 stream
// fp32 inputs: scores, softmax, P V and partials in float64.
// The same list with 16 rows per work-group and 32-key tiles.  The segment's
// queries and a tile's keys and values lie in LDS (rows padded by one float);
// row r belongs to the 16 lanes r * 16 ..: each forms two of its scores, its
// maximum and sum go over those lanes by shuffles, and each accumulates D / 16
// of its channels.  A tile is a chain of latencies (load 2.0 us, scores 2.5,
// softmax 0.5, P V 3.2 at 64 channels), which more loads in flight and values
// read whether they weigh or not shorten: 384 rows of each of 8 KV heads of 128
// over 4000 keys 1145 us without them, 721 so.
template <int D>
__global__ __launch_bounds__(256) void shared_stream_f32(SharedArgs a, int G) {
  constexpr int TK = kTileF32, R = kRowsF32, DS = D + 1;
  constexpr int PER = D / 16;                  // channels per lane
  __shared__ float qs[R * DS], ks[TK * DS], vs[TK * DS];
  __shared__ double ps[R][TK + 1];             // weights
  const int tid = threadIdx.x, r = tid >> 4, lane16 = tid & 15;
  const int wg = blockIdx.x;
  Cursor cu;
  int n1;
  if (!first_tile<R, TK>(a, wg, G, &cu, &n1)) return;
  const int kg = a.k * (a.Hq / a.Hkv);
  double o[PER], m = -INFINITY, l = 0.0;
  bool fresh = true;
  while (true) {
    const bool own = cu.u >= a.G;
    const int t0 = cu.t * TK, here = min(TK, cu.L - t0);
    const int row = cu.rt * R + r;             // of the unit
    __syncthreads();                           // the previous tile's reads are done
    if (fresh) {
      for (int i = tid; i < R * D; i += 256) {
        const int qr = cu.rt * R + i / D;
        qs[(i / D) * DS + i % D] =
            qr < cu.rows ? static_cast<const float*>(a.q)[(size_t)out_row(a, cu.first, cu.hk, qr) * D + i % D] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < PER; ++e) o[e] = 0.0;
      m = -INFINITY;
      l = 0.0;
    }
    const int seq = own ? cu.first : cu.u;
    const float* kb = static_cast<const float*>(own ? a.k_cache : a.k_prefix);
    const float* vb = static_cast<const float*>(own ? a.v_cache : a.v_prefix);
    const int32_t* table = own ? a.page_table : a.prefix_table;
    // all of a thread's loads are under way before the first is used
    constexpr int N = TK * D / 256;
    float kx[N], vx[N];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = tid + 256 * n;
      const int t = min(t0 + i / D, cu.L - 1);   // past the length: the last key, masked
      size_t off;
      if (table != nullptr) {
        const int pages = own ? a.num_pages : a.prefix_num_pages;
        const int page = min(max(table[(size_t)seq * (own ? a.max_pages : a.prefix_pages) + (t >> 4)], 0), pages - 1);
        off = (((size_t)page * a.Hkv + cu.hk) * 16 + (t & 15)) * D;
      } else {
        off = (((size_t)seq * (own ? a.Lmax : a.prefix_cap) + t) * a.Hkv + cu.hk) * D;
      }
      kx[n] = kb[off + i % D];
      vx[n] = vb[off + i % D];
    }
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int i = tid + 256 * n;
      ks[(i / D) * DS + i % D] = kx[n];
      vs[(i / D) * DS + i % D] = vx[n];
    }
    __syncthreads();
    const int lim = own ? cu.L - a.k + (row % kg) / (kg / a.k) : cu.L - 1;
    double s[2] = {0.0, 0.0};
#pragma unroll 16
    for (int e = 0; e < D; ++e) {
      const double q = (double)qs[r * DS + e];
#pragma unroll
      for (int i = 0; i < 2; ++i) s[i] = fma(q, (double)ks[(lane16 + 16 * i) * DS + e], s[i]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int t = lane16 + 16 * i;
      s[i] = t < here && t0 + t <= lim ? s[i] * (double)a.scale : -INFINITY;
    }
    double top = fmax(s[0], s[1]);
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) top = fmax(top, __shfl_xor(top, off, 64));
    top = fmax(m, top);
    const double keep = m == -INFINITY ? 0.0 : exp(m - top);
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const double p = s[i] == -INFINITY ? 0.0 : exp(s[i] - top);
      ps[r][lane16 + 16 * i] = p;
      sum += p;
    }
#pragma unroll
    for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor(sum, off, 64);
    l = l * keep + sum;
    m = top;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = keep != 0.0 ? o[e] * keep : 0.0;
#pragma unroll 8
    for (int t = 0; t < TK; ++t) {
      const double p = ps[r][t];
#pragma unroll
      for (int e = 0; e < PER; ++e) {
        const float v = vs[t * DS + lane16 + 16 * e];
        o[e] = fma(p, (double)(p != 0.0 ? v : 0.f), o[e]);   // a zero weight adds nothing
      }
    }
    fresh = cu.t + 1 == cu.nt;
    const bool end = place_behind<R>(cu) >= n1;
    if ((fresh || end) && row < cu.rows) {
      const size_t at = part_row<R>(a, own, cu.pair, wg) + r;
#pragma unroll
      for (int e = 0; e < PER; ++e)
        static_cast<double*>(a.part_o)[at * D + lane16 + 16 * e] = l != 0.0 ? o[e] / l : 0.0;
      // (a sum that is not a number may stand beside a maximum of none: never a partial without keys)
      if (lane16 == 0) static_cast<Vec<double, 2>*>(a.part_ml)[at] = {l == l ? m : l, l};
    }
    if (end) break;
    advance<R, TK>(a, cu);
  }
}

// ------------------------------------------------------------------ merge
// The tiles at places U, U + wt .. of a pair lie with work-groups owner(U) ..
// owner(U + (nt - 1) wt), owner(n) = floor(((n + 1) G - 1) / T), each of which
// wrote one partial (with few places, the owners of its tiles did).  A row's
// candidates are the partials of its prefix pair, then of its own pair.  A wave
// holds the row's channels (D / 64 per lane) and takes 8 candidates at a time:
// their (max, sum) are the same on every lane, so that their weights need no
// exchange between lanes.  Few rows have many candidates each and take the
// four waves of a work-group (SPLIT), joined in LDS; otherwise a wave takes
// `per` rows of one sequence, so that the scan over the units is made once for
// them.  Bound by latency while rows are few, by the partials' bytes beyond.
template <int ROWS, int TK, int D, bool SPLIT>
__global__ __launch_bounds__(256) void shared_merge(SharedArgs a, int G, int per, int wgs_seq) {
  constexpr int CH = D / 64, ROUND = 8;
  using F = PartT<ROWS>;
  // infinite values stay infinite: a zero weight (a round's spare places, too) adds
  // nothing.  On the matrix cores they are NaN already
  constexpr bool kExact = ROWS == kRowsF32;
  __shared__ F part[4][2 + D];                // SPLIT: each wave's max, sum and channels
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int b = blockIdx.x / wgs_seq;
  const int row0 = ((blockIdx.x - b * wgs_seq) * (SPLIT ? 1 : 4) + (SPLIT ? 0 : w)) * per;   // of the k Hq rows of b
  const int rows = a.k * a.Hq, row1 = min(row0 + per, rows);
  const int g = a.Hq / a.Hkv;

  // places before the unit, key tiles, pairs before it, row tiles and first row
  // of the sequence, for the group's prefix (0) and the sequence's own keys (1)
  int before[2] = {0, 0}, nt[2] = {0, 0}, wt[2] = {1, 1}, pairs[2] = {0, 0}, RT[2] = {1, 1}, base[2] = {0, 0};
  Carry c;
  for (int u0 = 0; u0 < a.G + a.B; u0 += 64) {
    const Span s = scan_units<ROWS, TK>(a, u0, c);
    const int u = u0 + lane;
    const bool is_group = u < a.G && s.un.first <= b && b < s.un.end;
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const unsigned long long hit = __ballot(kind == 0 ? is_group : u == a.G + b);
      if (hit == 0ull) continue;
      const int f = __builtin_ctzll(hit);
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, f); };
      RT[kind] = row_tiles(of(s.un.rows), ROWS);
      wt[kind] = tile_places(ROWS, of(s.un.rows));
      nt[kind] = tiles_of<TK>(of(s.un.L));
      before[kind] = of(s.n_before);
      pairs[kind] = kind == 0 ? of(s.p_before) : b * a.Hkv * RT[kind];
      base[kind] = kind == 0 ? (b - of(s.un.first)) * a.k * g : 0;
    }
  }
  const int T = c.places;
  // with fewer places than the work-groups need for a tile each, some between
  // two owners may have none: a candidate per tile, each owner's first one counts
  const bool sparse = T < G * most_places(ROWS);
  // ((n + 1) G - 1) / T: the float64 quotient is off by less than one
  const double inv_t = 1.0 / (double)max(T, 1);
  auto owner = [&](int n) {
    const long long x = (long long)(n + 1) * G - 1;
    const int q = (int)((double)x * inv_t);
    const long long r = x - (long long)q * T;
    return q + (r >= T) - (r < 0);
  };
  for (int row = row0; row < row1; ++row) {
    const int j = row / a.Hq, h = row - j * a.Hq, hk = h / g;
    int U[2], nc[2] = {0, 0}, wf[2] = {0, 0};
    long long first[2] = {0, 0};               // partial row that work-group 0 would write for the pair
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
      const int r = base[kind] + j * g + (h - hk * g);
      const int x = hk * RT[kind] + r / ROWS;
      U[kind] = before[kind] + x * (nt[kind] * wt[kind] + start_places(ROWS)) + start_places(ROWS);
      first[kind] = (long long)part_row<ROWS>(a, kind == 1, pairs[kind] + x, 0) + r % ROWS;
      if (nt[kind] == 0) continue;
      wf[kind] = owner(U[kind]);
      nc[kind] = sparse ? nt[kind] : owner(U[kind] + (nt[kind] - 1) * wt[kind]) - wf[kind] + 1;
    }
    const int ncand = nc[0] + nc[1];
    F mx = -INFINITY, wsum = 0, acc[CH];
#pragma unroll
    for (int e = 0; e < CH; ++e) acc[e] = 0;
    for (int c0 = SPLIT ? w * ROUND : 0; c0 < ncand; c0 += SPLIT ? 4 * ROUND : ROUND) {
      F ms[ROUND], ls[ROUND];                  // maximum and sum
      Vec<F, CH> po[ROUND];
#pragma unroll
      for (int i = 0; i < ROUND; ++i) {
        const int cand = min(c0 + i, ncand - 1);
        const int kind = cand >= nc[0], k = cand - (kind ? nc[0] : 0);
        int wv = wf[kind] + k, prev = -1;      // owners of this tile and of the one before
        if (sparse) {
          wv = owner(U[kind] + k * wt[kind]);
          if (k > 0) prev = owner(U[kind] + (k - 1) * wt[kind]);
        }
        const size_t prow = (size_t)(first[kind] + (long long)wv * (kind ? a.rows_own : ROWS));
        const Vec<F, 2> ml = static_cast<const Vec<F, 2>*>(a.part_ml)[prow];
        po[i] = *reinterpret_cast<const Vec<F, CH>*>(static_cast<const F*>(a.part_o) + prow * D + lane * CH);
        ms[i] = c0 + i < ncand && wv != prev ? ml[0] : -INFINITY;
        ls[i] = ml[1];
      }
      F nm = mx;
      bool none = mx == -INFINITY;
#pragma unroll
      for (int i = 0; i < ROUND; ++i) {
        nm = fmax(nm, ms[i]);
        none = none && ms[i] == -INFINITY;
      }
      if (none) continue;                      // no key in any partial so far
      const F keep = weight_of(mx - nm);       // (0 from -inf)
      wsum *= keep;
#pragma unroll
      for (int e = 0; e < CH; ++e) acc[e] = kExact && keep == 0 ? 0 : acc[e] * keep;
#pragma unroll
      for (int i = 0; i < ROUND; ++i) {
        const F wl = weight_of(ms[i] - nm) * ls[i];
        wsum += wl;
#pragma unroll
        for (int e = 0; e < CH; ++e) acc[e] = fma(wl, kExact && wl == 0 ? 0 : po[i][e], acc[e]);
      }
      mx = nm;
    }
    if constexpr (SPLIT) {
      __syncthreads();                         // the previous row's values are read
      part[w][0] = mx;
      part[w][1] = wsum;
#pragma unroll
      for (int e = 0; e < CH; ++e) part[w][2 + lane * CH + e] = acc[e];
      __syncthreads();
      if (w != 0) continue;
      F nm = mx;
#pragma unroll
      for (int v = 1; v < 4; ++v) nm = fmax(nm, part[v][0]);
      wsum = 0;
#pragma unroll
      for (int e = 0; e < CH; ++e) acc[e] = 0;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const F f = part[v][0] == nm ? 1 : weight_of(part[v][0] - nm);   // (-inf too)
        wsum = fma(f, part[v][1], wsum);
#pragma unroll
        for (int e = 0; e < CH; ++e)
          acc[e] = fma(f, kExact && f == 0 ? 0 : part[v][2 + lane * CH + e], acc[e]);
      }
      mx = nm;
    }
    const size_t orow = (size_t)b * rows + row;
    const F inv = wsum != 0 ? 1 / wsum : 0;
    if (ROWS != kRowsF32 && a.out_bf16) {
      Vec<__bf16, CH> v;
#pragma unroll
      for (int e = 0; e < CH; ++e) v[e] = float_to_bf16((float)(acc[e] * inv));
      *reinterpret_cast<Vec<__bf16, CH>*>(static_cast<__bf16*>(a.out) + orow * D + lane * CH) = v;
    } else {
      Vec<float, CH> v;
#pragma unroll
      for (int e = 0; e < CH; ++e) v[e] = (float)(acc[e] * inv);
      *reinterpret_cast<Vec<float, CH>*>(static_cast<float*>(a.out) + orow * D + lane * CH) = v;
    }
    if (a.lse != nullptr && lane == 0) a.lse[orow] = wsum != 0 ? lse_of(mx, wsum) : -INFINITY;
  }
}

template <int D, int RB, int TERMS>
hipError_t launch_bf16(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  hipLaunchKernelGGL((shared_stream_bf16<D, RB, TERMS>), dim3(p.wgs), dim3(512), 0, st, a, p.wgs);
  return hipGetLastError();
}

template <int ROWS, int TK, int D>
hipError_t merge_rows(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  const int rows = a.k * a.Hq;
  if ((long long)a.B * rows <= kSplitRows) {
    hipLaunchKernelGGL((shared_merge<ROWS, TK, D, true>), dim3((unsigned)(a.B * rows)), dim3(256), 0, st, a, p.wgs, 1,
                       rows);
  } else {
    // about kMergeWaves waves, a whole number of rows each
    const int per = (int)std::max(1LL, std::min((long long)rows, (long long)a.B * rows / kMergeWaves));
    const int wgs_seq = (rows + 4 * per - 1) / (4 * per);
    hipLaunchKernelGGL((shared_merge<ROWS, TK, D, false>), dim3((unsigned)(a.B * (long long)wgs_seq)), dim3(256), 0, st,
                       a, p.wgs, per, wgs_seq);
  }
  return hipGetLastError();
}
template <int ROWS, int TK>
hipError_t launch_merge(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  return a.D == 128 ? merge_rows<ROWS, TK, 128>(a, p, st) : merge_rows<ROWS, TK, 64>(a, p, st);
}

}  // namespace

SharedPlan plan_shared(int B, int k, int Hq, int Hkv, int D, int G, int prefix_cap, int cap, int dtype, bool out_bf16,
                       int cus) {
  SharedPlan p{};
  const int kg = k * (Hq / Hkv);
  const long long rows = (long long)B * kg;     // of a KV head
  cus = std::max(1, cus);
  int per_cu = 1;
  if (dtype == 0) {
    p.rows_wg = kRowsF32;
    per_cu = 2;
  } else {
    // 256 rows halve the copies and LDS reads per row: a tile of them takes 2.6 us
    // where two of 128 take 3.2, but twice the partials cost the call about 7.5 us.
    // So the places of the list decide (a third of a tile each, see above), with
    // groups of average size and every cache at capacity.  In tiles of 128 and of
    // 256: 256 rows over 16000 keys 47 and 50 us, over 65536 125 and 113; 384 rows
    // 59 and 63, 512 rows 70 and 69, 768 rows 92 and 89; 1024 over 65500 456 and 383.
    // fp32 outputs take three terms of P, for which 256 rows leave no registers.
    const long long avg = (rows + G - 1) / G;
    auto places = [&](int rows_wg) {
      auto of = [&](long long pairs, long long unit_rows, int keys) {
        return pairs * ((long long)((keys + kTile - 1) / kTile) *
                            tile_places(rows_wg, (int)std::min(unit_rows, (long long)rows_wg)) + start_places(rows_wg));
      };
      return Hkv * (of(G * ((avg + rows_wg - 1) / rows_wg), avg, prefix_cap) +
                    of(B * (long long)((kg + rows_wg - 1) / rows_wg), kg, cap));
    };
    p.rows_wg = out_bf16 && 52 * places(256) + 450LL * cus <= 32 * places(128) ? 256 : 128;   // (us * 60)
  }
  const int tk = dtype == 0 ? kTileF32 : kTile;
  p.rows_own = std::min((kg + 15) / 16 * 16, p.rows_wg);
  const long long prefix_pairs = Hkv * (rows / p.rows_wg + G);
  const long long own_pairs = (long long)B * Hkv * ((kg + p.rows_wg - 1) / p.rows_wg);
  const long long tiles = prefix_pairs * ((prefix_cap + tk - 1) / tk) + own_pairs * ((cap + tk - 1) / tk);
  p.ok = tiles < (1LL << 27);   // a pair has a tile or more: at most 9 places for each
  p.wgs = (int)std::max(1LL, std::min((long long)cus * per_cu, tiles));
  p.own_base = (prefix_pairs + p.wgs) * p.rows_wg;
  p.part_rows = (size_t)p.own_base + (size_t)(own_pairs + p.wgs) * p.rows_own;
  const size_t es = dtype == 0 ? sizeof(PartT<kRowsF32>) : sizeof(float);
  p.ml_offset = p.part_rows * D * es;
  p.workspace_bytes = p.ml_offset + p.part_rows * 2 * es;
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
    return e != hipSuccess ? e : launch_merge<kRowsF32, kTileF32>(a, p, st);
  }
  if (p.rows_wg == 256) {
    e = a.D == 128 ? launch_bf16<128, 2, 2>(a, p, st) : launch_bf16<64, 2, 2>(a, p, st);
    return e != hipSuccess ? e : launch_merge<256, kTile>(a, p, st);
  }
  if (a.out_bf16)
    e = a.D == 128 ? launch_bf16<128, 1, 2>(a, p, st) : launch_bf16<64, 1, 2>(a, p, st);
  else
    e = a.D == 128 ? launch_bf16<128, 1, 3>(a, p, st) : launch_bf16<64, 1, 3>(a, p, st);
  return e != hipSuccess ? e : launch_merge<128, kTile>(a, p, st);
}

}  // namespace sd
