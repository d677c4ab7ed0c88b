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


constexpr int kTileF32 = 32, kTile = 64;   // keys per tile (fp32, bf16)
// Places of the list in front of a pair's first tile: on the matrix cores
// starting a pair (its queries' latency with the ring drained, the partial of
// the one before) takes about as long as two tiles.
constexpr int kRowsF32 = 16;
constexpr int start_places(int rows_wg) { return rows_wg == kRowsF32 ? 0 : 2; }
constexpr int kMergeWaves = 4096;   // rows of a sequence share a wave beyond that many
constexpr float kHeadroom = 24.f;   // log2 of the largest weight before the maximum is raised

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
  s.places = s.un.L > 0 ? s.pairs * (tiles_of<TK>(s.un.L) + start_places(ROWS)) : 0;
  int ti = s.places, pi = s.pairs;
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) {
    const int x = __shfl_up(ti, off, 64), y = __shfl_up(pi, off, 64);
    if (lane >= off) {
      ti += x;
      pi += y;
    }
  }
  s.n_before = c.places + ti - s.places;
  s.p_before = c.pairs + pi - s.pairs;
  c.places += __shfl(ti, 63, 64);
  c.pairs += __shfl(pi, 63, 64);
  return s;
}

// length T of the list
template <int ROWS, int TK>
__device__ __forceinline__ int list_length(const SharedArgs& a) {
  Carry c;
  for (int u0 = 0; u0 < a.G + a.B; u0 += 64) scan_units<ROWS, TK>(a, u0, c);
  return c.places;
}

// cursor of the first tile at place n (0 <= n < T) or behind it.  The pair counts
// its kind only: own pairs start at 0 again (R rows each).
template <int ROWS, int TK>
__device__ __forceinline__ Cursor find_tile(const SharedArgs& a, int n) {
  Carry c;
  for (int u0 = 0; u0 < a.G + a.B; u0 += 64) {
    const Span s = scan_units<ROWS, TK>(a, u0, c);
    if (n >= c.places) continue;
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
    constexpr int kStart = start_places(ROWS);
    const int rem = n - of(s.n_before);
    const int x = rem / (cu.nt + kStart);
    cu.t = max(rem - x * (cu.nt + kStart) - kStart, 0);
    cu.n = of(s.n_before) + x * (cu.nt + kStart) + kStart + cu.t;
    cu.hk = x / cu.RT;
    cu.rt = x - cu.hk * cu.RT;
    cu.pair = cu.u < a.G ? of(s.p_before) + x : (cu.u - a.G) * a.Hkv * cu.RT + x;
    return cu;
  }
  return Cursor{};   // n >= T: not reached
}

// the same in scalar registers (the compiler cannot see that the search ends
// alike on every lane), so that its bookkeeping stays off the vector unit
template <int ROWS, int TK>
__device__ __forceinline__ Cursor locate(const SharedArgs& a, int n) {
  Cursor cu = find_tile<ROWS, TK>(a, n);
  int* f[] = {&cu.n, &cu.u, &cu.hk, &cu.rt, &cu.t, &cu.nt, &cu.RT, &cu.L, &cu.rows, &cu.first, &cu.end, &cu.pair};
#pragma unroll
  for (int* x : f) *x = __builtin_amdgcn_readfirstlane(*x);
  return cu;
}

// place of the tile behind cu
template <int ROWS>
__device__ __forceinline__ int place_behind(const Cursor& cu) {
  return cu.n + 1 + (cu.t + 1 == cu.nt ? start_places(ROWS) : 0);
}

// next tile of the list; the caller never steps past the last one
template <int ROWS, int TK>
__device__ __forceinline__ void advance(const SharedArgs& a, Cursor& cu) {
  ++cu.n;
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

// ------------------------------------------------- bf16 stream, many rows
// Eight waves of RB 16-row blocks on 64-key tiles, matrix-core bound.  A step
// computes the scores of tile x + 1 under the exponentials of tile x, then P V
// of tile x under the row maxima of tile x + 1, which are raised (rarely) after
// it.  It runs in groups of four LDS fragments each: a group's reads are issued
// one group ahead and waited for by count, and its matrix-core and vector
// operations alternate.  K and V have rings of four slots; the tile that a step
// copies lands two steps later.
template <int ID, int MFMAS, int VALUS>
__device__ __forceinline__ void alternate() {
  if constexpr (MFMAS > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, ID);
    __builtin_amdgcn_sched_group_barrier(0x002, VALUS, ID);
    alternate<ID, MFMAS - 1, VALUS>();
  }
}

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

template <int D, int RB, bool HILO>
__global__ __launch_bounds__(512, 2) void shared_wide_bf16(SharedArgs a, int G) {
  constexpr int NW = 8, TK = kTile, NBUF = 4;
  constexpr int DC = D / 32;                   // 32-channel slices (S^T = K Q^T)
  constexpr int DB = D / 16;                   // 16-channel blocks (O^T)
  constexpr int PK = D / 8;                    // 16-byte pieces per key row
  constexpr int ROW = D * 2;
  constexpr int HALF = TK * ROW;               // a tile's K (or V)
  constexpr int KEYS = 64 / PK;                // keys of one 64-lane copy
  constexpr int COPIES = TK / KEYS / NW;       // per wave and half
  constexpr int ROWS = NW * RB * 16;
  constexpr int KPG = 4 / DC;                  // 16-key blocks of a score group
  constexpr int NQK = 4 / KPG, NPVH = DB / 4, NG = NQK + 2 * NPVH;
  static_assert(NBUF * HALF <= 65536, "ring slots within the LDS instructions' offsets");
  __shared__ __align__(16) unsigned char ring[2][NBUF * HALF];   // K, V

  const int lane = threadIdx.x & 63, G4 = lane >> 4, c = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wg = blockIdx.x;
  const int T = __builtin_amdgcn_readfirstlane(list_length<ROWS, TK>(a));
  const int n0 = (int)((long long)T * wg / G), n1 = (int)((long long)T * (wg + 1) / G);
  if (n0 >= n1) return;
  Cursor cc = locate<ROWS, TK>(a, n0);
  if (cc.n >= n1) return;

  // copy i of this wave takes keys (w COPIES + i) KEYS .. of K and of V; a lane's
  // 16-byte piece goes to LDS slot piece ^ lds_swizzle(key).  A copy's keys lie in
  // one page.  Keys past the unit's length re-read its last key (masked).
  int ckey[COPIES];
  uint32_t cpiece[COPIES];
#pragma unroll
  for (int i = 0; i < COPIES; ++i) {
    ckey[i] = (w * COPIES + i) * KEYS + lane / PK;
    cpiece[i] = ((lane % PK) ^ lds_swizzle<PK>(ckey[i])) * 16;
  }
  // the tile that is copied next: its first keys' byte offsets in the caches
  // (found one step ahead, as page ids are loads) and its last key
  size_t cbase[COPIES];
  int clast = 0, cstep = 0;
  const unsigned char *ck = nullptr, *cv = nullptr;
  auto place = [&](const Cursor& cu) {
    const bool own = cu.u >= a.G;
    const int row = own ? cu.first : cu.u;
    ck = static_cast<const unsigned char*>(own ? a.k_cache : a.k_prefix);
    cv = static_cast<const unsigned char*>(own ? a.v_cache : a.v_prefix);
    const int32_t* table = own ? a.page_table : a.prefix_table;
    const int t0 = cu.t * TK;
    clast = cu.L - 1 - t0;
    if (table != nullptr) {
      const int pages = own ? a.num_pages : a.prefix_num_pages;
      cint32* pt = (cint32*)(table + (size_t)row * (own ? a.max_pages : a.prefix_pages));
      const int lastp = (cu.L - 1) >> 4;
      cstep = ROW;
#pragma unroll
      for (int i = 0; i < COPIES; ++i) {
        const int key0 = (w * COPIES + i) * KEYS;
        const int pi = min((t0 + key0) >> 4, lastp);
        const int page = min(max((int)pt[pi], 0), pages - 1);
        // offset of the tile's key 0 as if every key lay in this page
        cbase[i] = (((size_t)page * a.Hkv + cu.hk) * 16) * ROW - (size_t)(pi * 16 - t0) * ROW;
      }
    } else {
      cstep = a.Hkv * ROW;
#pragma unroll
      for (int i = 0; i < COPIES; ++i)
        cbase[i] = (((size_t)row * (own ? a.Lmax : a.prefix_cap) + t0) * a.Hkv + cu.hk) * ROW;
    }
  };
  auto issue = [&](int slot) {
#pragma unroll
    for (int i = 0; i < COPIES; ++i) {
      const uint32_t off = (uint32_t)min(ckey[i], clast) * (uint32_t)cstep + cpiece[i];
      const int at = slot * HALF + (w * COPIES + i) * 1024;
      __builtin_amdgcn_global_load_lds((gbl_cvoid*)(ck + cbase[i] + off), (lds_void*)(ring[0] + at), 16, 0, 0);
      __builtin_amdgcn_global_load_lds((gbl_cvoid*)(cv + cbase[i] + off), (lds_void*)(ring[1] + at), 16, 0, 0);
    }
  };

  // fragment addresses for the first 16 keys of slot 0 (the swizzle depends on
  // key % 16 only, so further blocks and slots are offsets)
  uint32_t kaddr[DC], vaddr[DB];
#pragma unroll
  for (int dc = 0; dc < DC; ++dc)
    kaddr[dc] = lds_addr(ring[0]) + c * ROW + (((dc * 4 + G4) ^ lds_swizzle<PK>(c)) * 16);
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int key = 4 * G4 + (c >> 2), ch = db * 16 + 4 * (c & 3);
    vaddr[db] = lds_addr(ring[1]) + key * ROW + (((ch >> 3) ^ lds_swizzle<PK>(key)) * 16) + (ch & 7) * 2;
  }

  // segment state (rows, maxima and sums as in the narrow kernel)
  bf16x8 qf[RB][DC];
  int lim[RB];
  float m[RB], l[RB];
  floatx4 o[RB][DB], sc[4][RB];                // sc: raw scores of the tile whose turn it is
  const bool neg = a.scale_log2 < 0.f;
  const float sl2 = fabsf(a.scale_log2);
  const int g = a.Hq / a.Hkv, kg = a.k * g;

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
          vr[gr & 1][d][0] = lds_read_tr16_b64_off<PH * HALF + hf * 32 * ROW>(vaddr[4 * pb + d] + dh);
          vr[gr & 1][d][1] = lds_read_tr16_b64_off<PH * HALF + hf * 32 * ROW + 16 * ROW>(vaddr[4 * pb + d] + dh);
        }
      });
    }
  };

  // maxima of the raw scores in s, raised where a weight would pass 2^24 (or at once)
  auto raise = [&](const floatx4 (&s)[4][RB], bool at_once) {
    float lm[RB];
    bool over = at_once;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      lm[rb] = s[0][rb][0];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) lm[rb] = fmaxf(lm[rb], s[kb][rb][i]);
      over = over || fmaf(lm[rb], sl2, -m[rb]) > kHeadroom;
    }
    if (__ballot(over) == 0ull) return;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float top = wave_max_across_groups(lm[rb]) * sl2;
      const float mnew = at_once ? top : fmaxf(m[rb], top);
      const float f = at_once ? 0.f : fast_exp2(m[rb] - mnew);   // O and l are 0 at the start
      l[rb] *= f;
#pragma unroll
      for (int db = 0; db < DB; ++db) o[rb][db] *= f;
      m[rb] = mnew;
    }
  };

  // One step, tile x of the segment: NEXT: there is a tile x + 1 in it; MASK: a
  // row's last visible key may lie in tile x (first key t0).  PH: ring phase of
  // x where known (the slots then sit in the instructions' offsets), else -1.
  auto step = [&](int n, int t0, auto ph_tag, auto next_tag, auto mask_tag) {
    constexpr int PH = decltype(ph_tag)::value;
    constexpr bool NEXT = decltype(next_tag)::value, MASK = decltype(mask_tag)::value;
    constexpr int PN0 = PH >= 0 ? (PH + 1) % NBUF : 0, PH0 = PH >= 0 ? PH : 0;
    const uint32_t dn = PH >= 0 ? 0u : (uint32_t)((n + 1) % NBUF) * HALF, dh = PH >= 0 ? 0u : (uint32_t)(n % NBUF) * HALF;
    constexpr int G0 = NEXT ? 0 : NQK;         // the last tile has no scores to form
    bf16x8 ph[2][RB], pl[2][RB];
    floatx4 sn[4][RB];
    auto weights = [&](int kb) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float p[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          p[i] = fast_exp2(fmaf(sc[kb][rb][i], sl2, -m[rb]));
          if constexpr (MASK) {
            if (t0 + kb * 16 + 4 * G4 + i > lim[rb]) p[i] = 0.f;
          }
          const __bf16 hi = float_to_bf16(p[i]);
          ph[kb >> 1][rb][(kb & 1) * 4 + i] = hi;
          if constexpr (HILO) pl[kb >> 1][rb][(kb & 1) * 4 + i] = float_to_bf16(p[i] - bf16_to_float(hi));
        }
        l[rb] += (p[0] + p[1]) + (p[2] + p[3]);
      }
    };
    reads(Const<G0>{}, Const<PN0>{}, Const<PH0>{}, dn, dh, Const<0>{});
    if constexpr (!NEXT) {
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) weights(kb);
    }
    unrolled<G0, NG>([&](auto gtag) {
      constexpr int gr = decltype(gtag)::value;
      reads(Const<gr + 1>{}, Const<PN0>{}, Const<PH0>{}, dn, dh, Const<0>{});
      lds_wait_n<(gr + 1 < NQK ? 4 : gr + 1 < NG ? 8 : 0)>();
      reads(gtag, Const<PN0>{}, Const<PH0>{}, dn, dh, Const<1>{});
      if constexpr (gr < NQK) {
#pragma unroll
        for (int kk = 0; kk < KPG; ++kk) {
          const int kb = gr * KPG + kk;
#pragma unroll
          for (int dc = 0; dc < DC; ++dc) {
            Pack8 pk;
            pk.u = xr[gr & 1][kk * DC + dc];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              sn[kb][rb] = mfma_bf16(pk.b, qf[rb][dc], dc == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : sn[kb][rb]);
          }
          weights(kb);
        }
        alternate<gr + 1, 4 * RB, HILO ? 6 : 3>();
      } else {
        constexpr int q = gr - NQK, hf = q / NPVH, pb = q % NPVH;
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          Pack8 vv;
          vv.u = u32x4{vr[gr & 1][d][0][0], vr[gr & 1][d][0][1], vr[gr & 1][d][1][0], vr[gr & 1][d][1][1]};
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) {
            o[rb][4 * pb + d] = mfma_bf16(vv.b, ph[hf][rb], o[rb][4 * pb + d]);
            if constexpr (HILO) o[rb][4 * pb + d] = mfma_bf16(vv.b, pl[hf][rb], o[rb][4 * pb + d]);
          }
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (NEXT) {
      raise(sn, false);
#pragma unroll
      for (int kb = 0; kb < 4; ++kb)
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) sc[kb][rb] = sn[kb][rb];
    }
  };

  // Ring: entering the step of tile n the copies of tiles n + 1 and n + 2 are
  // under way; the wait leaves tile n + 2's, the barrier frees tile n - 1's slot
  // for tile n + 3.  Past the range the last tile is copied again.
  Cursor ic = cc;
  place(ic);
  auto copy_next = [&](int slot) {
    issue(slot);
    if (place_behind<ROWS>(ic) < n1) {
      advance<ROWS, TK>(a, ic);
      place(ic);
    }
  };
#pragma unroll 1
  for (int i = 0; i < NBUF - 1; ++i) copy_next(i);
  wait_vm_then_barrier<2 * 2 * COPIES>();      // tile n0 is there
  auto begin = [&](int x) {                    // step x of the ring
    wait_vm_then_barrier<2 * COPIES>();
    copy_next((x + NBUF - 1) % NBUF);
  };

  int x = 0;                                   // ring step
  while (true) {
    const bool own = cc.u >= a.G;
    const int rt = cc.rt, rows = cc.rows, pair = cc.pair;
    const int steps = min(cc.nt - cc.t, n1 - cc.n);
    const int t_first = cc.t * TK;
    // tiles before the first with masked keys, and before the last
    const int unmasked = own ? cc.L - a.k : cc.L - 1;
    const int plain = max(0, min(steps - 1, (unmasked + 1) / TK - cc.t));
    const int r0 = rt * ROWS + w * RB * 16;
    if (r0 < rows) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const int r = r0 + rb * 16 + c;
        Pack8 pk;
        pk.u = u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int dc = 0; dc < DC; ++dc) qf[rb][dc] = pk.b;
        lim[rb] = -1;
        if (r < rows) {
          const u32x4* src = reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(a.q) +
                                                            (size_t)out_row(a, cc.first, cc.hk, r) * D);
#pragma unroll
          for (int dc = 0; dc < DC; ++dc) {
            pk.u = src[dc * 4 + G4];
            if (neg) pk.u ^= u32x4{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
            qf[rb][dc] = pk.b;
          }
          lim[rb] = own ? cc.L - a.k + (r % kg) / g : cc.L - 1;
        }
        l[rb] = 0.f;
        m[rb] = 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db) o[rb][db] = floatx4{0.f, 0.f, 0.f, 0.f};
      }
      __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // vmcnt(0): the counted waits only see copies
      // scores of the first tile
      const uint32_t d0 = (uint32_t)(x % NBUF) * HALF;
      unrolled<0, NQK>([&](auto gtag) {
        constexpr int gr = decltype(gtag)::value;
        reads(gtag, Const<0>{}, Const<0>{}, d0, 0u, Const<0>{});
        lds_wait();
        reads(gtag, Const<0>{}, Const<0>{}, d0, 0u, Const<1>{});
#pragma unroll
        for (int kk = 0; kk < KPG; ++kk)
#pragma unroll
          for (int dc = 0; dc < DC; ++dc) {
            Pack8 pk;
            pk.u = xr[gr & 1][kk * DC + dc];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
              sc[gr * KPG + kk][rb] =
                  mfma_bf16(pk.b, qf[rb][dc], dc == 0 ? floatx4{0.f, 0.f, 0.f, 0.f} : sc[gr * KPG + kk][rb]);
          }
      });
      raise(sc, true);
      int i = 0;                               // step of the segment
#define SD_STEP(PH, NEXT, MASK)                                                                 \
  {                                                                                             \
    begin(x);                                                                                   \
    step(x, t_first + i * TK, Const<PH>{}, Const<NEXT>{}, Const<MASK>{});                       \
    ++x;                                                                                        \
    ++i;                                                                                        \
  }
      while (i < plain && x % NBUF != 0) SD_STEP(-1, 1, 0)
      while (i + NBUF <= plain) {
        SD_STEP(0, 1, 0)
        SD_STEP(1, 1, 0)
        SD_STEP(2, 1, 0)
        SD_STEP(3, 1, 0)
      }
      while (i < plain) SD_STEP(-1, 1, 0)
      while (i < steps - 1) SD_STEP(-1, 1, 1)
      SD_STEP(-1, 0, 1)
#undef SD_STEP
      // the segment's partial
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const float lsum = wave_sum_across_groups(l[rb]);
        const int lr = (w * RB + rb) * 16 + c;
        if (rt * ROWS + lr >= rows) continue;
        const size_t prow = part_row<ROWS>(a, own, pair, wg) + lr;
        const float inv = lsum > 0.f ? 1.f / lsum : 0.f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
          *reinterpret_cast<floatx4*>(a.part_o + prow * D + db * 16 + 4 * G4) = o[rb][db] * inv;
        if (G4 == 0) a.part_lse[prow] = lsum > 0.f ? m[rb] + log2f(lsum) : -INFINITY;
      }
    } else {
      for (int i = 0; i < steps; ++i) begin(x++);   // no rows: its copies only
    }
    cc.t += steps - 1;
    cc.n += steps - 1;
    if (place_behind<ROWS>(cc) >= n1) break;
    advance<ROWS, TK>(a, cc);
  }
  __builtin_amdgcn_s_waitcnt((7 << 4) | (15 << 8));   // no copy may still write this LDS
}

// ------------------------------------------------------------- fp32 stream
// fp32 inputs: scores, softmax and P V in float64, as everywhere for fp32.
// The same list with 16 rows per work-group and 32-key tiles.  The segment's
// queries and a tile's keys and values lie in LDS (rows padded by one float);
// row r belongs to the 16 lanes r * 16 ..: each forms two of its scores, its
// maximum and sum go over those lanes by shuffles, and each accumulates D / 16
// of its channels.
template <int D>
__global__ __launch_bounds__(256) void shared_stream_f32(SharedArgs a, int G) {
  constexpr int TK = kTileF32, R = kRowsF32, DS = D + 1;
  constexpr int PER = D / 16;                  // channels per lane
  __shared__ float qs[R * DS], ks[TK * DS], vs[TK * DS];
  __shared__ double ps[R][TK + 1];             // weights
  const int tid = threadIdx.x, r = tid >> 4, lane16 = tid & 15;
  const int wg = blockIdx.x;
  const int T = list_length<R, TK>(a);
  const int n0 = (int)((long long)T * wg / G), n1 = (int)((long long)T * (wg + 1) / G);
  if (n0 >= n1) return;
  Cursor cu = locate<R, TK>(a, n0);
  if (cu.n >= n1) return;
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
#pragma unroll 4
    for (int i = tid; i < TK * D; i += 256) {
      const int t = min(t0 + i / D, cu.L - 1);   // past the length: the last key, masked
      size_t off;
      if (table != nullptr) {
        const int pages = own ? a.num_pages : a.prefix_num_pages;
        const int page = min(max(table[(size_t)seq * (own ? a.max_pages : a.prefix_pages) + (t >> 4)], 0), pages - 1);
        off = (((size_t)page * a.Hkv + cu.hk) * 16 + (t & 15)) * D;
      } else {
        off = (((size_t)seq * (own ? a.Lmax : a.prefix_cap) + t) * a.Hkv + cu.hk) * D;
      }
      ks[(i / D) * DS + i % D] = kb[off + i % D];
      vs[(i / D) * DS + i % D] = vb[off + i % D];
    }
    __syncthreads();
    const int lim = own ? cu.L - a.k + (row % kg) / (kg / a.k) : cu.L - 1;
    double s[2] = {0.0, 0.0};
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
    for (int e = 0; e < PER; ++e) o[e] *= keep;
    for (int t = 0; t < here; ++t) {
      const double p = ps[r][t];
#pragma unroll
      for (int e = 0; e < PER; ++e)
        o[e] = fma(p, p != 0.0 ? (double)vs[t * DS + lane16 + 16 * e] : 0.0, o[e]);   // a zero weight adds nothing
    }
    fresh = cu.t + 1 == cu.nt;
    const bool end = place_behind<R>(cu) >= n1;
    if ((fresh || end) && row < cu.rows) {
      const size_t at = part_row<R>(a, own, cu.pair, wg) + r;
#pragma unroll
      for (int e = 0; e < PER; ++e) a.part_o[at * D + lane16 + 16 * e] = l > 0.0 ? (float)(o[e] / l) : 0.f;
      if (lane16 == 0) a.part_lse[at] = l > 0.0 ? (float)((m + log(l)) * 1.4426950408889634) : -INFINITY;
    }
    if (end) break;
    advance<R, TK>(a, cu);
  }
}

// ------------------------------------------------------------------ merge
// One wave per output row.  The tiles at places [U, U + nt) lie with work-groups
// owner(U) .. owner(U + nt - 1), owner(n) = floor(((n + 1) G - 1) / T), each of
// which wrote one partial (with fewer places than work-groups, each owner did).  Candidates of the prefix pair, then of the own pair,
// are taken 32 at a time: lanes 0..31 load their lse while each half-wave loads
// the outputs of 16 of them (4 channels per lane), and the chunk's weights
// 2^(lse - max) rescale a running sum.  Every shuffle runs on all lanes.
// A wave takes `per` rows of one sequence, so that the scan over the units is
// made once for them.
template <int ROWS, int TK>
__global__ __launch_bounds__(256) void shared_merge(SharedArgs a, int G, int per, int wgs_seq) {
  const int w = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int b = blockIdx.x / wgs_seq;
  const int row0 = ((blockIdx.x - b * wgs_seq) * 4 + w) * per;   // of the k Hq rows of sequence b
  if (row0 >= a.k * a.Hq) return;
  const int D = a.D, g = a.Hq / a.Hkv;

  // places before the unit, key tiles, pairs before it, row tiles and first row
  // of the sequence, for the group's prefix (0) and the sequence's own keys (1)
  int before[2] = {0, 0}, nt[2] = {0, 0}, pairs[2] = {0, 0}, RT[2] = {1, 1}, base[2] = {0, 0};
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
      nt[kind] = tiles_of<TK>(of(s.un.L));
      before[kind] = of(s.n_before);
      pairs[kind] = kind == 0 ? of(s.p_before) : b * a.Hkv * RT[kind];
      base[kind] = kind == 0 ? (b - of(s.un.first)) * a.k * g : 0;
    }
  }
  const int T = c.places;
  auto owner = [&](int n) { return (int)((((long long)n + 1) * G - 1) / T); };
  const bool sparse = T < G;   // then a work-group has one place or none: a candidate per tile
  for (int row = row0; row < min(row0 + per, a.k * a.Hq); ++row) {
  const int j = row / a.Hq, h = row - j * a.Hq, hk = h / g;
  const size_t orow = (size_t)b * a.k * a.Hq + row;
  int U[2], pair[2], lr[2], wf[2] = {0, 0}, nc[2] = {0, 0};
#pragma unroll
  for (int kind = 0; kind < 2; ++kind) {
    const int r = base[kind] + j * g + (h - hk * g);
    const int x = hk * RT[kind] + r / ROWS;
    U[kind] = before[kind] + x * (nt[kind] + start_places(ROWS)) + start_places(ROWS);
    pair[kind] = pairs[kind] + x;
    lr[kind] = r % ROWS;
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
      *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(a.out) + orow * D + d4 * 4) = u32x2{pk.u[0], pk.u[1]};
    } else {
      *reinterpret_cast<floatx4*>(static_cast<float*>(a.out) + orow * D + d4 * 4) = v;
    }
  }
  if (a.lse != nullptr && lane == 0) a.lse[orow] = wsum > 0.f ? (mx + log2f(wsum)) * kLn2 : -INFINITY;
  }
}

template <int D, int RB>
hipError_t launch_wide(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  if (a.out_bf16)
    hipLaunchKernelGGL((shared_wide_bf16<D, RB, false>), dim3(p.wgs), dim3(512), 0, st, a, p.wgs);
  else
    hipLaunchKernelGGL((shared_wide_bf16<D, RB, true>), dim3(p.wgs), dim3(512), 0, st, a, p.wgs);
  return hipGetLastError();
}

template <int ROWS, int TK>
hipError_t launch_merge(const SharedArgs& a, const SharedPlan& p, hipStream_t st) {
  // about kMergeWaves waves, a whole number of rows each
  const int rows = a.k * a.Hq;
  const int per = (int)std::max(1LL, std::min((long long)rows, (long long)a.B * rows / kMergeWaves));
  const int wgs_seq = (rows + 4 * per - 1) / (4 * per);
  hipLaunchKernelGGL((shared_merge<ROWS, TK>), dim3((unsigned)(a.B * (long long)wgs_seq)), dim3(256), 0, st, a, p.wgs, per,
                     wgs_seq);
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
    per_cu = 2;
  } else {
    // rows of an average group; a wave of two 16-row blocks halves the LDS reads
    // per product, eight such waves halve the HBM reads per row again
    const long long avg = (rows + G - 1) / G;
    p.rows_wg = 128;
    auto places = [&](int rows_wg) {
      return Hkv * (G * ((avg + rows_wg - 1) / rows_wg) * ((prefix_cap + kTile - 1) / kTile) +
                    B * (long long)((kg + rows_wg - 1) / rows_wg) * ((cap + kTile - 1) / kTile + start_places(rows_wg)));
    };
    if (places(256) * 8 <= places(128) * 5) p.rows_wg = 256;
    per_cu = 1;
  }
  p.rows_own = std::min((kg + 15) / 16 * 16, p.rows_wg);
  const int own_tiles = (kg + p.rows_wg - 1) / p.rows_wg;
  const long long prefix_pairs = Hkv * (rows / p.rows_wg + G);
  const long long own_pairs = (long long)B * Hkv * own_tiles;
  const int tk = p.rows_wg >= 128 ? kTile : kTileF32;
  const long long prefix_tiles = prefix_pairs * ((prefix_cap + tk - 1) / tk);
  const long long own_tiles_cap = own_pairs * ((cap + tk - 1) / tk);
  p.ok = prefix_tiles + own_tiles_cap + start_places(p.rows_wg) * (prefix_pairs + own_pairs) < (1LL << 30);
  p.wgs = (int)std::max(1LL, std::min((long long)cus * per_cu, prefix_tiles + own_tiles_cap));
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
    return e != hipSuccess ? e : launch_merge<kRowsF32, kTileF32>(a, p, st);
  }
  if (p.rows_wg == 128) {
    e = a.D == 128 ? launch_wide<128, 1>(a, p, st) : launch_wide<64, 1>(a, p, st);
    return e != hipSuccess ? e : launch_merge<128, kTile>(a, p, st);
  }
  e = a.D == 128 ? launch_wide<128, 2>(a, p, st) : launch_wide<64, 2>(a, p, st);
  return e != hipSuccess ? e : launch_merge<256, kTile>(a, p, st);
}

}  // namespace sd
