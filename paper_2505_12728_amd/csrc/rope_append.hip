// Rotary positions with one to four axes, alone (sd_rope) or on the way of
// new keys and values into the cache (sd_kv_append).
//
// Mathematics.  The first 2P channels of a head are P pairs (i, i + P); pair
// i belongs to axis a (consecutive runs of pairs, one per axis) and turns by
//   ang = pos[a] f_i,  f_i = theta^(-i / P)            (running), or
//                      f_i = theta^(-(i - i0) / n_a)   (per axis),
//   y1 = x1 cos ang - x2 sin ang,  y2 = x1 sin ang + x2 cos ang;
// the rest of the channels and the values are copied.  The inverse turns by
// -ang; the map being orthogonal, it is also the gradient.
//
// Angles are formed in float64 as turns, pos * f_i / (2 pi), and reduced
// there (fp32 would leave 0.008 rad at position 10^5).  For fp32 outputs sine and
// cosine are taken there too and rounded once: fp32 functions of the rounded
// fraction are off by up to 1.5e-7 and save nothing from 16 heads on (20736 rows of
// 16 heads of 80: 36 us with either; 65536 rows of a single head of 128: 27 us, 25
// with those).  bf16 outputs, whose rounding is 2^16 times theirs, take the fp32
// functions.  Products are fp32 and each output is rounded once.
//
// Bound by HBM: every element is read once and written once, 3 operations
// between.  One wave takes one token at a time (or a share of its heads while
// tokens are fewer than the waves the device holds): a lane forms the
// frequency of its pair once and the sine and cosine once per token, for all
// heads, and passes them through LDS; then the wave walks the token's heads
// in units of VE pairs (two 16-byte reads and writes: VE = 8 for bf16, 4 for
// fp32), with kBatch units of every lane in flight.  Measured: 65536 rows of 80
// heads of 128 into a cache 527 us, 5.1 TB/s; 6272 rows of 32 heads 18.2 us;
// 8 rows 3.6 us, the launch and three dependent latencies (a copy of 2 GiB
// runs at 4.9 TB/s).
#include <math.h>

#include <algorithm>

#include "device_common.hpp"
#include "launch.hpp"

namespace sd {
namespace {

constexpr int kWavesWg = 4;
// Units in flight per lane: two leave few enough registers for eight waves a
// SIMD (26111 rows of a video prompt 104 -> 97 us against four; eight units 148).
constexpr int kBatch = 2;
constexpr int kWgsCu = 16;     // work-groups per compute unit, two rounds of those waves
constexpr double kInv2Pi = 0.15915494309189533577;

// VE values of type T at p as floats, with the widest loads that VE allows
template <typename T, int VE>
__device__ __forceinline__ void load_vec(const T* p, float (&x)[VE]) {
  constexpr int W = VE * (int)sizeof(T) / 4;   // 32-bit words
  if constexpr (W >= 2 && W % 2 == 0) {
    uint32_t w[W];
    if constexpr (W % 4 == 0) {
#pragma unroll
      for (int k = 0; k < W / 4; ++k) {
        const u32x4 u = reinterpret_cast<const u32x4*>(p)[k];
#pragma unroll
        for (int e = 0; e < 4; ++e) w[4 * k + e] = u[e];
      }
    } else {
      const u32x2 u = *reinterpret_cast<const u32x2*>(p);
      w[0] = u[0];
      w[1] = u[1];
    }
#pragma unroll
    for (int e = 0; e < VE; ++e) {
      if constexpr (sizeof(T) == 4)
        x[e] = __uint_as_float(w[e]);
      else
        x[e] = __uint_as_float((e & 1) ? (w[e / 2] & 0xffff0000u) : (w[e / 2] << 16));
    }
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) x[e] = (float)p[e];
  }
}

template <typename T, int VE>
__device__ __forceinline__ void store_vec(T* p, const float (&x)[VE]) {
  constexpr int W = VE * (int)sizeof(T) / 4;
  if constexpr (W >= 2 && W % 2 == 0) {
    union {
      T t[VE];
      uint32_t w[W];
    } o;
#pragma unroll
    for (int e = 0; e < VE; ++e) o.t[e] = (T)x[e];   // to nearest even
    if constexpr (W % 4 == 0) {
#pragma unroll
      for (int k = 0; k < W / 4; ++k)
        reinterpret_cast<u32x4*>(p)[k] = u32x4{o.w[4 * k], o.w[4 * k + 1], o.w[4 * k + 2], o.w[4 * k + 3]};
    } else {
      *reinterpret_cast<u32x2*>(p) = u32x2{o.w[0], o.w[1]};
    }
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) p[e] = (T)x[e];
  }
}

// Sequence of row t: the largest b < B with row_start[b] <= t, by a search of
// 64 probes per step (one step up to 64 sequences); wave-uniform.
__device__ __forceinline__ int sequence_of(const int32_t* row_start, int B, int t) {
  const int lane = threadIdx.x & 63;
  int lo = 0, hi = B;
  while (true) {
    const int step = (hi - lo + 63) / 64;
    const int i = lo + lane * step;
    const unsigned long long hit = __ballot(i < hi && row_start[min(i, B - 1)] <= t);
    lo += max((int)__popcll(hit) - 1, 0) * step;
    if (step == 1) return min(lo, B - 1);
    hi = min(hi, lo + step);
  }
}

template <typename TS, typename TD, int VE, bool APPEND>
__global__ __launch_bounds__(kWavesWg * 64) void rope_rows(RopeArgs a) {
  __shared__ __align__(16) float2 table[kWavesWg][kRopeMaxPairs];
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int P = a.pairs, D = a.D;

  // frequencies of pairs lane and lane + 64, in turns per position, and their axes
  double f[2] = {0.0, 0.0};
  int axis[2] = {0, 0};
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int i = lane + 64 * k;
    if (i < P) {
      int ax = 0, first = 0, n = a.end[0];
#pragma unroll
      for (int x = 0; x + 1 < kRopeMaxAxes; ++x) {
        if (x + 1 < a.axes && i >= a.end[x]) {
          ax = x + 1;
          first = a.end[x];
          n = a.end[x + 1] - first;
        }
      }
      if (!a.per_axis) {
        first = 0;
        n = P;
      }
      axis[k] = ax;
      f[k] = exp(-(double)(i - first) / (double)n * a.log_theta) * kInv2Pi;
    }
  }

  // units of a head: P / VE of two vectors that turn, then the copied rest
  const int turning = P / VE;
  const int units = turning + (D - 2 * P) / VE;
  const int heads = a.Hq + 2 * a.Hkv;
  const int share = a.share;                       // waves per token
  const int slots = gridDim.x * kWavesWg / share;  // tokens in flight
  const int wave = blockIdx.x * kWavesWg + w;
  const int part = wave % share;
  for (int t = wave / share; t < a.T; t += slots) {
    // the token's place in the cache: -1 where there is none
    TD* kdst = nullptr;
    TD* vdst = nullptr;
    int p = 0, head_step = D;
    if constexpr (APPEND) {
      int b, j, n;
      if (a.row_start != nullptr) {
        if (t < a.row_start[0] || t >= a.row_start[a.B]) continue;
        b = __builtin_amdgcn_readfirstlane(sequence_of(a.row_start, a.B, t));
        j = t - a.row_start[b];
        n = a.row_start[b + 1] - a.row_start[b];
      } else {
        n = a.rows;
        b = t / n;
        j = t - b * n;
      }
      p = a.kv_len[b] - n + j;
      size_t at = 0;
      bool ok = p >= 0 && p < a.capacity;
      if (ok) {
        if (a.page_table != nullptr) {
          const int page = a.page_table[(size_t)b * a.max_pages + (p >> 4)];
          ok = page >= 0 && page < a.num_pages;
          at = ((size_t)page * a.Hkv * 16 + (p & 15)) * D;
          head_step = 16 * D;
        } else {
          at = ((size_t)b * a.capacity + p) * a.Hkv * D;
        }
      }
      if (ok) {
        kdst = static_cast<TD*>(a.k_cache) + at;
        vdst = static_cast<TD*>(a.v_cache) + at;
      }
    }
    // sines and cosines of this token, for every head
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = lane + 64 * k;
      if (i < P) {
        const int q = a.pos != nullptr ? a.pos[(size_t)axis[k] * a.T + t] : p;
        double turn = (double)q * f[k];
        turn -= rint(turn);
        float sn, cs;
        if constexpr (sizeof(TD) == 4) {
          double s64, c64;
          sincospi(2.0 * turn, &s64, &c64);
          sn = (float)s64;
          cs = (float)c64;
        } else {
          sincospif((float)(2.0 * turn), &sn, &cs);
        }
        table[w][i] = make_float2(cs, a.inverse ? -sn : sn);
      }
    }
    // one wave writes and reads its own row of the table: LDS operations of a
    // wave complete in order, the barrier only holds the compiler
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");

    int h = (part * 64 + lane) / units;
    int c = (part * 64 + lane) - h * units;
    while (h < heads) {
      float x1[kBatch][VE], x2[kBatch][VE];
      TD* dst[kBatch];
      int unit[kBatch];
      bool turns[kBatch];
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        dst[k] = nullptr;
        unit[k] = c;
        turns[k] = false;
        if (h < heads) {
          const TS* src;
          if (h < a.Hq) {
            src = static_cast<const TS*>(a.q) + (size_t)t * a.q_stride + (size_t)h * D;
            dst[k] = static_cast<TD*>(a.q_out) + (size_t)t * a.q_out_stride + (size_t)h * D;
          } else if (h < a.Hq + a.Hkv) {
            src = static_cast<const TS*>(a.k) + (size_t)t * a.k_stride + (size_t)(h - a.Hq) * D;
            if (kdst != nullptr) dst[k] = kdst + (size_t)(h - a.Hq) * head_step;
          } else {
            src = static_cast<const TS*>(a.v) + (size_t)t * a.v_stride + (size_t)(h - a.Hq - a.Hkv) * D;
            if (vdst != nullptr) dst[k] = vdst + (size_t)(h - a.Hq - a.Hkv) * head_step;
          }
          if (c < turning) {
            turns[k] = h < a.Hq + a.Hkv;
            load_vec<TS, VE>(src + c * VE, x1[k]);
            load_vec<TS, VE>(src + P + c * VE, x2[k]);
          } else {
            load_vec<TS, VE>(src + 2 * P + (c - turning) * VE, x1[k]);
          }
        }
        c += a.step_unit;
        h += a.step_head;
        if (c >= units) {
          c -= units;
          ++h;
        }
      }
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        if (dst[k] == nullptr) continue;
        const int u = unit[k];
        if (u >= turning) {
          store_vec<TD, VE>(dst[k] + 2 * P + (u - turning) * VE, x1[k]);
          continue;
        }
        if (turns[k]) {
#pragma unroll
          for (int e = 0; e < VE; ++e) {
            const float2 cs = table[w][u * VE + e];
            const float y1 = x1[k][e] * cs.x - x2[k][e] * cs.y;
            const float y2 = x1[k][e] * cs.y + x2[k][e] * cs.x;
            x1[k][e] = y1;
            x2[k][e] = y2;
          }
        }
        store_vec<TD, VE>(dst[k] + u * VE, x1[k]);
        store_vec<TD, VE>(dst[k] + P + u * VE, x2[k]);
      }
    }
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();   // the next token's table overwrites this one's
  }
}

template <typename TS, typename TD, int VE, bool APPEND>
hipError_t launch(RopeArgs a, int cus, hipStream_t st) {
  const int units = a.pairs / VE + (a.D - 2 * a.pairs) / VE;
  const long long items = (long long)(a.Hq + 2 * a.Hkv) * units;
  // while the tokens are fewer than the grid's waves, several share a token's
  // heads, down to one unit per lane (8 rows of 32 heads: 5.1 us in one wave each,
  // 3.6 so)
  const long long waves = (long long)std::max(cus, 1) * kWgsCu * kWavesWg;
  long long share = std::min(waves / a.T, (items + 63) / 64);
  a.share = 1;
  while (a.share * 2 <= share && a.share < 64) a.share *= 2;
  a.step_head = (int)(64 * a.share / units);
  a.step_unit = (int)(64 * a.share % units);
  const long long wgs = std::min(((long long)a.T * a.share + kWavesWg - 1) / kWavesWg, waves / kWavesWg);
  // slots = work-groups x waves / share must be whole
  const long long per = std::max(1, a.share / kWavesWg);
  hipLaunchKernelGGL((rope_rows<TS, TD, VE, APPEND>), dim3((unsigned)((wgs + per - 1) / per * per)),
                     dim3(kWavesWg * 64), 0, st, a);
  return hipGetLastError();
}

template <typename TS, typename TD, bool APPEND>
hipError_t by_width(const RopeArgs& a, int width, int cus, hipStream_t st) {
  // (eight fp32 outputs would be two stores of 16 bytes 32 bytes apart on the
  // lanes: 20736 rows of 16 heads of 80 51 us, 44 with four)
  if constexpr (sizeof(TD) == 2)
    if (width >= 8) return launch<TS, TD, 8, APPEND>(a, cus, st);
  if (width >= 4) return launch<TS, TD, 4, APPEND>(a, cus, st);
  return launch<TS, TD, 1, APPEND>(a, cus, st);
}

}  // namespace

// Values per vector that every address and every run of channels allows: 8 or
// 4 (16-byte accesses where that is at least 16 bytes), or single values.
static int vector_width(const RopeArgs& a, int src_size, int dst_size) {
  for (int ve = 8; ve > 1; ve /= 2) {
    const size_t sb = std::min(16, ve * src_size), db = std::min(16, ve * dst_size);
    auto on = [](const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; };
    auto whole = [](long long stride, int size, size_t n) { return (size_t)stride * size % n == 0; };
    if (a.D % ve != 0 || a.pairs % ve != 0) continue;
    if (!on(a.q, sb) || !on(a.k, sb) || !on(a.v, sb) || !on(a.q_out, db) || !on(a.k_cache, db) || !on(a.v_cache, db))
      continue;
    if (!whole(a.q_stride, src_size, sb) || !whole(a.k_stride, src_size, sb) || !whole(a.v_stride, src_size, sb) ||
        !whole(a.q_out_stride, dst_size, db))
      continue;
    return ve;
  }
  return 1;
}

hipError_t launch_rope(const RopeArgs& a, int dtype, int cus, hipStream_t st) {
  if (dtype == 0) return by_width<float, float, false>(a, vector_width(a, 4, 4), cus, st);
  return by_width<__bf16, __bf16, false>(a, vector_width(a, 2, 2), cus, st);
}

hipError_t launch_kv_append(const RopeArgs& a, int src_dtype, int dtype, int cus, hipStream_t st) {
  if (src_dtype == 0 && dtype == 0) return by_width<float, float, true>(a, vector_width(a, 4, 4), cus, st);
  if (src_dtype == 0) return by_width<float, __bf16, true>(a, vector_width(a, 4, 2), cus, st);
  return by_width<__bf16, __bf16, true>(a, vector_width(a, 2, 2), cus, st);
}

}  // namespace sd
