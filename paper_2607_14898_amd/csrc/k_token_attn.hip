// Attention of new tokens over the slots of a token cache, and the weight that every
// slot receives.
//
// Rows (query tokens x heads of a KV group) meet keys on the 32x32 MFMA as
// S^T = K Q^T, so a lane holds one row and 16 keys of a 32-key block: the row maximum
// takes one exchange between the wave's halves and the row sum stays in the lane until
// the end. Keys go to the MFMA in the order that makes the scores' registers exactly
// the B operand of O^T += V^T P^T, so probabilities never leave the registers. V
// stays as it lies in the cache, [slot][dim]: the 16-bit kernels read its transposed
// fragments from LDS with the transposing read, the fp32 ones element by element.
// The fp32 MFMA takes one key (one dim) of each half a step, so eight of them are one
// 16-bit MFMA and everything else is the same code.
//
// What a row sees goes by positions: slot s is visible to row r if 0 <= pos[s] < lim[r]
// (lim = query position + 1 if causal, 2^31 if not, 0 for padding), one unsigned
// comparison. Tiles of slots that no row sees are skipped before their keys are loaded,
// and tiles that every row sees need no mask.
//
// Whatever empty and hidden slots hold must not matter. Scores are replaced, not added
// to. Empty slots are left out (many rows) or their V is zeroed as it is staged (few). V
// of slots hidden from some rows alone may hold infinities or NaN, which 0 x V would spread: rows that end up not finite are
// computed once more with such elements as zeros, and if there were any, those of visible
// slots are then added. Finite data comes here only where its unnormalised sums overflow; the
// second time they do not.
#include "fd_token.h"

#include <stdint.h>

#include <algorithm>
#include <initializer_list>
#include <type_traits>

namespace fd {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Values of fp32's range may overflow the sums, whose probabilities reach 2^8 for up to 2^24
// slots. Rows that end not finite are computed again, and then these are 2^-40 of that.
constexpr float kBelow = 40.f;

template <typename T> struct Op;
template <> struct Op<_Float16> {
  using V = f16x8;
  // Probabilities are kept below 2^15 and, with the running maximum at 2^6, above the
  // subnormal f16 values down to 2^-20 of it.
  static constexpr float kShift = 6.f;
  static constexpr float kDown = 0.f;  // (f16 values times those sums are far from fp32's end)
  static __device__ __forceinline__ f32x16 mma(V a, V b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Op<__bf16> {
  using V = bf16x8;
  static constexpr float kShift = 0.f;
  static constexpr float kDown = kBelow;
  static __device__ __forceinline__ f32x16 mma(V a, V b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Op<float> {
  using V = f32x8;
  static constexpr float kShift = 0.f;
  static constexpr float kDown = kBelow;
  static __device__ __forceinline__ f32x16 mma(V a, V b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

// Adding n terms one by one in fp32 is off by up to n half steps, and equal terms come close to
// that: a sum over 2^19 of them in a row was off by 5e-3. So no sum runs on for long: those of
// single keys or MFMAs end after this many slots (rows) and are added up in turn (folds: 1% of a
// chunk of 4096 tokens x 4 heads, 8 groups, 65536 slots, 128 dims, bf16; every 8192 slots 2.5%).
constexpr int kPartSlots = 16384;       // of a part of attend_keys_kernel (four waves)
template <typename T> constexpr int kFoldSlots = sizeof(T) == 4 ? 4096 : 16384;  // of attend_rows_kernel
constexpr int kPartRows = 32768;        // of a part of weights_kernel (32 lanes)

constexpr f32x16 kZero = {};
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr float kRaise = 8.f;  // the running shift rises when a score passes it by 2^8

// Key that A row i of the score MFMA holds (i = 8a + 4b + c: key 16 (a / 2) + 8 b +
// 4 (a % 2) + c): register r of lane l is then key 16 (r / 8) + 8 (l / 32) + r % 8.
__device__ __forceinline__ int key_of_row(int i) {
  return 16 * (i >> 4) + 8 * ((i >> 2) & 1) + 4 * ((i >> 3) & 1) + (i & 3);
}

// 16-byte chunk ch of row `row` of a [rows][D] tile in LDS. K fragments read one chunk
// of 16 different rows at a time, so chunks are permuted by the row (rows that share
// 256 bytes alike); transposing V reads take 64 bytes of four rows at a time, which are
// spread over the four 64-byte parts of 256 bytes.
template <typename T, int D> struct Tile {
  static constexpr int CPR = D * (int)sizeof(T) / 16;
  static constexpr int EPC = 16 / (int)sizeof(T);
  static __device__ __forceinline__ int k(int row, int ch) {
    constexpr int RP = CPR < 16 ? 16 / CPR : 1, M = (CPR < 16 ? CPR : 16) - 1;
    return row * CPR + (ch ^ ((row / RP) & M));
  }
  static __device__ __forceinline__ int v(int row, int ch) {
    if constexpr (sizeof(T) == 4 || CPR == 4) return row * CPR + ch;
    if constexpr (CPR == 8) return row * CPR + (ch ^ (((row >> 1) & 1) << 2));
    return row * CPR + (ch ^ ((row & 3) << 2));
  }
  // dims 16 ks + 8 lh .. + 7 of key row `row`
  static __device__ __forceinline__ typename Op<T>::V k_frag(const u32x4* t, int row, int ks, int lh) {
    typename Op<T>::V f;
    if constexpr (sizeof(T) == 2) {
      const u32x4 x = t[k(row, 2 * ks + lh)];
      f = *reinterpret_cast<const typename Op<T>::V*>(&x);
    } else {
      const u32x4 x = t[k(row, 4 * ks + 2 * lh)], y = t[k(row, 4 * ks + 2 * lh + 1)];
      const float4 a = *reinterpret_cast<const float4*>(&x), b = *reinterpret_cast<const float4*>(&y);
      f = typename Op<T>::V{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    }
    return f;
  }
  // dim 32 d + lane % 32 of keys row0 + 8 (lane / 32) .. + 7
  static __device__ __forceinline__ typename Op<T>::V v_frag(const u32x4* t, int row0, int d, int lane) {
    typename Op<T>::V f;
    if constexpr (sizeof(T) == 2) {
      // lane j of 16 hands in 4 dims of key j / 4 and gets dim j of four keys
      const int j = lane & 15, q = lane >> 4;
      const int row = row0 + 8 * (q >> 1) + (j >> 2), ch = 4 * d + 2 * (q & 1) + ((j & 3) >> 1);
      union {
        i16x4 h[2];
        typename Op<T>::V v;
      } u;
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const char* p = (const char*)(t + v(row + 4 * x, ch)) + 8 * (j & 1);
        u.h[x] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(p));
      }
      f = u.v;
    } else {
      const float* p = reinterpret_cast<const float*>(t) + (row0 + 8 * (lane >> 5)) * D + 32 * d + (lane & 31);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = p[e * D];
    }
    return f;
  }
};

__device__ __forceinline__ float other_half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float other_half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
// Sum over the 32 lanes of a half, in its last lane.
__device__ __forceinline__ float half_sum(float x) {
  auto moved = [](float y, auto ctrl, auto rows) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(y), decltype(ctrl)::value, decltype(rows)::value,
                                                      0xf, false));
  };
  using std::integral_constant;
  x += moved(x, integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});  // 1, 2, 4, 8 lanes up in 16
  x += moved(x, integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
  x += moved(x, integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});  // rows 0, 2 into 1, 3
  return x;
}
__device__ __forceinline__ uint32_t lanes_max(uint32_t x) {
  for (int o = 32; o > 0; o >>= 1) x = max(x, (uint32_t)__shfl_xor((int)x, o));
  return __builtin_amdgcn_readfirstlane(x);
}
__device__ __forceinline__ uint32_t lanes_min(uint32_t x) {
  for (int o = 32; o > 0; o >>= 1) x = min(x, (uint32_t)__shfl_xor((int)x, o));
  return __builtin_amdgcn_readfirstlane(x);
}

// 16 bytes of V with its infinities and NaN as zeros.
template <typename T> __device__ __forceinline__ u32x4 finite_part(u32x4 x) {
  union {
    u32x4 u;
    T e[16 / sizeof(T)];
  } w;
  w.u = x;
#pragma unroll
  for (int i = 0; i < (int)(16 / sizeof(T)); ++i)
    if (!isfinite((float)w.e[i])) w.e[i] = (T)0.f;
  return w.u;
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, bytes, 0x00020000);
}
__device__ __forceinline__ uint32_t lds_address(const u32x4* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const u32x4*)p;
}

// The rows of a call: where a row's query lies, and the first position it does not see.
struct Row {
  int i, head;     // query token, head
  uint32_t lim;
};
// r / rep: below 2^24 and for rep <= 256 the high word of r ceil(2^32 / rep) is exact
// (the multiplier is less than rep / 2^32 too large, and r rep < 2^32).
__device__ __forceinline__ int token_of(const TokenAttend& a, int r) {
  return a.rep == 1 ? r : (int)__umulhi((uint32_t)r, a.rep_inv);
}
__device__ __forceinline__ Row row_of(const TokenAttend& a, int b, int g, int64_t r, int64_t R) {
  Row w{0, g * a.rep, 0};
  if (r < R) {
    w.i = token_of(a, (int)r);
    w.head = g * a.rep + (int)r - w.i * a.rep;
    const int p = a.pos[(int64_t)b * a.n + w.i];
    w.lim = p < 0 ? 0u : a.causal ? (uint32_t)p + 1u : 0x80000000u;
  }
  return w;
}
template <typename T> __device__ __forceinline__ const T* q_of(const TokenAttend& a, int b, const Row& w) {
  return (const T*)a.q + b * a.qs[0] + w.i * a.qs[1] + w.head * a.qs[2];
}
template <typename T> __device__ __forceinline__ T* out_of(const TokenAttend& a, int b, const Row& w) {
  return (T*)a.out + b * a.os[0] + w.i * a.os[1] + w.head * a.os[2];
}

// One row of a wave's 32 (held by lanes lr and lr + 32): running shift, sum and output.
template <typename T, int D, bool EXACT> struct Softmax {
  using O = Op<T>;
  f32x16 acc[D / 32];  // O^T: dims 32 d + 8 (r / 4) + 4 (lane / 32) + r % 4 of the lane's row
  float m, l;          // shift in log2 units (-inf: nothing seen), sum over this half's keys
  __device__ __forceinline__ void reset() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
  }
  // Scores of KB 32-key blocks (hidden ones -inf) and their values in LDS. Probabilities
  // enter 2^-down of what the shift says.
  template <int KB>
  __device__ __forceinline__ void add(f32x16 (&s)[KB], float c, float down, const u32x4* vt, int row0, int lane) {
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    mx = other_half_max(mx) * c;
    // The shift need not be the maximum: it only keeps the probabilities in range, so it
    // follows a rising maximum when that is 2^8 ahead (and from the first visible key on).
    if (__ballot(mx > m + kRaise) != 0) {
      const float mn = fmaxf(m, mx);
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= f;
    }
    const float sub = m == -INFINITY ? 0.f : O::kShift - down - m;
    // 16 keys at a time where registers are short, else all the exponentials before all
    // the MFMAs (which then run at raised priority in one go)
    constexpr int NX = KB * 2, GX = D == 128 ? 1 : NX;
#pragma unroll
    for (int x0 = 0; x0 < NX; x0 += GX) {
      // (V's fragments are on their way while the exponentials are taken)
      typename O::V ph[GX], pl[GX], vf[GX][D / 32];
      float add = 0.f;  // (a sum of its own: see kPartSlots)
#pragma unroll
      for (int y = 0; y < GX; ++y)
#pragma unroll
        for (int d = 0; d < D / 32; ++d) vf[y][d] = Tile<T, D>::v_frag(vt, row0 + 16 * (x0 + y), d, lane);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int y = 0; y < GX; ++y)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int x = x0 + y;
          const float p = __builtin_amdgcn_exp2f(fmaf(s[x / 2][8 * (x % 2) + e], c, sub));
          add += p;
          // P enters the second MFMA in the cache's type. Where memory bounds the kernel
          // (EXACT) what that rounding loses goes in by a second MFMA; elsewhere, where it would
          // be half as many MFMAs again, its half step per key, as large as the output's own
          // rounding, is kept (the sum that it is divided by is of unrounded ones). Error against
          // 64 bits, all in: the bf16 long chunk 2.3e-3 (the output's rounding alone 1.7e-3), the fp16
          // frame 2.9e-4 (2.1e-4).
          ph[y][e] = (T)p;
          if constexpr (EXACT && sizeof(T) == 2) pl[y][e] = (T)(p - (float)ph[y][e]);
        }
      l += add;
      __builtin_amdgcn_s_setprio(2);
#pragma unroll
      for (int y = 0; y < GX; ++y)
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          acc[d] = O::mma(vf[y][d], ph[y], acc[d]);
          if constexpr (EXACT && sizeof(T) == 2) acc[d] = O::mma(vf[y][d], pl[y], acc[d]);
        }
      __builtin_amdgcn_s_setprio(0);
    }
  }
  __device__ __forceinline__ bool finite() const {
    float t = 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) t += 0.f * acc[d][r];  // NaN if any is not finite
    return t == 0.f;
  }
  // A row whose scores were all NaN has no maximum, but it has seen something.
  __device__ __forceinline__ void close(float sum) {
    if (m == -INFINITY && sum != sum) m = 0.f;
  }
  // Adds the infinities and NaN among the values of slots s0 .. s1 - 1 that the row sees.
  // The wave looks through several slots at a load; only those that hold some are added.
  __device__ __forceinline__ void add_unbounded(const T* v, int64_t step, const int* pos, int s0, int s1, uint32_t lim,
                                                int lane) {
    using TL = Tile<T, D>;
    constexpr int SL = 64 / TL::CPR, U = 8;  // slots of a load, loads under way
    for (int x0 = s0; x0 < s1; x0 += SL * U) {
      u32x4 c[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        c[u] = *reinterpret_cast<const u32x4*>(v + min(x0 + u * SL + lane / TL::CPR, s1 - 1) * step +
                                               lane % TL::CPR * TL::EPC);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const u32x4 f = finite_part<T>(c[u]);
        uint64_t bad = __ballot(f.x != c[u].x || f.y != c[u].y || f.z != c[u].z || f.w != c[u].w);
        while (bad) {
          const int x = x0 + u * SL + __builtin_ctzll(bad) / TL::CPR;
          bad &= ~0ull << (__builtin_ctzll(bad) / TL::CPR * TL::CPR + TL::CPR - 1) << 1;
          if (x >= s1 || (uint32_t)pos[x] >= lim) continue;
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float y = (float)v[x * step + 32 * d + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3)];
              if (!isfinite(y)) acc[d][r] += y;
            }
        }
      }
    }
  }
};

// A part's output on the joined shift. A factor that underflows takes a part out, but not
// the infinities and NaN of values that the row sees: they reach it however slots are parted.
__device__ __forceinline__ float on_shift(float x, float f) {
  return f != 0.f ? x * f : isfinite(x) ? 0.f : x;
}

// Stores 4 consecutive dims.
template <typename T> __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
  struct alignas(4 * sizeof(T)) Q { T e[4]; };
  *reinterpret_cast<Q*>(p) = Q{(T)a, (T)b, (T)c, (T)d};
}

// (part_ml holds shift and sum of each part's rows, part_o their output.)

// Few rows (serving): memory bounds it, so the keys are parted among as many waves as it
// takes. A wave walks 32-slot tiles of its workgroup's part on its own: it stages a
// tile's keys, then its values, through 32 rows of LDS that no other wave touches, so the
// loop has no barrier and a CU's waves drift apart. Both loads of a tile go out together;
// with 8 to 12 waves on a CU up to 128 KB are in flight. The four waves' results meet in
// LDS, the parts' in finish_kernel. 16 requests, 8 groups, 4 heads each, 128 dims, 16384 slots
// (30 to 100% full), bf16: 168 us, 4.2 TB/s with the scores written for the weights, 5.2 to
// 5.5 TB/s without.
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D == 512 ? 1 : 2) void attend_keys_kernel(TokenCacheArgs c,
                                                                                        TokenAttend a,
                                                                                        TokenAttendPlan pl) {
  using TL = Tile<T, D>;
  constexpr int NV = 32 * TL::CPR / 64;  // 16-byte loads of a lane per tile
  constexpr int kTileB = 32 * D * (int)sizeof(T), kJoinB = 32 * 33 * 4;
  __shared__ u32x4 buf[4][(kTileB > kJoinB ? kTileB : kJoinB) / 16];
  __shared__ int spos[4][32];
  __shared__ float sm[4][32], sl[4][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int split = blockIdx.x, rt = blockIdx.y, bg = blockIdx.z, b = bg / c.G, g = bg - b * c.G;
  const int64_t R = (int64_t)a.n * a.rep;
  const int64_t row = (int64_t)rt * 32 + lr;
  const Row w = row_of(a, b, g, row, R);
  const uint32_t lim_max = lanes_max(w.lim), lim_min = lanes_min(w.lim ? w.lim : ~0u);
  const float cs = a.scale * kLog2e;

  typename Op<T>::V qf[D / 16];
  {
    const T* q = q_of<T>(a, b, w);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[ks][e] = (T)0.f;
      if (row < R) qf[ks] = *reinterpret_cast<const typename Op<T>::V*>(q + 16 * ks + 8 * lh);
    }
  }
  const T* kb = (const T*)c.k + b * c.ks[0] + g * c.ks[1];
  const T* vb = (const T*)c.v + b * c.vs[0] + g * c.vs[1];
  const int* ps = c.pos + (int64_t)bg * c.C;

  // Tiles are dealt to the parts' waves in turn: used slots lie in front in a cache that has
  // room, and contiguous parts behind them would have nothing to do.
  const int tiles = (c.C + 31) / 32, hop = 4 * pl.splits, t0 = 4 * split + wave;
  u32x4* tile = buf[wave];
  Softmax<T, D, true> sx;
  bool changed = false;  // some value of this wave's slots is not finite
  for (int scrub = 0;; scrub = 1) {
    sx.reset();
    for (int tc = t0; tc < tiles; tc += hop * 64) {
      // which of the wave's next 64 tiles any row sees, two tiles a load: walked one by one,
      // an empty tile would cost a wait for memory
      uint64_t live = 0;
#pragma unroll 8
      for (int x = 0; x < 32; ++x) {
        const int t = tc + hop * (2 * x + lh), sp = t * 32 + lr;
        const uint64_t m = __ballot((t < tiles && sp < c.C ? (uint32_t)ps[sp] : ~0u) < lim_max);
        live |= (uint64_t)((uint32_t)m != 0) << (2 * x) | (uint64_t)((uint32_t)(m >> 32) != 0) << (2 * x + 1);
        if (tc + 2 * hop * (x + 1) >= tiles) break;
      }
      while (live) {
        const int t = tc + hop * __builtin_ctzll(live);
        live &= live - 1;
        const int p = t * 32 + lr < c.C ? ps[t * 32 + lr] : -1;
        const uint32_t taken = (uint32_t)__ballot(p >= 0);
        const bool all = (uint32_t)__ballot((uint32_t)p < lim_min) == ~0u;
        u32x4 kr[NV], vr[NV];
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int idx = j * 64 + lane, kr_ = idx / TL::CPR, ch = idx % TL::CPR;
          const int64_t s = min(t * 32 + kr_, c.C - 1);
          kr[j] = *reinterpret_cast<const u32x4*>(kb + s * c.ks[2] + ch * TL::EPC);
          vr[j] = *reinterpret_cast<const u32x4*>(vb + s * c.vs[2] + ch * TL::EPC);
        }
        if (!all) spos[wave][lr] = p;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int idx = j * 64 + lane;
          tile[TL::k(idx / TL::CPR, idx % TL::CPR)] = kr[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        f32x16 s[1];
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          s[0] = Op<T>::mma(TL::k_frag(tile, key_of_row(lr), ks, lh), qf[ks], ks ? s[0] : kZero);
        if (a.weight_out && row < R) {  // [tile][row][32]: whole lines, however few the rows
          float* score = (float*)a.ws + pl.scores + (((int64_t)bg * tiles + t) * R + row) * 32 + 8 * lh;
#pragma unroll
          for (int r = 0; r < 16; r += 4)
            store4(score + 16 * (r >> 3) + (r & 4), s[0][r], s[0][r + 1], s[0][r + 2], s[0][r + 3]);
        }
        if (!all) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((uint32_t)spos[wave][16 * (r >> 3) + 8 * lh + (r & 7)] >= w.lim) s[0][r] = -INFINITY;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int idx = j * 64 + lane, vrow = idx / TL::CPR;
          u32x4 x = vr[j];
          if (!(taken >> vrow & 1)) x = u32x4{0, 0, 0, 0};
          if (scrub) {
            const u32x4 f = finite_part<T>(x);
            changed |= f.x != x.x || f.y != x.y || f.z != x.z || f.w != x.w;
            x = f;
          }
          tile[TL::v(vrow, idx % TL::CPR)] = x;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        sx.template add<1>(s, cs, scrub ? Op<T>::kDown : 0.f, tile, 0, lane);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      }
    }
    if (scrub) {
      sx.m += Op<T>::kDown;
      if (__ballot(changed))
        for (int t = t0; t < tiles; t += hop)
          sx.add_unbounded(vb, c.vs[2], ps, t * 32, min(t * 32 + 32, c.C), w.lim, lane);
      break;
    }
    if (__ballot(w.lim != 0 && !sx.finite()) == 0) break;
  }

  if (w.lim == 0) {  // padding: what tiles without a mask gave it does not count
    sx.m = -INFINITY;
    sx.l = 0.f;
  }
  // the four waves' rows on one shift
  const float lsum = other_half_sum(sx.l);
  sx.close(lsum);
  if (lh == 0) {
    sm[wave][lr] = sx.m;
    sl[wave][lr] = lsum;
  }
  __syncthreads();
  const float M = fmaxf(fmaxf(sm[0][lr], sm[1][lr]), fmaxf(sm[2][lr], sm[3][lr]));
  const float f = sx.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(sx.m - M);
  float L = 0.f;
#pragma unroll
  for (int x = 0; x < 4; ++x) L += sm[x][lr] == -INFINITY ? 0.f : sl[x][lr] * __builtin_amdgcn_exp2f(sm[x][lr] - M);
  // (normalised before they are added up: sums of parts could overflow where their mean does not)
  const float part = f == 0.f ? 0.f : f / L;
  const bool direct = pl.splits == 1 && !a.weight_out;
  float* ml = (float*)a.ws + pl.part_ml + (((int64_t)bg * pl.splits + split) * R + row) * 2;
  if (wave == 0 && lh == 0 && row < R) {
    if (!direct) {
      ml[0] = M;
      ml[1] = L;
    } else if (a.lse) {
      a.lse[((int64_t)b * c.G * a.rep + w.head) * a.n + w.i] =
          M == -INFINITY ? -INFINITY : (M - Op<T>::kShift + __builtin_amdgcn_logf(L)) * kLn2;
    }
  }
  // outputs of 32 dims at a time: thread -> row tid / 8, 4 dims
  const int orow = tid >> 3, od = 4 * (tid & 7);
  const int64_t orow_g = (int64_t)rt * 32 + orow;
  const Row ow = row_of(a, b, g, orow_g, R);
  const bool none = fmaxf(fmaxf(sm[0][orow], sm[1][orow]), fmaxf(sm[2][orow], sm[3][orow])) == -INFINITY;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    float* so = (float*)buf[wave];
#pragma unroll
    for (int r = 0; r < 16; ++r) so[lr * 33 + 8 * (r >> 2) + 4 * lh + (r & 3)] = on_shift(sx.acc[d][r], part);
    __syncthreads();
    float o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      o[e] = 0.f;
#pragma unroll
      for (int x = 0; x < 4; ++x) o[e] += ((const float*)buf[x])[orow * 33 + od + e];
    }
    if (orow_g < R) {
      if (direct) {
        if (none) store4(out_of<T>(a, b, ow) + 32 * d + od, 0.f, 0.f, 0.f, 0.f);
        else store4(out_of<T>(a, b, ow) + 32 * d + od, o[0], o[1], o[2], o[3]);
      } else {
        store4((float*)a.ws + pl.part_o + (((int64_t)bg * pl.splits + split) * R + orow_g) * D + 32 * d + od, o[0], o[1],
               o[2], o[3]);
      }
    }
    __syncthreads();
  }
}

// Many rows (a chunk of tokens): the matrix cores and the exponentials bound it. A
// workgroup's four waves own 32 rows each and share tiles of KT slots through LDS, two
// of them in turn: the next tile's 16-byte loads fly while a tile is computed.
//
// Slots are taken through a list. In a cache that has turned over, a chunk's own tokens
// lie scattered among the old ones and every tile of consecutive slots would need a mask,
// so the workgroup first sorts kScan slots' indices by what its rows see of them: those
// that all rows see, those that some see (the chunk's own tokens, later ones left out),
// nothing else. Only the second kind is masked, and empty slots cost no tile.
//
// 4096 tokens x 4 heads, 8 groups, 128 dims, 12288 old and 4096 own slots, bf16: 975 us on the
// fastest machine seen and 1056 on the slowest, 987 and 911 TFLOP/s (a large library product on
// the former: 1187); the sorting took it from 1275 to 1134.
// 1560 x 8 rows, 3 groups, 64 dims, 4680 slots, fp16: 85 to 88 us, 529 to 511 TFLOP/s. In two of five
// cycles there neither an MFMA nor a vector instruction issues: every tile waits for its
// maximum (over its scores, then the other half's, then the vote) before its first exponential,
// and 588 workgroups lie uneven on 768 places.
constexpr int kScan = 4096, kBlock = 64;
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D == 512 ? 1 : 2) void attend_rows_kernel(TokenCacheArgs c,
                                                                                        TokenAttend a,
                                                                                        TokenAttendPlan pl) {
  using TL = Tile<T, D>;
  constexpr int KB = sizeof(T) == 2 ? 2 : 1, KT = 32 * KB;
  constexpr int NV = KT * TL::CPR / 256;
  __shared__ u32x4 sk[2][KT * TL::CPR], sv[2][KT * TL::CPR];
  __shared__ int spos[2][KT];
  __shared__ uint16_t list[kScan];
  __shared__ uint32_t slim[2][4];
  __shared__ int scount[2][4];
  __shared__ int schanged;  // some staged value is not finite
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  // Workgroups are dealt to the 8 XCDs in turn; each XCD takes a contiguous range of
  // (request and group, part, row tile), so that its L2 holds few groups' keys at once.
  const int n_wg = gridDim.x, lin = blockIdx.x;
  const int xq = n_wg / 8, xr = n_wg % 8, xcd = lin % 8;
  const int wid = (xcd < xr ? xcd * (xq + 1) : xr * (xq + 1) + (xcd - xr) * xq) + lin / 8;
  const int rt = wid % pl.row_tiles, rest = wid / pl.row_tiles;
  const int split = rest % pl.splits, bg = rest / pl.splits, b = bg / c.G, g = bg - b * c.G;
  const int64_t R = (int64_t)a.n * a.rep;
  const int64_t row = (int64_t)rt * 128 + wave * 32 + lr;
  const Row w = row_of(a, b, g, row, R);
  const uint32_t lim_max = lanes_max(w.lim), lim_min = lanes_min(w.lim ? w.lim : ~0u);
  if (tid == 0) schanged = 0;
  if (lane == 0) {
    slim[0][wave] = lim_max;
    slim[1][wave] = lim_min;
  }
  const float cs = a.scale * kLog2e;
  typename Op<T>::V qf[D / 16];
  {
    const T* q = q_of<T>(a, b, w);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
#pragma unroll
      for (int e = 0; e < 8; ++e) qf[ks][e] = (T)0.f;
      if (row < R) qf[ks] = *reinterpret_cast<const typename Op<T>::V*>(q + 16 * ks + 8 * lh);
    }
  }
  const T* kbase = (const T*)c.k + b * c.ks[0] + g * c.ks[1];
  const T* vbase = (const T*)c.v + b * c.vs[0] + g * c.vs[1];
  const int* ps = c.pos + (int64_t)bg * c.C;
  __syncthreads();
  const uint32_t wg_lim = max(max(slim[0][0], slim[0][1]), max(slim[0][2], slim[0][3]));
  const uint32_t wg_min = min(wg_lim, min(min(slim[1][0], slim[1][1]), min(slim[1][2], slim[1][3])));

  // Blocks of kBlock slots are dealt to the parts in turn (used slots lie in front in a
  // cache that has room). Place l of a scan is slot c0 + l + (l / kBlock) skip.
  const int skip = kBlock * (pl.splits - 1), span = pl.scan * pl.splits;
  auto from_c0 = [&](uint32_t l) { return __umul24(l / kBlock, (uint32_t)skip) + l; };
  const uint32_t kstep = (uint32_t)c.ks[2] * sizeof(T), vstep = (uint32_t)c.vs[2] * sizeof(T);  // below 2^24
  const uint32_t lds_k = lds_address(&sk[0][0]), lds_v = lds_address(&sv[0][0]);
  auto pos_of = [&](int s) { return *(const int*)((const char*)ps + 4u * (uint32_t)s); };
  int pr = -1;
  int c0 = 0, m = 0, seen = 0;  // the scanned range's first slot, its list's length, those that all rows see
  __amdgpu_buffer_rsrc_t rk, rv;
  // Tile t goes to LDS by DMA, 16 bytes a lane in lane order, so the lane picks the chunk
  // that belongs where it writes (both permutations are their own inverses).
  auto load = [&](int t, int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int idx = j * 256 + tid, r = idx / TL::CPR, e = t * KT + r;
      const uint32_t s = from_c0(list[min(e, m - 1)]);
      const uint32_t ok = __umul24(s, kstep) + 16 * (TL::k(r, idx % TL::CPR) - r * TL::CPR);
      const uint32_t ov = __umul24(s, vstep) + 16 * (TL::v(r, idx % TL::CPR) - r * TL::CPR);
      const uint32_t at = 16u * (uint32_t)(buf * KT * TL::CPR + j * 256 + wave * 64);
      // M0 is reserved by the compiler, but nothing else in this kernel reads it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
      asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :
                   : "s"(lds_k + at), "v"(ok), "s"(rk)
                   : "m0");
      asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                   :
                   : "s"(lds_v + at), "v"(ov), "s"(rv)
                   : "m0");
#pragma clang diagnostic pop
    }
    if ((t + 1) * KT > seen && tid < KT) {
      const int e = t * KT + tid;
      pr = e < m ? pos_of(c0 + (int)from_c0(list[e])) : -1;
    }
  };
  // the DMA of tile t is complete and its readers may begin, those of the one before are done
  auto arrive = [&](int t, int buf, bool scrub) __attribute__((always_inline)) {
    if ((t + 1) * KT > seen && tid < KT) spos[buf][tid] = pr;
    __builtin_amdgcn_s_waitcnt(0);
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (scrub) {
#pragma unroll 1
      for (int idx = tid; idx < KT * TL::CPR; idx += 256) {
        const u32x4 x = sv[buf][idx], f = finite_part<T>(x);
        if (f.x != x.x || f.y != x.y || f.z != x.z || f.w != x.w) schanged = 1;
        sv[buf][idx] = f;
      }
      __syncthreads();
    }
  };

  Softmax<T, D, false> sx;
  // Moves what has been added up to the row's total in the workspace, scaled to the shift that
  // has been reached since, or (last) takes that total in. Both lanes of a row keep its shift and sum.
  bool folded = false;
  auto fold = [&](bool last) __attribute__((always_inline)) {
    const float L = other_half_sum(sx.l);
    if (row < R) {
      const int64_t at = ((int64_t)bg * pl.splits + split) * R + row;
      float* ml = (float*)a.ws + pl.part_ml + at * 2;
      float* o = (float*)a.ws + pl.part_o + at * D + 4 * lh;
      const float f = folded && ml[0] != -INFINITY ? __builtin_amdgcn_exp2f(ml[0] - sx.m) : 0.f;
      const float l = folded ? ml[1] * f : 0.f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
          float4* t = reinterpret_cast<float4*>(o + 32 * d + 2 * r);
          const float4 x = folded ? *t : make_float4(0.f, 0.f, 0.f, 0.f);
          const float y[4] = {fmaf(x.x, f, sx.acc[d][r]), fmaf(x.y, f, sx.acc[d][r + 1]),
                              fmaf(x.z, f, sx.acc[d][r + 2]), fmaf(x.w, f, sx.acc[d][r + 3])};
          if (!last) *t = make_float4(y[0], y[1], y[2], y[3]);
#pragma unroll
          for (int e = 0; e < 4; ++e) sx.acc[d][r + e] = last ? y[e] : 0.f;
        }
      if (!last) {
        ml[0] = sx.m;
        ml[1] = L + l;
        sx.l = 0.f;
      } else if (lh == 0) {
        sx.l += l;
      }
    }
    folded = true;
  };
  for (int scrub = 0;; scrub = 1) {
    sx.reset();
    folded = false;
    int since = 0;  // ranges
    for (c0 = split * kBlock; c0 < c.C; c0 += span) {
      const int c1 = min(c.C, c0 + span);
      auto scanned = [&](int x) {
        const int l = wave * (kScan / 4) + x * 64 + lane, s = c0 + (int)from_c0((uint32_t)l);
        return (uint32_t)(l < pl.scan && s < c1 ? pos_of(s) : -1);
      };
      int n0 = 0, n1 = 0;
#pragma unroll 8
      for (int x = 0; x < kScan / 256; ++x) {
        const uint32_t p = scanned(x);
        n0 += (int)__popcll(__ballot(p < wg_min));
        n1 += (int)__popcll(__ballot(p - wg_min < wg_lim - wg_min));
      }
      __syncthreads();  // the last range's readers are done
      if (lane == 0) {
        scount[0][wave] = n0;
        scount[1][wave] = n1;
      }
      __syncthreads();
      seen = scount[0][0] + scount[0][1] + scount[0][2] + scount[0][3];
      m = seen + scount[1][0] + scount[1][1] + scount[1][2] + scount[1][3];
      if (m == 0) continue;
      if (pl.fold != 0 && since == pl.fold) {
        fold(false);
        since = 0;
      }
      ++since;
      int at0 = 0, at1 = seen;
      for (int x = 0; x < wave; ++x) {
        at0 += scount[0][x];
        at1 += scount[1][x];
      }
      const uint64_t below = (1ull << lane) - 1;
#pragma unroll 8
      for (int x = 0; x < kScan / 256; ++x) {
        const uint32_t p = scanned(x);
        const bool k0 = p < wg_min, k1 = p - wg_min < wg_lim - wg_min;
        const uint64_t b0 = __ballot(k0), b1 = __ballot(k1);
        const uint16_t s = (uint16_t)(wave * (kScan / 4) + x * 64 + lane);
        if (k0) list[at0 + (int)__popcll(b0 & below)] = s;
        if (k1) list[at1 + (int)__popcll(b1 & below)] = s;
        at0 += (int)__popcll(b0);
        at1 += (int)__popcll(b1);
      }
      __syncthreads();
      seen = __builtin_amdgcn_readfirstlane(seen);
      m = __builtin_amdgcn_readfirstlane(m);
      rk = buffer_of(kbase + (int64_t)c0 * c.ks[2], (uint32_t)(c1 - c0 - 1) * kstep + D * (uint32_t)sizeof(T));
      rv = buffer_of(vbase + (int64_t)c0 * c.vs[2], (uint32_t)(c1 - c0 - 1) * vstep + D * (uint32_t)sizeof(T));
      const int tiles = (m + KT - 1) / KT;
      load(0, 0);
      arrive(0, 0, scrub);
      for (int t = 0; t < tiles; ++t) {
        const int cur = t & 1;
        if (t + 1 < tiles) load(t + 1, cur ^ 1);
        bool any = lim_max != 0, all = true;
        if ((t + 1) * KT > seen) {
          const int q = spos[cur][lane % KT];
          any = __ballot((uint32_t)q < lim_max) != 0;
          all = __ballot((uint32_t)q < lim_min) == ~0ull;
        }
        if (any) {
          f32x16 s[KB];
          // (a wave at its MFMAs issues them ahead of the other waves on the SIMD, whose
          // exponentials fill in between: 10% at 64 dims, 1% at 128)
          __builtin_amdgcn_s_setprio(3);
          typename Op<T>::V kf[D / 16][KB];
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) kf[ks][kb] = TL::k_frag(sk[cur], 32 * kb + key_of_row(lr), ks, lh);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) s[kb] = Op<T>::mma(kf[ks][kb], qf[ks], ks ? s[kb] : kZero);
          __builtin_amdgcn_s_setprio(0);
          if (!all) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if ((uint32_t)spos[cur][32 * kb + 16 * (r >> 3) + 8 * lh + (r & 7)] >= w.lim) s[kb][r] = -INFINITY;
          }
          sx.template add<KB>(s, cs, scrub ? Op<T>::kDown : 0.f, sv[cur], 0, lane);
        }
        if (t + 1 < tiles) arrive(t + 1, cur ^ 1, scrub);
      }
    }
    __syncthreads();
    if (folded) fold(true);
    if (scrub) {
      sx.m += Op<T>::kDown;
      if (schanged)
        for (int s = split * kBlock; s < c.C; s += kBlock * pl.splits)
          sx.add_unbounded(vbase, c.vs[2], ps, s, min(s + kBlock, c.C), w.lim, lane);
      break;
    }
    if (!__syncthreads_or(w.lim != 0 && !sx.finite())) break;
  }

  if (w.lim == 0) {  // padding: what tiles without a mask gave it does not count
    sx.m = -INFINITY;
    sx.l = 0.f;
  }
  const float L = other_half_sum(sx.l);
  sx.close(L);
  // (the row's place is worked out again, from a lane the compiler takes for another:
  // kept through the loop it would cost registers that 128 dims do not have)
  int lane_ = lane;
  asm volatile("" : "+v"(lane_));
  const int64_t row_ = (int64_t)rt * 128 + wave * 32 + (lane_ & 31);
  const int lh_ = lane_ >> 5;
  if (row_ >= R) return;
  const Row w_ = row_of(a, b, g, row_, R);
  const bool none = sx.m == -INFINITY;
  const float l2 = none ? -INFINITY : sx.m - Op<T>::kShift + __builtin_amdgcn_logf(L);
  if (pl.splits > 1) {
    const int64_t pr_ = ((int64_t)bg * pl.splits + split) * R + row_;
    float* ml = (float*)a.ws + pl.part_ml + pr_ * 2;
    if (lh_ == 0) {
      ml[0] = sx.m;
      ml[1] = L;
    }
    const float inv = none ? 0.f : 1.f / L;
    float* o = (float*)a.ws + pl.part_o + pr_ * D;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        store4(o + 32 * d + 2 * r + 4 * lh_, on_shift(sx.acc[d][r], inv), on_shift(sx.acc[d][r + 1], inv),
               on_shift(sx.acc[d][r + 2], inv), on_shift(sx.acc[d][r + 3], inv));
    return;
  }
  if (lh_ == 0) {
    if (a.weight_out) ((float*)a.ws)[pl.lse2 + (int64_t)bg * R + row_] = l2;
    if (a.lse) a.lse[((int64_t)b * c.G * a.rep + w_.head) * a.n + w_.i] = none ? -INFINITY : l2 * kLn2;
  }
  const float inv = none ? 0.f : 1.f / L;
  T* o = out_of<T>(a, b, w_);
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : sx.acc[d][r + e] * inv;
      store4(o + 32 * d + 2 * r + 4 * lh_, x[0], x[1], x[2], x[3]);
    }
}

// What is left when the parts are done: workgroups below row_blocks join the parts of
// rows (D / 4 threads each), the others add up what rows gave 256 NS slots each,
// from the scores that attend_keys_kernel kept (4 bytes a row and slot, beside 4 D of a
// 16-bit key and value). Each of those works out its rows' log-sums from the parts by
// itself, 16 threads a row (64 for 256 parts: a call of 4 rows 19.7 us against 20.4, of 28 rows
// 35.5 against 29.7). Parts are read side by side throughout: a chain of dependent
// loads per part cost 0.7 us each.
// Four slots a thread once that still leaves two workgroups a CU (2^19 slots in all; a whole call
// of one token, 8 x 8 groups of 2048 slots 14.9 us with one and 15.8 with four, of 8192 34.8 and 33.4).
constexpr int kFinishRows = 64;
template <typename T, int D, int NS>
__global__ __launch_bounds__(256) void finish_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl,
                                                     int row_blocks, int slot_blocks) {
  __shared__ float s_l2[kFinishRows];
  __shared__ uint32_t s_lim[kFinishRows];
  const float* ws = (const float*)a.ws;
  const int R = a.n * a.rep;
  const int S = pl.splits;
  const int tid = threadIdx.x;
  // shift and sum of row r of (b, g) over the parts, by W neighbouring threads (j: this one's place)
  auto total = [&](int64_t bg, int r, int j, auto width, float& M, float& L) {
    constexpr int W = decltype(width)::value;
    const float2* ml = reinterpret_cast<const float2*>(ws + pl.part_ml) + bg * S * R + r;
    M = -INFINITY;
    L = 0.f;
    for (int s = j; s < S; s += 4 * W) {
      float2 x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = ml[(int64_t)min(s + e * W, S - 1) * R];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (s + e * W >= S) break;
        const float m = fmaxf(M, x[e].x);
        if (m != -INFINITY) L = L * __builtin_amdgcn_exp2f(M - m) + x[e].y * __builtin_amdgcn_exp2f(x[e].x - m);
        M = m;
      }
    }
#pragma unroll
    for (int o = 1; o < W; o <<= 1) {
      const float M2 = __shfl_xor(M, o), L2 = __shfl_xor(L, o), m = fmaxf(M, M2);
      if (m != -INFINITY) {
        // (the lower lane's share first, so that all of them round alike)
        const float x = L * __builtin_amdgcn_exp2f(M - m), y = L2 * __builtin_amdgcn_exp2f(M2 - m);
        L = j & o ? y + x : x + y;
      }
      M = m;
    }
  };
  if ((int)blockIdx.x < row_blocks) {
    // (many parts are shared by pl.join groups of a row's threads, which meet in LDS)
    constexpr int TPR = D / 4, RPB = 256 / TPR;
    __shared__ float4 s_o[256];
    const int64_t rows = (int64_t)c.B * c.G * R;
    const int group = tid / TPR % pl.join;
    const int64_t row_ = (int64_t)blockIdx.x * (RPB / pl.join) + tid / TPR / pl.join, row = min(row_, rows - 1);
    const int j = tid % TPR, d = 4 * j;
    const int64_t bg = row / R;
    const int r = (int)(row - bg * R);
    const int b = (int)(bg / c.G), g = (int)(bg - (int64_t)b * c.G);
    float M, L;
    total(bg, r, j, std::integral_constant<int, TPR>{}, M, L);
    const float inv = M == -INFINITY ? 0.f : 1.f / L;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const float* po = ws + pl.part_o + (bg * S * R + r) * D + d;
    const float2* ml = reinterpret_cast<const float2*>(ws + pl.part_ml) + bg * S * R + r;
    for (int s0 = group; s0 < S; s0 += 4 * pl.join) {
      float2 x[4];
      float4 p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int64_t s = min(s0 + e * pl.join, S - 1);
        x[e] = ml[s * R];
        p[e] = *reinterpret_cast<const float4*>(po + s * R * D);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float f = s0 + e * pl.join >= S || x[e].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(x[e].x - M) * x[e].y * inv;
        if (f != 0.f) {
          o.x = fmaf(f, p[e].x, o.x);
          o.y = fmaf(f, p[e].y, o.y);
          o.z = fmaf(f, p[e].z, o.z);
          o.w = fmaf(f, p[e].w, o.w);
        } else {
          o.x += on_shift(p[e].x, 0.f);
          o.y += on_shift(p[e].y, 0.f);
          o.z += on_shift(p[e].z, 0.f);
          o.w += on_shift(p[e].w, 0.f);
        }
      }
    }
    if (pl.join > 1) {
      s_o[tid] = o;
      __syncthreads();
      if (group == 0)
        for (int y = 1; y < pl.join; ++y) {
          const float4 p = s_o[tid + y * TPR];
          o = make_float4(o.x + p.x, o.y + p.y, o.z + p.z, o.w + p.w);
        }
    }
    if (row_ >= rows || group != 0) return;
    const Row w = row_of(a, b, g, r, R);
    if (M == -INFINITY) o = make_float4(0.f, 0.f, 0.f, 0.f);
    store4(out_of<T>(a, b, w) + d, o.x, o.y, o.z, o.w);
    if (j == 0) {
      const float l2 = M == -INFINITY ? -INFINITY : M - Op<T>::kShift + __builtin_amdgcn_logf(L);
      if (a.weight_out && !pl.by_keys) ((float*)a.ws)[pl.lse2 + row] = l2;
      if (a.lse) a.lse[((int64_t)b * c.G * a.rep + w.head) * a.n + w.i] = M == -INFINITY ? -INFINITY : l2 * kLn2;
    }
    return;
  }
  const int y = blockIdx.x - row_blocks;
  const int64_t bg = y / slot_blocks;
  const int b = (int)(bg / c.G), g = (int)(bg - (int64_t)b * c.G);
  const int s0 = (y % slot_blocks) * 256 * NS + tid;
  const int tiles = (c.C + 31) / 32;
  uint32_t p[NS];
  float sum[NS];
#pragma unroll
  for (int x = 0; x < NS; ++x) {
    p[x] = s0 + 256 * x < c.C ? (uint32_t)c.pos[bg * c.C + s0 + 256 * x] : ~0u;
    sum[x] = 0.f;
  }
  const float cs = a.scale * kLog2e;
  for (int r0 = 0; r0 < R; r0 += kFinishRows) {
    const int m = min(kFinishRows, R - r0);
    __syncthreads();
    constexpr int W = 16, RG = 256 / W;
    for (int q = tid / W; q < (m + RG - 1) / RG * RG; q += RG) {
      float M, L;
      total(bg, r0 + min(q, m - 1), tid % W, std::integral_constant<int, W>{}, M, L);
      if (tid % W == 0 && q < m) {
        s_l2[q] = M - Op<T>::kShift + __builtin_amdgcn_logf(L);
        s_lim[q] = M == -INFINITY ? 0u : row_of(a, b, g, r0 + q, R).lim;
      }
    }
    __syncthreads();
    const float* sc[NS];
#pragma unroll
    for (int x = 0; x < NS; ++x) {
      const int s = min(s0 + 256 * x, c.C - 1);
      sc[x] = ws + pl.scores + ((bg * tiles + s / 32) * R + r0) * 32 + s % 32;
    }
    for (int r = 0; r < m; r += 4) {
      float v[NS][4];  // (of tiles that no row sees, whatever the workspace held: not used)
#pragma unroll
      for (int x = 0; x < NS; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) v[x][e] = sc[x][min(r + e, m - 1) * 32];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t lim = r + e < m ? s_lim[min(r + e, m - 1)] : 0u;
        const float l2 = s_l2[min(r + e, m - 1)];
#pragma unroll
        for (int x = 0; x < NS; ++x)
          if (p[x] < lim) sum[x] += __builtin_amdgcn_exp2f(fmaf(v[x][e], cs, -l2));
      }
    }
  }
#pragma unroll
  for (int x = 0; x < NS; ++x)
    if (s0 + 256 * x < c.C) {
      const int64_t at = bg * c.C + s0 + 256 * x;
      a.weight_out[at] = p[x] >= 0x80000000u ? 0.f : fmaf(a.decay, c.weight[at], sum[x]);
    }
}

// The weights of a chunk of tokens: p = exp2(score - lse) needs the rows' log-sums, so
// the scores are computed again, with the keys held and the rows streaming past: a wave
// keeps the fragments of KB blocks of 32 keys in registers and the four waves share tiles of 64 rows
// through LDS. Half the matrix work of the attention, and its exponentials. A
// workgroup's slots are taken in the order seen by every row, by some rows, empty, so
// that a mask costs the waves with the call's own tokens alone. Where whole workgroups would
// leave CUs idle, RW = 2 waves share their keys and take every other 32 rows (61 tokens x 4
// heads, 6 groups, 1531 slots, fp32: 15 us against 19.5). The long chunk above: 678 to
// 717 us, 709 to 670 TFLOP/s; the frame 53 us.
template <typename T, int D, int RW>
__global__ __launch_bounds__(256, D == 128 || RW == 2 ? 2 : 3) void weights_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl) {
  using TL = Tile<T, D>;
  constexpr int KB = sizeof(T) == 2 ? 2 : 1;  // 32-key blocks of a wave
  constexpr int KW = 128 * KB / RW;           // slots of a workgroup
  constexpr int RT = 64;                      // rows of a tile
  constexpr int NV = RT * TL::CPR / 256;
  __shared__ u32x4 sq[2][RT * TL::CPR];
  __shared__ float sl2[2][RT];
  __shared__ uint32_t slim[2][RT];
  __shared__ int lslot[KW];       // the workgroup's slots in that order
  __shared__ uint32_t lpos[KW];   // and their positions (empty: from 2^31 on)
  __shared__ uint32_t smin;
  __shared__ int scount[3][4];
  __shared__ float spart[4 / RW][KB][16][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int kwave = wave / RW, rwave = wave % RW;
  const int slot_blocks = (c.C + KW - 1) / KW;
  const int kbk = blockIdx.x % slot_blocks, part = blockIdx.x / slot_blocks;
  const int bg = blockIdx.y, b = bg / c.G, g = bg - b * c.G;
  const int64_t R = (int64_t)a.n * a.rep;
  const T* kbase = (const T*)c.k + b * c.ks[0] + g * c.ks[1];
  const T* qbase = (const T*)a.q + b * a.qs[0] + g * a.rep * a.qs[2];
  const float* l2 = (const float*)a.ws + pl.lse2 + (int64_t)bg * R;
  const float cs = a.scale * kLog2e;
  const int64_t row_tiles = (R + RT - 1) / RT, per = (row_tiles + pl.weight_parts - 1) / pl.weight_parts;
  const int64_t t0 = part * per, t1 = min(row_tiles, t0 + per);

  // the first position that some row of this part does not see
  if (tid == 0) smin = ~0u;
  __syncthreads();
  if (t0 < t1) {
    uint32_t lim = ~0u;
    const int i1 = token_of(a, (int)min(R, t1 * RT) - 1);
    for (int i = token_of(a, (int)(t0 * RT)) + tid; i <= i1; i += 256) {
      const uint32_t l = row_of(a, b, g, (int64_t)i * a.rep, R).lim;
      lim = l ? min(lim, l) : lim;
    }
    lim = lanes_min(lim);
    if (lane == 0) atomicMin(&smin, lim);
  }
  __syncthreads();
  {
    const int s = kbk * KW + tid;
    const uint32_t p = tid < KW && s < c.C ? (uint32_t)c.pos[(int64_t)bg * c.C + s] : ~0u;
    const int cls = p < smin ? 0 : p < 0x80000000u ? 1 : 2;
    uint64_t m[3];
#pragma unroll
    for (int x = 0; x < 3; ++x) {
      m[x] = __ballot(cls == x);
      if (lane == 0) scount[x][wave] = (int)__popcll(m[x]);
    }
    __syncthreads();
    int at = (int)__popcll(m[cls] & ((1ull << lane) - 1));
    for (int x = 0; x <= cls; ++x)
      for (int w = 0; w < (x < cls ? 4 : wave); ++w) at += scount[x][w];
    if (at < KW) {  // (threads beyond the slots come last)
      lslot[at] = min(s, c.C - 1);
      lpos[at] = p;
    }
    int used = 0;
    for (int x = 0; x < 2; ++x)
      for (int w = 0; w < 4; ++w) used += scount[x][w];
    if (used == 0) {  // (the whole workgroup)
      if (tid < KW && s < c.C) {
        if (pl.weight_parts > 1)
          ((float*)a.ws)[pl.weights + ((int64_t)bg * pl.weight_parts + part) * c.C + s] = 0.f;
        else a.weight_out[(int64_t)bg * c.C + s] = 0.f;
      }
      return;
    }
  }
  __syncthreads();

  typename Op<T>::V kf[KB][D / 16];
  uint32_t p_max = 0, p_min = ~0u;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const int at = (kwave * KB + kb) * 32 + lr;
    const uint32_t p = lpos[at];
    p_max = p < 0x80000000u ? max(p_max, p) : p_max;  // (what empty slots add up is not stored)
    p_min = min(p_min, p);
    const T* k = kbase + (int64_t)lslot[at] * c.ks[2];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kf[kb][ks] = *reinterpret_cast<const typename Op<T>::V*>(k + 16 * ks + 8 * lh);
  }
  p_max = lanes_max(p_max);
  p_min = lanes_min(p_min);

  u32x4 qr[NV];
  float l2r = 0.f;
  uint32_t limr = 0;
  // Where this thread's chunks of the next tile lie: head and address of each, carried on by
  // RT rows a tile (4096 tokens x 4 heads, 8 groups, 16384 slots, 128 dims: 686 us; with
  // the products of rows and strides in every tile 726).
  const int d_tok = token_of(a, RT), d_head = RT - d_tok * a.rep;
  const int64_t step = d_tok * a.qs[1] + d_head * a.qs[2], wrap = a.qs[1] - a.rep * a.qs[2];
  int head[NV];
  const T* qp[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int idx = j * 256 + tid, r = (int)t0 * RT + idx / TL::CPR, i = token_of(a, r);
    head[j] = r - i * a.rep;
    qp[j] = qbase + i * a.qs[1] + head[j] * a.qs[2] + idx % TL::CPR * TL::EPC;
  }
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    if ((t + 1) * RT <= R) {
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        qr[j] = *reinterpret_cast<const u32x4*>(qp[j]);
        head[j] += d_head;
        const bool c = head[j] >= a.rep;
        head[j] -= c ? a.rep : 0;
        qp[j] += step + (c ? wrap : 0);
      }
    } else {  // the last tile repeats the last row
#pragma unroll
      for (int j = 0; j < NV; ++j) {
        const int idx = j * 256 + tid, ch = idx % TL::CPR;
        const int r = min((int)t * RT + idx / TL::CPR, (int)R - 1), i = token_of(a, r);
        qr[j] = *reinterpret_cast<const u32x4*>(qbase + i * a.qs[1] + (r - i * a.rep) * a.qs[2] + ch * TL::EPC);
      }
    }
    if (tid < RT) {
      const int64_t r = t * RT + tid;
      l2r = r < R ? l2[r] : 0.f;
      limr = r < R && l2r != -INFINITY ? row_of(a, b, g, r, R).lim : 0u;
    }
  };
  auto stage = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int idx = j * 256 + tid;
      sq[buf][TL::k(idx / TL::CPR, idx % TL::CPR)] = qr[j];
    }
    if (tid < RT) {
      sl2[buf][tid] = l2r;
      slim[buf][tid] = limr;
    }
  };
  float sum[KB][16];
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[kb][r] = 0.f;
  if (t0 < t1) {
    load(t0);
    stage(0);
  }
  __syncthreads();
  for (int64_t t = t0; t < t1; ++t) {
    const int cur = (int)(t - t0) & 1;
    if (t + 1 < t1) load(t + 1);
#pragma unroll 1
    for (int rb = rwave; rb < RT / 32; rb += RW) {
      const uint32_t lim = slim[cur][32 * rb + lr];
      if (__ballot(lim > p_min) == 0) continue;
      const bool all = __ballot(lim > p_max) == ~0ull;
      const float nl = -sl2[cur][32 * rb + lr];
      f32x16 s[KB];
      // (all fragments are on their way before the first MFMA: left to itself the compiler
      // waits for each of them in turn)
      typename Op<T>::V q[D / 16];
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) q[ks] = TL::k_frag(sq[cur], 32 * rb + lr, ks, lh);
      if constexpr (sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) s[kb] = Op<T>::mma(kf[kb][ks], q[ks], ks ? s[kb] : kZero);
      if (all) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sum[kb][r] += __builtin_amdgcn_exp2f(fmaf(s[kb][r], cs, nl));
      } else {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const uint32_t p = lpos[(kwave * KB + kb) * 32 + 8 * (r >> 2) + 4 * lh + (r & 3)];
            const float x = __builtin_amdgcn_exp2f(fmaf(s[kb][r], cs, nl));
            sum[kb][r] += p < lim ? x : 0.f;
          }
      }
    }
    if (t + 1 < t1) stage(cur ^ 1);
    __syncthreads();
  }
  // over the 32 rows of a half, then over the waves that shared the rows
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[kb][r] = half_sum(sum[kb][r]);
  if constexpr (RW > 1) {
    if (rwave == 1 && lr == 31)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) spart[kwave][kb][r][lh] = sum[kb][r];
    __syncthreads();
    if (rwave == 1) return;
  }
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = RW > 1 ? sum[kb][r] + spart[kwave][kb][r][lh] : sum[kb][r];
      const int at = (kwave * KB + kb) * 32 + 8 * (r >> 2) + 4 * lh + (r & 3);
      // (the list's end repeats no slot: a last, short block leaves its surplus out)
      if (lr == 31 && at < min(KW, c.C - kbk * KW)) {
        const int64_t s = lslot[at], slot = (int64_t)bg * c.C + s;
        if (pl.weight_parts > 1) ((float*)a.ws)[pl.weights + ((int64_t)bg * pl.weight_parts + part) * c.C + s] = x;
        else a.weight_out[slot] = lpos[at] >= 0x80000000u ? 0.f : fmaf(a.decay, c.weight[slot], x);
      }
    }
}

__global__ __launch_bounds__(256) void weights_join_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl) {
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (int64_t)c.B * c.G * c.C) return;
  const int64_t bg = at / c.C;
  const float* w = (const float*)a.ws + pl.weights + bg * pl.weight_parts * c.C + (at - bg * c.C);
  float x = 0.f;
  for (int i = 0; i < pl.weight_parts; ++i) x += w[(int64_t)i * c.C];
  a.weight_out[at] = c.pos[at] < 0 ? 0.f : fmaf(a.decay, c.weight[at], x);
}

template <typename T, int D>
hipError_t attend_launch(const TokenCacheArgs& c, TokenAttend a, const TokenAttendPlan& pl, hipStream_t s) {
  a.rep_inv = (uint32_t)((((uint64_t)1 << 32) + a.rep - 1) / a.rep);
  const int64_t R = (int64_t)a.n * a.rep;
  const int BG = c.B * c.G;
  if (a.n == 0) {  // no rows: the weights only fade
    if (a.weight_out) {  // (a plan of no parts)
      TokenAttendPlan none;
      none.weight_parts = 0;
      hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)(((int64_t)BG * c.C + 255) / 256)), dim3(256), 0, s, c, a,
                         none);
    }
    return hipGetLastError();
  }
  const int rows_each = 256 / (D / 4) / pl.join;
  const int64_t row_blocks = ((int64_t)BG * R + rows_each - 1) / rows_each;
  const bool wide = (int64_t)BG * c.C >= 1 << 19;
  const int slot_blocks = (c.C + (wide ? 1023 : 255)) / (wide ? 1024 : 256);
  auto finish = [&](bool slots) {
    const dim3 grid((unsigned)(row_blocks + (slots ? (int64_t)BG * slot_blocks : 0)));
    if (wide) hipLaunchKernelGGL((finish_kernel<T, D, 4>), grid, dim3(256), 0, s, c, a, pl, (int)row_blocks, slot_blocks);
    else hipLaunchKernelGGL((finish_kernel<T, D, 1>), grid, dim3(256), 0, s, c, a, pl, (int)row_blocks, slot_blocks);
  };
  if (pl.by_keys) {
    hipLaunchKernelGGL((attend_keys_kernel<T, D>), dim3(pl.splits, pl.row_tiles, BG), dim3(256), 0, s, c, a, pl);
    if (pl.splits > 1 || a.weight_out) finish(a.weight_out != nullptr);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((attend_rows_kernel<T, D>), dim3((unsigned)(pl.row_tiles * pl.splits * BG)), dim3(256), 0, s, c, a,
                     pl);
  if (pl.splits > 1) finish(false);
  if (a.weight_out) {
    const int kw = (sizeof(T) == 2 ? 256 : 128) / pl.row_waves;
    const dim3 grid((unsigned)((c.C + kw - 1) / kw * pl.weight_parts), (unsigned)BG);
    if (pl.row_waves == 2) hipLaunchKernelGGL((weights_kernel<T, D, 2>), grid, dim3(256), 0, s, c, a, pl);
    else hipLaunchKernelGGL((weights_kernel<T, D, 1>), grid, dim3(256), 0, s, c, a, pl);
    if (pl.weight_parts > 1)
      hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)(((int64_t)BG * c.C + 255) / 256)), dim3(256), 0, s, c, a,
                         pl);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t attend_dim(const TokenCacheArgs& c, const TokenAttend& a, const TokenAttendPlan& pl, hipStream_t s) {
  if (c.D == 32) return attend_launch<T, 32>(c, a, pl, s);
  if (c.D == 64) return attend_launch<T, 64>(c, a, pl, s);
  return attend_launch<T, 128>(c, a, pl, s);
}

}  // namespace

TokenAttendPlan token_attend_plan(const TokenCacheArgs& c, int n, int rep, int kind, bool weights) {
  TokenAttendPlan p;
  const int64_t R = (int64_t)n * rep, BG = (int64_t)c.B * c.G;
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  auto clamp = [](int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; };
  // (8 groups, 32768 slots, 128 dims, bf16, with weights: 64 rows 60 us by keys against 73,
  // 96 rows 105 against 81; 3 groups, 4680 slots, 64 dims, fp32: 26 against 36, 32 against 39)
  p.by_keys = R <= 64;
  p.row_tiles = (int)up(R, p.by_keys ? 32 : 128);
  const int64_t wgs = BG * p.row_tiles;
  // workgroups that the chip holds at once, by the kernels' registers (LDS allows as many):
  // attend_keys_kernel, and weights_kernel for one and two waves that share keys. (One token, 8
  // groups x 4 heads, 65536 slots, 64 dims, fp32: 67 us by the two a CU that fit, 84 by three. Of
  // 32 dims four fit, but three are as fast or faster: 131072 slots, bf16, 37 us against 38.)
  const int fp32 = kind == 2;
  const int64_t held = 256 * (c.D == 128 ? 2 - fp32 : c.D == 64 ? 3 - fp32 : 3);
  const int64_t held_w1 = 256 * (c.D == 128 ? 2 : 3 + (fp32 && c.D == 32));
  const int64_t held_w2 = 256 * (fp32 ? (c.D == 128 ? 2 : c.D == 64 ? 3 : 4) : c.D == 32 ? 3 : 2);
  if (p.by_keys) {
    // whole rounds of what is held, of parts that are long beside what a part costs by
    // itself (about 96 slots' time) but leave two tiles of 32 slots a wave
    int64_t best = INT64_MAX;
    const int64_t least = up(c.C, kPartSlots), most = std::max(clamp(up(c.C, 256), 1, 256), least);
    for (int64_t round = 1; round <= 8; ++round) {
      const int64_t s = clamp(held * round / wgs, least, most);
      const int64_t cost = up(wgs * s, held) * (up(c.C, s) + 96);
      if (cost < best) {
        best = cost;
        p.splits = (int)s;
      }
    }
  } else {
    // byte offsets of a scan's slots from its first fit 32 bits
    const int64_t step = (kind == 2 ? 4 : 2) * (c.ks[2] > c.vs[2] ? c.ks[2] : c.vs[2]);
    const int64_t blocks = ((int64_t)1 << 32) / ((c.C > 1 && step > 0 ? step : 1) * kBlock);  // >= 4
    // Parts by a model of what was measured, in us: a tile of 64 slots takes a workgroup
    // alone on its CU t, L of them on one CU 0.65 L t, a workgroup's ends six tiles' time, and
    // joining parts a launch and its traffic. (1560 tokens x 8 heads, 3 groups, 4680 slots, 64
    // dims: one part 118 us, two 87 + 9, three 88 + 12. 61 tokens x 4, 6 groups, 1531 slots,
    // fp32: two parts 64 us, eleven 21.) More parts only where they gain 5%.
    const double t = kind == 2 ? 0.065 * c.D : c.D == 128 ? 1.75 : c.D == 64 ? 1.2 : 0.9;
    double best = 0.0;
    const int64_t most = clamp(c.C / kBlock, 1, blocks < 64 ? blocks : 64);
    for (const int64_t parts : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64}) {
      const int64_t s = parts < most ? parts : most;
      const double load = 0.65 * (double)up(wgs * s, 256);
      const double cost = ((double)c.C / (64.0 * s) + 6.0) * t * (load < 1.0 ? 1.0 : load) +
                          (s > 1 ? 4.0 + (double)(s * BG * R * c.D) * 8.0 / 5e6 : 0.0);
      if (s == 1 || cost < 0.95 * best) {
        best = cost;
        p.splits = (int)s;
      }
    }
    p.scan = (int)clamp(blocks / p.splits, 1, kScan / kBlock) * kBlock;
    const int64_t fold = kind == 2 ? kFoldSlots<float> : kFoldSlots<_Float16>;
    if (up(up(c.C, kBlock), p.splits) * kBlock > fold) p.fold = (int)std::max<int64_t>(1, fold / p.scan);
    const int64_t blk = up(c.C, kind == 2 ? 128 : 256), kw = blk * BG;
    p.weight_parts = (int)clamp(held_w1 / kw, 1, clamp(R / 256, 1, 64));
    // (kPartRows, within 2^23 workgroups)
    p.weight_parts = (int)std::max<int64_t>(p.weight_parts, clamp(up(R, kPartRows), 1, std::max<int64_t>(1, (1 << 23) / blk)));
    p.row_waves = p.weight_parts == 1 && kw * 2 <= held_w2 ? 2 : 1;
  }
  int64_t at = 0;
  auto take = [&](int64_t floats) {
    const int64_t o = at;
    at += up(floats, 64) * 64;
    return o;
  };
  // Groups of a row's threads in a workgroup of finish_kernel (4 rows, 64 dims: 64 parts by one
  // group 32 us in all, by four 16, by sixteen 12; 256 parts 100, 36 and 20).
  const int groups = 256 / (c.D / 4);
  p.join = p.splits >= 32 ? groups : p.splits >= 8 ? 4 : 1;
  if (p.splits > 1 || p.fold || (p.by_keys && weights)) {
    p.part_o = take(BG * p.splits * R * c.D);
    p.part_ml = take(BG * p.splits * R * 2);
  }
  if (weights && p.by_keys) p.scores = take(BG * R * up(c.C, 32) * 32);
  if (weights && !p.by_keys) {
    p.lse2 = take(BG * R);
    if (p.weight_parts > 1) p.weights = take(BG * p.weight_parts * c.C);
  }
  p.bytes = at * 4;
  return p;
}

hipError_t token_attend(const TokenCacheArgs& c, const TokenAttend& a, const TokenAttendPlan& pl, int kind,
                        hipStream_t s) {
  if (kind == 0) return attend_dim<_Float16>(c, a, pl, s);
  if (kind == 1) return attend_dim<__bf16>(c, a, pl, s);
  return attend_dim<float>(c, a, pl, s);
}

}  // namespace fd
