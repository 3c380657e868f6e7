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
// to. V of empty slots is zeroed as it is staged. V of slots hidden from some rows alone
// may hold infinities or NaN, which 0 x V would spread: rows that end up not finite are
// computed once more with such elements as zeros, and those of visible slots are then
// added (slow, and never taken by finite data).
#include "fd_token.h"

#include <type_traits>

namespace fd {
namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T> struct Op;
template <> struct Op<_Float16> {
  using V = f16x8;
  // Probabilities are kept below 2^15 and, with the running maximum at 2^6, above the
  // subnormal f16 values down to 2^-20 of it.
  static constexpr float kShift = 6.f;
  static __device__ __forceinline__ f32x16 mma(V a, V b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
};
template <> struct Op<__bf16> {
  using V = bf16x8;
  static constexpr float kShift = 0.f;
  static __device__ __forceinline__ f32x16 mma(V a, V b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
  }
};
template <> struct Op<float> {
  using V = f32x8;
  static constexpr float kShift = 0.f;
  static __device__ __forceinline__ f32x16 mma(V a, V b, f32x16 c) {
#pragma unroll
    for (int j = 0; j < 8; ++j) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], c, 0, 0, 0);
    return c;
  }
};

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

// The rows of a call: where a row's query lies, and the first position it does not see.
struct Row {
  int i, head;     // query token, head
  uint32_t lim;
};
__device__ __forceinline__ Row row_of(const TokenAttend& a, int b, int g, int64_t r, int64_t R) {
  Row w{0, g * a.rep, 0};
  if (r < R) {
    w.i = (int)(r / a.rep);
    w.head = g * a.rep + (int)(r - (int64_t)w.i * a.rep);
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
  // Scores of KB 32-key blocks (hidden ones -inf) and their values in LDS.
  template <int KB>
  __device__ __forceinline__ void add(f32x16 (&s)[KB], float c, const u32x4* vt, int row0, int lane) {
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
    const float sub = m == -INFINITY ? 0.f : O::kShift - m;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int st = 0; st < 2; ++st) {
        typename O::V ph, pl;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][8 * st + e], c, sub));
          l += p;
          // P enters the second MFMA in the cache's type. Where memory bounds the kernel
          // (EXACT) what that rounding loses goes in by a second MFMA; elsewhere its half
          // step per key, as large as the output's own rounding, is kept.
          ph[e] = (T)p;
          if constexpr (EXACT && sizeof(T) == 2) pl[e] = (T)(p - (float)ph[e]);
        }
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const typename O::V vf = Tile<T, D>::v_frag(vt, row0 + 32 * kb + 16 * st, d, lane);
          acc[d] = O::mma(vf, ph, acc[d]);
          if constexpr (EXACT && sizeof(T) == 2) acc[d] = O::mma(vf, pl, acc[d]);
        }
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
  // Adds the infinities and NaN of one slot's value.
  __device__ __forceinline__ void add_unbounded(const T* v, int lh) {
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float x = (float)v[32 * d + 8 * (r >> 2) + 4 * lh + (r & 3)];
        if (!isfinite(x)) acc[d][r] += x;
      }
  }
};

// Stores 4 consecutive dims.
template <typename T> __device__ __forceinline__ void store4(T* p, float a, float b, float c, float d) {
  struct alignas(4 * sizeof(T)) Q { T e[4]; };
  *reinterpret_cast<Q*>(p) = Q{(T)a, (T)b, (T)c, (T)d};
}

// (part_ml holds shift and sum of each part's rows, part_o their unnormalised output.)

// Few rows (serving): memory bounds it, so the keys are parted among as many waves as it
// takes. A wave walks 32-slot tiles of its workgroup's part on its own: it stages a
// tile's keys, then its values, through 32 rows of LDS that no other wave touches, so the
// loop has no barrier and a CU's waves drift apart. Both loads of a tile go out together;
// with 8 to 12 waves on a CU up to 128 KB are in flight. The four waves' results meet in
// LDS, the parts' in finish_kernel.
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D == 512 ? 1 : 2) void attend_keys_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl) {
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
  float* score = a.weight_out ? (float*)a.ws + pl.scores + ((int64_t)bg * R + row) * c.C : nullptr;

  const int tiles = (c.C + 31) / 32, per = (tiles + pl.splits - 1) / pl.splits;
  const int t0 = split * per + wave, t1 = min(tiles, (split + 1) * per);
  auto pos_at = [&](int t) {
    const int s = t * 32 + lr;
    return t < t1 && s < c.C ? ps[s] : -1;
  };
  u32x4* tile = buf[wave];
  Softmax<T, D, true> sx;
  for (int scrub = 0;; scrub = 1) {
    sx.reset();
    int p_next = pos_at(t0);
    for (int t = t0; t < t1; t += 4) {
      const int p = p_next;
      p_next = pos_at(t + 4);
      if ((uint32_t)__ballot((uint32_t)p < lim_max) == 0) continue;
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
      for (int r = 0; r < 16; ++r) s[0][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) s[0] = Op<T>::mma(TL::k_frag(tile, key_of_row(lr), ks, lh), qf[ks], s[0]);
      if (score && row < R) {
        const int s0 = t * 32 + 8 * lh;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int sl_ = s0 + 16 * (r >> 3) + (r & 7);
          if (sl_ < c.C) score[sl_] = s[0][r];
        }
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
        if (scrub) x = finite_part<T>(x);
        tile[TL::v(vrow, idx % TL::CPR)] = x;
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      sx.template add<1>(s, cs, tile, 0, lane);
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }
    if (scrub || __ballot(w.lim != 0 && !sx.finite()) == 0) {
      if (scrub)
        for (int t = t0; t < t1; t += 4)
          for (int x = t * 32; x < min(t * 32 + 32, c.C); ++x)
            if ((uint32_t)ps[x] < w.lim) sx.add_unbounded(vb + x * c.vs[2], lh);
      break;
    }
  }

  if (w.lim == 0) {  // padding: what tiles without a mask gave it does not count
    sx.m = -INFINITY;
    sx.l = 0.f;
  }
  // the four waves' rows on one shift
  const float lsum = other_half_sum(sx.l);
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
  float inv = 0.f;
  {
    const float oM = fmaxf(fmaxf(sm[0][orow], sm[1][orow]), fmaxf(sm[2][orow], sm[3][orow]));
    float oL = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x)
      oL += sm[x][orow] == -INFINITY ? 0.f : sl[x][orow] * __builtin_amdgcn_exp2f(sm[x][orow] - oM);
    inv = oM == -INFINITY ? 0.f : 1.f / oL;
  }
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    float* so = (float*)buf[wave];
#pragma unroll
    for (int r = 0; r < 16; ++r) so[lr * 33 + 8 * (r >> 2) + 4 * lh + (r & 3)] = f == 0.f ? 0.f : sx.acc[d][r] * f;
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
        if (inv == 0.f) store4(out_of<T>(a, b, ow) + 32 * d + od, 0.f, 0.f, 0.f, 0.f);
        else store4(out_of<T>(a, b, ow) + 32 * d + od, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
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
template <typename T, int D>
__global__ __launch_bounds__(256, sizeof(T) * D == 512 ? 1 : 2) void attend_rows_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl) {
  using TL = Tile<T, D>;
  constexpr int KB = sizeof(T) == 2 ? 2 : 1, KT = 32 * KB;
  constexpr int NV = KT * TL::CPR / 256;
  __shared__ u32x4 sk[2][KT * TL::CPR], sv[2][KT * TL::CPR];
  __shared__ int spos[2][KT];
  __shared__ uint32_t slim[4];
  __shared__ uint32_t slive[4];
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
  if (lane == 0) slim[wave] = lim_max;
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
  const uint32_t wg_lim = max(max(slim[0], slim[1]), max(slim[2], slim[3]));

  const int tiles = (c.C + KT - 1) / KT, per = (tiles + pl.splits - 1) / pl.splits;
  const int t_lo = split * per, t_hi = min(tiles, t_lo + per);
  u32x4 kr[NV], vr[NV];
  int pr = -1;
  auto load = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int idx = j * 256 + tid, kr_ = idx / TL::CPR, ch = idx % TL::CPR;
      const int64_t s = min(t * KT + kr_, c.C - 1);
      kr[j] = *reinterpret_cast<const u32x4*>(kbase + s * c.ks[2] + ch * TL::EPC);
      vr[j] = *reinterpret_cast<const u32x4*>(vbase + s * c.vs[2] + ch * TL::EPC);
    }
    const int s = t * KT + lane;
    pr = (KT == 64 || lane < KT) && s < c.C ? ps[s] : -1;
  };
  auto stage = [&](int buf, bool scrub) __attribute__((always_inline)) {
    const uint64_t taken = __ballot(pr >= 0);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int idx = j * 256 + tid, r = idx / TL::CPR, ch = idx % TL::CPR;
      u32x4 x = vr[j];
      if (!(taken >> r & 1)) x = u32x4{0, 0, 0, 0};
      if (scrub) x = finite_part<T>(x);
      sk[buf][TL::k(r, ch)] = kr[j];
      sv[buf][TL::v(r, ch)] = x;
    }
    if (tid < KT) spos[buf][tid] = pr;
  };

  Softmax<T, D, false> sx;
  for (int scrub = 0;; scrub = 1) {
    sx.reset();
    for (int c0 = t_lo; c0 < t_hi; c0 += 64) {
      // which of the next 64 tiles any row of the workgroup sees: 16 tiles a wave
      uint32_t mine = 0;
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        const int t = c0 + wave * 16 + x, s = t * KT + lane;
        const int p = t < t_hi && (KT == 64 || lane < KT) && s < c.C ? ps[s] : -1;
        mine |= __ballot((uint32_t)p < wg_lim) ? 1u << x : 0u;
      }
      __syncthreads();  // the last tiles' readers are done, and slive's
      if (lane == 0) slive[wave] = mine;
      __syncthreads();
      uint64_t live = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) live |= (uint64_t)__builtin_amdgcn_readfirstlane(slive[x]) << (16 * x);
      if (live == 0) continue;
      auto next = [&]() __attribute__((always_inline)) {
        const int x = __builtin_ctzll(live);
        live &= live - 1;
        return c0 + x;
      };
      load(next());
      stage(0, scrub);
      __syncthreads();
      for (int cur = 0;; cur ^= 1) {
        const bool more = live != 0;
        if (more) load(next());
        const int p = spos[cur][lane % KT];
        if (__ballot((uint32_t)p < lim_max) != 0) {
          const bool all = __ballot((uint32_t)p < lim_min) == ~0ull;
          f32x16 s[KB];
#pragma unroll
          for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
          for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
              s[kb] = Op<T>::mma(TL::k_frag(sk[cur], 32 * kb + key_of_row(lr), ks, lh), qf[ks], s[kb]);
          if (!all) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
              for (int r = 0; r < 16; ++r)
                if ((uint32_t)spos[cur][32 * kb + 16 * (r >> 3) + 8 * lh + (r & 7)] >= w.lim) s[kb][r] = -INFINITY;
          }
          sx.template add<KB>(s, cs, sv[cur], 0, lane);
        }
        if (!more) break;
        stage(cur ^ 1, scrub);
        __syncthreads();
      }
    }
    __syncthreads();
    if (scrub) {
      for (int x = t_lo * KT; x < min(t_hi * KT, c.C); ++x)
        if ((uint32_t)ps[x] < w.lim) sx.add_unbounded(vbase + x * c.vs[2], lh);
      break;
    }
    if (!__syncthreads_or(w.lim != 0 && !sx.finite())) break;
  }

  if (w.lim == 0) {  // padding: what tiles without a mask gave it does not count
    sx.m = -INFINITY;
    sx.l = 0.f;
  }
  const float L = other_half_sum(sx.l);
  if (row >= R) return;
  const bool none = sx.m == -INFINITY;
  const float l2 = none ? -INFINITY : sx.m - Op<T>::kShift + __builtin_amdgcn_logf(L);
  if (pl.splits > 1) {
    const int64_t pr_ = ((int64_t)bg * pl.splits + split) * R + row;
    float* ml = (float*)a.ws + pl.part_ml + pr_ * 2;
    if (lh == 0) {
      ml[0] = sx.m;
      ml[1] = L;
    }
    float* o = (float*)a.ws + pl.part_o + pr_ * D;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4)
        store4(o + 32 * d + 2 * r + 4 * lh, sx.acc[d][r], sx.acc[d][r + 1], sx.acc[d][r + 2], sx.acc[d][r + 3]);
    return;
  }
  if (lh == 0) {
    if (a.weight_out) ((float*)a.ws)[pl.lse2 + (int64_t)bg * R + row] = l2;
    if (a.lse) a.lse[((int64_t)b * c.G * a.rep + w.head) * a.n + w.i] = none ? -INFINITY : l2 * kLn2;
  }
  const float inv = none ? 0.f : 1.f / L;
  T* o = out_of<T>(a, b, w);
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = none ? 0.f : sx.acc[d][r + e] * inv;
      store4(o + 32 * d + 2 * r + 4 * lh, x[0], x[1], x[2], x[3]);
    }
}

// What is left when the parts are done: workgroups below row_blocks join the parts of
// rows (D / 4 threads each), the others add up what rows gave 256 slots each, from the
// scores that attend_keys_kernel kept (4 bytes a row and slot, beside 4 D of a 16-bit key
// and value). Each of those works out its rows' log-sums from the parts by itself.
constexpr int kFinishRows = 64;
template <typename T, int D>
__global__ __launch_bounds__(256) void finish_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl,
                                                     int row_blocks, int slot_blocks) {
  __shared__ float s_l2[kFinishRows];
  __shared__ uint32_t s_lim[kFinishRows];
  const float* ws = (const float*)a.ws;
  const int64_t R = (int64_t)a.n * a.rep;
  const int S = pl.splits;
  const int tid = threadIdx.x;
  // shift and sum of row r of (b, g) over the parts
  auto total = [&](int64_t bg, int64_t r, float& M, float& L) {
    M = -INFINITY;
    L = 0.f;
    for (int s = 0; s < S; ++s) M = fmaxf(M, ws[pl.part_ml + ((bg * S + s) * R + r) * 2]);
    if (M == -INFINITY) return;
    for (int s = 0; s < S; ++s) {
      const float2 ml = *reinterpret_cast<const float2*>(ws + pl.part_ml + ((bg * S + s) * R + r) * 2);
      if (ml.x != -INFINITY) L += ml.y * __builtin_amdgcn_exp2f(ml.x - M);
    }
  };
  if ((int)blockIdx.x < row_blocks) {
    constexpr int TPR = D / 4, RPB = 256 / TPR;
    const int64_t x = (int64_t)blockIdx.x * RPB + tid / TPR;  // row over all (b, g)
    const int d = 4 * (tid % TPR);
    if (x >= (int64_t)c.B * c.G * R) return;
    const int64_t bg = x / R, r = x - bg * R;
    const int b = (int)(bg / c.G), g = (int)(bg - (int64_t)b * c.G);
    float M, L;
    total(bg, r, M, L);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    if (M != -INFINITY) {
      for (int s = 0; s < S; ++s) {
        const int64_t pr = (bg * S + s) * R + r;
        const float ms = ws[pl.part_ml + pr * 2];
        if (ms == -INFINITY) continue;
        const float f = __builtin_amdgcn_exp2f(ms - M);
        const float4 p = *reinterpret_cast<const float4*>(ws + pl.part_o + pr * D + d);
        o.x += f * p.x;
        o.y += f * p.y;
        o.z += f * p.z;
        o.w += f * p.w;
      }
      const float inv = 1.f / L;
      o = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
    }
    const Row w = row_of(a, b, g, r, R);
    store4(out_of<T>(a, b, w) + d, o.x, o.y, o.z, o.w);
    if (d == 0) {
      const float l2 = M == -INFINITY ? -INFINITY : M - Op<T>::kShift + __builtin_amdgcn_logf(L);
      if (a.weight_out && !pl.by_keys) ((float*)a.ws)[pl.lse2 + x] = l2;
      if (a.lse) a.lse[((int64_t)b * c.G * a.rep + w.head) * a.n + w.i] = M == -INFINITY ? -INFINITY : l2 * kLn2;
    }
    return;
  }
  const int y = blockIdx.x - row_blocks;
  const int64_t bg = y / slot_blocks;
  const int b = (int)(bg / c.G), g = (int)(bg - (int64_t)b * c.G);
  const int s = (y % slot_blocks) * 256 + tid;
  const int p = s < c.C ? c.pos[bg * c.C + s] : -1;
  float sum = 0.f;
  const float cs = a.scale * kLog2e;
  for (int64_t r0 = 0; r0 < R; r0 += kFinishRows) {
    const int m = (int)min((int64_t)kFinishRows, R - r0);
    __syncthreads();
    if (tid < m) {
      float M, L;
      total(bg, r0 + tid, M, L);
      s_l2[tid] = M - Op<T>::kShift + __builtin_amdgcn_logf(L);
      s_lim[tid] = M == -INFINITY ? 0u : row_of(a, b, g, r0 + tid, R).lim;
    }
    __syncthreads();
    if (p >= 0)
      for (int r = 0; r < m; ++r)
        if ((uint32_t)p < s_lim[r])
          sum += __builtin_amdgcn_exp2f(fmaf(ws[pl.scores + (bg * R + r0 + r) * c.C + s], cs, -s_l2[r]));
  }
  if (s < c.C) {
    const int64_t at = bg * c.C + s;
    a.weight_out[at] = p < 0 ? 0.f : fmaf(a.decay, c.weight[at], sum);
  }
}

// The weights of a chunk of tokens: p = exp2(score - lse) needs the rows' log-sums, so
// the scores are computed again, with the keys held and the rows streaming past: a wave
// keeps 32 KB keys' fragments in registers and the four waves share tiles of 32 rows
// through LDS. Half the matrix work of the attention, and its exponentials.
template <typename T, int D>
__global__ __launch_bounds__(256, 2) void weights_kernel(TokenCacheArgs c, TokenAttend a, TokenAttendPlan pl) {
  using TL = Tile<T, D>;
  constexpr int KB = sizeof(T) == 2 ? 2 : 1;  // 32-key blocks of a wave
  constexpr int NV = (32 * TL::CPR + 255) / 256;
  __shared__ u32x4 sq[2][32 * TL::CPR];
  __shared__ float sl2[2][32];
  __shared__ uint32_t slim[2][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int lr = lane & 31, lh = lane >> 5;
  const int slot_blocks = (c.C + 128 * KB - 1) / (128 * KB);
  const int kbk = blockIdx.x % slot_blocks, part = blockIdx.x / slot_blocks;
  const int bg = blockIdx.y, b = bg / c.G, g = bg - b * c.G;
  const int64_t R = (int64_t)a.n * a.rep;
  const int s0 = kbk * 128 * KB + wave * 32 * KB;
  const int* ps = c.pos + (int64_t)bg * c.C;
  const T* kbase = (const T*)c.k + b * c.ks[0] + g * c.ks[1];
  const float* l2 = (const float*)a.ws + pl.lse2 + (int64_t)bg * R;
  const float cs = a.scale * kLog2e;

  typename Op<T>::V kf[KB][D / 16];
  int kp[KB][16];          // positions of the lane's 16 keys a block (register r: key 8 (r / 4) + 4 lh + r % 4)
  uint32_t p_max = 0, p_min = ~0u;
#pragma unroll
  for (int kb = 0; kb < KB; ++kb) {
    const T* k = kbase + (int64_t)min(s0 + 32 * kb + lr, c.C - 1) * c.ks[2];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) kf[kb][ks] = *reinterpret_cast<const typename Op<T>::V*>(k + 16 * ks + 8 * lh);
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int s = s0 + 32 * kb + 8 * (r >> 2) + 4 * lh + (r & 3);
      kp[kb][r] = s < c.C ? ps[s] : -1;
      p_max = max(p_max, (uint32_t)kp[kb][r]);
      p_min = min(p_min, (uint32_t)kp[kb][r]);
    }
  }
  p_max = lanes_max(p_max);  // an empty slot among them: >= 2^31, so that no row sees them all
  p_min = lanes_min(p_min);

  const int64_t row_tiles = (R + 31) / 32, per = (row_tiles + pl.weight_parts - 1) / pl.weight_parts;
  const int64_t t0 = part * per, t1 = min(row_tiles, t0 + per);
  u32x4 qr[NV];
  float l2r = 0.f;
  uint32_t limr = 0;
  auto load = [&](int64_t t) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int idx = j * 256 + tid, ch = idx % TL::CPR;
      if (32 * TL::CPR % 256 == 0 || idx < 32 * TL::CPR) {
        const int64_t r = min(t * 32 + idx / TL::CPR, R - 1);
        const int i = (int)(r / a.rep);
        qr[j] = *reinterpret_cast<const u32x4*>((const T*)a.q + b * a.qs[0] + i * a.qs[1] +
                                                (g * a.rep + (int)(r - (int64_t)i * a.rep)) * a.qs[2] + ch * TL::EPC);
      }
    }
    if (tid < 32) {
      const int64_t r = t * 32 + tid;
      l2r = r < R ? l2[r] : 0.f;
      limr = r < R && l2r != -INFINITY ? row_of(a, b, g, r, R).lim : 0u;
    }
  };
  auto stage = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int idx = j * 256 + tid;
      if (32 * TL::CPR % 256 == 0 || idx < 32 * TL::CPR) sq[buf][TL::k(idx / TL::CPR, idx % TL::CPR)] = qr[j];
    }
    if (tid < 32) {
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
    const uint32_t lim = slim[cur][lr];
    if (__ballot(lim > p_min) != 0) {
      const bool all = __ballot(lim > p_max) == ~0ull;
      const float nl = -sl2[cur][lr];
      f32x16 s[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[kb][r] = 0.f;
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const typename Op<T>::V q = TL::k_frag(sq[cur], lr, ks, lh);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) s[kb] = Op<T>::mma(kf[kb][ks], q, s[kb]);
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[kb][r], cs, nl));
          sum[kb][r] += all || (uint32_t)kp[kb][r] < lim ? p : 0.f;
        }
    }
    if (t + 1 < t1) stage(cur ^ 1);
    __syncthreads();
  }
  // over the 32 rows of a half
#pragma unroll
  for (int kb = 0; kb < KB; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = sum[kb][r];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) x += __shfl_xor(x, o);
      const int s = s0 + 32 * kb + 8 * (r >> 2) + 4 * lh + (r & 3);
      if (lr == 0 && s < c.C) {
        const int64_t at = (int64_t)bg * c.C + s;
        if (pl.weight_parts > 1) ((float*)a.ws)[pl.weights + ((int64_t)bg * pl.weight_parts + part) * c.C + s] = x;
        else a.weight_out[at] = kp[kb][r] < 0 ? 0.f : fmaf(a.decay, c.weight[at], x);
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
hipError_t attend_launch(const TokenCacheArgs& c, const TokenAttend& a, int kind, hipStream_t s) {
  const int64_t R = (int64_t)a.n * a.rep;
  const int BG = c.B * c.G;
  if (a.n == 0) {  // no rows: the weights only fade
    if (a.weight_out) {
      TokenAttendPlan none;
      none.weight_parts = 0;
      hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)(((int64_t)BG * c.C + 255) / 256)), dim3(256), 0, s, c, a,
                         none);
    }
    return hipGetLastError();
  }
  const TokenAttendPlan pl = token_attend_plan(c, a.n, a.rep, kind, a.weight_out != nullptr);
  const int slot_blocks = (c.C + 255) / 256;
  const int64_t row_blocks = ((int64_t)BG * R * (D / 4) + 255) / 256;
  if (pl.by_keys) {
    hipLaunchKernelGGL((attend_keys_kernel<T, D>), dim3(pl.splits, pl.row_tiles, BG), dim3(256), 0, s, c, a, pl);
    if (pl.splits > 1 || a.weight_out)
      hipLaunchKernelGGL((finish_kernel<T, D>),
                         dim3((unsigned)(row_blocks + (a.weight_out ? (int64_t)BG * slot_blocks : 0))), dim3(256), 0, s, c,
                         a, pl, (int)row_blocks, slot_blocks);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((attend_rows_kernel<T, D>), dim3((unsigned)(pl.row_tiles * pl.splits * BG)), dim3(256), 0, s, c, a,
                     pl);
  if (pl.splits > 1)
    hipLaunchKernelGGL((finish_kernel<T, D>), dim3((unsigned)row_blocks), dim3(256), 0, s, c, a, pl, (int)row_blocks,
                       slot_blocks);
  if (a.weight_out) {
    constexpr int KW = sizeof(T) == 2 ? 256 : 128;
    hipLaunchKernelGGL((weights_kernel<T, D>), dim3((unsigned)((c.C + KW - 1) / KW * pl.weight_parts), (unsigned)BG),
                       dim3(256), 0, s, c, a, pl);
    if (pl.weight_parts > 1)
      hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)(((int64_t)BG * c.C + 255) / 256)), dim3(256), 0, s, c, a,
                         pl);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t attend_dim(const TokenCacheArgs& c, const TokenAttend& a, int kind, hipStream_t s) {
  if (c.D == 32) return attend_launch<T, 32>(c, a, kind, s);
  if (c.D == 64) return attend_launch<T, 64>(c, a, kind, s);
  return attend_launch<T, 128>(c, a, kind, s);
}

}  // namespace

TokenAttendPlan token_attend_plan(const TokenCacheArgs& c, int n, int rep, int kind, bool weights) {
  TokenAttendPlan p;
  const int64_t R = (int64_t)n * rep, BG = (int64_t)c.B * c.G;
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  auto clamp = [](int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; };
  p.by_keys = R <= 64;
  p.row_tiles = (int)up(R, p.by_keys ? 32 : 128);
  const int64_t wgs = BG * p.row_tiles;
  if (p.by_keys) {
    // three workgroups a CU, but at least two tiles of 32 slots a wave
    p.splits = (int)clamp(up(768, wgs), 1, clamp(up(c.C, 256), 1, 128));
  } else {
    // enough workgroups for two a CU, parts of at least 512 slots
    p.splits = wgs >= 384 ? 1 : (int)clamp(512 / wgs, 1, clamp(c.C / 512, 1, 16));
    const int64_t kw = up(c.C, kind == 2 ? 128 : 256) * BG;
    p.weight_parts = kw >= 384 ? 1 : (int)clamp(512 / kw, 1, clamp(R / 256, 1, 64));
  }
  int64_t at = 0;
  auto take = [&](int64_t floats) {
    const int64_t o = at;
    at += up(floats, 64) * 64;
    return o;
  };
  if (p.splits > 1 || (p.by_keys && weights)) {
    p.part_o = take(BG * p.splits * R * c.D);
    p.part_ml = take(BG * p.splits * R * 2);
  }
  if (weights && p.by_keys) p.scores = take(BG * R * c.C);
  if (weights && !p.by_keys) {
    p.lse2 = take(BG * R);
    if (p.weight_parts > 1) p.weights = take(BG * p.weight_parts * c.C);
  }
  p.bytes = at * 4;
  return p;
}

hipError_t token_attend(const TokenCacheArgs& c, const TokenAttend& a, int kind, hipStream_t s) {
  if (kind == 0) return attend_dim<_Float16>(c, a, kind, s);
  if (kind == 1) return attend_dim<__bf16>(c, a, kind, s);
  return attend_dim<float>(c, a, kind, s);
}

}  // namespace fd
