// The choice of slots for new tokens of a token cache: for every request and KV
// group the m slots that come first by (class, weight, slot), where m is the number
// of the request's valid new tokens and a slot's class is 0 empty, 1 free to go,
// 2 recent, 3 first. The chosen slots, in rising order, go to the valid tokens in
// order. New tokens then overwrite what they replace where it lies, so an eviction
// moves no key or value: 8 bytes are read per slot, and nothing else.
//
// One workgroup of 16 waves per (request, group). A wave owns a contiguous segment of
// slots, so that ranks in slot order are ballots inside the wave and one scan over
// the 16 waves. The m-th smallest weight of the class in which the count runs out
// is found by three histograms of its 11, 11 and 10 highest bits (a radix select:
// three passes whatever the weights and m), and equal weights go in slot order by
// their rank. Up to 16384 slots the keys stay in registers, so memory is read once
// (64 keys a thread would spill); above that each pass reads them again, out of L2.
// Integer counts only: the result does not depend on the order of the atomics.
// One new token (serving) is a plain minimum of (class, weight, slot).
#include "fd_token.h"

namespace fd {
namespace {

constexpr int kThreads = 1024, kWaves = 16, kBins = 2048;
constexpr int kWords = kMaxSlotTokens / 64;

// Weights as unsigned integers in the same order; NaN as the lowest, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  w = w != w ? -INFINITY : w + 0.f;
  const uint32_t u = __float_as_uint(w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int slot_class(int p, int64_t recent_from, int first) {
  return p < 0 ? 0 : (p < first ? 3 : ((int64_t)p > recent_from ? 2 : 1));
}

// Inclusive sum over the lanes of a wave.
__device__ __forceinline__ int wave_scan(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  return x;
}

// Adds one to hist[bin] for every lane with `on`. Lanes that agree on one bin (empty
// or fresh slots all weigh the same) make one addition instead of 64 in a row.
__device__ __forceinline__ void count_bin(int* hist, int bin, bool on, int lane) {
  const uint64_t m = __ballot(on);
  if (m == 0) return;
  const int lead = __ffsll((unsigned long long)m) - 1;
  const int b0 = __shfl(bin, lead);
  const uint64_t same = __ballot(on && bin == b0);
  if (lane == lead) atomicAdd(&hist[b0], (int)__popcll(same));
  if (on && bin != b0) atomicAdd(&hist[bin], 1);
}

template <int PER>  // keys of a thread held in registers; 0: read again for every pass
__global__ __launch_bounds__(kThreads) void slots_kernel(TokenSlots a) {
  __shared__ int hist[3][kBins];
  __shared__ uint64_t masks[kWords];
  __shared__ int before[kWords];
  __shared__ int part[kWaves][4];
  __shared__ int found[4];  // bin, slots before it; newest; last valid token
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.x / a.G;
  const int64_t base = (int64_t)blockIdx.x * a.C;
  const int* tok_pos = a.pos + (int64_t)b * a.n;
  int* out = a.slots + (int64_t)blockIdx.x * a.n;

  // the valid tokens: 64 of them a word, with the count before it
  const int words = (a.n + 63) / 64;
  if (tid < 4) found[tid] = -1;
  __syncthreads();
  int newest = -1, last = -1;
  for (int w = wave; w < words; w += kWaves) {
    const int i = w * 64 + lane;
    const int p = i < a.n ? tok_pos[i] : -1;
    const uint64_t m = __ballot(p >= 0);
    if (lane == 0) masks[w] = m;
    if (p >= 0) {
      newest = max(newest, p);
      last = i;
    } else if (i < a.n) {
      out[i] = -1;
    }
  }
  if (newest >= 0) {
    atomicMax(&found[2], newest);
    atomicMax(&found[3], last);
  }
  __syncthreads();
  newest = found[2];
  last = found[3];
  if (last < 0) return;  // (the whole workgroup)
  {
    const int c = tid < words ? (int)__popcll(masks[tid]) : 0;
    const int inc = wave_scan(c, lane);
    if (lane == 63) part[wave][0] = inc;
    __syncthreads();
    int off = 0;
    for (int w = 0; w < wave; ++w) off += part[w][0];
    if (tid < words) before[tid] = off + inc - c;
  }
  for (int i = tid; i < 3 * kBins; i += kThreads) (&hist[0][0])[i] = 0;
  __syncthreads();
  const int m = before[words - 1] + (int)__popcll(masks[words - 1]);
  const bool dense = last == m - 1;  // the valid tokens are the first m
  const int64_t recent_from = (int64_t)newest - a.keep_recent;

  const int steps = PER ? PER : ((a.C + kWaves - 1) / kWaves + 63) / 64;
  const int seg = wave * steps * 64;
  uint32_t key[PER ? PER : 1];
  uint32_t cls[PER ? (PER + 7) / 8 : 1];
  auto load = [&](int j, uint32_t& k, int& c) {
    const int s = seg + j * 64 + lane;
    c = 4;  // no slot
    k = 0;
    if (s < a.C) {
      c = slot_class(a.slot_pos[base + s], recent_from, a.keep_first);
      k = c ? weight_key(a.weight[base + s]) : 0;
    }
  };
  if constexpr (PER > 0) {
#pragma unroll
    for (int j = 0; j < (PER + 7) / 8; ++j) cls[j] = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      int c;
      load(j, key[j], c);
      cls[j / 8] |= (uint32_t)c << (4 * (j % 8));
    }
  }
  // f(slot of lane 0, class, key of this lane's slot)
  auto each = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j) f(seg + j * 64, (int)(cls[j / 8] >> (4 * (j % 8))) & 15, key[j]);
    } else {
      for (int j = 0; j < steps; ++j) {
        uint32_t k;
        int c;
        load(j, k, c);
        f(seg + j * 64, c, k);
      }
    }
  };

  // counts of the classes, and the first histogram of each that has weights
  int cnt[4] = {0, 0, 0, 0};
  each([&](int, int c, uint32_t k) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const bool on = c == q;
      cnt[q] += (int)__popcll(__ballot(on));
      if (q) count_bin(hist[q - 1], (int)(k >> 21), on, lane);
    }
  });
  if (lane == 0)
    for (int q = 0; q < 4; ++q) part[wave][q] = cnt[q];
  __syncthreads();
  int rem = m, cut = 0;  // the class in which the count runs out, and what is left to take there
  for (; cut < 3; ++cut) {
    int c = 0;
    for (int w = 0; w < kWaves; ++w) c += part[w][cut];
    if (rem <= c) break;
    rem -= c;
  }
  __syncthreads();  // part is written again below

  // the bin of h in which the count reaches `rem`, and rem less what lies before it
  auto find = [&](const int* h, int bins) {
    const int i0 = 2 * tid;
    const int h0 = i0 < bins ? h[i0] : 0, h1 = i0 + 1 < bins ? h[i0 + 1] : 0;
    const int inc = wave_scan(h0 + h1, lane);
    if (lane == 63) part[wave][0] = inc;
    __syncthreads();
    int off = 0;
    for (int w = 0; w < wave; ++w) off += part[w][0];
    const int ex = off + inc - h0 - h1;
    if (ex < rem && rem <= ex + h0 + h1) {
      const bool second = rem > ex + h0;
      found[0] = i0 + second;
      found[1] = second ? ex + h0 : ex;
    }
    __syncthreads();
    rem -= found[1];
    return (uint32_t)found[0];
  };
  uint32_t cut_key = 0;
  if (cut > 0) {
    const uint32_t b1 = find(hist[cut - 1], kBins);
    int* h = hist[cut % 3];  // another class's histogram is free now
    for (int pass = 0; pass < 2; ++pass) {
      const int sh = pass ? 0 : 10, bits = pass ? 10 : 11;
      for (int i = tid; i < kBins; i += kThreads) h[i] = 0;
      if (pass == 0) cut_key = b1;
      __syncthreads();
      each([&](int, int c, uint32_t k) {
        count_bin(h, (int)((k >> sh) & ((1u << bits) - 1)), c == cut && (k >> (sh + bits)) == cut_key, lane);
      });
      __syncthreads();
      cut_key = (cut_key << bits) | find(h, 1 << bits);
    }
  }

  // ranks in slot order: below the cut all, at the cut the first `rem`
  int n_lt = 0, n_eq = 0;
  each([&](int, int c, uint32_t k) {
    n_lt += (int)__popcll(__ballot(c < cut || (c == cut && k < cut_key)));
    n_eq += (int)__popcll(__ballot(c == cut && k == cut_key));
  });
  if (lane == 0) {
    part[wave][1] = n_lt;
    part[wave][2] = n_eq;
  }
  __syncthreads();
  int lt0 = 0, eq0 = 0;
  for (int w = 0; w < wave; ++w) {
    lt0 += part[w][1];
    eq0 += part[w][2];
  }
  int rank0 = lt0 + min(eq0, rem);
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0;
  each([&](int s0, int c, uint32_t k) {
    const bool lt = c < cut || (c == cut && k < cut_key), eq = c == cut && k == cut_key;
    const uint64_t em = __ballot(eq);
    const bool take = lt || (eq && eq0 + (int)__popcll(em & below) < rem);
    const uint64_t tm = __ballot(take);
    if (take) {
      const int r = rank0 + (int)__popcll(tm & below);
      int t = r;
      if (!dense && r < m) {  // token of rank r: its word, then its bit
        int lo = 0, hi = words - 1;
        while (lo < hi) {
          const int mid = (lo + hi + 1) / 2;
          if (before[mid] <= r) lo = mid;
          else hi = mid - 1;
        }
        uint64_t w = masks[lo];
        for (int i = r - before[lo]; i > 0; --i) w &= w - 1;
        t = lo * 64 + __ffsll((unsigned long long)w) - 1;
      }
      if (r < m) out[t] = s0 + lane;
    }
    eq0 += (int)__popcll(em);
    rank0 += (int)__popcll(tm);
  });
}

// One new token: the least (class, weight, slot).
__global__ __launch_bounds__(kThreads) void slot_least_kernel(TokenSlots a) {
  __shared__ uint64_t part[kWaves];
  const int tid = threadIdx.x;
  const int64_t base = (int64_t)blockIdx.x * a.C;
  const int p = a.pos[blockIdx.x / a.G];
  const int64_t recent_from = (int64_t)p - a.keep_recent;
  uint64_t best = ~0ull;
  for (int s = tid; s < a.C; s += kThreads) {
    const int c = slot_class(a.slot_pos[base + s], recent_from, a.keep_first);
    const uint64_t k = (((uint64_t)c << 32 | (c ? weight_key(a.weight[base + s]) : 0)) << 24) | (uint32_t)s;
    best = k < best ? k : best;
  }
  for (int o = 32; o > 0; o >>= 1) {
    const uint64_t y = __shfl_xor((unsigned long long)best, o);
    best = y < best ? y : best;
  }
  if ((tid & 63) == 0) part[tid >> 6] = best;
  __syncthreads();
  if (tid == 0) {
    for (int w = 1; w < kWaves; ++w) best = part[w] < best ? part[w] : best;
    a.slots[blockIdx.x] = p < 0 ? -1 : (int)(best & 0xFFFFFF);
  }
}

}  // namespace

hipError_t token_slots(const TokenSlots& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.G));
  if (a.n == 1) hipLaunchKernelGGL(slot_least_kernel, grid, dim3(kThreads), 0, s, a);
  else if (a.C <= 4 * kThreads) hipLaunchKernelGGL(slots_kernel<4>, grid, dim3(kThreads), 0, s, a);
  else if (a.C <= 16 * kThreads) hipLaunchKernelGGL(slots_kernel<16>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(slots_kernel<0>, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace fd
