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
// is found by histograms of its 11, 11 and 10 highest bits (a radix select: at most
// three passes whatever the weights and m, fewer if a bin is taken whole), and equal
// weights go in slot order by their rank. Up to 16384 keys stay in registers, so memory
// is read once (64 keys a thread would spill). Above that a first launch chooses the best
// m of every 16384 slots and a second one among those, as long as that halves the keys
// at least; else each pass reads all keys again, out of L2. 4 requests x 8 groups, 131072
// slots, 1560 tokens each: 26 + 19 us (203 in one launch when that was all there was),
// where one workgroup's instructions and barriers are the limit and not memory.
// Integer counts only: the result does not depend on the order of the atomics.
// One new token (serving) is a plain minimum of (class, weight, slot): 2.7 us at 1024 slots.
// The one workgroup of a pair reads what a CU can (8 bytes a slot at 37 GB/s): 28 us at 131072
// slots, 107 at 524288; there chunks are faster while they find idle CUs (chunks_of).
#include "fd_token.h"

#include <type_traits>

namespace fd {
namespace {

constexpr int kThreads = 1024, kWaves = 16, kBins = 2048, kChunk = 16 * kThreads;
constexpr int kWords = kMaxSlotTokens / 64;
// The highest 11 bits of weights (sign, exponent, two more) fall into a few dozen bins;
// lanes add to eight copies of the first histogram, in banks of their own.
constexpr int kCopies = 8;

// Weights as unsigned integers in the same order; NaN as the lowest, -0 as 0.
__device__ __forceinline__ uint32_t weight_key(float w) {
  w = w != w ? -INFINITY : w + 0.f;
  const uint32_t u = __float_as_uint(w);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ int slot_class(int p, int recent_from, int first) {
  return p < 0 ? 0 : (p < first ? 3 : (p > recent_from ? 2 : 1));
}

// Inclusive sum over the lanes of a wave: within rows of 16, then row 0 into 1 and 2
// into 3, then the lower half into the upper (no LDS round trips).
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// Adds one to hist[bin] for every lane with `on`. Lanes that agree on one bin (empty
// or fresh slots all weigh the same) make one addition instead of 64 in a row.
__device__ __forceinline__ void count_bin(int* hist, int bin, bool on, int lane) {
  const uint64_t m = __ballot(on);
  if (m == 0) return;
  const int lead = __ffsll((unsigned long long)m) - 1;
  const int b0 = __builtin_amdgcn_readlane(bin, lead);
  const uint64_t same = __ballot(on && bin == b0);
  if (lane == lead) atomicAdd(&hist[b0], (int)__popcll(same));
  if (on && bin != b0) atomicAdd(&hist[bin], 1);
}

// Sum of column q over the waves before `wave` (all loads at once).
__device__ __forceinline__ int before_wave(const int (*part)[4], int q, int wave) {
  int s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int x = part[w][q];
    s += w < wave ? x : 0;
  }
  return s;
}

template <int PER>  // keys of a thread held in registers; 0: read again for every pass
__global__ __launch_bounds__(kThreads) void slots_kernel(TokenSlots a) {
  __shared__ int hist0[kBins * kCopies], hist[2][kBins];
  __shared__ uint64_t masks[kWords];
  __shared__ int before[kWords];
  __shared__ int part[kWaves][4];
  __shared__ int found[4];  // bin, slots before it; newest; last valid token
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  // this workgroup's slots: all of its (request, group), or (a.chunks) one chunk of them,
  // or (a.list) the ones that the chunks chose
  const bool chunked = a.chunks > 0 && !a.list_in;
  const int bg = chunked ? blockIdx.x / a.chunks : blockIdx.x, b = bg / a.G;
  const int first = chunked ? (int)(blockIdx.x % a.chunks) * kChunk : 0;
  const int count = a.list_in ? a.chunks * a.n : chunked ? min(kChunk, a.C - first) : a.C;
  const int* spos = a.slot_pos + (int64_t)bg * a.C;
  const float* swt = a.weight + (int64_t)bg * a.C;
  const int* list = a.list_in ? a.list_in + (int64_t)bg * count : nullptr;
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
    } else if (i < a.n && !chunked) {
      out[i] = -1;
    }
  }
  // (one atomic a wave: those of 64 lanes on one address take their turns)
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    newest = max(newest, __shfl_xor(newest, o));
    last = max(last, __shfl_xor(last, o));
  }
  if (lane == 0 && last >= 0) {
    atomicMax(&found[2], newest);
    atomicMax(&found[3], last);
  }
  __syncthreads();
  newest = found[2];
  last = found[3];
  if (last < 0) {  // (the whole workgroup)
    if (chunked)
      for (int i = tid; i < a.n; i += kThreads) out[i] = -1;
    return;
  }
  {
    const int c = tid < words ? (int)__popcll(masks[tid]) : 0;
    const int inc = wave_scan(c);
    if (lane == 63) part[wave][0] = inc;
    __syncthreads();
    const int off = before_wave(part, 0, wave);
    if (tid < words) before[tid] = off + inc - c;
  }
  for (int i = tid; i < kBins * kCopies; i += kThreads) hist0[i] = 0;
  for (int i = tid; i < 2 * kBins; i += kThreads) (&hist[0][0])[i] = 0;
  __syncthreads();
  const int tokens = before[words - 1] + (int)__popcll(masks[words - 1]);
  const int m = min(tokens, count);
  const bool dense = chunked || last == tokens - 1;  // the valid tokens are the first ones
  if (chunked)
    for (int i = m + tid; i < a.n; i += kThreads) out[i] = -1;
  const int recent_from = newest - a.keep_recent;  // (both are >= 0)

  const int steps = PER ? PER : ((count + kWaves - 1) / kWaves + 63) / 64;
  const int seg = wave * steps * 64;
  uint32_t key[PER ? PER : 1];
  uint32_t cls[PER ? (PER + 7) / 8 : 1];
  // N places from step j on: class and key of this lane's slots (all loads at once)
  auto load = [&](int j, auto places, int* c, uint32_t* k) __attribute__((always_inline)) {
    constexpr int N = decltype(places)::value;
    int s[N], p[N];
    float w[N];
    if (list) {
#pragma unroll
      for (int x = 0; x < N; ++x) s[x] = list[min(seg + (j + x) * 64 + lane, count - 1)];
    } else {
#pragma unroll
      for (int x = 0; x < N; ++x) s[x] = first + min(seg + (j + x) * 64 + lane, count - 1);
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      p[x] = spos[max(s[x], 0)];
      w[x] = swt[max(s[x], 0)];
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      const bool none = s[x] < 0 || j + x >= steps || seg + (j + x) * 64 + lane >= count;
      c[x] = none ? 4 : slot_class(p[x], recent_from, a.keep_first);  // 4: no slot
      k[x] = weight_key(w[x]);
    }
  };
  // f(first lane's place, class, key) of all places, eight of a lane at a time
  auto stream = [&](auto f) {
    for (int j = 0; j < steps; j += 8) {
      uint32_t k[8];
      int c[8];
      load(j, std::integral_constant<int, 8>{}, c, k);
#pragma unroll
      for (int x = 0; x < 8; ++x) f(seg + (j + x) * 64, c[x], k[x]);
    }
  };

  // the class in which the count runs out, and what is left to take there
  int cnt[4] = {0, 0, 0, 0};
  auto count_class = [&](int c) {
#pragma unroll
    for (int q = 0; q < 4; ++q) cnt[q] += (int)__popcll(__ballot(c == q));
  };
  if constexpr (PER > 0) {
    int c[PER];
    load(0, std::integral_constant<int, PER>{}, c, key);
#pragma unroll
    for (int j = 0; j < (PER + 7) / 8; ++j) cls[j] = 0;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      count_class(c[j]);
      cls[j / 8] |= (uint32_t)c[j] << (4 * (j % 8));
    }
  } else {
    stream([&](int, int c, uint32_t) { count_class(c); });
  }
  if (lane == 0)
    for (int q = 0; q < 4; ++q) part[wave][q] = cnt[q];
  __syncthreads();
  int rem = m, cut = 0;
  for (; cut < 3; ++cut) {
    const int c = before_wave(part, cut, kWaves);
    if (rem <= c) break;
    rem -= c;
  }
  rem = m;
  __syncthreads();  // part is written again below

  // From here on one key: 0 before that class, ~0 behind it (weights lie between the two),
  // and 1 for all empty slots, which take no order but their index.
  auto final_key = [&](int c, uint32_t k) { return c < cut ? 0u : c > cut ? ~0u : cut ? k : 1u; };
  if constexpr (PER > 0) {
#pragma unroll
    for (int j = 0; j < PER; ++j) key[j] = final_key((int)(cls[j / 8] >> (4 * (j % 8))) & 15, key[j]);
  }
  auto each = [&](auto f) {
    if constexpr (PER > 0) {
#pragma unroll
      for (int j = 0; j < PER; ++j) f(seg + j * 64, key[j]);
    } else {
      stream([&](int s0, int c, uint32_t k) { f(s0, final_key(c, k)); });
    }
  };
  // cut_key: the least key of which not all are taken; `rem` of those are
  uint32_t cut_key = 1;
  if (cut == 0) {
    // (nothing has key 0: the first m empty slots)
  } else {
    uint32_t prefix = 0;
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int sh = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
      if (pass == 0)
        each([&](int, uint32_t k) { atomicAdd(&hist0[(k >> 21) * kCopies + lane % kCopies], 1); });
      else
        each([&](int, uint32_t k) {
          count_bin(hist[pass - 1], (int)((k >> sh) & ((1u << bits) - 1)), (k >> sh >> bits) == prefix, lane);
        });
      __syncthreads();
      // the bin in which the count reaches `rem`, and rem less what lies before it
      const int i0 = 2 * tid;
      int h0 = 0, h1 = 0;
      if (pass == 0) {
#pragma unroll
        for (int x = 0; x < kCopies; ++x) {
          h0 += hist0[i0 * kCopies + x];
          h1 += hist0[(i0 + 1) * kCopies + x];
        }
      } else {
        h0 = hist[pass - 1][i0];
        h1 = hist[pass - 1][i0 + 1];
      }
      const int inc = wave_scan(h0 + h1);
      if (lane == 63) part[wave][0] = inc;
      __syncthreads();
      const int ex = before_wave(part, 0, wave) + inc - h0 - h1;
      if (ex < rem && rem <= ex + h0 + h1) {
        const bool second = rem > ex + h0;
        found[0] = i0 + second;
        found[1] = second ? ex + h0 : ex;
        found[2] = second ? h1 : h0;
      }
      __syncthreads();
      rem -= found[1];
      prefix = (prefix << bits) | (uint32_t)found[0];
      if (rem == found[2] || pass == 2) {  // the whole bin is taken, or it is one key
        const bool all = rem == found[2];
        cut_key = all ? (prefix + 1) << sh : prefix;
        if (all) rem = 0;
        break;
      }
    }
  }

  // ranks in slot order: below the cut all, at the cut the first `rem`
  int n_lt = 0, n_eq = 0;
  each([&](int, uint32_t k) {
    n_lt += (int)__popcll(__ballot(k < cut_key));
    n_eq += (int)__popcll(__ballot(k == cut_key));
  });
  if (lane == 0) {
    part[wave][1] = n_lt;
    part[wave][2] = n_eq;
  }
  __syncthreads();
  const int lt0 = before_wave(part, 1, wave);
  int eq0 = before_wave(part, 2, wave);
  int rank0 = lt0 + min(eq0, rem);
  const uint64_t below = lane ? ~0ull >> (64 - lane) : 0;
  // token of rank r among the valid ones: its word, then its bit
  auto token_at = [&](int r) {
    if (dense) return r;
    int lo = 0, hi = words - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (before[mid] <= r) lo = mid;
      else hi = mid - 1;
    }
    uint64_t w = masks[lo];
    for (int i = r - before[lo]; i > 0; --i) w &= w - 1;
    return lo * 64 + __ffsll((unsigned long long)w) - 1;
  };
  each([&](int s0, uint32_t k) {
    const uint64_t em = __ballot(k == cut_key), lm = __ballot(k < cut_key);
    if ((em | lm) == 0) return;
    const bool take = (lm >> lane & 1) || ((em >> lane & 1) && eq0 + (int)__popcll(em & below) < rem);
    const uint64_t tm = __ballot(take);
    const int r = rank0 + (int)__popcll(tm & below);
    if (take && r < m) out[token_at(r)] = first + s0 + lane;
    eq0 += (int)__popcll(em);
    rank0 += (int)__popcll(tm);
  });
  if (list) {  // from places in the list to slots
    __syncthreads();
    for (int i = tid; i < a.n; i += kThreads) {
      const int e = out[i];
      if (e >= 0) out[i] = list[e];
    }
  }
}

// One new token: the least (class, weight, slot). U loads of each array are under way (a
// few thousand slots are one to four a thread, and eight would load the last one over and
// over: 1024 slots 2.8 us against 4.1, 4096 3.0 to 3.6 against 3.8 to 4.3, 8192 alike; from
// there on eight are faster, 17.7 us against 28.5 for 128 pairs of 65536).
template <int U>
__global__ __launch_bounds__(kThreads) void slot_least_kernel(TokenSlots a) {
  __shared__ uint64_t part[kWaves];
  const int tid = threadIdx.x;
  const int64_t base = (int64_t)blockIdx.x * a.C;
  const int p = a.pos[blockIdx.x / a.G];
  const int recent_from = max(p, 0) - a.keep_recent;
  uint64_t best = ~0ull;
  for (int s0 = tid; s0 < a.C; s0 += U * kThreads) {
    int q[U];
    float w[U];
#pragma unroll
    for (int x = 0; x < U; ++x) {
      const int64_t at = base + min(s0 + x * kThreads, a.C - 1);
      q[x] = a.slot_pos[at];
      w[x] = a.weight[at];
    }
#pragma unroll
    for (int x = 0; x < U; ++x) {  // (the last slot may come twice: the least is the same)
      const int c = slot_class(q[x], recent_from, a.keep_first);
      const int s = min(s0 + x * kThreads, a.C - 1);
      const uint64_t k = (((uint64_t)c << 32 | (c ? weight_key(w[x]) : 0)) << 24) | (uint32_t)s;
      best = k < best ? k : best;
    }
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

namespace {
hipError_t choose(const TokenSlots& a, unsigned blocks, int keys, hipStream_t s) {
  const dim3 grid(blocks);
  if (keys <= 4 * kThreads) hipLaunchKernelGGL(slots_kernel<4>, grid, dim3(kThreads), 0, s, a);
  else if (keys <= 16 * kThreads) hipLaunchKernelGGL(slots_kernel<16>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(slots_kernel<0>, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

// Chunks of a first launch, or 0: one launch. For one token that is a plain minimum, 3.5 us a
// chunk of its pair, while chunks cost 15 us a round of 256 workgroups and 10 to join (measured: 8
// pairs of 131072 slots 24 us against 28, of 2^20 42 against 224; 32 of 262144 43 against 59; but 64
// pairs of 131072 43 against 32).
int64_t chunks_of(int64_t pairs, int capacity, int n) {
  const int64_t chunks = ((int64_t)capacity + kChunk - 1) / kChunk;
  if (n == 1) return 3.5 * (double)chunks > 15.0 * (double)((pairs * chunks + 255) / 256) + 10.0 ? chunks : 0;
  return capacity > kChunk && n > 1 && chunks * n <= capacity / 2 ? chunks : 0;
}
}  // namespace

int64_t token_slots_workspace(int batch, int groups, int capacity, int n) {
  const int64_t pairs = (int64_t)batch * groups;
  return pairs * chunks_of(pairs, capacity, n) * n * 4;
}

hipError_t token_slots(TokenSlots a, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.G));
  const int64_t chunks = chunks_of((int64_t)a.B * a.G, a.C, a.n);
  if (chunks > 0) {
    TokenSlots f = a;
    f.chunks = a.chunks = (int)chunks;
    f.slots = (int*)a.ws;
    const hipError_t e = choose(f, (unsigned)(a.B * a.G * chunks), kChunk, s);
    if (e != hipSuccess) return e;
    a.list_in = (const int*)a.ws;
    return choose(a, (unsigned)(a.B * a.G), (int)chunks * a.n, s);
  }
  if (a.n > 1) return choose(a, (unsigned)(a.B * a.G), a.C, s);
  if (a.C <= 4 * kThreads) hipLaunchKernelGGL(slot_least_kernel<1>, grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL(slot_least_kernel<8>, grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace fd
