// Rotary positions on rows of head vectors, and the append of rotated keys and
// of values to a token cache.
//
// Pair i of a vector turns by the angle coordinate x frequency_i:
//   (x0, x1) -> m (x0 cos - x1 sin, x0 sin + x1 cos).
// The angle is taken in 64 bits as a number of turns less the nearest whole one
// (at position 2^23 an fp32 product would be off by up to half a radian), and only
// then goes to fp32 for the sine and cosine; what that rounding took off the angle is
// turned in afterwards, to first order. All heads of a token share its angles:
// a workgroup computes each (cos, sin) of its tokens once, into LDS, and then
// streams the heads' vectors past them, 16 bytes a thread. Both kernels read every
// element once and write it once, so memory bounds them, and for single tokens the
// launch does. 8160 tokens x 32 heads x 128, bf16, 96 rotated: 34 us (3.9 TB/s with fresh
// memory every time); 3600 tokens x 3 groups appended: 5.8 us; one token: 2.2 us.
#include "fd_token.h"

namespace fd {
namespace {

constexpr int kPairs = 256;  // (cos, sin) of one workgroup

template <typename T> struct Vec16 { T e[16 / sizeof(T)]; };

// One pair turned, with the same roundings in every path.
template <typename T>
__device__ __forceinline__ void turn(T& x0, T& x1, float2 c) {
  const float u = (float)x0, w = (float)x1;
  x0 = (T)fmaf(u, c.x, -(w * c.y));
  x1 = (T)fmaf(u, c.y, w * c.x);
}

// The (cos, sin) of tokens tok0 .. tok0 + nt - 1, one thread a pair.
__device__ __forceinline__ void fill_angles(const RopeArgs& r, int64_t tok0, int nt, float2* cs) {
  for (int i = threadIdx.x; i < nt * r.half; i += 256) {
    const int t = i / r.half, pair = i - t * r.half;
    const int ax = r.axis ? min(max(r.axis[pair], 0), r.axes - 1) : 0;
    const double turns = (double)r.coords[(tok0 + t) * r.axes + ax] * r.freq[pair] * 0.15915494309189533577;
    const double rest = turns - rint(turns);  // -1/2 .. 1/2
    const float part = (float)rest, lost = (float)((rest - part) * 6.28318530717958647693);
    float sn, cn;
    sincospif(2.f * part, &sn, &cn);
    cs[i] = make_float2(fmaf(-sn, lost, cn) * r.mag, fmaf(cn, lost, sn) * r.mag * r.sign);
  }
}

// Work items of one head vector: VEC: 16 bytes (half layout: 16 bytes of each
// half); else single pairs, then single elements of the part that is not rotated.
template <typename T, bool IL, bool VEC>
__host__ __device__ inline int row_items(int dim, int half) {
  constexpr int V = 16 / sizeof(T);
  if (VEC) return IL ? dim / V : (dim - half) / V;
  return dim - half;
}

template <typename T, bool IL, bool VEC>
__device__ __forceinline__ void turn_item(const T* x, T* o, int item, int half, const float2* cs) {
  constexpr int V = 16 / sizeof(T);
  if constexpr (VEC && IL) {
    Vec16<T> a = *reinterpret_cast<const Vec16<T>*>(x + item * V);
    const int p0 = item * (V / 2);
#pragma unroll
    for (int e = 0; e < V / 2; ++e)
      if (p0 + e < half) turn(a.e[2 * e], a.e[2 * e + 1], cs[p0 + e]);
    *reinterpret_cast<Vec16<T>*>(o + item * V) = a;
  } else if constexpr (VEC) {
    const int np = half / V;
    if (item < np) {
      Vec16<T> a = *reinterpret_cast<const Vec16<T>*>(x + item * V);
      Vec16<T> b = *reinterpret_cast<const Vec16<T>*>(x + half + item * V);
#pragma unroll
      for (int e = 0; e < V; ++e) turn(a.e[e], b.e[e], cs[item * V + e]);
      *reinterpret_cast<Vec16<T>*>(o + item * V) = a;
      *reinterpret_cast<Vec16<T>*>(o + half + item * V) = b;
    } else {
      const int d = half + item * V;  // 2 half + (item - np) V
      *reinterpret_cast<uint4*>(o + d) = *reinterpret_cast<const uint4*>(x + d);
    }
  } else {
    if (item < half) {
      const int i0 = IL ? 2 * item : item, i1 = IL ? 2 * item + 1 : item + half;
      T a = x[i0], b = x[i1];
      turn(a, b, cs[item]);
      o[i0] = a;
      o[i1] = b;
    } else {
      o[half + item] = x[half + item];
    }
  }
}

// A thread's walk over [tokens][rows][items] in steps of 256: divided once, then carried.
struct Walk {
  int t, row, item;
  int dt, drow, ditem, rows, items;
  __device__ __forceinline__ Walk(int rows_, int items_) : rows(rows_), items(items_) {
    const int per = rows * items;
    t = threadIdx.x / per;
    const int rem = threadIdx.x - t * per;
    row = rem / items;
    item = rem - row * items;
    dt = 256 / per;
    const int drem = 256 - dt * per;
    drow = drem / items;
    ditem = drem - drow * items;
  }
  __device__ __forceinline__ void next() {
    item += ditem;
    const bool c = item >= items;
    item -= c ? items : 0;
    row += drow + c;
    const bool d = row >= rows;
    row -= d ? rows : 0;
    t += dt + d;
  }
};

// Workgroup: nt tokens x a range of the heads (gridDim.y ranges).
template <typename T, bool IL, bool VEC>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs r, RopeRows x, int nt) {
  __shared__ float2 cs[kPairs];
  const int items = row_items<T, IL, VEC>(x.dim, r.half);
  const int h0 = (int)((int64_t)x.heads * blockIdx.y / gridDim.y);
  const int h1 = (int)((int64_t)x.heads * (blockIdx.y + 1) / gridDim.y);
  for (int64_t t0 = (int64_t)blockIdx.x * nt; t0 < x.tokens; t0 += (int64_t)gridDim.x * nt) {
    const int m = (int)min((int64_t)nt, x.tokens - t0);
    __syncthreads();  // the previous tokens' angles are no longer read
    fill_angles(r, t0, m, cs);
    __syncthreads();
    for (Walk w(h1 - h0, items); w.t < m; w.next())
      turn_item<T, IL, VEC>((const T*)x.x + (t0 + w.t) * x.x_token + (h0 + w.row) * x.x_head,
                            (T*)x.out + (t0 + w.t) * x.o_token + (h0 + w.row) * x.o_head, w.item, r.half,
                            cs + w.t * r.half);
  }
}

// Tokens run over the whole batch (token b n + i). Slots are checked here: they
// come from device memory.
template <typename T, bool IL, bool VEC>
__global__ __launch_bounds__(256) void append_kernel(TokenCacheArgs c, RopeArgs r, TokenAppend a, int nt) {
  __shared__ float2 cs[kPairs];
  constexpr int V = 16 / sizeof(T);
  const int items = row_items<T, IL, VEC>(c.D, r.half), vch = c.D / V;
  const int per_row = items + vch + 1;
  const int64_t tokens = (int64_t)c.B * a.n;
  for (int64_t t0 = (int64_t)blockIdx.x * nt; t0 < tokens; t0 += (int64_t)gridDim.x * nt) {
    const int m = (int)min((int64_t)nt, tokens - t0);
    __syncthreads();
    fill_angles(r, t0, m, cs);
    __syncthreads();
    for (Walk w(c.G, per_row); w.t < m; w.next()) {
      const int t = w.t, g = w.row, item = w.item;
      const int64_t tok = t0 + t;
      const int b = (int)(tok / a.n), j = (int)(tok - (int64_t)b * a.n);
      const int p = a.pos[tok], slot = a.slots[((int64_t)b * c.G + g) * a.n + j];
      if (p < 0 || slot < 0 || slot >= c.C) continue;
      if (item < items) {
        turn_item<T, IL, VEC>((const T*)a.k + b * a.ks[0] + j * a.ks[1] + g * a.ks[2],
                              (T*)c.k + b * c.ks[0] + g * c.ks[1] + slot * c.ks[2], item, r.half, cs + t * r.half);
      } else if (item < items + vch) {
        const int d = (item - items) * V;
        *reinterpret_cast<uint4*>((T*)c.v + b * c.vs[0] + g * c.vs[1] + slot * c.vs[2] + d) =
            *reinterpret_cast<const uint4*>((const T*)a.v + b * a.vs[0] + j * a.vs[1] + g * a.vs[2] + d);
      } else {
        const int64_t at = ((int64_t)b * c.G + g) * c.C + slot;
        c.pos[at] = p;
        c.weight[at] = 0.f;
      }
    }
  }
}

// Tokens of a workgroup: as many as 256 pairs allow, but no more than leaves
// the launch 1024 workgroups.
int tokens_per_group(int64_t tokens, int half) {
  const int64_t most = half ? kPairs / half : 8;
  int64_t nt = (tokens + 1023) / 1024;
  if (nt > most) nt = most;
  return (int)(nt < 1 ? 1 : nt);
}

template <typename T, bool IL, bool VEC>
hipError_t rope_launch(const RopeArgs& r, const RopeRows& x, hipStream_t s) {
  const int nt = tokens_per_group(x.tokens, r.half);
  int64_t gx = (x.tokens + nt - 1) / nt;
  if (gx > 65536) gx = 65536;
  // few tokens: their heads are shared among workgroups of at least one item a thread
  int64_t gy = (int64_t)x.heads * row_items<T, IL, VEC>(x.dim, r.half) / 256;
  const int64_t room = 1024 / gx;
  gy = gy < 1 || room < 1 ? 1 : (gy < room ? gy : room);
  if (gy > x.heads) gy = x.heads;
  hipLaunchKernelGGL((rope_kernel<T, IL, VEC>), dim3((unsigned)gx, (unsigned)gy), dim3(256), 0, s, r, x, nt);
  return hipGetLastError();
}

template <typename T, bool IL, bool VEC>
hipError_t append_launch(const TokenCacheArgs& c, const RopeArgs& r, const TokenAppend& a, hipStream_t s) {
  const int64_t tokens = (int64_t)c.B * a.n;
  const int nt = tokens_per_group(tokens, r.half);
  int64_t gx = (tokens + nt - 1) / nt;
  if (gx > 65536) gx = 65536;
  hipLaunchKernelGGL((append_kernel<T, IL, VEC>), dim3((unsigned)gx), dim3(256), 0, s, c, r, a, nt);
  return hipGetLastError();
}

template <int ES>
bool pairs_by_16(const RopeArgs& r, int dim) {  // whole 16-byte pieces of both halves, and of the rest
  constexpr int V = 16 / ES;
  return dim % V == 0 && (r.interleaved || r.half % V == 0);
}

template <typename T>
hipError_t rope_type(const RopeArgs& r, const RopeRows& x, hipStream_t s) {
  constexpr int V = 16 / sizeof(T);
  const bool aligned = ((uintptr_t)x.x | (uintptr_t)x.out) % 16 == 0 &&
                       (x.x_token | x.x_head | x.o_token | x.o_head) % V == 0;
  const bool vec = aligned && pairs_by_16<sizeof(T)>(r, x.dim);
  if (r.interleaved) return vec ? rope_launch<T, true, true>(r, x, s) : rope_launch<T, true, false>(r, x, s);
  return vec ? rope_launch<T, false, true>(r, x, s) : rope_launch<T, false, false>(r, x, s);
}

template <typename T>
hipError_t append_type(const TokenCacheArgs& c, const RopeArgs& r, const TokenAppend& a, hipStream_t s) {
  // (rows are 16-byte aligned by the host's checks)
  const bool vec = pairs_by_16<sizeof(T)>(r, c.D);
  if (r.interleaved) return append_launch<T, true, true>(c, r, a, s);
  return vec ? append_launch<T, false, true>(c, r, a, s) : append_launch<T, false, false>(c, r, a, s);
}

}  // namespace

hipError_t rope_rows(const RopeArgs& r, const RopeRows& x, int kind, hipStream_t s) {
  if (kind == 0) return rope_type<_Float16>(r, x, s);
  if (kind == 1) return rope_type<__bf16>(r, x, s);
  return rope_type<float>(r, x, s);
}

hipError_t token_append(const TokenCacheArgs& c, const RopeArgs& r, const TokenAppend& a, int kind, hipStream_t s) {
  if (kind == 0) return append_type<_Float16>(c, r, a, s);
  if (kind == 1) return append_type<__bf16>(c, r, a, s);
  return append_type<float>(c, r, a, s);
}

}  // namespace fd
