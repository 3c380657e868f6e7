// Internal interface between the host checks of the token cache and of rotary
// positions (fd_token.cpp) and their gfx950 kernels. Every launcher enqueues on
// `stream` and returns the hipError_t of the launch; shapes are checked before.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fd {

// Rotation of the first 2 half elements of a head vector.
struct RopeArgs {
  const double* freq = nullptr;   // [half] angular frequency of each pair
  const int* axis = nullptr;      // [half] coordinate that turns the pair, or null (all 0)
  const int* coords = nullptr;    // [tokens][axes]
  int axes = 1, half = 0;
  int interleaved = 1;            // pairs (2 i, 2 i + 1); else (i, i + half)
  float mag = 1.f;                // cos and sin are multiplied by this
  float sign = 1.f;               // -1: the inverse rotation
};

struct RopeRows {
  const void* x = nullptr;
  void* out = nullptr;
  int64_t tokens = 0;
  int heads = 1, dim = 64;
  int64_t x_token = 0, x_head = 0, o_token = 0, o_head = 0;  // strides in elements
};

// kind: 0 f16, 1 bf16, 2 fp32
hipError_t rope_rows(const RopeArgs& r, const RopeRows& x, int kind, hipStream_t stream);

// A token cache's memory (strides in elements: batch, group, slot).
struct TokenCacheArgs {
  void* k = nullptr;
  void* v = nullptr;
  int* pos = nullptr;        // [B][G][C], < 0: empty
  float* weight = nullptr;   // [B][G][C]
  int64_t ks[3] = {}, vs[3] = {};
  int B = 1, G = 1, C = 1, D = 64;
};

struct TokenAppend {
  const void* k = nullptr;   // [B][n][G][D] by strides (batch, token, group)
  const void* v = nullptr;
  int64_t ks[3] = {}, vs[3] = {};
  int n = 0;
  const int* pos = nullptr;    // [B][n]
  const int* slots = nullptr;  // [B][G][n]
};
// Rotated keys (r.half 0: as they are) and values into their slots.
hipError_t token_append(const TokenCacheArgs& c, const RopeArgs& r, const TokenAppend& a, int kind,
                        hipStream_t stream);

struct TokenSlots {
  const int* slot_pos = nullptr;   // [B][G][C]
  const float* weight = nullptr;   // [B][G][C]
  const int* pos = nullptr;        // [B][n]
  int* slots = nullptr;            // [B][G][n]
  int B = 1, G = 1, C = 1, n = 1;
  int keep_first = 0, keep_recent = 0;
  void* ws = nullptr;              // token_slots_workspace bytes
  // of the two launches of a large choice (set by the launcher)
  int chunks = 0;                  // chunks of slots
  const int* list_in = nullptr;    // [B G][chunks][n] what they chose (second launch)
};
constexpr int kMaxSlotTokens = 65536;  // new tokens of one choice
int64_t token_slots_workspace(int batch, int groups, int capacity, int n);
hipError_t token_slots(TokenSlots a, hipStream_t stream);

// Attention over a token cache. Row r = i rep + h of a (request, group) is query
// token i of the group's head h (R = n rep rows), so that a tile of rows covers
// neighbouring tokens of every head that shares the keys.
struct TokenAttend {
  const void* q = nullptr;     // [B][n][N][D] by strides (batch, token, head)
  void* out = nullptr;
  int64_t qs[3] = {}, os[3] = {};
  const int* pos = nullptr;    // [B][n], < 0: padding
  int n = 0, rep = 1;
  uint32_t rep_inv = 0;        // ceil(2^32 / rep), set by the launcher
  float scale = 1.f;
  int causal = 1;
  float* lse = nullptr;        // [B][N][n] or null
  float* weight_out = nullptr; // [B][G][C] or null
  float decay = 1.f;
  void* ws = nullptr;          // token_attend_plan().bytes
};

// How a call is laid out, from its sizes alone.
struct TokenAttendPlan {
  int by_keys = 0;      // few rows: waves share a row tile and part the keys
  int row_tiles = 1;    // tiles of 32 rows (by_keys) or 128
  int splits = 1;       // parts of the slots
  int scan = 1;         // slots that a workgroup sorts at a time (not by_keys)
  int fold = 0;         // such ranges between folds of its sums (0: none, not by_keys)
  int weight_parts = 1; // parts of the rows in the pass over the weights
  int row_waves = 1;    // waves that share keys in that pass
  int join = 1;         // groups of threads that share a row's parts when they are joined
  // offsets into the workspace, in floats
  int64_t part_o = 0, part_ml = 0, lse2 = 0, scores = 0, weights = 0;
  int64_t bytes = 0;
};
TokenAttendPlan token_attend_plan(const TokenCacheArgs& c, int n, int rep, int kind, bool weights);
// pl: token_attend_plan of the call's sizes (unused where a.n is 0).
hipError_t token_attend(const TokenCacheArgs& c, const TokenAttend& a, const TokenAttendPlan& pl, int kind,
                        hipStream_t stream);

}  // namespace fd
