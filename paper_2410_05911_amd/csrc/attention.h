// Cross attention and its gradient: what attention_host.cpp hands to the kernels.
#pragma once

#include <cstddef>
#include <cstdint>

#include <hip/hip_runtime.h>

namespace aecct {

// [batch][length][heads][d], strides in values (d's is 1), none negative.
struct Heads {
  const void *p;
  int64_t batch, row, head;
  bool packed = false;         // zeros behind each row's d values, up to a whole 16-byte piece
};
// The queries of the heads that share a key head are the rows of one problem: row r is query r % queries of head
// key head * (heads / kv_heads) + r / queries.  A pair is a sequence and a key head.
struct Attention {
  int64_t batch, queries, keys;
  int heads, kv_heads, d;
  float scale;
  Heads q, k, v, o;            // o: out; in the gradient an input
  const int32_t *lengths;      // [batch], or null
  const uint8_t *mask;         // [queries][ldmask], or null
  int64_t ldmask;
  uint32_t *words;             // the mask packed, 32 keys a word: [queries][words_of(keys)]
  uint8_t *flags;              // whether any of 32 queries may attend any of 64 keys: [tiles of queries][tiles of keys]
  float *lse;                  // [batch][heads][queries]; in the gradient an input
  int splits;
  float *part_o, *part_ml;     // [splits][pairs][rows][d_of(d)], [splits][pairs][rows][2]
};
// Copies of up to four tensors [batch][length][heads][d] as [batch][length][heads][line], zeros behind d.  What lies past a sequence's
// length is not read (lengths: or null).
struct PackHeads {
  Heads from;
  int64_t batch, length;       // length 0: not asked for
  int heads, d, line;
  const int32_t *lengths;
  void *to;
};
struct PackHeadsAll {
  PackHeads t[4];
};
hipError_t launch_pack_heads(int type, const PackHeadsAll &p, hipStream_t s);
// Whether the tiles of such a tensor go past the registers as it is (its address apart).
inline bool ragged_heads(int size, int64_t batch, int64_t row, int64_t head, int d) {
  const int64_t e = 16 / size;
  return d % e != 0 || batch % e != 0 || row % e != 0 || head % e != 0;
}

struct AttentionPlan {
  bool few;                    // 32 rows a block, its wavefronts share the keys; else 128 rows
  int splits;
  size_t words, flags, part_o, part_ml;   // bytes
};
__host__ __device__ inline int64_t words_of(int64_t keys) { return (keys + 63) / 64 * 2; }
__host__ __device__ inline int d_of(int d) { return d <= 32 ? 32 : d <= 64 ? 64 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }
AttentionPlan plan_attention(int type, int64_t batch, int64_t queries, int64_t keys, int heads, int kv_heads, int d, bool masked);
hipError_t launch_mask(const Attention &a, hipStream_t s);
hipError_t launch_attention(int type, const Attention &a, const AttentionPlan &p, hipStream_t s);

struct AttentionGrad {
  Attention a;
  Heads dout, dq, dk, dv;      // dq, dk, dv: out
  float *rows;                 // [pairs][rows][2]: lse (16-bit types: times log2(e)), and the sum of dout o
  int splits;                  // of the rows, for dk and dv
  float *part;                 // [splits][2][pairs][keys][d_of(d)], or null
  int splits_q;                // of the keys, for dq
  float *part_q;               // [splits_q][pairs][rows][d_of(d)], or null
};
struct AttentionGradPlan {
  int splits, splits_q;
  size_t words, flags, rows, part, part_q;   // bytes
};
AttentionGradPlan plan_attention_grad(int type, int64_t batch, int64_t queries, int64_t keys, int heads, int kv_heads, int d,
                                      bool masked);
hipError_t launch_attention_grad(int type, const AttentionGrad &a, hipStream_t s);

}  // namespace aecct
