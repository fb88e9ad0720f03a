// vc_q8.h -- plans and host launchers of the 8-bit cache (append, read back,
// attention) and of the rotary positions.  Internal.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace vc {

constexpr int kQ8Block = 64;  // rows that share a scale (VC_Q8_BLOCK)
constexpr int kQ8SplitTiles = 256;  // most column tiles of a prompt that are cut along their rows
constexpr int kQ8SplitBlocks = 4;   // fewest blocks a cut leaves together

// Row (l, b, i, h) of a strided tensor starts at base + l*layer + b*seq +
// i*token + h*head elements.
struct RowsDesc {
  uint64_t base;
  int64_t layer, seq, token, head;
};

// The cache, as in vc_q8cache.
struct Q8Cache {
  uint8_t *kc, *vc;
  float *ks, *vs;
  uint16_t *kt, *vt;
  const int64_t *row_off;
  const int32_t *cap;
  int32_t *len;
  const int32_t *order;  // may be null
};

struct Q8Rows {  // append (k, v read) and read back (k, v written)
  Q8Cache c;
  RowsDesc k, v;
  const int64_t *unit_off;  // element offset of each unit's first row; null: the strides
  const int32_t *count;     // append: rows per (layer, sequence); null: n
  int32_t B, Hkv, d, units;
  int32_t n;    // append: rows per unit; read: row bound
  int32_t nj;   // workgroups per unit
  int32_t fp32; // read: element type
};

constexpr int kRopeMaxHalf = 64;
struct RopeTable {
  int32_t rot, adjacent;   // rotated channels (0: no rotation); pairs (2i, 2i+1) or (i, i + rot/2)
  uint64_t axis1, axis2;   // bit i: frequency i turns with the height / the width
  float scale, sgn;
  double turns[kRopeMaxHalf];  // frequency i over 2 pi
};

struct Q8Attn {
  Q8Cache c;
  RowsDesc q, out;
  const int32_t *count;  // queries per sequence; null: n
  int32_t L, B, Hq, Hkv, G, d, units;
  int32_t wgs;           // workgroups of the attention launch
  int32_t n, cols;       // queries per sequence; cols = n * G
  int32_t causal, fp32;
  int32_t max_rows;
  float sc;              // scale * log2(e)
  // One token at a time (cols <= 16): pieces of `piece` blocks, at most npmax
  // a unit (qcols 16).  Prompts (npmax 1): nqt column tiles of qcols columns,
  // each in as many key splits as the launch's workgroups allow (ns 1: whole).
  int32_t piece, npmax;
  int32_t qcols, nqt, ns;
  float *part_o;         // partial results: [part][qcols][d], [part][qcols]
  float2 *part_ml;
  // A step (step = 1; else attention alone): the new rows, the rotation of queries and
  // new keys.
  int32_t step;
  RowsDesc k, v;
  RopeTable rope;
  const int32_t *pos;    // [3][B]
  // For the join: a step's pieces of each unit, whose lengths it then advances
  // (bit 30: by a row); a prompt's first part and number of parts of each tile.
  int32_t *np;
};

struct RopePlan {
  RowsDesc qi, qo, ki, ko;
  const int32_t *pos;    // [3][B][n]
  const int32_t *count;  // tokens per sequence; null: n
  int32_t B, L, Hq, Hkv, d, n;  // Hq (Hkv) is 0 where there are no queries (keys)
  int32_t fp32;
  RopeTable t;
};

hipError_t launch_q8_append(const Q8Rows &p, int format, hipStream_t st);
hipError_t launch_q8_read(const Q8Rows &p, int format, hipStream_t st);
hipError_t launch_q8_decode(const Q8Attn &p, int format, hipStream_t st);
hipError_t launch_q8_prompt(const Q8Attn &p, int format, hipStream_t st);
hipError_t launch_q8_join(const Q8Attn &p, hipStream_t st);  // called by the two above
hipError_t launch_rope(const RopePlan &p, hipStream_t st);

}  // namespace vc
