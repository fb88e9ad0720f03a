// vc_mass.h -- plans and host launchers of the cache that keeps its rows' attention
// weight: attention (single tokens, prompts) and eviction.  Internal.
#pragma once
#include "vc_q8.h"

namespace vc {

constexpr int kMassTile = 32;         // rows of a single token's tile
constexpr int kMassHeld4 = 10112;     // logits that a workgroup of four waves keeps in LDS
constexpr int kMassHeld8 = 30 * 1024; // one of eight
constexpr int kMassChunk = 1024;      // threads of a workgroup of k_finish, of one row or four
constexpr int kMassKeys = 256;        // rows of a workgroup of k_mass_cols
constexpr int kEvictBytes = 32768;    // keys (and as many values) of a workgroup of k_move
constexpr int kMassMaxRows = INT32_MAX - 1024;  // so that the end of a row's tile is a row index

// The cache, as in vc_mass_cache.
struct MassPool {
  uint16_t *kp, *vp;
  float *mass;
  const int64_t *row_off;
  const int32_t *cap;
  int32_t *len;
};

struct MassAttn {
  MassPool c;
  RowsDesc q, out, k, v;  // k, v: the rows to append
  const int32_t *count;   // queries per sequence; null: n
  int32_t L, B, Hq, Hkv, G, d, units;
  int32_t wgs;            // workgroups of the attention launch
  int32_t n, cols;        // queries per sequence; cols = n * G
  int32_t append, fp32, causal;  // causal: always 1
  int32_t max_rows;
  float sc, decay;        // sc = scale * log2(e)
  // Single tokens (cols <= 16): workgroups of `waves` waves take the units in `order`
  // (null: as they are), in pieces of `piece` tiles, at most npmax a unit.  The logits of
  // every column wait for its maximum and sum: of a unit in one piece those of rows below
  // `here` in LDS, all others in [unit][cols][ldr], from row `here` on.
  const int32_t *order;
  int32_t waves, piece, npmax, here, ldr;
  int32_t finish, finish_wgs;  // the second launch, of cut units: rows a thread (1 or 4), workgroups
  float *logits;
  // Prompts (npmax 1): nqt column tiles of qcols columns, each in as many key splits
  // as the launch's workgroups allow (ns 1: whole).
  int32_t qcols, nqt, ns;
  float *part_o;          // partial results: [part][qcols][d], [part][qcols]
  float2 *part_ml;
  // Prompts' masses: `ktiles` tiles of kMassKeys rows a unit, each tile's columns shared by
  // csplit workgroups, and what each of several adds: [unit][tile][csplit][row].
  int32_t ktiles, csplit;
  float *part_mass;
  float2 *stat;           // prompts: [unit][cols] maximum and 1 / sum of the weights
  // Per unit (rows before the call, rows now, queries, pieces): of single tokens in
  // several pieces, and of prompts that append.
  int4 *state;
  int32_t *np;            // prompts: first part and number of parts of each tile
};

struct EvictPlan {
  MassPool c, to;  // to: not read in place
  const int32_t *keep;
  int32_t units, d, inplace, sinks, recent, max_rows;
  int32_t chunks;    // workgroups of a unit's move
  int32_t ldl;       // rows of a unit's list
  int32_t *list;     // [unit][ldl] kept rows, ascending
  int32_t *count;    // [unit] how many
  uint32_t *flags;   // [unit][chunks]: the chunk's rows are read (in place)
  uint32_t *ticket;  // [unit]: chunks handed out (in place)
  int32_t *index;    // the caller's: [unit][index_rows], or null
  int32_t index_rows;
};

// launch_mass_token: attention (and append) in one launch, or two where units are cut.
// launch_mass_prompt: append, attention, join where tiles are cut, and the rows' weights.
hipError_t launch_mass_token(const MassAttn &p, hipStream_t st);
hipError_t launch_mass_prompt(const MassAttn &p, hipStream_t st);
hipError_t launch_mass_cols(const MassAttn &p, hipStream_t st);  // called by launch_mass_prompt
hipError_t launch_mass_evict(const EvictPlan &p, hipStream_t st);

}  // namespace vc
