// shared_prefix_layout.h -- what lies where in the shared memory of
// shared_prefix_split_kernel, and how many ring slots that leaves room for.  Plain
// integer code, so that it also compiles for the host, where it is checked.
#pragma once

#include <stdint.h>

#ifdef __CUDACC__
#define SF_HOST_DEVICE __host__ __device__
#else
#define SF_HOST_DEVICE
#endif

namespace sf {

constexpr int kSpTile = 128;  // keys per tile, query rows per row tile
constexpr int kSpItems = 2;   // pieces published ahead (four took the plan's room)
constexpr int kSpInfo = 5;    // words that a softmax warp keeps about its piece
constexpr int kSpSmemMax = 227 * 1024;

// A piece, as its CTA's warps read it from shared memory.
struct SpItem {
  int n, t0, keys;  // key tiles t0 .. t0 + n - 1 of the segment's keys; n = 0: no more pieces
  int own, row, h;  // row of block_table (own) or prefix_table
  int dual, again;  // both streams read every tile; the keys are read again by other pieces
  int duo;          // key tiles t of head h + t % 2, a stream a head
  int pad;
  struct {
    int two;               // the first key tile's weights go to P V as two bf16 terms
    int n, first, step;    // the stream's key tiles within the piece (n = 0: none)
    int token, rows;       // first query token and rows of its row tile
    uint32_t slot;         // first row of its partial
  } s[2];
};

template <int D, int STAGES>
struct SpSmem {
  static constexpr int kTileBytes = kSpTile * D * 2;  // a K, V or Q tile
  static constexpr int kQOffset = STAGES * kTileBytes;
  static constexpr int kBarOffset = kQOffset + 2 * kTileBytes;
  // full[S], empty[S], then per stream q_full, q_empty, s_full, p_full[2], o_done, fin, turn;
  // item_full, item_empty per published piece; joint, read per stream
  static constexpr int kNumBars = 2 * STAGES + 16 + 2 * kSpItems + 4;
  static constexpr int kMiscOffset = kBarOffset + 8 * kNumBars;  // TMEM base, abort word
  static constexpr int kItemOffset = kMiscOffset + 16;
  static constexpr int kMlOffset = kItemOffset + kSpItems * static_cast<int>(sizeof(SpItem));  // float2 [2][128]
  static constexpr int kInfoOffset = kMlOffset + 2 * 8 * kSpTile;  // int [8 warps][kSpInfo], int [2][2]
  static constexpr int kPlanOffset = kInfoOffset + 8 * 4 * kSpInfo + 16;
};

// Bytes of shared memory behind that: lengths of all entities, the groups' first
// sequences, costs and partial rows.
SF_HOST_DEVICE constexpr int sp_plan_bytes(int B, int num_groups) { return 4 * (B + 4 * num_groups + 1); }

template <int D, int STAGES>
constexpr int sp_smem_bytes(int B, int num_groups) {
  return SpSmem<D, STAGES>::kPlanOffset + sp_plan_bytes(B, num_groups);
}

// The deepest ring that leaves room for the plan of B sequences.  With 128-wide heads
// five slots leave 368 bytes (87 sequences of one group, 59 of eight), and four suffice
// for two key tiles: 59 sequences of 212 to 916 own tokens, 32 heads, a prefix of 140
// take 115 us with five and 120 with four, a prefix of 8 131 and 140, 64 sequences over
// 32768 tokens 186 and 188, but 8 sequences of 5 rows over 3008 tokens 24.6 and 24.3.
constexpr int sp_stages(int D, int B, int num_groups) {
  return D == 128 ? (sp_smem_bytes<128, 5>(B, num_groups) <= kSpSmemMax ? 5 : 4)
                  : (sp_smem_bytes<64, 10>(B, num_groups) <= kSpSmemMax ? 10 : 8);
}

}  // namespace sf
