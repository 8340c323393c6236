// Drafted trees: arguments and launchers of the kernels in tree_kernels.hip (attention, scores) and walk_kernels.hip (the walk
// against the target's probabilities, the kept path).
#pragma once
#include "tkv_internal.h"

namespace tkv {

constexpr int TREE_MAX = 128;        // nodes of a tree: their ancestors fit four words
constexpr int TREE_WORDS = TREE_MAX / 32;

// One layer's attention of a tree, and (q_all, several layers) the scores of the nodes kept.
struct TreeArgs {
  const char* fpK; const char* fpV;   // layer bases, as in AttnArgs
  const char* c2K; const char* c2V; const char* s2K; const char* s2V;
  const void* q; void* out;           // [B][n][Hq][D]
  const int* parents;                 // [B][n]
  const int* f_loc; const int* f_pos; const int* q_loc; const int* q_pos;
  const int* cnt;
  float* part_ml;                     // [B][Hkv][S][2][C]: maximum (of logits times log2 e) and sum of a split, per column
  float* part_o;                      // [B][Hkv][S][C][D]
  float2* stat; int stat_stride;      // [B][Hkv][stat_stride] maximum and 1 / sum of a column: what the scores are made with later
  int* here;                          // [B][n] whether a node is there
  int B, Hq, Hkv, G, n, C;            // C = n * G columns of a kv head, column = node * G + head of the group
  int S, groups;                      // splits of a pair's tiles, groups of columns
  int waves_c, blocks;                // the workgroup's shape (TreeShape)
  int Nmax, capF, cap2, cb, sb, t2fmt, out_kind;
  float scale2;                       // softmax_scale * log2 e
  int nF[ATTN_ARG_SEQS], nQ[ATTN_ARG_SEQS];
};

// The kept queries' weights, layer0 .. layer0 + layers - 1: gain[layer][B][stride] by list index (list F, then list Q).
struct TreeScoreArgs {
  const char* fpK; const char* c2K; const char* s2K;   // layer layer0's bases
  const void* q;                      // [layers][B][n][Hq][D]
  const int* path; int n_path;        // [B][n_path]
  const int* kept;                    // [B] nodes kept
  const int* f_loc; const int* f_pos; const int* q_loc; const int* q_pos;
  const int* cnt;
  const float2* stat; int stat_stride; // [layers][B][Hkv][stat_stride]
  const float* vnorm;                 // [layers][B][Hkv][Nmax], or NULL
  float* gain; float* score;
  int stride, layers;
  int B, Hq, Hkv, G, n, Nmax, capF, cap2, cb, sb, t2fmt;
  float scale2, score_scale;
};

// Shapes of a workgroup: waves side by side over columns and over rows, a wave's blocks of 16 columns; groups of columns that a tree of C
// columns then takes.  The narrowest comes first; false: there are no more.
struct TreeShape { int waves_c, waves_r, blocks, groups; };
bool tree_shape(int kt, int C, int which, TreeShape& s);
hipError_t launch_tree_attend(const TreeArgs& a, int D, int kt, hipStream_t st);
hipError_t launch_tree_scores(const TreeScoreArgs& a, int D, int kt, int max_rows, hipStream_t st);

// The walk (tkv_verify_tree)
constexpr int WALK_MAX_PARTS = 32;
struct WalkArgs {
  const int* parents; const int* tokens;          // [B][n]
  const char* p; const char* q;                   // [B][n] rows of vocab probabilities, q or NULL
  const float* u; const float* u_draw;            // [B][n], [B]
  int* path; int* n_path; int* next;              // [B][n], [B], [B]
  double* part; int* arrived;                     // [B][WALK_MAX_PARTS], [B] (0 between calls)
  long long p_stride, q_stride;                   // elements from row to row
  int B, n, vocab, W;
};
int walk_parts(int B, int vocab, int cus);
hipError_t launch_walk(const WalkArgs& a, int kt, hipStream_t st);
hipError_t launch_walk_init(int* arrived, int B, hipStream_t st);

// The kept path (tkv_accept_tree): counts and checks, then the change.  info: [B][2] nodes kept, rows of the range that hold a slot
// (negative: a bad path).
hipError_t launch_accept_check(const DevView& v, int base, int n, const int* path, int n_path, int* info, hipStream_t st);
hipError_t launch_accept(const DevView& v, int base, int n, int keep, const int* path, int n_path, const int* info, hipStream_t st);

}  // namespace tkv
