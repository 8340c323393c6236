// Attention of a drafted tree over the tiered KV cache, and the scores of the nodes that are kept.
//
//   k_tree_attend : node i of a tree of n sees the live context and, of the tree's own rows (the last n entries of list F), its
//                 ancestors and itself.  The n * G columns (node, head of the group) of a kv head go side by side over the lanes;
//                 a workgroup of WC x WR waves walks a run of the pair's tiles of 32 * WR rows, and every tile, brought once into
//                 the LDS, serves the workgroup's columns.  S^T = K q^T and O^T = V^T P^T on the matrix cores.
//   k_tree_merge : joins a pair's splits, where it has more than one, into the output and the columns' statistics.
//   k_tree_scores : the kept queries' weights once more, from K, q and those statistics, summed over heads: one float per layer
//                 and position, which k_tree_gain adds up over the layers into the scores.
// Tiles, splits and orders of addition depend on the lists' lengths and logical order alone, never on the slot a row lies in.
#include <algorithm>
#include <utility>

#include "device_common.h"
#include "tree.h"

namespace tkv {

typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

enum RowMode : int { R_FULL = 0, R_INT8 = 1, R_INT4 = 2 };

template <int KT>
__device__ __forceinline__ f32x16 mfma_32x32x16(const u32x4& x, const u32x4& y, f32x16 c) {
  if constexpr (KT == KT_BF16)
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
__device__ __forceinline__ float max_swap32(float x) {         // maximum over lanes l and l + 32, in both
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// Two weights as a sum of NT 16-bit terms, each the nearest to what the terms before it left (16-bit outputs: one).  Binary32 outputs: three bfloat16
// terms hold a weight whole (two leave up to 2^-18 of it: outputs 1.7e-6 from 64 bits, where binary32 arithmetic is 6e-7), two
// binary16 terms to 2^-23.
template <int KT, int NT>
__device__ __forceinline__ void weight_terms(float p0, float p1, uint32_t (&t)[NT]) {
  // (Opaque: a caller's multiplication would be taken into one use of a rounded value and not into the other, and the rest would be that of
  // a neighbour.)
  if constexpr (NT > 1) asm("" : "+v"(p0), "+v"(p1));
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const f32x2 p = {p0, p1};
    if constexpr (KT == KT_BF16) {
      const bf16x2 h = __builtin_convertvector(p, bf16x2);
      t[i] = __builtin_bit_cast(uint32_t, h);
      if (i + 1 < NT) {
        uint32_t first = 0xbf80u, second = 0xbf800000u;    // (-1, 0) and (0, -1); in registers: as an instruction's own constant the first is another number
        asm("" : "+s"(first), "+s"(second));
        p0 = __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, first), p0, false);       // p0 - h.x
        p1 = __builtin_amdgcn_fdot2_f32_bf16(h, __builtin_bit_cast(bf16x2, second), p1, false);
      }
    } else {
      const f16x2 h = __builtin_convertvector(p, f16x2);
      t[i] = __builtin_bit_cast(uint32_t, h);
      if (i + 1 < NT) { p0 = fmaf((float)h.x, -1.f, p0); p1 = fmaf((float)h.y, -1.f, p1); }
    }
  }
}

// ---- rows in the LDS, where they come through registers --------------------------------------------------------------------
// Bytes from row to row.  K rows are read by 32 lanes with a row each, the same 16 bytes of all: a piece more than the row, and any 16
// consecutive rows are on 16 different bank groups.  Binary32 V rows are read along the row, the wave's halves four rows apart: 32 bytes
// more.  A lane's addresses then differ by immediates.
template <int D, int ES = 4>
struct Pitch { static constexpr int K = D * ES + 16, V = D * ES + 32; };

// What a thread brings in of a tile: 16 bytes of a row as the LDS holds it, from as many bytes of the stored row.
template <int MODE, int KT>
struct Piece { using type = u32x4; };
template <int KT> struct Piece<R_INT8, KT> { using type = u32x2; };
template <int KT> struct Piece<R_INT4, KT> { using type = uint32_t; };
template <> struct Piece<R_INT8, KT_F32> { using type = uint32_t; };
template <> struct Piece<R_INT4, KT_F32> { using type = uint16_t; };

// ... and as the LDS holds it.  Codes become 16-bit values (scales stay outside the products), or binary32 ones times their scale.
template <int KT> __device__ __forceinline__ u32x4 row_piece(const u32x4& x, float) { return x; }
template <int KT> __device__ __forceinline__ u32x4 row_piece(const u32x2& x, float) {
  u32x4 y; uint32_t a, b;
  widen_int8<KT>(x.x, a, b); y.x = a; y.y = b;
  widen_int8<KT>(x.y, a, b); y.z = a; y.w = b;
  return y;
}
template <int KT> __device__ __forceinline__ u32x4 row_piece(const uint32_t& x, float sc) {
  if constexpr (KT == KT_F32) {
    const f32x4 y = {sbyte_f(x, 0) * sc, sbyte_f(x, 1) * sc, sbyte_f(x, 2) * sc, sbyte_f(x, 3) * sc};
    return __builtin_bit_cast(u32x4, y);
  } else return widen_int4<KT>(x);
}
template <int KT> __device__ __forceinline__ u32x4 row_piece(const uint16_t& x, float sc) {
  const f32x4 y = {snib_f(x, 0) * sc, snib_f(x, 1) * sc, snib_f(x, 2) * sc, snib_f(x, 3) * sc};
  return __builtin_bit_cast(u32x4, y);
}

// A list's rows of one (layer, sequence, kv head)
struct RowSrc { const char* k; const char* v; const char* sk; const char* sv; const int* list; int n, cap, code_bytes, scale_bytes; };

#if TKV_TREE_PART < 6
// ---- attention: what the two kernels share ---------------------------------------------------------------------------------
// A workgroup's share: a group of columns of one (sequence, kv head) pair, and a run of the pair's tiles (list F's, then list Q's).
struct Run {
  int grp, u, pair, b, kvh, nF, nQ, tF, t0, t1, tail0;      // u = pair * S + split; tail0: the tree's first entry of list F
  bool tail;                                               // the run has tree rows
};
template <int TR, int QW>                                  // QW: time of a tile of list Q, in quarters of one of list F
__device__ __forceinline__ bool run_of(const TreeArgs& a, Run& r) {
  // Groups of columns of one run of tiles are eight workgroups apart: on one XCD, whose L2 then serves all but the first of them.
  // (Divisions are made on the vector ALUs; their results are the same in every lane, and the row descriptors have to be known to be.)
  const auto same = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  const int id = blockIdx.x;
  r.grp = same((id >> 3) % a.groups); r.u = same((id >> 3) / a.groups) * 8 + (id & 7);
  if (r.u >= a.B * a.Hkv * a.S) return false;
  r.pair = same(r.u / a.S); r.b = same(r.pair / a.Hkv); r.kvh = r.pair - r.b * a.Hkv;
  const int sp = r.u - r.pair * a.S;
  if (a.B <= ATTN_ARG_SEQS) { r.nF = a.nF[r.b]; r.nQ = a.nQ[r.b]; }
  else { r.nF = a.cnt[r.b * CNT_N + C_NF]; r.nQ = a.cnt[r.b * CNT_N + C_NQ]; }
  r.tF = (r.nF + TR - 1) / TR;
  const int tQ = (r.nQ + TR - 1) / TR;
  const long long work = 4ll * r.tF + (long long)QW * tQ;
  const auto tile_at = [&](int s) {
    const int w = (int)(work * s / a.S);
    return s == a.S ? r.tF + tQ : w <= 4 * r.tF ? w / 4 : r.tF + (w - 4 * r.tF) / QW;
  };
  r.t0 = same(tile_at(sp)); r.t1 = same(tile_at(sp + 1));
  r.tail0 = r.nF - a.n;
  r.tail = r.t0 < r.tF && r.t1 * TR > r.tail0;
  return true;
}

// Who sees whom: a node's set is its own bit and its parent's set; in log2(n) rounds every node takes over the set of the node it
// points at and points where that one pointed.  A node whose chain meets a bad parent is not there: its set is empty.  sm_up: scratch.
using Sees = uint32_t[TREE_WORDS];
__device__ __forceinline__ void who_sees(const TreeArgs& a, const Run& r, Sees* sm_sees, int* sm_up) {
  const int t = threadIdx.x, p = t < a.n ? a.parents[r.b * a.n + t] : -1;
  bool off = t < a.n && (p < -1 || p >= t);
  int up = off ? -1 : p;
  Sees sees;
#pragma unroll
  for (int w = 0; w < TREE_WORDS; ++w) sees[w] = t < a.n && (t >> 5) == w ? 1u << (t & 31) : 0u;
  const auto put = [&] {
    if (t < TREE_MAX) {
#pragma unroll
      for (int w = 0; w < TREE_WORDS; ++w) sm_sees[t][w] = off ? 0u : sees[w];
      sm_up[t] = off ? -2 : up;
    }
  };
  put();
  __syncthreads();
  for (int d = 1; d < a.n; d *= 2) {
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < TREE_WORDS; ++w) sees[w] |= sm_sees[up][w];
      up = sm_up[up];
      off = off || up == -2;
    }
    __syncthreads();
    put();
    __syncthreads();
  }
  if (r.t1 >= r.tF && r.grp == 0 && r.kvh == 0 && t < a.n) a.here[r.b * a.n + t] = !off;
}
__device__ __forceinline__ bool is_there(const Sees* sm_sees, int i) { return (sm_sees[i][i >> 5] >> (i & 31)) & 1; }

// Rows e0 .. e0 + 31 of a list of n, of which those from tail0 on are the tree's (list Q: tail0 beyond the end): the ones `node` sees
__device__ __forceinline__ uint32_t seen_rows(const Sees* sm_sees, int node, int e0, int n, int tail0) {
  uint32_t vis = e0 + 32 <= n ? ~0u : e0 < n ? (1u << (n - e0)) - 1 : 0u;
  if (e0 + 32 > tail0) {
    const int nb = e0 - tail0, w = nb >> 5, sh = nb & 31;               // node of the first row (-31 .. n)
    const uint32_t lo = w < 0 ? ~0u : w < TREE_WORDS ? sm_sees[node][w] : 0u, hi = w + 1 < TREE_WORDS ? sm_sees[node][w + 1] : 0u;
    vis &= sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
  }
  return vis;
}

// A 32 x 32 result has column `lane & 31`, and in register r row 8 * (r / 4) + 4 * h + r % 4 (h = lane / 32).
// The column's maximum m (of logits times scale2: in units of log 2) after N tiles of logits.  It is followed up only where they exceed it
// 2^LAG times: l and the outputs need a product each then, for all lanes.
template <int N, int NDB, int LAG>
__device__ __forceinline__ void follow_maximum(const f32x16 (&s)[N], float scale2, float& m, float& l, f32x16 (&o)[NDB]) {
  float tm = s[0][0];
#pragma unroll
  for (int r = 1; r < 16 * N; ++r) tm = fmaxf(tm, s[r / 16][r % 16]);
  const float mn = fmaxf(m, max_swap32(tm) * scale2);
  if (__builtin_amdgcn_ballot_w64(mn > m + (float)LAG)) {
    const float al = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
    l *= al;
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] *= al;
    m = mn;
  }
}
// logits to weights 2^(s * scale2 + sub), which l takes the sum of
__device__ __forceinline__ void tile_weights(const f32x16& s, float scale2, float sub, float& l, float (&p)[16]) {
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], scale2, sub));
    sum[r & 3] += p[r];
  }
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// The row waves' shares joined (by way of the LDS, the upper half of the waves to the lower one each time), and the result written: the
// output and the column's statistics, or a split's share for k_tree_merge.
template <int D, int WC, int WR>
__device__ __forceinline__ void finish_columns(const TreeArgs& a, const Run& r, const Sees* sm_sees, char* sm_a, char* sm_b, int wc, int wr, int lane, int col, int node, bool live,
                                               f32x16 (&o)[D / 32], float m, float l) {
  constexpr int NDB = D / 32, SHARE = NDB * 16 + 2;        // floats of a lane
  const int h = lane >> 5;
  if constexpr (WR > 1) {
    for (int half = WR / 2; half >= 1; half /= 2) {
      float* so = (float*)((wr & (half - 1)) * WC + wc ? sm_b : sm_a) + lane;      // (two shares at a time)
      __syncthreads();
      if (wr >= half && wr < 2 * half) {
#pragma unroll
        for (int i = 0; i < NDB * 16; ++i) so[i * 64] = o[i / 16][i % 16];
        so[(SHARE - 2) * 64] = m; so[(SHARE - 1) * 64] = l;
      }
      __syncthreads();
      if (wr < half) {
        const float m1 = so[(SHARE - 2) * 64], mx = fmaxf(m, m1), mu = mx == -INFINITY ? 0.f : mx;
        const float f0 = __builtin_amdgcn_exp2f(m - mu), f1 = __builtin_amdgcn_exp2f(m1 - mu);
        l = fmaf(l, f0, so[(SHARE - 1) * 64] * f1);
#pragma unroll
        for (int i = 0; i < NDB * 16; ++i) o[i / 16][i % 16] = fmaf(o[i / 16][i % 16], f0, so[i * 64] * f1);
        m = mx;
      }
    }
  }
  if (!live || wr > 0) return;
  if (a.S > 1) {
    float* po = a.part_o + ((size_t)r.u * a.C + col) * D + 4 * h;
#pragma unroll
    for (int i = 0; i < NDB * 4; ++i) *(f32x4*)(po + 8 * i) = f32x4{o[i / 4][4 * (i % 4)], o[i / 4][4 * (i % 4) + 1], o[i / 4][4 * (i % 4) + 2], o[i / 4][4 * (i % 4) + 3]};
    if (h == 0) { a.part_ml[(size_t)r.u * 2 * a.C + col] = m; a.part_ml[((size_t)r.u * 2 + 1) * a.C + col] = l; }
    return;
  }
  const float il = is_there(sm_sees, node) && l > 0.f ? 1.0f / l : 0.f;
  const size_t at = (((size_t)r.b * a.n + node) * a.Hq + r.kvh * a.G + (col - node * a.G)) * D + 4 * h;
  // register k of o[i] is element 32 i + 8 (k / 4) + 4 h + k % 4; the caller's tensor may begin anywhere
  const auto each = [&](auto store) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
      for (int k = 0; k < 16; ++k) store(at + 32 * i + 8 * (k / 4) + k % 4, il > 0.f ? o[i][k] * il : 0.f);
  };
  if (a.out_kind == KT_F32) each([&](size_t e, float y) { ((float*)a.out)[e] = y; });
  else if (a.out_kind == KT_BF16) each([&](size_t e, float y) { ((uint16_t*)a.out)[e] = f32_to_bf16(y); });
  else each([&](size_t e, float y) { ((_Float16*)a.out)[e] = (_Float16)y; });
  if (h == 0) a.stat[(size_t)r.pair * a.stat_stride + col] = float2{m, il};
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t row_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), 0, (int)bytes, 0x00020000);
}
typedef __attribute__((address_space(3))) void lds_void;
// 16 bytes a lane from base + off to the 1 KB at `to`, in lane order; zeros from beyond the end
__device__ __forceinline__ void to_lds(const __amdgpu_buffer_rsrc_t& rs, char* to, uint32_t off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void*)to, 16, off, 0, 0, 0);
}
// At most N requests of this wave still under way, its LDS accesses done; with BAR for all waves of the workgroup.  (A wait that the
// compiler knows: it counts requests on from there.)
template <int N, bool BAR>
__device__ __forceinline__ void wait_rows() {
  asm volatile("" : : : "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0070);
  if constexpr (BAR) asm volatile("s_barrier" : : : "memory");
  else asm volatile("" : : : "memory");
}
template <bool BAR>
__device__ __forceinline__ void lds_barrier() {
  if constexpr (BAR) asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
  else asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");
}

// ---- attention, 16-bit rows ----------------------------------------------------------------------------------------------
// A wave has NB blocks of 16 columns.  S^T = K q^T and O^T = V^T P^T in 16x16x32 products: a lane owns one column of every block (lane & 15;
// its rows are 16 rb + 4 kb + r, kb = lane / 16), so that maximum, sum and their corrections need no exchange but between the wave's four
// quarters (and the maximum only where a lane's own logits pass it 2^LAG times), and the weights leave the first product as the second
// one's operand.  With 32x32x16 products, whose columns come in 32s, five blocks of 32 for 160 columns left one SIMD the load of two.
// Rows of list F go straight to the LDS (1 KB an instruction: 4 rows of 256 bytes, 8 of 128), two stages in turn: the next tile's are
// under way while one is computed on.  The LDS order is lane order, so a row's 16-byte pieces are rotated by fetching them so: K rows are
// read by 16 lanes with a row each, the same piece of all; V rows transposed, four rows x 32 bytes at a time; with a piece's width (V: two)
// between blocks of 1 KB neither meets a bank twice.  Every stage is an array of its own and the loop is unrolled over them: reads of one do
// not wait for what is on its way to the other.
// Rows of list Q come through registers, a tile or two ahead, and are widened into the stages.  Their codes are exact in 16 bits, and scales
// stay outside the products: K's on the logits, V's on the weights, which then go to the matrix cores in binary16 whatever the rows' type
// (two terms hold a weight to 2^-23, where bfloat16 takes three).
// Eight waves a workgroup (two a SIMD) and one workgroup a CU.  What bounds it depends: 32 sequences x 16384 in int4, 895 MB, 205 us: the
// memory (4.4 TB/s; a large copy reads and writes 4.8).  4 x 8201 in binary16, 42 us: the rows at 3 TB/s, beginning, end and the splits'
// join being 12 of them.  8 x 4133 with 160 columns, 67 us: the matrix cores have 51 GFLOP with three terms a weight, 0.8 PFLOP/s over the
// launch's 63 us (a large product here: 1.2), and of that time neither leaving out the weights (-16 us), two of three terms (-12) nor the
// fetches (-8) would free much.  One user's 1422 rows, 15 us a layer: one tile a workgroup, beginning and end.
// Not kept: the waves of a SIMD in opposite phases (two barriers a tile: 79 us for the 160 columns against 78; one: 83), blocks of columns dealt
// out 3 / 2 over the waves (126: two bodies of code).
template <int D>
struct Block {
  static constexpr int RB = 2 * D, ROWS = 1024 / RB, KPITCH = 1040, VPITCH = 1056, N = 32 / ROWS;      // rows of a block; blocks of 32 rows
  // piece p of row x of a block: K's pieces 4 ks + kb lie with kb on top, so that lanes of different kb are in different quarters of a row
  static __device__ __forceinline__ int k_place(int x, int p) { return D == 128 ? ((p & 3) << 2 | p >> 2) ^ (x << 2) : ((p & 3) << 1 | p >> 2) ^ (x & 6); }
  static __device__ __forceinline__ int k_piece(int x, int at) {          // and the piece that lies there
    const int y = at ^ (D == 128 ? x << 2 : x & 6);
    return D == 128 ? (y & 3) << 2 | y >> 2 : (y & 1) << 2 | y >> 1;
  }
  static __device__ __forceinline__ int v_place(int x, int p) { return D == 128 ? p ^ (x << 2) : p ^ ((x & 2) << 1) ^ ((x & 4) >> 1); }
};
template <int KT>
__device__ __forceinline__ f32x4 mfma_16x16x32(const u32x4& x, const u32x4& y, f32x4 c) {
  if constexpr (KT == KT_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, x), __builtin_bit_cast(f16x8, y), c, 0, 0, 0);
}
__device__ __forceinline__ float max_swap16(float x) {         // maximum over lanes l and l ^ 16, in both
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}
__device__ __forceinline__ float add_swap16(float x) {         // the sum likewise
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (uint32_t)r[0]) + __builtin_bit_cast(float, (uint32_t)r[1]);
}
constexpr f32x4 ZERO4 = {0.f, 0.f, 0.f, 0.f};
__device__ __forceinline__ int exponent_of(float x) {          // |x| < 2^exponent_of(x); the same for all lanes, from the first's
  const int e = (int)((__builtin_bit_cast(uint32_t, x) >> 23) & 255u) - 126;
  return __builtin_amdgcn_readfirstlane(e < -100 ? -100 : e);
}

template <int D, int KT, int WC, int WR, int NB, int NT, int QM>
__global__ __launch_bounds__(64 * WC * WR, WC == 1 ? 1 : 2) void k_tree_attend(const TreeArgs a) {
  using BL = Block<D>;
  constexpr int RB = BL::RB, PPR = RB / 16, TR = 32 * WR, NBW = BL::N / WC, NPT = 32 * PPR / (64 * WC);
  constexpr int ND = D / 16, NKS = D / 32, NG = QM == R_INT4 ? D / 32 : 1, KT32 = BL::N * BL::KPITCH, VT32 = BL::N * BL::VPITCH;
  // Weights are up to 2^LAG of what the column's maximum would make of them, which is followed up only from there on (a product for every
  // output then).  They and their sums are held times 2^oex: in binary16 up to 2^15 (times the largest V scale so far), to use its range.
  constexpr int LAG = 4, TOP = 15 - LAG;
  constexpr int NTQ = NT == 1 ? 1 : 2;                     // terms of a weight beside V codes, in binary16 always (codes are exact in it)
  static_assert(64 * WC * WR >= TREE_MAX && NBW >= 1 && NPT >= 1, "a thread per node");
  // Two stages of K and of V rows, 32 of each row wave
  __shared__ __attribute__((aligned(16))) char sm_k0[WR * KT32], sm_k1[WR * KT32], sm_v0[WR * VT32], sm_v1[WR * VT32];
  __shared__ __attribute__((aligned(16))) float sm_sc[2][2][NG][TR];           // [stage][K, V][group][row]
  __shared__ Sees sm_sees[TREE_MAX];

  Run r;
  if (!run_of<TR, QM == R_INT4 ? 6 : 5>(a, r)) return;
  const int t = threadIdx.x, lane = t & 63, n = lane & 15, kb = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wc = wave % WC, wr = wave / WC;
  // Where the rows of list F's next two tiles begin, that the wave is to fetch: asked for before anything else
  const int te = r.t1 < r.tF ? r.t1 : r.tF, end = te * TR < r.nF ? te * TR : r.nF, lr = lane / PPR, lp = lane % PPR;       // the lane's row of a block, and the place of its piece
  uint32_t row[2][NBW];
  const auto rows_of = [&](int tile, uint32_t (&y)[NBW]) __attribute__((always_inline)) {
    const int* list = a.f_loc + (size_t)r.b * a.Nmax;
#pragma unroll
    for (int i = 0; i < NBW; ++i) {
      const int e = tile * TR + 32 * wr + (wc + WC * i) * BL::ROWS + lr;
      y[i] = (uint32_t)list[e < end ? e : end - 1];
    }
  };
  if (r.t0 < te) { rows_of(r.t0, row[0]); rows_of(r.t0 + 1, row[1]); }
  // The wave's columns c0 .. (blocks of them are dealt out evenly over the groups), the group's end c1; one past the last repeats the last
  const auto block_of = [&](int g) { return __builtin_amdgcn_readfirstlane((a.C + 15) / 16 * g / a.groups); };
  const int c0 = 16 * (block_of(r.grp) + wc * NB), c1 = 16 * block_of(r.grp + 1) < a.C ? 16 * block_of(r.grp + 1) : a.C;
  const auto column = [&](int cb) { return c0 + 16 * cb + n < a.C ? c0 + 16 * cb + n : a.C - 1; };
  u32x4 qf[NB][NKS];                                       // elements 32 ks + 8 kb .. of the queries
#pragma unroll
  for (int cb = 0; cb < NB; ++cb) {
    const int col = column(cb), node = col / a.G;
    const char* q = (const char*)a.q + (((size_t)r.b * a.n + node) * a.Hq + r.kvh * a.G + (col - node * a.G)) * RB + 16 * kb;
#pragma unroll
    for (int i = 0; i < NKS; ++i) qf[cb][i] = ((const PackedU32x4*)(q + 64 * i))->v;
  }
  if (r.tail) {
    who_sees(a, r, sm_sees, (int*)sm_k0);
    __syncthreads();
  }
  f32x4 o[NB][ND];
  float m[NB], l[NB];                                      // maximum (of logits times scale2) and the lane's share of the sum
#pragma unroll
  for (int cb = 0; cb < NB; ++cb) {
    m[cb] = -INFINITY; l[cb] = 0.f;
#pragma unroll
    for (int i = 0; i < ND; ++i) o[cb][i] = ZERO4;
  }
  int oex = KT == KT_F16 ? TOP : -LAG;
  bool codes = false;                                      // (V scales have been seen)
  const auto scale_o = [&](int cb, float f) __attribute__((always_inline)) {
    l[cb] *= f;
#pragma unroll
    for (int i = 0; i < ND; ++i) o[cb][i] *= f;
  };

  // LDS addresses of a lane within 32 rows: row n (K, rows 16 further on: N / 2 blocks), row 4 kb + j (V)
  constexpr int NVA = D == 128 ? 4 : ND;
  int ka[NKS], va[NVA];
  {
    const int x = n % BL::ROWS, base = wr * KT32 + n / BL::ROWS * BL::KPITCH + x * RB;
#pragma unroll
    for (int i = 0; i < NKS; ++i) ka[i] = base + 16 * BL::k_place(x, 4 * i + kb);
    const int j = 4 * kb + ((lane >> 2) & 3), vx = j % BL::ROWS, vb = wr * VT32 + j / BL::ROWS * BL::VPITCH + vx * RB + 8 * (lane & 1);
#pragma unroll
    for (int i = 0; i < NVA; ++i) va[i] = vb + 16 * BL::v_place(vx, (D == 128 ? 4 : 2) * i + ((lane >> 1) & 1));
  }
  const auto scales4 = [&](int sc, int which, int g, int rb) __attribute__((always_inline)) {
    return *(const f32x4*)&sm_sc[sc][which][g][32 * wr + 16 * rb + 4 * kb];
  };

  // ---- a tile of 32 rows in three parts.  Logits: ----
  f32x4 s[NB][2];
  const auto logits = [&](auto mode_c, const char* sm, int sc) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode_c)::value;
#pragma unroll
    for (int rb = 0; rb < 2; ++rb) {
#pragma unroll
      for (int cb = 0; cb < NB; ++cb) s[cb][rb] = ZERO4;
#pragma unroll
      for (int ks = 0; ks < NKS; ++ks) {
        const u32x4 x = *(const u32x4*)(sm + ka[ks] + rb * (BL::N / 2) * BL::KPITCH);
        if constexpr (MODE == R_INT4) {
          const f32x4 f = scales4(sc, 0, ks, rb);          // (a product is a group deep)
#pragma unroll
          for (int cb = 0; cb < NB; ++cb) {
            const f32x4 part = mfma_16x16x32<KT>(x, qf[cb][ks], ZERO4);
#pragma unroll
            for (int j = 0; j < 4; ++j) s[cb][rb][j] = fmaf(f[j], part[j], s[cb][rb][j]);
          }
        } else {
#pragma unroll
          for (int cb = 0; cb < NB; ++cb) s[cb][rb] = mfma_16x16x32<KT>(x, qf[cb][ks], s[cb][rb]);
        }
      }
    }
  };
  // ---- weights, in s: of rows e0 .. ----
  const auto weights = [&](auto mode_c, int sc, int e0, int n_list) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode_c)::value;
    if constexpr (MODE == R_INT8) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) {
        const f32x4 f = scales4(sc, 0, 0, rb);
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) s[cb][rb] *= f;
      }
    }
    const int tail0 = MODE == R_FULL ? r.tail0 : 0x7fffffff - 64;
    if (e0 + 32 > n_list || (MODE == R_FULL && e0 + 32 > tail0)) {      // the list's end, and the tree's rows
#pragma unroll
      for (int cb = 0; cb < NB; ++cb) {
        const uint32_t vis = seen_rows(sm_sees, column(cb) / a.G, e0, n_list, tail0) >> (4 * kb);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[cb][rb][j] = (vis >> (16 * rb + j)) & 1 ? s[cb][rb][j] : -INFINITY;
      }
    }
    float tm[NB];                                          // the lane's own largest; the column's is looked for only if one of them calls for it
    bool up = false;
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) {
      tm[cb] = s[cb][0][0];
#pragma unroll
      for (int j = 1; j < 8; ++j) tm[cb] = fmaxf(tm[cb], s[cb][j / 4][j % 4]);
      up = up || fmaf(tm[cb], a.scale2, -(float)LAG) > m[cb];
    }
    if (__builtin_amdgcn_ballot_w64(up)) {
#pragma unroll
      for (int cb = 0; cb < NB; ++cb) {
        const float mn = fmaxf(m[cb], max_swap16(max_swap32(tm[cb])) * a.scale2);
        scale_o(cb, mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[cb] - mn));
        m[cb] = mn;
      }
    }
    if constexpr (MODE != R_FULL) {
      float vmax = 0.f;
#pragma unroll
      for (int g = 0; g < NG; ++g) vmax = fmaxf(vmax, sm_sc[sc][1][g][32 * wr + (lane & 31)]);
#pragma unroll
      for (int x = 1; x < 32; x *= 2) vmax = fmaxf(vmax, __shfl_xor(vmax, x));
      const int ex = exponent_of(vmax);
      if (vmax > 0.f && (!codes || TOP - ex < oex)) {
        int now = TOP - ex;
        if (!codes) {                                      // from what rows of list F left: not so far up that it overflows
          float big = 0.f;
#pragma unroll
          for (int cb = 0; cb < NB; ++cb) {
            big = fmaxf(big, l[cb]);
#pragma unroll
            for (int i = 0; i < D / 4; ++i) big = fmaxf(big, fabsf(o[cb][i / 4][i % 4]));
          }
#pragma unroll
          for (int x = 1; x < 64; x *= 2) big = fmaxf(big, __shfl_xor(big, x));
          const int room = oex + 100 - exponent_of(big);
          if (big > 0.f && now > room) now = room > oex ? room : oex < now ? oex : now;
          codes = true;
        }
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) scale_o(cb, ldexpf(1.f, now - oex));
        oex = now;
      }
    }
#pragma unroll
    for (int cb = 0; cb < NB; ++cb) {
      const float sub = (float)oex - (m[cb] == -INFINITY ? 0.f : m[cb]);       // (nothing seen yet: every weight is 2^-inf)
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float x = __builtin_amdgcn_exp2f(fmaf(s[cb][i / 4][i % 4], a.scale2, sub));
        s[cb][i / 4][i % 4] = x;
        sum = i ? sum + x : x;
      }
      l[cb] += sum;
    }
  };
  // ---- and the weights, times V scales of group g, as the second product takes them ----
  const auto terms = [&](auto mode_c, auto& w, int sc, int g) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode_c)::value, N = MODE == R_FULL ? NT : NTQ;
    f32x4 f[2];
    if constexpr (MODE != R_FULL) {
#pragma unroll
      for (int rb = 0; rb < 2; ++rb) f[rb] = scales4(sc, 1, g, rb);
    }
#pragma unroll
    for (int cb = 0; cb < NB; ++cb)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float p0 = s[cb][i / 2][2 * (i & 1)], p1 = s[cb][i / 2][2 * (i & 1) + 1];
        if constexpr (MODE != R_FULL) { p0 *= f[i / 2][2 * (i & 1)]; p1 *= f[i / 2][2 * (i & 1) + 1]; }
        uint32_t tw[N];
        weight_terms<(MODE == R_FULL ? KT : KT_F16), N>(p0, p1, tw);
#pragma unroll
        for (int k = 0; k < N; ++k) w[cb][k][i] = tw[k];
      }
  };
  const auto outputs = [&](auto mode_c, auto& w, const char* sm, int sc) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode_c)::value, N = MODE == R_FULL ? NT : NTQ;
#pragma unroll
    for (int db = 0; db < ND; ++db) {
      if constexpr (MODE == R_INT4) {
        if ((db & 1) == 0) { __builtin_amdgcn_sched_barrier(0); terms(mode_c, w, sc, db / 2); }      // (one group's at a time: registers)
      }
      union { s16x4 half[2]; u32x4 v; } x;                 // rows 4 kb + j, then 16 + 4 kb + j
#pragma unroll
      for (int rb = 0; rb < 2; ++rb)
        x.half[rb] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(sm + (D == 128 ? va[db >> 1] + 32 * (db & 1) : va[db]) + rb * (BL::N / 2) * BL::VPITCH));
#pragma unroll
      for (int k = 0; k < N; ++k)
#pragma unroll
        for (int cb = 0; cb < NB; ++cb) o[cb][db] = mfma_16x16x32<(MODE == R_FULL ? KT : KT_F16)>(x.v, w[cb][k], o[cb][db]);
    }
  };
  // A list's tiles from t0 to t1 (32 rows of every row wave each), with a barrier a tile; fetch brings the next one into the other stage.
  const auto tiles = [&](auto mode_c, int t0, int t1, int n_list, auto fetch) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode_c)::value;
    const auto step = [&](auto ic, int tile) __attribute__((always_inline)) {
      constexpr int i = decltype(ic)::value;
      fetch(ic, tile);
      if (c0 < c1) {
        u32x4 w[NB][MODE == R_FULL ? NT : NTQ];
        logits(mode_c, i ? sm_k1 : sm_k0, i);
        weights(mode_c, i, tile * TR + 32 * wr, n_list);
        if constexpr (MODE != R_INT4) terms(mode_c, w, i, 0);
        outputs(mode_c, w, i ? sm_v1 : sm_v0, i);
      }
      if constexpr (MODE == R_FULL) wait_rows<0, (WC > 1)>();
      else lds_barrier<(WC > 1)>();
      return tile + 1 < t1;
    };
    for (int tile = t0;; tile += 2) {
      if (!step(std::integral_constant<int, 0>{}, tile)) break;
      if (!step(std::integral_constant<int, 1>{}, tile + 1)) break;
    }
    wait_rows<0, true>();
  };

  // ---- list F: straight to the LDS.  While a tile's weights are made, the K rows of the next but one and the V rows of the next are asked for
  // (the places of those just used) ----
  if (r.t0 < te) {
    const size_t at = (size_t)r.pair * a.capF * RB;
    const __amdgpu_buffer_rsrc_t rk = row_rsrc(a.fpK + at, (uint32_t)a.capF * RB), rv = row_rsrc(a.fpV + at, (uint32_t)a.capF * RB);
    const uint32_t kc = 16 * BL::k_piece(lr, lp), vc = 16 * BL::v_place(lr, lp);
    const int whole = r.tail && r.tail0 < end ? r.tail0 : end;      // entries before it are there
    const auto ask = [&](const __amdgpu_buffer_rsrc_t& rs, char* sm, int pitch, int tile32, uint32_t piece, int tile, const uint32_t (&y)[NBW]) __attribute__((always_inline)) {
      if (tile * TR + TR <= whole) {
#pragma unroll
        for (int i = 0; i < NBW; ++i) to_lds(rs, sm + wr * tile32 + (wc + WC * i) * pitch, y[i] * (uint32_t)RB + piece);
      } else {
#pragma unroll
        for (int i = 0; i < NBW; ++i) {
          const int blk = wc + WC * i, e = tile * TR + 32 * wr + blk * BL::ROWS + lr;
          const bool none = e >= end || (e >= whole && !is_there(sm_sees, e - r.tail0));           // zeros arrive
          to_lds(rs, sm + wr * tile32 + blk * pitch, none ? 0xffffffffu : y[i] * (uint32_t)RB + piece);
        }
      }
    };
    const auto ask_k = [&](char* sm, int tile, const uint32_t (&y)[NBW]) __attribute__((always_inline)) { ask(rk, sm, BL::KPITCH, KT32, kc, tile, y); };
    const auto ask_v = [&](char* sm, int tile, const uint32_t (&y)[NBW]) __attribute__((always_inline)) { ask(rv, sm, BL::VPITCH, VT32, vc, tile, y); };
    ask_k(sm_k0, r.t0, row[0]);
    ask_v(sm_v0, r.t0, row[0]);
    wait_rows<0, true>();
    tiles(std::integral_constant<int, R_FULL>{}, r.t0, te, r.nF,
          [&](auto ic, int tile) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            if (tile + 1 >= te) return;
            ask_k(i ? sm_k0 : sm_k1, tile + 1, row[i ^ 1]);
            ask_v(i ? sm_v0 : sm_v1, tile + 1, row[i ^ 1]);
            rows_of(tile + 2, row[i]);
          });
  }
  // ---- list Q: through registers, asked for AHEAD tiles before they are widened into the LDS, a row wave's rows by its WC waves ----
  if (const int qb = r.t0 > r.tF ? r.t0 - r.tF : 0, qe = r.t1 - r.tF; qb < qe) {
    using P = typename Piece<QM, KT>::type;
    const size_t rows = (size_t)r.pair * a.cap2;
    const char* const k = a.c2K + rows * a.cb; const char* const v = a.c2V + rows * a.cb;
    const char* const ksc = a.s2K + rows * a.sb; const char* const vsc = a.s2V + rows * a.sb;
    const int* list = a.q_loc + (size_t)r.b * a.Nmax;
    const int tt = wc * 64 + lane;
    constexpr int AHEAD = NB == 3 || WC == 2 ? 1 : 2;      // (registers)
    struct Ahead {                                         // a tile on its way, AHEAD of them in turn
      int slot[NPT], slot_s;                               // slots of the one after the next
      P k[NPT], v[NPT];
      u32x2 sk, sv;                                        // scales of row tt
      uint32_t none;                                       // bit i: piece i has no row; bit 31: row tt
    } on[AHEAD];
    const auto load_slots = [&](Ahead& y, int tile) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int e = tile * TR + 32 * wr + (tt + i * 64 * WC) / PPR;
        y.slot[i] = e < r.nQ ? list[e] : -1;
      }
      const int e = tile * TR + 32 * wr + tt;
      y.slot_s = tt < 32 && e < r.nQ ? list[e] : -1;
    };
    const auto load_rows = [&](Ahead& y) __attribute__((always_inline)) {
      y.none = 0;
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const bool off = (uint32_t)y.slot[i] >= (uint32_t)a.cap2;
        y.none |= (uint32_t)off << i;
        const uint32_t at = (off ? 0u : (uint32_t)y.slot[i]) * (uint32_t)a.cb + (uint32_t)((tt + i * 64 * WC) % PPR) * (uint32_t)sizeof(P);
        y.k[i] = *(const P*)(k + at); y.v[i] = *(const P*)(v + at);
      }
      const bool off = (uint32_t)y.slot_s >= (uint32_t)a.cap2;
      y.none |= (uint32_t)off << 31;
      const uint32_t at = (off ? 0u : (uint32_t)y.slot_s) * (uint32_t)a.sb;
      if constexpr (QM == R_INT4 && D == 128) { y.sk = *(const u32x2*)(ksc + at); y.sv = *(const u32x2*)(vsc + at); }
      else { y.sk.x = *(const uint32_t*)(ksc + at); y.sv.x = *(const uint32_t*)(vsc + at); }
    };
    const auto store_rows = [&](const Ahead& y, char* sk, char* sv, int sc) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int idx = tt + i * 64 * WC, row = idx / PPR, p = idx % PPR, x = row % BL::ROWS;
        u32x4 yk = row_piece<KT>(y.k[i], 0.f), yv = row_piece<KT_F16>(y.v[i], 0.f);
        if ((y.none >> i) & 1) yk = yv = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(sk + wr * KT32 + row / BL::ROWS * BL::KPITCH + x * RB + 16 * BL::k_place(x, p)) = yk;
        *(u32x4*)(sv + wr * VT32 + row / BL::ROWS * BL::VPITCH + x * RB + 16 * BL::v_place(x, p)) = yv;
      }
      if (tt < 32) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const float fk = QM == R_INT8 ? __builtin_bit_cast(float, y.sk.x) : half_of(g < 2 ? y.sk.x : y.sk.y, g & 1);
          const float fv = QM == R_INT8 ? __builtin_bit_cast(float, y.sv.x) : half_of(g < 2 ? y.sv.x : y.sv.y, g & 1);
          sm_sc[sc][0][g][32 * wr + tt] = y.none >> 31 ? 0.f : fk;
          sm_sc[sc][1][g][32 * wr + tt] = y.none >> 31 ? 0.f : fv;
        }
      }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load_slots(on[i], qb + i);
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) { load_rows(on[i]); load_slots(on[i], qb + AHEAD + i); }
    store_rows(on[0], sm_k0, sm_v0, 0);
    load_rows(on[0]);
    load_slots(on[0], qb + 2 * AHEAD);
    lds_barrier<true>();
    tiles(std::integral_constant<int, QM>{}, qb, qe, r.nQ,
          [&](auto ic, int tile) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;         // the next tile, into the places of the last
            store_rows(on[(i + 1) % AHEAD], i ? sm_k0 : sm_k1, i ? sm_v0 : sm_v1, i ^ 1);
            load_rows(on[(i + 1) % AHEAD]);
            load_slots(on[(i + 1) % AHEAD], tile + 1 + 2 * AHEAD);
          });
  }
  // ---- the columns' sums: quarters joined, then the row waves' shares (by way of the LDS, the upper half of the waves to the lower one
  // each time, a block of columns at a time), then the output and the statistics, or a split's share for k_tree_merge ----
#pragma unroll
  for (int cb = 0; cb < NB; ++cb) {
    scale_o(cb, ldexpf(1.f, -oex));
    l[cb] = add_swap16(add_swap32(l[cb], l[cb]));
  }
  if constexpr (WR > 1) {
    constexpr int HALF = D / 8;                            // a lane's outputs of a block of columns, halved over the K and V places; maximum and sum in the scales'
    static_assert(HALF * 256 * (WR / 2) * WC <= WR * KT32 && 2 * 16 * (WR / 2) * WC <= 2 * NG * TR, "shares fit a stage");
#pragma unroll
    for (int half = WR / 2; half >= 1; half /= 2)
#pragma unroll
      for (int cb = 0; cb < NB; ++cb) {
        const int sh = (wr & (half - 1)) * WC + wc;
        float* so0 = (float*)(cb & 1 ? sm_k1 : sm_k0) + sh * HALF * 64 + lane;
        float* so1 = (float*)(cb & 1 ? sm_v1 : sm_v0) + sh * HALF * 64 + lane;
        float* sl = &sm_sc[cb & 1][0][0][0] + sh * 32 + n;
        __syncthreads();
        if (wr >= half && wr < 2 * half) {
#pragma unroll
          for (int i = 0; i < HALF; ++i) { so0[i * 64] = o[cb][i / 4][i % 4]; so1[i * 64] = o[cb][ND / 2 + i / 4][i % 4]; }
          if (kb == 0) { sl[0] = m[cb]; sl[16] = l[cb]; }
        }
        __syncthreads();
        if (wr < half) {
          const float m1 = sl[0], mx = fmaxf(m[cb], m1), mu = mx == -INFINITY ? 0.f : mx;
          const float f0 = __builtin_amdgcn_exp2f(m[cb] - mu), f1 = __builtin_amdgcn_exp2f(m1 - mu);
          l[cb] = fmaf(l[cb], f0, sl[16] * f1);
#pragma unroll
          for (int i = 0; i < HALF; ++i) {
            o[cb][i / 4][i % 4] = fmaf(o[cb][i / 4][i % 4], f0, so0[i * 64] * f1);
            o[cb][ND / 2 + i / 4][i % 4] = fmaf(o[cb][ND / 2 + i / 4][i % 4], f0, so1[i * 64] * f1);
          }
          m[cb] = mx;
        }
      }
  }
  if (wr > 0) return;
#pragma unroll
  for (int cb = 0; cb < NB; ++cb) {
    const int col = c0 + 16 * cb + n, node = col / a.G;
    if (col >= c1) continue;
    if (a.S > 1) {
      float* po = a.part_o + ((size_t)r.u * a.C + col) * D + 4 * kb;
#pragma unroll
      for (int i = 0; i < ND; ++i) *(f32x4*)(po + 16 * i) = o[cb][i];
      if (kb == 0) { a.part_ml[(size_t)r.u * 2 * a.C + col] = m[cb]; a.part_ml[((size_t)r.u * 2 + 1) * a.C + col] = l[cb]; }
      continue;
    }
    const float il = is_there(sm_sees, node) && l[cb] > 0.f ? 1.0f / l[cb] : 0.f;
    const size_t at = (((size_t)r.b * a.n + node) * a.Hq + r.kvh * a.G + (col - node * a.G)) * D + 4 * kb;
    const auto each = [&](auto store) __attribute__((always_inline)) {           // (the caller's tensor may begin anywhere)
#pragma unroll
      for (int i = 0; i < ND; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) store(at + 16 * i + k, il > 0.f ? o[cb][i][k] * il : 0.f);
    };
    if (a.out_kind == KT_F32) each([&](size_t e, float y) { ((float*)a.out)[e] = y; });
    else if (a.out_kind == KT_BF16) each([&](size_t e, float y) { ((uint16_t*)a.out)[e] = f32_to_bf16(y); });
    else each([&](size_t e, float y) { ((_Float16*)a.out)[e] = (_Float16)y; });
    if (kb == 0) a.stat[(size_t)r.pair * a.stat_stride + col] = float2{m[cb], il};
  }
}

// ---- attention, binary32 rows ----------------------------------------------------------------------------------------------
// The same walk with binary32 products, four at a time along the row; rows of both lists through registers, one tile ahead, codes times
// their scales on the way.  Bound by the matrix cores' binary32 rate, a sixteenth of the 16-bit one: 10 x 14520 rows of 4 kv heads under
// 42 columns, 213 us (19 GFLOP in 64 columns: 90 TFLOP/s, a large product here 154; 510 with one workgroup of two waves a CU).
template <int D, int WC, int WR, int QM>
__global__ __launch_bounds__(64 * WC * WR) void k_tree_attend_f32(const TreeArgs a) {
  constexpr int RB = D * 4, PPR = RB / 16, NTH = 64 * WC * WR, TR = 32 * WR, NPT = TR * PPR / NTH, KP = Pitch<D>::K, VP = Pitch<D>::V, NDB = D / 32;
  static_assert(NTH >= TREE_MAX && TR * PPR % NTH == 0, "a thread per node");
  __shared__ __attribute__((aligned(16))) char sm_kv[2][TR * (KP + VP)];       // [buffer]: K rows, then V rows
  __shared__ Sees sm_sees[TREE_MAX];

  Run r;
  if (!run_of<TR, 4>(a, r)) return;
  const int t = threadIdx.x, lane = t & 63, ln = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wc = wave % WC, wr = wave / WC;
  if (r.tail) {
    who_sees(a, r, sm_sees, (int*)sm_kv[0]);
    __syncthreads();
  }
  const int c0 = (r.grp * WC + wc) * 32;
  const bool active = c0 < a.C;
  const int col = c0 + ln < a.C ? c0 + ln : a.C - 1, node = col / a.G, head = r.kvh * a.G + (col - node * a.G);
  f32x4 qf[D / 8];                                         // elements 4 * (2 i + h) .. of the query
  {
    const char* q = (const char*)a.q + (((size_t)r.b * a.n + node) * a.Hq + head) * RB + 16 * h;
#pragma unroll
    for (int i = 0; i < D / 8; ++i) qf[i] = __builtin_bit_cast(f32x4, ((const PackedU32x4*)(q + 32 * i))->v);
  }
  f32x16 o[NDB];
#pragma unroll
  for (int i = 0; i < NDB; ++i) o[i] = zero16();
  float m = -INFINITY, l = 0.f;
  int buf = 0;

  const auto walk = [&](auto mode_c, const RowSrc& src, int tb, int te) {
    constexpr int MODE = decltype(mode_c)::value;
    using P = typename Piece<MODE, KT_F32>::type;
    if (tb >= te) return;
    int slot[NPT];
    P rk[NPT], rv[NPT];
    float fk[NPT], fv[NPT];                                // the pieces' scales
    uint32_t none = 0;
    const auto load_slots = [&](int tile) {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int e = tile * TR + (t + i * NTH) / PPR;
        slot[i] = e < src.n ? src.list[e] : -1;
        if (MODE == R_FULL && r.tail && e >= r.tail0 && e < r.nF && !is_there(sm_sees, e - r.tail0)) slot[i] = -1;   // not there: zeros, whatever it holds
      }
    };
    const auto load_rows = [&] {
      none = 0;
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const bool off = (uint32_t)slot[i] >= (uint32_t)src.cap;
        const uint32_t s = off ? 0u : (uint32_t)slot[i];
        const int p = (t + i * NTH) % PPR;
        none |= (uint32_t)off << i;
        const uint32_t at = s * (uint32_t)src.code_bytes + (uint32_t)p * (uint32_t)sizeof(P);
        rk[i] = *(const P*)(src.k + at); rv[i] = *(const P*)(src.v + at);
        if constexpr (MODE == R_INT8) { fk[i] = *(const float*)(src.sk + 4 * s); fv[i] = *(const float*)(src.sv + 4 * s); }
        if constexpr (MODE == R_INT4) { fk[i] = (float)*(const _Float16*)(src.sk + s * src.scale_bytes + 2 * (p / 8)); fv[i] = (float)*(const _Float16*)(src.sv + s * src.scale_bytes + 2 * (p / 8)); }
      }
    };
    const auto store_rows = [&] {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int idx = t + i * NTH, row = idx / PPR, p = idx % PPR;
        u32x4 k = row_piece<KT_F32>(rk[i], fk[i]), v = row_piece<KT_F32>(rv[i], fv[i]);
        if ((none >> i) & 1) k = v = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(sm_kv[buf] + row * KP + 16 * p) = k;
        *(u32x4*)(sm_kv[buf] + TR * KP + row * VP + 16 * p) = v;
      }
    };
    const auto compute = [&](int tile) {
      const char* kt = sm_kv[buf] + (32 * wr + ln) * KP + 16 * h;
      const char* vt = sm_kv[buf] + TR * KP + (32 * wr + 4 * h) * VP + 4 * ln;
      f32x16 s = zero16();
#pragma unroll
      for (int c = 0; c < D / 8; ++c) {
        const f32x4 x = *(const f32x4*)(kt + 32 * c);
#pragma unroll
        for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], qf[c][j], s, 0, 0, 0);
      }
      const int e0 = tile * TR + 32 * wr, tail0 = MODE == R_FULL ? r.tail0 : 0x7fffffff - 64;
      if (e0 + 32 > src.n || (MODE == R_FULL && e0 + 32 > tail0)) {
        const uint32_t vis = seen_rows(sm_sees, node, e0, src.n, tail0) >> (4 * h);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (vis >> (8 * (i / 4) + i % 4)) & 1 ? s[i] : -INFINITY;
      }
      const f32x16 ss[1] = {s};
      follow_maximum<1, NDB, 8>(ss, a.scale2, m, l, o);
      float p[16];
      tile_weights(s, a.scale2, m == -INFINITY ? 0.f : -m, l, p);      // (nothing seen yet: every weight is 2^-inf)
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int db = 0; db < NDB; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(*(const float*)(vt + (8 * (i / 4) + i % 4) * VP + 128 * db), p[i], o[db], 0, 0, 0);
    };
    load_slots(tb);
    load_rows();
    load_slots(tb + 1);
    for (int tile = tb; tile < te; ++tile) {
      store_rows();
      if (tile + 1 < te) { load_rows(); load_slots(tile + 2); }
      __syncthreads();                                     // the buffer is full; the other one's readers are through
      if (active) compute(tile);
      buf ^= 1;
    }
  };
  {
    const size_t at = (size_t)r.pair * a.capF * RB;
    const RowSrc src{a.fpK + at, a.fpV + at, nullptr, nullptr, a.f_loc + (size_t)r.b * a.Nmax, r.nF, a.capF, RB, 0};
    walk(std::integral_constant<int, R_FULL>{}, src, r.t0, r.t1 < r.tF ? r.t1 : r.tF);
  }
  {
    const size_t rows = (size_t)r.pair * a.cap2;
    const RowSrc src{a.c2K + rows * a.cb, a.c2V + rows * a.cb, a.s2K + rows * a.sb, a.s2V + rows * a.sb, a.q_loc + (size_t)r.b * a.Nmax, r.nQ, a.cap2, a.cb, a.sb};
    walk(std::integral_constant<int, QM>{}, src, r.t0 > r.tF ? r.t0 - r.tF : 0, r.t1 - r.tF);
  }
  l = add_swap32(l, l);
  finish_columns<D, WC, WR>(a, r, sm_sees, sm_kv[0], sm_kv[1], wc, wr, lane, col, node, active && c0 + ln < a.C, o, m, l);
}

// ---- the kept queries' weights ---------------------------------------------------------------------------------------------
// Grid (runs of 128 list entries, B, layers).  A wave has 32 rows of list F or list Q, for one kv head after the other, and the kept
// columns of that head in blocks of 32; 4 waves a workgroup, each on its own.  Bound by the latency of the K rows, which arrive once, and of
// the queries: eight layers of 8 x 4133 rows (0.49 GB, 101 us at the rate of a copy) take 115 us with two waves a SIMD and the next block's queries asked for early, 137
// without that, 209 with one wave (both code formats in one kernel); three waves spill (146).  Binary32 rows: one wave (three layers of
// 10 x 14520 rows, 0.7 GB: 280 us; two spill, 509).
template <int D, int KT, int QM>
__global__ __launch_bounds__(256, KT == KT_F32 ? 1 : 2) void k_tree_scores(const TreeScoreArgs a) {
  constexpr int ES = KT == KT_F32 ? 4 : 2, RB = D * ES, PPR = RB / 16, NPT = 32 * PPR / 64;
  constexpr int NG = D / 32, NQF = KT == KT_F32 ? D / 8 : D / 16, KP = Pitch<D, ES>::K;
  __shared__ __attribute__((aligned(16))) char sm_k[4][32 * KP];
  __shared__ __attribute__((aligned(16))) float sm_sc[4][NG][32], sm_vn[4][32];
  const int b = blockIdx.y, layer = blockIdx.z, lane = threadIdx.x & 63, ln = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int kept = a.kept[2 * b];
  if (kept <= 0) return;
  const int nF = a.cnt[b * CNT_N + C_NF], nQ = a.cnt[b * CNT_N + C_NQ], tF = (nF + 31) / 32, tQ = (nQ + 31) / 32;
  const int tile = blockIdx.x * 4 + wave;
  if (tile >= tF + tQ) return;
  const size_t lb = (size_t)layer * a.B + b;
  char* const tk = sm_k[wave];

  const auto rows = [&](auto mode_c, const RowSrc& src0, const int* pos, int e0) {
    constexpr int MODE = decltype(mode_c)::value;
    using P = typename Piece<MODE, KT>::type;
    constexpr bool SCALED = MODE != R_FULL && KT != KT_F32;
    RowSrc src = src0;
    uint32_t at[NPT], dead = 0;
#pragma unroll
    for (int i = 0; i < NPT; ++i) {
      const int e = e0 + (lane + 64 * i) / PPR, s = e < src.n ? src.list[e] : -1;
      const bool none = (uint32_t)s >= (uint32_t)src.cap;
      dead |= (uint32_t)none << i;
      at[i] = none ? 0u : (uint32_t)s;
    }
    int slot_s = -1;
    if constexpr (SCALED) {
      slot_s = e0 + ln < src.n ? src.list[e0 + ln] : -1;
      if ((uint32_t)slot_s >= (uint32_t)src.cap) slot_s = -1;
    }
    const int at_pos = a.vnorm && e0 + ln < src.n ? pos[e0 + ln] : -1;       // row ln's value norm, of one kv head after the other
    const float* vnorm = a.vnorm + lb * a.Hkv * a.Nmax;
    float vn = 0.f;
    float sum[16];
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[r] = 0.f;
    P rk[NPT];
    float fk[NPT];
    u32x2 sk = {0u, 0u};
    const auto load = [&] {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int p = (lane + 64 * i) % PPR;
        rk[i] = *(const P*)(src.k + (size_t)at[i] * src.code_bytes + p * sizeof(P));
        if constexpr (MODE == R_INT8 && KT == KT_F32) fk[i] = *(const float*)(src.sk + (size_t)4 * at[i]);
        if constexpr (MODE == R_INT4 && KT == KT_F32) fk[i] = (float)*(const _Float16*)(src.sk + (size_t)at[i] * src.scale_bytes + 2 * (p / 8));
      }
      if constexpr (SCALED) {
        const char* s = src.sk + (size_t)(slot_s < 0 ? 0 : slot_s) * src.scale_bytes;
        if constexpr (MODE == R_INT4 && D == 128) sk = *(const u32x2*)s;
        else sk.x = *(const uint32_t*)s;
      }
      if (at_pos >= 0) vn = vnorm[at_pos];
    };
    load();
    // A block's queries and statistics are asked for while the one before it is weighed
    u32x4 qf[NQF];
    float2 st;
    int j = 0;                                             // the column's token
    const auto load_q = [&](int kvh, int c0) __attribute__((always_inline)) {
      const int c = c0 + ln < kept * a.G ? c0 + ln : kept * a.G - 1, g = c - c / a.G * a.G;
      j = c / a.G;
      const int node = a.path[(size_t)b * a.n_path + j];
      st = a.stat[(lb * a.Hkv + kvh) * a.stat_stride + node * a.G + g];
      const char* q = (const char*)a.q + ((lb * a.n + node) * a.Hq + kvh * a.G + g) * RB + 16 * h;
#pragma unroll
      for (int i = 0; i < NQF; ++i) qf[i] = ((const PackedU32x4*)(q + 32 * i))->v;
    };
    load_q(0, 0);
    for (int kvh = 0; kvh < a.Hkv; ++kvh) {
      // (a wave's LDS accesses are served in order: the last head's reads come before these writes)
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int idx = lane + 64 * i, row = idx / PPR, p = idx % PPR;
        u32x4 k = row_piece<KT>(rk[i], fk[i]);
        if ((dead >> i) & 1) k = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(tk + row * KP + 16 * p) = k;
      }
      if constexpr (SCALED) {
        if (lane < 32) {
          if constexpr (MODE == R_INT8) sm_sc[wave][0][ln] = slot_s < 0 ? 0.f : __builtin_bit_cast(float, sk.x);
          else {
#pragma unroll
            for (int g = 0; g < NG; ++g) sm_sc[wave][g][ln] = slot_s < 0 ? 0.f : half_of(g < 2 ? sk.x : sk.y, g & 1);
          }
        }
      }
      if (a.vnorm && lane < 32) sm_vn[wave][ln] = vn;
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (kvh + 1 < a.Hkv) {
        vnorm += a.Nmax;
        src.k += (size_t)src.cap * src.code_bytes; src.sk += (size_t)src.cap * src.scale_bytes;
        load();
      }
      float own[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) own[r] = 0.f;
      for (int c0 = 0; c0 < kept * a.G; c0 += 32) {
        const bool on = c0 + ln < kept * a.G;
        f32x16 s = zero16();
        if constexpr (KT == KT_F32) {
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const f32x4 x = *(const f32x4*)(tk + ln * KP + 16 * h + 32 * i), y = __builtin_bit_cast(f32x4, qf[i]);
#pragma unroll
            for (int k = 0; k < 4; ++k) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[k], y[k], s, 0, 0, 0);
          }
        } else {
#pragma unroll
          for (int gr = 0; gr < (MODE == R_INT4 ? NG : 1); ++gr) {
            constexpr int N = MODE == R_INT4 ? 2 : D / 16;
            f32x16 part = zero16();
#pragma unroll
            for (int k = 0; k < N; ++k) {
              const int ks = gr * N + k;
              part = mfma_32x32x16<KT>(*(const u32x4*)(tk + ln * KP + 16 * h + 32 * ks), qf[ks], part);
            }
            if constexpr (MODE == R_FULL) s = part;
            else {
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const f32x4 f = *(const f32x4*)&sm_sc[wave][gr][8 * i + 4 * h];
#pragma unroll
                for (int k = 0; k < 4; ++k) s[4 * i + k] = fmaf(f[k], part[4 * i + k], s[4 * i + k]);
              }
            }
          }
        }
        // the column's token sees entries up to its own; the kept nodes are the last `kept` entries of list F
        const int lim = MODE == R_FULL ? nF - kept + j + 1 : src.n;
        const float2 of = st;
        if (c0 + 32 < kept * a.G) load_q(kvh, c0 + 32);
        else if (kvh + 1 < a.Hkv) load_q(kvh + 1, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = e0 + 8 * (r / 4) + 4 * h + r % 4;
          const float w = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, -of.x)) * of.y;
          own[r] += on && e < lim ? w : 0.f;
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 f = {1.f, 1.f, 1.f, 1.f};
        if (a.vnorm) f = *(const f32x4*)&sm_vn[wave][8 * i + 4 * h];
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[4 * i + k] = fmaf(own[4 * i + k], f[k], sum[4 * i + k]);
      }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int x = 1; x < 32; x *= 2) sum[r] += __shfl_xor(sum[r], x);
    float* gain = a.gain + lb * a.stride + (MODE == R_FULL ? 0 : tF * 32) + e0;
    if (ln == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) *(f32x4*)(gain + 8 * i + 4 * h) = f32x4{sum[4 * i], sum[4 * i + 1], sum[4 * i + 2], sum[4 * i + 3]};
    }
  };
  const size_t pl = lb * a.Hkv;
  if (tile < tF) {
    const RowSrc src{a.fpK + pl * a.capF * RB, nullptr, nullptr, nullptr, a.f_loc + (size_t)b * a.Nmax, nF, a.capF, RB, 0};
    rows(std::integral_constant<int, R_FULL>{}, src, a.f_pos + (size_t)b * a.Nmax, tile * 32);
  } else {
    const RowSrc src{a.c2K + pl * a.cap2 * a.cb, nullptr, a.s2K + pl * a.cap2 * a.sb, nullptr, a.q_loc + (size_t)b * a.Nmax, nQ, a.cap2, a.cb, a.sb};
    rows(std::integral_constant<int, QM>{}, src, a.q_pos + (size_t)b * a.Nmax, (tile - tF) * 32);
  }
}

template <int D, int KT, int WC, int WR, int NB>
static hipError_t run_attend(const TreeArgs& a, hipStream_t st) {
  if (a.n < 1 || a.n > TREE_MAX || a.C != a.n * a.G || a.S < 1 || a.groups < 1 || ((a.C + 15) / 16 + a.groups - 1) / a.groups > NB * WC) return hipErrorInvalidValue;
  const dim3 grid((unsigned)((a.B * a.Hkv * a.S + 7) / 8 * 8) * a.groups), block(64 * WC * WR);
  if constexpr (KT == KT_F32) {
    hipLaunchKernelGGL((a.t2fmt == 0 ? k_tree_attend_f32<D, WC, WR, R_INT8> : k_tree_attend_f32<D, WC, WR, R_INT4>), grid, block, 0, st, a);
  } else {
    constexpr int MANY = KT == KT_BF16 ? 3 : 2;            // terms of a weight for binary32 outputs; else one
    const bool many = a.out_kind == KT_F32;
    const auto kernel = a.t2fmt == 0 ? (many ? k_tree_attend<D, KT, WC, WR, NB, MANY, R_INT8> : k_tree_attend<D, KT, WC, WR, NB, 1, R_INT8>)
                                     : (many ? k_tree_attend<D, KT, WC, WR, NB, MANY, R_INT4> : k_tree_attend<D, KT, WC, WR, NB, 1, R_INT4>);
    hipLaunchKernelGGL(kernel, grid, block, 0, st, a);
  }
  return hipGetLastError();
}
template <int D, int KT>
hipError_t tree_attend_by_type(const TreeArgs& a, hipStream_t st);
template <int D, int KT>
hipError_t tree_scores_by_type(const TreeScoreArgs& a, int max_rows, hipStream_t st);

#define TKV_TREE_PART_OF(D_, KT_)                                                                                       \
  template <>                                                                                                           \
  hipError_t tree_attend_by_type<D_, KT_>(const TreeArgs& a, hipStream_t st) {                                          \
    if constexpr (KT_ == KT_F32) {                                                                                      \
      if (a.waves_c == 1) return run_attend<D_, KT_, 1, 2, 2>(a, st);                                                   \
      if (a.waves_c == 2) return run_attend<D_, KT_, 2, 1, 2>(a, st);                                                   \
      return run_attend<D_, KT_, 4, 1, 2>(a, st);                                                                       \
    } else {                                                                                                            \
      if (a.waves_c == 1) return a.blocks == 1 ? run_attend<D_, KT_, 1, 4, 1>(a, st) : run_attend<D_, KT_, 1, 4, 2>(a, st); \
      if (a.waves_c == 2) return run_attend<D_, KT_, 2, 4, 2>(a, st);                                                   \
      return a.blocks <= 2 ? run_attend<D_, KT_, 4, 2, 2>(a, st) : run_attend<D_, KT_, 4, 2, 3>(a, st);                 \
    }                                                                                                                   \
  }                                                                                                                     \
  template <>                                                                                                           \
  hipError_t tree_scores_by_type<D_, KT_>(const TreeScoreArgs& a, int max_rows, hipStream_t st) {                       \
    const dim3 grid((unsigned)(max_rows + 127) / 128 + 1, a.B, a.layers);                                               \
    hipLaunchKernelGGL((a.t2fmt == 0 ? k_tree_scores<D_, KT_, R_INT8> : k_tree_scores<D_, KT_, R_INT4>), grid, dim3(256), 0, st, a); \
    return hipGetLastError();                                                                                           \
  }
#if TKV_TREE_PART == 0
TKV_TREE_PART_OF(128, KT_BF16)
#elif TKV_TREE_PART == 1
TKV_TREE_PART_OF(128, KT_F16)
#elif TKV_TREE_PART == 2
TKV_TREE_PART_OF(128, KT_F32)
#elif TKV_TREE_PART == 3
TKV_TREE_PART_OF(64, KT_BF16)
#elif TKV_TREE_PART == 4
TKV_TREE_PART_OF(64, KT_F16)
#else
TKV_TREE_PART_OF(64, KT_F32)
#endif

#else
template <int D, int KT> hipError_t tree_attend_by_type(const TreeArgs& a, hipStream_t st);
template <int D, int KT> hipError_t tree_scores_by_type(const TreeScoreArgs& a, int max_rows, hipStream_t st);
#define TKV_TREE_DECLARE(D_, KT_)                                                              \
  template <> hipError_t tree_attend_by_type<D_, KT_>(const TreeArgs& a, hipStream_t st);      \
  template <> hipError_t tree_scores_by_type<D_, KT_>(const TreeScoreArgs& a, int max_rows, hipStream_t st);
TKV_TREE_DECLARE(128, KT_BF16) TKV_TREE_DECLARE(128, KT_F16) TKV_TREE_DECLARE(128, KT_F32)
TKV_TREE_DECLARE(64, KT_BF16) TKV_TREE_DECLARE(64, KT_F16) TKV_TREE_DECLARE(64, KT_F32)

// ---- splits joined: D / 4 lanes per (pair, column), eight splits at a time --------------------------------------------------
// Bound by latency: 21 MB in 6.8 us (9.6 with a wave per column, maximum and sum before the rest).
template <int D>
__global__ __launch_bounds__(256) void k_tree_merge(const TreeArgs a) {
  constexpr int LANES = D / 4, COLS = 256 / LANES, MANY = 8;
  const int i = threadIdx.x % LANES, c = blockIdx.x * COLS + threadIdx.x / LANES, pair = blockIdx.y;
  if (c >= a.C) return;
  const int b = pair / a.Hkv, kvh = pair - b * a.Hkv, node = c / a.G;
  const float* ml = a.part_ml + (size_t)pair * a.S * 2 * a.C + c;
  const float* po = a.part_o + ((size_t)pair * a.S * a.C + c) * D + 4 * i;
  const bool here = a.here[b * a.n + node] != 0;
  float mx = -INFINITY, sum = 0.f;
  f32x4 x = {0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < a.S; s0 += MANY) {
    float m[MANY], l[MANY];
    f32x4 o[MANY];
#pragma unroll
    for (int k = 0; k < MANY; ++k) {                       // (past the last: the last again, at no weight)
      const size_t s = s0 + k < a.S ? s0 + k : a.S - 1;
      m[k] = ml[2 * s * a.C]; l[k] = ml[(2 * s + 1) * a.C]; o[k] = *(const f32x4*)(po + s * a.C * D);
    }
    float mn = mx;
#pragma unroll
    for (int k = 0; k < MANY; ++k) { if (s0 + k >= a.S) m[k] = -INFINITY; mn = fmaxf(mn, m[k]); }
    const float mu = mn > -INFINITY ? mn : 0.f, f = __builtin_amdgcn_exp2f(mx - mu);
    sum *= f; x *= f;
#pragma unroll
    for (int k = 0; k < MANY; ++k) {
      const float w = __builtin_amdgcn_exp2f(m[k] - mu);
      sum = fmaf(l[k], w, sum);
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = fmaf(o[k][j], w, x[j]);
    }
    mx = mn;
  }
  const float il = here && sum > 0.f ? 1.0f / sum : 0.f;
  const size_t at = (((size_t)b * a.n + node) * a.Hq + kvh * a.G + (c - node * a.G)) * D + 4 * i;
#pragma unroll
  for (int j = 0; j < 4; ++j) {                            // (the caller's tensor may begin anywhere)
    const float y = il > 0.f ? x[j] * il : 0.f;
    if (a.out_kind == KT_F32) ((float*)a.out)[at + j] = y;
    else if (a.out_kind == KT_BF16) ((uint16_t*)a.out)[at + j] = f32_to_bf16(y);
    else ((_Float16*)a.out)[at + j] = (_Float16)y;
  }
  if (i == 0) a.stat[(size_t)pair * a.stat_stride + c] = float2{mx, il};
}

// one thread per list entry: its weights, layer after layer, into the score of its position
__global__ __launch_bounds__(256) void k_tree_gain(const TreeScoreArgs a) {
  const int b = blockIdx.y, i = blockIdx.x * 256 + threadIdx.x;
  if (a.kept[2 * b] <= 0) return;
  const int nF = a.cnt[b * CNT_N + C_NF], nQ = a.cnt[b * CNT_N + C_NQ], colq = (nF + 31) / 32 * 32;
  int pos = -1;
  if (i < nF) pos = a.f_pos[(size_t)b * a.Nmax + i];
  else if (i >= colq && i < colq + nQ) pos = a.q_pos[(size_t)b * a.Nmax + (i - colq)];
  if (pos < 0) return;
  float s = 0.f;
#pragma unroll 4
  for (int l = 0; l < a.layers; ++l) s += a.gain[((size_t)l * a.B + b) * a.stride + i];
  a.score[(size_t)b * a.Nmax + pos] += a.score_scale * s;
}

bool tree_shape(int kt, int C, int which, TreeShape& s) {
  constexpr int WIDE[5][2] = {{1, 1}, {1, 2}, {2, 2}, {4, 2}, {4, 3}}, WIDE32[3] = {1, 2, 4};
  if (which >= (kt == KT_F32 ? 3 : 5)) return false;
  s.waves_c = kt == KT_F32 ? WIDE32[which] : WIDE[which][0];
  s.waves_r = kt == KT_F32 ? (s.waves_c == 1 ? 2 : 1) : s.waves_c == 1 ? 4 : 8 / s.waves_c;
  s.blocks = kt == KT_F32 ? 2 : WIDE[which][1];
  s.groups = ((C + 15) / 16 + s.waves_c * s.blocks - 1) / (s.waves_c * s.blocks);
  return true;
}

hipError_t launch_tree_attend(const TreeArgs& a, int D, int kt, hipStream_t st) {
  hipError_t e = hipErrorInvalidValue;
  if (D == 128) e = kt == KT_BF16 ? tree_attend_by_type<128, KT_BF16>(a, st) : kt == KT_F16 ? tree_attend_by_type<128, KT_F16>(a, st) : tree_attend_by_type<128, KT_F32>(a, st);
  else if (D == 64) e = kt == KT_BF16 ? tree_attend_by_type<64, KT_BF16>(a, st) : kt == KT_F16 ? tree_attend_by_type<64, KT_F16>(a, st) : tree_attend_by_type<64, KT_F32>(a, st);
  if (e != hipSuccess || a.S == 1) return e;
  const dim3 grid((unsigned)(a.C * (D / 4) + 255) / 256, (unsigned)(a.B * a.Hkv));
  if (D == 128) hipLaunchKernelGGL((k_tree_merge<128>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_tree_merge<64>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_tree_scores(const TreeScoreArgs& a, int D, int kt, int max_rows, hipStream_t st) {
  hipError_t e = hipErrorInvalidValue;
  if (D == 128) e = kt == KT_BF16 ? tree_scores_by_type<128, KT_BF16>(a, max_rows, st) : kt == KT_F16 ? tree_scores_by_type<128, KT_F16>(a, max_rows, st) : tree_scores_by_type<128, KT_F32>(a, max_rows, st);
  else if (D == 64) e = kt == KT_BF16 ? tree_scores_by_type<64, KT_BF16>(a, max_rows, st) : kt == KT_F16 ? tree_scores_by_type<64, KT_F16>(a, max_rows, st) : tree_scores_by_type<64, KT_F32>(a, max_rows, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_tree_gain, dim3((unsigned)(max_rows + 32 + 255) / 256, a.B), dim3(256), 0, st, a);
  return hipGetLastError();
}
#endif

}  // namespace tkv
