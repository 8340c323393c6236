// Attention of a drafted tree over the tiered KV cache, and the scores of the nodes that are kept.
//
//   k_tree_attend : node i of a tree of n sees the live context and, of the tree's own rows (the last n entries of list F), its
//                 ancestors and itself.  The n * G columns (node, head of the group) of a kv head go side by side, 32 per wave;
//                 a workgroup of WC x WR waves walks a run of the pair's tiles of 32 * WR rows, and every tile, brought once into
//                 the LDS, serves the 32 * WC columns of the workgroup.  S^T = K q^T and O^T = V^T P^T on the matrix cores
//                 (32x32 instructions): a lane owns one column, so that maximum, sum and their corrections need no exchange but
//                 one between the wave's halves, and the weights leave the first product as the second one's operand.
//   k_tree_merge : joins a pair's splits, where it has more than one, into the output and the columns' statistics.
//   k_tree_scores : the kept queries' weights once more, from K, q and those statistics, summed over heads: one float per layer
//                 and position, which k_tree_gain adds up over the layers into the scores.
// Tiles, splits and orders of addition depend on the lists' lengths and logical order alone, never on the slot a row lies in.
#include <algorithm>

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

// Two weights as a sum of NT 16-bit terms, each the nearest to what the terms before it left.  Binary32 outputs: three bfloat16
// terms hold a weight whole (two leave up to 2^-18 of it: outputs 1.7e-6 from 64 bits, where binary32 arithmetic is 6e-7), two
// binary16 terms to 2^-23.
template <int KT, int NT>
__device__ __forceinline__ void weight_terms(float p0, float p1, uint32_t (&t)[NT]) {
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    if constexpr (KT == KT_BF16) {
      const f32x2 p = {p0, p1};
      t[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
      if (i + 1 < NT) { p0 -= __builtin_bit_cast(float, t[i] << 16); p1 -= __builtin_bit_cast(float, t[i] & 0xffff0000u); }
    } else {
      const f16x2 h = {(_Float16)p0, (_Float16)p1};
      t[i] = __builtin_bit_cast(uint32_t, h);
      if (i + 1 < NT) { p0 -= (float)h.x; p1 -= (float)h.y; }
    }
  }
}

// ---- rows in the LDS ---------------------------------------------------------------------------------------------------
// A row's 16-byte pieces are rotated among each other by its number.  K rows are read by 32 lanes with a row each, the same piece
// of all (any 16 consecutive rows on 16 different bank groups); 16-bit V rows by transposing reads of four rows x 64 bytes, binary32
// ones along the row, the wave's halves four rows apart.
template <int D, int KT>
__device__ __forceinline__ int k_place(int row, int p) { return KT == KT_F32 || D == 128 ? p ^ (row & 15) : p ^ ((row >> 1) & 7); }
template <int D, int KT>
__device__ __forceinline__ int v_place(int row, int p) {
  return KT == KT_F32 ? p ^ (((row >> 2) & 1) << 3) : D == 128 ? p ^ ((row & 3) << 2) : p ^ (((row >> 1) & 1) << 2);
}

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
// ---- attention -----------------------------------------------------------------------------------------------------------
template <int D, int KT, int WC, int WR, int NT>
__global__ __launch_bounds__(64 * WC * WR) void k_tree_attend(const TreeArgs a) {
  constexpr int ES = KT == KT_F32 ? 4 : 2, RB = D * ES, PPR = RB / 16, NW = WC * WR, NTH = 64 * NW, TR = 32 * WR;
  constexpr int PIECES = TR * PPR, NPT = (PIECES + NTH - 1) / NTH, TILE = TR * RB;
  constexpr int NDB = D / 32, NG = D / 32, NQF = KT == KT_F32 ? D / 8 : D / 16;
  constexpr float SHIFT = KT == KT_F16 ? 14.f : 0.f;       // weights are taken times 2^SHIFT: small ones stay clear of binary16's least exponent
  static_assert(NTH >= TREE_MAX && TR <= NTH, "a thread per node, and per row");
  __shared__ __attribute__((aligned(16))) char sm_kv[2][2][TILE];
  __shared__ __attribute__((aligned(16))) float sm_sc[2][2][KT == KT_F32 ? 1 : NG][TR];     // [buffer][K, V][group][row]
  __shared__ uint32_t sm_sees[TREE_MAX][TREE_WORDS];
  __shared__ int sm_up[TREE_MAX], sm_off[TREE_MAX];
  __shared__ float sm_ml[NW][2][32];

  // Groups of columns of one run of tiles are eight workgroups apart: on one XCD, whose L2 then serves all but the first of them.
  const int id = blockIdx.x, grp = (id >> 3) % a.groups, u = ((id >> 3) / a.groups) * 8 + (id & 7);
  if (u >= a.B * a.Hkv * a.S) return;
  const int pair = u / a.S, sp = u - pair * a.S, b = pair / a.Hkv, kvh = pair - b * a.Hkv;
  const int t = threadIdx.x, lane = t & 63, ln = lane & 31, h = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(t >> 6), wc = wave % WC, wr = wave / WC;
  int nF, nQ;
  if (a.B <= ATTN_ARG_SEQS) { nF = a.nF[b]; nQ = a.nQ[b]; }
  else { nF = a.cnt[b * CNT_N + C_NF]; nQ = a.cnt[b * CNT_N + C_NQ]; }
  const int tF = (nF + TR - 1) / TR, tQ = (nQ + TR - 1) / TR, T = tF + tQ;
  const int t0 = (int)((long long)T * sp / a.S), t1 = (int)((long long)T * (sp + 1) / a.S);
  const int tail0 = nF - a.n;                              // the tree's first entry of list F
  const bool tail = t0 < tF && t1 * TR > tail0;            // this run has tree rows

  // Who sees whom: a node's set is its own bit and its parent's set; in log2(n) rounds every node takes over the set of the node it
  // points at and points where that one pointed.  A node whose chain meets a bad parent is not there: its set is empty.
  if (tail) {
    const int p = t < a.n ? a.parents[b * a.n + t] : -1;
    bool off = t < a.n && (p < -1 || p >= t);
    int up = off ? -1 : p;
    uint32_t sees[TREE_WORDS];
#pragma unroll
    for (int w = 0; w < TREE_WORDS; ++w) sees[w] = t < a.n && (t >> 5) == w ? 1u << (t & 31) : 0u;
    const auto put = [&] {
      if (t < TREE_MAX) {
#pragma unroll
        for (int w = 0; w < TREE_WORDS; ++w) sm_sees[t][w] = off ? 0u : sees[w];
        sm_up[t] = up; sm_off[t] = off;
      }
    };
    put();
    __syncthreads();
    for (int d = 1; d < a.n; d *= 2) {
      if (up >= 0) {
#pragma unroll
        for (int w = 0; w < TREE_WORDS; ++w) sees[w] |= sm_sees[up][w];
        off = off || sm_off[up];
        up = sm_up[up];
      }
      __syncthreads();
      put();
      __syncthreads();
    }
    if (t1 >= tF && grp == 0 && kvh == 0 && t < a.n) a.here[b * a.n + t] = !off;
  }

  // the wave's columns; one past the last repeats the last
  const int c0 = (grp * WC + wc) * 32;
  const bool active = c0 < a.C;
  const int col = c0 + ln < a.C ? c0 + ln : a.C - 1, node = col / a.G, head = kvh * a.G + (col - node * a.G);
  u32x4 qf[NQF];                                           // elements 8 * (2 ks + h) .. of the query (binary32: 4 * (2 ks + h) ..)
  {
    const char* q = (const char*)a.q + (((size_t)b * a.n + node) * a.Hq + head) * RB + 16 * h;
#pragma unroll
    for (int i = 0; i < NQF; ++i) qf[i] = ((const PackedU32x4*)(q + 32 * i))->v;
  }
  f32x16 o[NDB];
#pragma unroll
  for (int i = 0; i < NDB; ++i) o[i] = zero16();
  float m = -INFINITY, l = 0.f;                            // maximum (times scale2) and the lane's share of the sum
  float osc = 0.f;                                         // binary16: power of two that o is held times (0: nothing in it yet)
  int buf = 0;

  const size_t prow = (size_t)pair;
  const auto walk = [&](auto mode_c, const RowSrc& src, int tb, int te) {
    constexpr int MODE = decltype(mode_c)::value;
    using P = typename Piece<MODE, KT>::type;
    constexpr bool SCALED = MODE != R_FULL && KT != KT_F32;        // scales go to the LDS
    if (tb >= te) return;
    int slot[NPT], slot_s = -1;
    P rk[NPT], rv[NPT];
    float fk[NPT], fv[NPT];                                // binary32: the pieces' scales
    u32x2 sk = {0u, 0u}, sv = {0u, 0u};                    // the scales of row t
    uint32_t dead = 0;
    bool dead_s = true;
    const auto slot_of = [&](int tile, int row) {
      const int e = tile * TR + row;
      int s = e < src.n ? src.list[e] : -1;
      if (MODE == R_FULL && tail && e >= tail0 && e < nF && sm_off[e - tail0]) s = -1;      // not there: counts as zeros, whatever it holds
      return s;
    };
    const auto load_slots = [&](int tile) {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int idx = t + i * NTH;
        slot[i] = PIECES % NTH == 0 || idx < PIECES ? slot_of(tile, idx / PPR) : -1;
      }
      if constexpr (SCALED) slot_s = t < TR ? slot_of(tile, t) : -1;
    };
    const auto load_rows = [&] {
      dead = 0;
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const bool none = (uint32_t)slot[i] >= (uint32_t)src.cap;
        const uint32_t s = none ? 0u : (uint32_t)slot[i];
        const int p = (t + i * NTH) % PPR;
        dead |= (uint32_t)none << i;
        const uint32_t at = s * (uint32_t)src.code_bytes + (uint32_t)p * (uint32_t)sizeof(P);
        rk[i] = *(const P*)(src.k + at); rv[i] = *(const P*)(src.v + at);
        if constexpr (MODE == R_INT8 && KT == KT_F32) { fk[i] = *(const float*)(src.sk + 4 * s); fv[i] = *(const float*)(src.sv + 4 * s); }
        if constexpr (MODE == R_INT4 && KT == KT_F32) {
          fk[i] = (float)*(const _Float16*)(src.sk + s * src.scale_bytes + 2 * (p / 8)); fv[i] = (float)*(const _Float16*)(src.sv + s * src.scale_bytes + 2 * (p / 8));
        }
      }
      if constexpr (SCALED) {
        dead_s = (uint32_t)slot_s >= (uint32_t)src.cap;
        const uint32_t at = (dead_s ? 0u : (uint32_t)slot_s) * (uint32_t)src.scale_bytes;
        if constexpr (MODE == R_INT4 && D == 128) { sk = *(const u32x2*)(src.sk + at); sv = *(const u32x2*)(src.sv + at); }
        else { sk.x = *(const uint32_t*)(src.sk + at); sv.x = *(const uint32_t*)(src.sv + at); }
      }
    };
    const auto store_rows = [&] {
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int idx = t + i * NTH, row = idx / PPR, p = idx % PPR;
        if (PIECES % NTH != 0 && idx >= PIECES) break;
        u32x4 k = row_piece<KT>(rk[i], fk[i]), v = row_piece<KT>(rv[i], fv[i]);
        if ((dead >> i) & 1) k = v = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(sm_kv[buf][0] + row * RB + 16 * k_place<D, KT>(row, p)) = k;
        *(u32x4*)(sm_kv[buf][1] + row * RB + 16 * v_place<D, KT>(row, p)) = v;
      }
      if constexpr (SCALED) {
        if (t < TR) {
          if constexpr (MODE == R_INT8) {
            sm_sc[buf][0][0][t] = dead_s ? 0.f : __builtin_bit_cast(float, sk.x); sm_sc[buf][1][0][t] = dead_s ? 0.f : __builtin_bit_cast(float, sv.x);
          } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              sm_sc[buf][0][g][t] = dead_s ? 0.f : half_of(g < 2 ? sk.x : sk.y, g & 1); sm_sc[buf][1][g][t] = dead_s ? 0.f : half_of(g < 2 ? sv.x : sv.y, g & 1);
            }
          }
        }
      }
    };
    // register r of a 32 x 32 result is row 8 * (r / 4) + 4 * h + r % 4
    const auto row_scales = [&](int which, int g, float (&f)[16]) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x4 x = *(const f32x4*)&sm_sc[buf][which][g][32 * wr + 8 * i + 4 * h];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[4 * i + j] = x[j];
      }
    };
    const auto compute = [&](int tile) {
      const char* kt = sm_kv[buf][0] + 32 * wr * RB;
      const char* vt = sm_kv[buf][1] + 32 * wr * RB;
      f32x16 s = zero16();
      if constexpr (KT == KT_F32) {
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
          const f32x4 x = *(const f32x4*)(kt + ln * RB + 16 * k_place<D, KT>(ln, 2 * c + h)), y = __builtin_bit_cast(f32x4, qf[c]);
#pragma unroll
          for (int j = 0; j < 4; ++j) s = __builtin_amdgcn_mfma_f32_32x32x2f32(x[j], y[j], s, 0, 0, 0);
        }
      } else if constexpr (MODE == R_INT4) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          f32x16 part = zero16();
#pragma unroll
          for (int ks = 2 * g; ks < 2 * g + 2; ++ks)
            part = mfma_32x32x16<KT>(*(const u32x4*)(kt + ln * RB + 16 * k_place<D, KT>(ln, 2 * ks + h)), qf[ks], part);
          float f[16];
          row_scales(0, g, f);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] = fmaf(f[r], part[r], s[r]);
        }
      } else {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) s = mfma_32x32x16<KT>(*(const u32x4*)(kt + ln * RB + 16 * k_place<D, KT>(ln, 2 * ks + h)), qf[ks], s);
        if constexpr (MODE == R_INT8) {
          float f[16];
          row_scales(0, 0, f);
#pragma unroll
          for (int r = 0; r < 16; ++r) s[r] *= f[r];
        }
      }
      // the list's end, and the tree's rows
      const int e0 = tile * TR + 32 * wr;
      if (e0 + 32 > src.n || (MODE == R_FULL && e0 + 32 > tail0)) {
        uint32_t vis = e0 + 32 <= src.n ? ~0u : e0 < src.n ? (1u << (src.n - e0)) - 1 : 0u;
        if (MODE == R_FULL && e0 + 32 > tail0) {
          const int nb = e0 - tail0, w = nb >> 5, sh = nb & 31;         // node of the first row (-31 .. n)
          const uint32_t lo = w < 0 ? ~0u : w < TREE_WORDS ? sm_sees[node][w] : 0u, hi = w + 1 < TREE_WORDS ? sm_sees[node][w + 1] : 0u;
          vis &= sh ? (lo >> sh) | (hi << (32 - sh)) : lo;
        }
        vis >>= 4 * h;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = (vis >> (8 * (r / 4) + r % 4)) & 1 ? s[r] : -INFINITY;
      }
      float tm = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) tm = fmaxf(tm, s[r]);
      const float mn = fmaxf(m, max_swap32(tm) * a.scale2);
      const float mu = mn == -INFINITY ? 0.f : mn;                      // nothing seen yet: every weight is 2^-inf
      if (__builtin_amdgcn_ballot_w64(mn > m)) {
        const float al = __builtin_amdgcn_exp2f(m - mu);
        l *= al;
#pragma unroll
        for (int i = 0; i < NDB; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[i][r] *= al;
        m = mn;
      }
      float p[16], sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        p[r] = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, SHIFT - mu));
        sum[r & 3] += p[r];
      }
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      if constexpr (KT == KT_F32) {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int row = 8 * (r / 4) + 4 * h + r % 4;
#pragma unroll
          for (int db = 0; db < NDB; ++db) {
            const float x = *(const float*)(vt + row * RB + 16 * v_place<D, KT>(row, 8 * db + (ln >> 2)) + 4 * (ln & 3));
            o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, p[r], o[db], 0, 0, 0);
          }
        }
      } else {
        if constexpr (KT == KT_F16) {
          // weights times V scales stay within binary16 for the largest scale so far, and use its range
          float vmax = 1.f;
          if constexpr (MODE != R_FULL) {
            vmax = 0.f;
#pragma unroll
            for (int g = 0; g < (MODE == R_INT4 ? NG : 1); ++g) vmax = fmaxf(vmax, sm_sc[buf][1][g][32 * wr + ln]);
#pragma unroll
            for (int x = 1; x < 32; x *= 2) vmax = fmaxf(vmax, __shfl_xor(vmax, x));
          }
          if (vmax > 0.f && (osc == 0.f || vmax * osc > 2.f)) {
            int ex;
            (void)frexpf(vmax, &ex);
            const float now = ldexpf(1.f, MODE == R_FULL ? 0 : -ex), f = osc == 0.f ? 1.f : now / osc;
            osc = now;
#pragma unroll
            for (int i = 0; i < NDB; ++i)
#pragma unroll
              for (int r = 0; r < 16; ++r) o[i][r] *= f;
          }
        }
        u32x4 w[2][NT];
        const auto terms = [&](int g) {                    // the weights, times V scales of group g, as the second product takes them
          float f[16];
          if constexpr (MODE != R_FULL) row_scales(1, g, f);
#pragma unroll
          for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int r = 8 * st + 2 * i;
              float p0 = p[r], p1 = p[r + 1];
              if constexpr (KT == KT_F16) { p0 *= osc; p1 *= osc; }
              if constexpr (MODE != R_FULL) { p0 *= f[r]; p1 *= f[r + 1]; }
              uint32_t tw[NT];
              weight_terms<KT, NT>(p0, p1, tw);
#pragma unroll
              for (int k = 0; k < NT; ++k) w[st][k][i] = tw[k];
            }
        };
        if constexpr (MODE != R_INT4) terms(0);
        const int j = (lane >> 2) & 3, cq = lane & 3, hi16 = (lane >> 4) & 1;
#pragma unroll
        for (int db = 0; db < NDB; ++db) {
          if constexpr (MODE == R_INT4) terms(db);
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            union { s16x4 half[2]; u32x4 v; } x;
#pragma unroll
            for (int rr = 0; rr < 2; ++rr) {
              const int row = 16 * st + 8 * rr + 4 * h + j;
              const char* src_v = vt + row * RB + 16 * v_place<D, KT>(row, 4 * db + 2 * hi16 + (cq >> 1)) + 8 * (cq & 1);
              x.half[rr] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)src_v);
            }
#pragma unroll
            for (int k = 0; k < NT; ++k) o[db] = mfma_32x32x16<KT>(x.v, w[st][k], o[db]);
          }
        }
      }
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
    const size_t at = prow * a.capF * RB;
    const RowSrc src{a.fpK + at, a.fpV + at, nullptr, nullptr, a.f_loc + (size_t)b * a.Nmax, nF, a.capF, RB, 0};
    walk(std::integral_constant<int, R_FULL>{}, src, t0, t1 < tF ? t1 : tF);
  }
  {
    const size_t rows = prow * a.cap2;
    const RowSrc src{a.c2K + rows * a.cb, a.c2V + rows * a.cb, a.s2K + rows * a.sb, a.s2V + rows * a.sb, a.q_loc + (size_t)b * a.Nmax, nQ, a.cap2, a.cb, a.sb};
    const int qb = t0 > tF ? t0 - tF : 0, qe = t1 - tF;
    if (a.t2fmt == 0) walk(std::integral_constant<int, R_INT8>{}, src, qb, qe);
    else walk(std::integral_constant<int, R_INT4>{}, src, qb, qe);
  }

  // ---- the columns' sums ----
  l = add_swap32(l, l);
  if constexpr (KT == KT_F16) {
    const float f = osc > 0.f ? 0x1p-14f / osc : 0.f;
    l *= 0x1p-14f;
#pragma unroll
    for (int i = 0; i < NDB; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[i][r] *= f;
  }
  // one split: the output itself; else its share, and the column's maximum and sum
  const auto finish = [&](int c, int nd, float mx, float sum, int d, auto x) {       // x: consecutive elements from d on
    constexpr int N = sizeof(x) / 4;
    if (a.S > 1) {
      __builtin_memcpy(a.part_o + ((size_t)u * a.C + c) * D + d, &x, sizeof x);
      if (d == 0) { a.part_ml[(size_t)u * 2 * a.C + c] = mx; a.part_ml[((size_t)u * 2 + 1) * a.C + c] = sum; }
      return;
    }
    const float il = !sm_off[nd] && sum > 0.f ? 1.0f / sum : 0.f;
    const size_t at = (((size_t)b * a.n + nd) * a.Hq + kvh * a.G + (c - nd * a.G)) * D + d;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const float y = il > 0.f ? ((const float*)&x)[i] * il : 0.f;
      if (a.out_kind == KT_F32) ((float*)a.out)[at + i] = y;
      else if (a.out_kind == KT_BF16) ((uint16_t*)a.out)[at + i] = f32_to_bf16(y);
      else ((_Float16*)a.out)[at + i] = (_Float16)y;
    }
    if (d == 0) a.stat[(size_t)pair * a.stat_stride + c] = float2{mx, il};
  };
  if constexpr (WR == 1) {
    if (active && c0 + ln < a.C) {
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          finish(col, node, m, l, 32 * db + 8 * i + 4 * h, f32x4{o[db][4 * i], o[db][4 * i + 1], o[db][4 * i + 2], o[db][4 * i + 3]});
    }
  } else {
    // the row waves' shares side by side in the LDS, [element][column], columns rotated by element for the reads along a column
    static_assert(NW * 32 * D * 4 <= (int)sizeof(sm_kv), "shares fit the tiles' place");
    __syncthreads();
    float* so = (float*)sm_kv;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int d = 32 * db + 8 * (r / 4) + 4 * h + r % 4;
        so[(wave * D + d) * 32 + (ln ^ (d & 31))] = o[db][r];
      }
    if (lane < 32) { sm_ml[wave][0][ln] = m; sm_ml[wave][1][ln] = l; }
    __syncthreads();
    for (int i = t; i < WC * 32 * D; i += NTH) {
      const int d = i % D, cw = i / (32 * D), cl = (i / D) & 31, c = (grp * WC + cw) * 32 + cl;
      if (c >= a.C) continue;
      float mx = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll
      for (int r = 0; r < WR; ++r) mx = fmaxf(mx, sm_ml[r * WC + cw][0][cl]);
      if (mx > -INFINITY) {
#pragma unroll
        for (int r = 0; r < WR; ++r) {
          const float f = __builtin_amdgcn_exp2f(sm_ml[r * WC + cw][0][cl] - mx);
          sum = fmaf(sm_ml[r * WC + cw][1][cl], f, sum);
          x = fmaf(so[((r * WC + cw) * D + d) * 32 + (cl ^ (d & 31))], f, x);
        }
      }
      finish(c, c / a.G, mx, sum, d, x);
    }
  }
}

// ---- the kept queries' weights ---------------------------------------------------------------------------------------------
// Grid (runs of 128 list entries, B, layers).  A wave has 32 rows of list F or list Q, for one kv head after the other, and the kept
// columns of that head in blocks of 32.  Bound by the K rows, which arrive once; 4 waves a workgroup, each on its own.
template <int D, int KT>
__global__ __launch_bounds__(256) void k_tree_scores(const TreeScoreArgs a) {
  constexpr int ES = KT == KT_F32 ? 4 : 2, RB = D * ES, PPR = RB / 16, NPT = 32 * PPR / 64;
  constexpr int NG = D / 32, NQF = KT == KT_F32 ? D / 8 : D / 16;
  __shared__ __attribute__((aligned(16))) char sm_k[4][32 * RB];
  __shared__ __attribute__((aligned(16))) float sm_sc[4][NG][32];
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
    };
    load();
    for (int kvh = 0; kvh < a.Hkv; ++kvh) {
      // (a wave's LDS accesses are served in order: the last head's reads come before these writes)
#pragma unroll
      for (int i = 0; i < NPT; ++i) {
        const int idx = lane + 64 * i, row = idx / PPR, p = idx % PPR;
        u32x4 k = row_piece<KT>(rk[i], fk[i]);
        if ((dead >> i) & 1) k = u32x4{0u, 0u, 0u, 0u};
        *(u32x4*)(tk + row * RB + 16 * k_place<D, KT>(row, p)) = k;
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
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
      if (kvh + 1 < a.Hkv) {
        src.k += (size_t)src.cap * src.code_bytes; src.sk += (size_t)src.cap * src.scale_bytes;
        load();
      }
      float own[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) own[r] = 0.f;
      for (int c0 = 0; c0 < kept * a.G; c0 += 32) {
        const bool on = c0 + ln < kept * a.G;
        const int c = on ? c0 + ln : kept * a.G - 1, j = c / a.G, g = c - j * a.G;
        const int node = a.path[(size_t)b * a.n_path + j];
        const float2 st = a.stat[(lb * a.Hkv + kvh) * a.stat_stride + node * a.G + g];
        const char* q = (const char*)a.q + ((lb * a.n + node) * a.Hq + kvh * a.G + g) * RB + 16 * h;
        u32x4 qf[NQF];
#pragma unroll
        for (int i = 0; i < NQF; ++i) qf[i] = ((const PackedU32x4*)(q + 32 * i))->v;
        f32x16 s = zero16();
        if constexpr (KT == KT_F32) {
#pragma unroll
          for (int i = 0; i < D / 8; ++i) {
            const f32x4 x = *(const f32x4*)(tk + ln * RB + 16 * k_place<D, KT>(ln, 2 * i + h)), y = __builtin_bit_cast(f32x4, qf[i]);
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
              part = mfma_32x32x16<KT>(*(const u32x4*)(tk + ln * RB + 16 * k_place<D, KT>(ln, 2 * ks + h)), qf[ks], part);
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
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const int e = e0 + 8 * (r / 4) + 4 * h + r % 4;
          const float w = __builtin_amdgcn_exp2f(fmaf(s[r], a.scale2, -st.x)) * st.y;
          own[r] += on && e < lim ? w : 0.f;
        }
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (a.vnorm) {
          const int e = e0 + 8 * (r / 4) + 4 * h + r % 4;
          own[r] *= e < src.n ? a.vnorm[(lb * a.Hkv + kvh) * a.Nmax + pos[e]] : 0.f;
        }
        sum[r] += own[r];
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
    if (a.t2fmt == 0) rows(std::integral_constant<int, R_INT8>{}, src, a.q_pos + (size_t)b * a.Nmax, (tile - tF) * 32);
    else rows(std::integral_constant<int, R_INT4>{}, src, a.q_pos + (size_t)b * a.Nmax, (tile - tF) * 32);
  }
}

template <int D, int KT, int WC, int WR>
static hipError_t run_attend(const TreeArgs& a, hipStream_t st) {
  constexpr int TERMS = KT == KT_BF16 ? 3 : 2;             // for binary32 outputs
  if (a.n < 1 || a.n > TREE_MAX || a.C != a.n * a.G || a.S < 1 || a.groups != (a.C + 32 * WC - 1) / (32 * WC)) return hipErrorInvalidValue;
  const int units = (a.B * a.Hkv * a.S + 7) / 8 * 8;
  const dim3 grid((unsigned)units * a.groups), block(64 * WC * WR);
  if (KT == KT_F32 || a.out_kind == KT_F32) hipLaunchKernelGGL((k_tree_attend<D, KT, WC, WR, TERMS>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((k_tree_attend<D, KT, WC, WR, 1>), grid, block, 0, st, a);
  return hipGetLastError();
}
template <int D, int KT>
hipError_t tree_attend_by_type(const TreeArgs& a, hipStream_t st);
template <int D, int KT>
hipError_t tree_scores_by_type(const TreeScoreArgs& a, int max_rows, hipStream_t st);

#define TKV_TREE_PART_OF(D_, KT_)                                                                                       \
  template <>                                                                                                           \
  hipError_t tree_attend_by_type<D_, KT_>(const TreeArgs& a, hipStream_t st) {                                          \
    const TreeShape s = tree_shape(D_, KT_, a.C);                                                                       \
    if constexpr (KT_ == KT_F32) {                                                                                      \
      if (s.waves_c == 1) return run_attend<D_, KT_, 1, 2>(a, st);                                                      \
      if (s.waves_c == 2) return run_attend<D_, KT_, 2, 1>(a, st);                                                      \
      return run_attend<D_, KT_, 4, 1>(a, st);                                                                          \
    } else {                                                                                                            \
      if (s.waves_c == 1) return run_attend<D_, KT_, 1, 4>(a, st);                                                      \
      if (s.waves_c == 2) return run_attend<D_, KT_, 2, 2>(a, st);                                                      \
      if (s.waves_c == 4) return run_attend<D_, KT_, 4, 1>(a, st);                                                      \
      return run_attend<D_, KT_, 8, 1>(a, st);                                                                          \
    }                                                                                                                   \
  }                                                                                                                     \
  template <>                                                                                                           \
  hipError_t tree_scores_by_type<D_, KT_>(const TreeScoreArgs& a, int max_rows, hipStream_t st) {                       \
    hipLaunchKernelGGL((k_tree_scores<D_, KT_>), dim3((unsigned)(max_rows + 127) / 128 + 1, a.B, a.layers), dim3(256), 0, st, a); \
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

// ---- splits joined: a wave per (pair, column) ------------------------------------------------------------------------------
template <int D>
__global__ __launch_bounds__(256) void k_tree_merge(const TreeArgs a) {
  constexpr int N = D / 64;
  const int lane = threadIdx.x & 63, c = blockIdx.x * 4 + (threadIdx.x >> 6), pair = blockIdx.y;
  if (c >= a.C) return;
  const int b = pair / a.Hkv, kvh = pair - b * a.Hkv, node = c / a.G;
  const float* ml = a.part_ml + (size_t)pair * a.S * 2 * a.C + c;
  const float* po = a.part_o + ((size_t)pair * a.S * a.C + c) * D + N * lane;
  float mx = -INFINITY, sum = 0.f, x[N];
  for (int s = lane; s < a.S; s += 64) mx = fmaxf(mx, ml[(size_t)2 * s * a.C]);
#pragma unroll
  for (int k = 1; k < 64; k *= 2) mx = fmaxf(mx, __shfl_xor(mx, k));
  const float mu = mx > -INFINITY ? mx : 0.f;
  for (int s = lane; s < a.S; s += 64) sum = fmaf(ml[((size_t)2 * s + 1) * a.C], __builtin_amdgcn_exp2f(ml[(size_t)2 * s * a.C] - mu), sum);
#pragma unroll
  for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = 0.f;
#pragma unroll 8
  for (int s = 0; s < a.S; ++s) {
    const float f = __builtin_amdgcn_exp2f(ml[(size_t)2 * s * a.C] - mu);
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = fmaf(po[(size_t)s * a.C * D + i], f, x[i]);
  }
  const float il = a.here[b * a.n + node] && sum > 0.f ? 1.0f / sum : 0.f;
  const size_t at = (((size_t)b * a.n + node) * a.Hq + kvh * a.G + (c - node * a.G)) * D + N * lane;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = il > 0.f ? x[i] * il : 0.f;
    if (a.out_kind == KT_F32) ((float*)a.out)[at + i] = y;
    else if (a.out_kind == KT_BF16) ((uint16_t*)a.out)[at + i] = f32_to_bf16(y);
    else ((_Float16*)a.out)[at + i] = (_Float16)y;
  }
  if (lane == 0) a.stat[(size_t)pair * a.stat_stride + c] = float2{mx, il};
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

TreeShape tree_shape(int D, int kt, int C) {
  TreeShape s;
  if (kt == KT_F32) { s.waves_c = C <= 32 ? 1 : C <= 64 ? 2 : 4; s.waves_r = s.waves_c == 1 ? 2 : 1; }
  else { s.waves_c = C <= 32 ? 1 : C <= 64 ? 2 : C <= 128 ? 4 : 8; s.waves_r = s.waves_c < 4 ? 4 / s.waves_c : 1; }
  s.groups = (C + 32 * s.waves_c - 1) / (32 * s.waves_c);
  return s;
}
int tree_tile_rows(const TreeShape& s) { return 32 * s.waves_r; }
int tree_units(int kt, const TreeShape& s, int cus) { return s.waves_c == 1 || kt == KT_F32 ? cus : 2 * cus; }

hipError_t launch_tree_attend(const TreeArgs& a, int D, int kt, hipStream_t st) {
  hipError_t e = hipErrorInvalidValue;
  if (D == 128) e = kt == KT_BF16 ? tree_attend_by_type<128, KT_BF16>(a, st) : kt == KT_F16 ? tree_attend_by_type<128, KT_F16>(a, st) : tree_attend_by_type<128, KT_F32>(a, st);
  else if (D == 64) e = kt == KT_BF16 ? tree_attend_by_type<64, KT_BF16>(a, st) : kt == KT_F16 ? tree_attend_by_type<64, KT_F16>(a, st) : tree_attend_by_type<64, KT_F32>(a, st);
  if (e != hipSuccess || a.S == 1) return e;
  const dim3 grid((unsigned)(a.C + 3) / 4, (unsigned)(a.B * a.Hkv));
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
