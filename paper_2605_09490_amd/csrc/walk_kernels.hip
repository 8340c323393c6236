// The end of a speculative step: the walk of a drafted tree against the target's probabilities, and the cache's change to the path
// that it keeps.
//
//   k_walk : W workgroups per sequence.  Whether a child is taken depends on single elements of its parent's rows, which the lanes of
//            a wave gather for all nodes at once; only the sum of a residual, and the draw of the next token, read whole rows.  Every
//            workgroup walks the tree (the same steps in each) up to the first such sum and takes its part of the row; the last to
//            arrive adds the parts, walks on, and draws.  Sums and residuals are held in 64 bits: which token is drawn, and whether
//            one is taken, is decided by comparing them.  Bound by the chain of dependent steps: a gather, a sum, the parts'
//            meeting, the draw (16 us for one line), and a pass of one workgroup over a row (8 us for 100003 pairs in binary32, with
//            32 elements of a lane on their way; 16 with four) for every further rejection of a drawn child.  A barrier of a
//            sequence's workgroups instead would need them all on the chip at once, which nobody can promise.
//   k_accept_check, k_accept : one workgroup per sequence.  Slots change hands, no row moves.
#include "device_common.h"
#include "tree.h"

namespace tkv {

constexpr int WALK_THREADS = 1024, WALK_WAVES = WALK_THREADS / 64;

template <int PT>
__device__ __forceinline__ double prob(const char* row, long long x) {
  if constexpr (PT == KT_F32) return (double)((const float*)row)[x];
  else if constexpr (PT == KT_BF16) return (double)__builtin_bit_cast(float, (uint32_t)((const uint16_t*)row)[x] << 16);
  else return (double)(float)((const _Float16*)row)[x];
}
// element e of 16 bytes of a row
template <int PT>
__device__ __forceinline__ double prob_of(const u32x4& v, int e) {
  if constexpr (PT == KT_F32) { const uint32_t w = v[e]; return (double)__builtin_bit_cast(float, w); }
  else if constexpr (PT == KT_BF16) return (double)__builtin_bit_cast(float, e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
  else return (double)half_of(v[e / 2], e & 1);
}

// The distribution a child of `cur` is tested against, and the next token drawn from, after the rejections at `cur`: p[cur], less
// total * q[cur] for each of them, never below 0 (q given), or with their tokens' elements 0.
struct Residual {
  const char* p; const char* q;
  int subs;                        // subtractions made (q given), or tokens taken out
  const double* total;             // [subs] the sum before each subtraction
  const int* out;                  // [subs] tokens taken out
  __device__ __forceinline__ double at(double pv, double qv, int x) const {
    if (q) {
      for (int k = 0; k < subs; ++k) pv = fmax(pv - total[k] * qv, 0.0);
    } else {
      for (int k = 0; k < subs; ++k) pv = out[k] == x ? 0.0 : pv;
    }
    return pv;
  }
};

// elements x .. of a row, as `at` makes them, added up
template <int PT, int VE>
__device__ __forceinline__ double piece_sum(const Residual& r, const u32x4& pv, const u32x4& qv, int x) {
  double v[VE];
#pragma unroll
  for (int e = 0; e < VE; ++e) v[e] = prob_of<PT>(pv, e);
  for (int k = 0; k < r.subs; ++k) {
    if (r.q) {
      const double total = r.total[k];
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = fmax(v[e] - total * prob_of<PT>(qv, e), 0.0);
    } else {
      const int out = r.out[k] - x;
#pragma unroll
      for (int e = 0; e < VE; ++e) v[e] = out == e ? 0.0 : v[e];
    }
  }
  double s = 0.0;
#pragma unroll
  for (int e = 0; e < VE; ++e) s += v[e];
  return s;
}
// sum of elements lo .. hi - 1, by the lanes t, t + stride, ... of `stride`.  32 elements of a lane (of either row) are on their way at
// once: one workgroup alone waits for memory otherwise.
template <int PT>
__device__ __forceinline__ double part_sum(const Residual& r, int lo, int hi, int t, int stride) {
  constexpr int ES = PT == KT_F32 ? 4 : 2, VE = 16 / ES, MANY = 32 / VE;
  double s = 0.0;
  const int whole = lo + (hi > lo ? (hi - lo) / VE * VE : 0);
  for (int x = lo + t * VE; x < whole; x += MANY * stride * VE) {
    u32x4 pv[MANY], qv[MANY];
#pragma unroll
    for (int i = 0; i < MANY; ++i) {
      const int y = x + i * stride * VE < whole ? x + i * stride * VE : x;
      pv[i] = ((const PackedU32x4*)(r.p + (size_t)y * ES))->v;
      qv[i] = u32x4{0u, 0u, 0u, 0u};
      if (r.q) qv[i] = ((const PackedU32x4*)(r.q + (size_t)y * ES))->v;
    }
#pragma unroll
    for (int i = 0; i < MANY; ++i) {
      const int y = x + i * stride * VE;
      if (y < whole) s += piece_sum<PT, VE>(r, pv[i], qv[i], y);
    }
  }
  if (whole + t < hi) s += r.at(prob<PT>(r.p, whole + t), r.q ? prob<PT>(r.q, whole + t) : 0.0, whole + t);      // (fewer than VE of them)
  return s;
}
__device__ __forceinline__ double wave_sum_f64(double x) {
#pragma unroll
  for (int k = 1; k < 64; k *= 2) x += __shfl_xor(x, k);
  return x;
}

template <int PT>
__global__ __launch_bounds__(WALK_THREADS) void k_walk(const WalkArgs a) {
  constexpr int ES = PT == KT_F32 ? 4 : 2;
  __shared__ double sm_total[TREE_MAX], sm_part[WALK_MAX_PARTS], sm_wave[WALK_WAVES];
  __shared__ int sm_out[TREE_MAX], sm_path[TREE_MAX];
  __shared__ int sm_cur, sm_subs, sm_want, sm_last, sm_token, sm_chunk;
  __shared__ double sm_base;
  const int b = blockIdx.y, w0 = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6, n = a.n;
  const int cl = ((a.vocab + a.W - 1) / a.W + 7) & ~7;      // elements of a part, whole 16-byte pieces
  const auto row = [&](const char* base, long long stride, int node) { return base + ((size_t)b * n + node) * (size_t)stride * ES; };

  // wave 0: what the tests need of every node, nodes `lane` and `lane + 64`
  int par[2] = {-1, -1}, tok[2] = {-1, -1};
  double node_u[2] = {0.0, 0.0}, node_p[2] = {0.0, 0.0}, node_q[2] = {0.0, 0.0};
  if (wave == 0) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = lane + 64 * k;
      if (i < n && i > 0) par[k] = a.parents[b * n + i];
      if (par[k] >= i) par[k] = -1;
      if (i < n) {
        const int x = a.tokens[b * n + i];
        const bool ok = par[k] >= 0 && x >= 0 && x < a.vocab;
        tok[k] = x;
        node_u[k] = (double)a.u[b * n + i];
        if (ok) node_p[k] = prob<PT>(row(a.p, a.p_stride, par[k]), x);
        if (ok && a.q) node_q[k] = prob<PT>(row(a.q, a.q_stride, par[k]), x);
        sm_path[i] = -1;
      }
    }
    if (lane == 0) sm_path[0] = 0;
  }
  __syncthreads();

  // Walk state, the same in all lanes of wave 0
  int cur = 0, last = 0, subs = 0, depth = 1;
  double total = 1.0;
  // a node's value, from its lane
  const auto int_of = [](const int (&v)[2], int i) { return __builtin_amdgcn_readlane(i < 64 ? v[0] : v[1], i & 63); };
  const auto value_of = [](const double (&v)[2], int i) {
    const uint64_t x = __builtin_bit_cast(uint64_t, i < 64 ? v[0] : v[1]);
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)x, i & 63), hi = __builtin_amdgcn_readlane((uint32_t)(x >> 32), i & 63);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
  };
  // On from here: up to a rejection whose residual has to be summed (q given; subs counts it then), or to the end.
  const auto walk = [&]() -> bool {
    for (;;) {
      const uint64_t lo = __builtin_amdgcn_ballot_w64(par[0] == cur && lane > last), hi = __builtin_amdgcn_ballot_w64(par[1] == cur && lane + 64 > last);
      if (!(lo | hi)) return false;
      const int i = lo ? __builtin_ctzll(lo) : 64 + __builtin_ctzll(hi);
      last = i;
      const double qv = a.q ? value_of(node_q, i) : 1.0;
      double left = value_of(node_p, i);
      if (a.q) left = Residual{a.p, a.q, subs, sm_total, sm_out}.at(left, qv, 0);
      if (value_of(node_u, i) * total * qv < left) {
        cur = i; subs = 0; total = 1.0;
        if (lane == 0) sm_path[depth] = i;
        ++depth;
      } else if (a.q) {
        if (lane == 0) sm_total[subs] = total;
        ++subs;
        return true;
      } else {
        const double mass = total - left;
        if (mass > 0.0) {
          const int x = int_of(tok, i);
          if (lane == 0) sm_out[subs] = x;
#pragma unroll
          for (int k = 0; k < 2; ++k) node_p[k] = par[k] == cur && tok[k] == x ? 0.0 : node_p[k];
          ++subs; total = mass;
        }
      }
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
  };
  const auto say = [&](bool more) {       // wave 0 to all: the residual to be summed, and whether the walk goes on after it
    if (t == 0) { sm_cur = cur; sm_subs = subs; sm_want = more; }
    __syncthreads();
  };
  if (wave == 0) { const bool more = walk(); say(more); } else __syncthreads();

  // this workgroup's part
  Residual r{row(a.p, a.p_stride, sm_cur), a.q ? row(a.q, a.q_stride, sm_cur) : nullptr, sm_subs, sm_total, sm_out};
  {
    const int lo = w0 * cl, hi = lo + cl < a.vocab ? lo + cl : a.vocab;
    const double s = wave_sum_f64(part_sum<PT>(r, lo, hi, t, WALK_THREADS));
    if (lane == 0) sm_wave[wave] = s;
    __syncthreads();
    if (t == 0) {
      double x = 0.0;
      for (int w = 0; w < WALK_WAVES; ++w) x += sm_wave[w];
      __hip_atomic_store(&a.part[b * WALK_MAX_PARTS + w0], x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sm_last = __hip_atomic_fetch_add(&a.arrived[b], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == a.W - 1;
    }
    __syncthreads();
    if (!sm_last) return;
    if (t < a.W) sm_part[t] = __hip_atomic_load(&a.part[b * WALK_MAX_PARTS + t], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (t == 0) __hip_atomic_store(&a.arrived[b], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
  }

  // the last workgroup: on with the walk; residuals that are still to be summed it takes alone, a wave per part
  const auto all_parts = [&] {
    r = Residual{row(a.p, a.p_stride, sm_cur), a.q ? row(a.q, a.q_stride, sm_cur) : nullptr, sm_subs, sm_total, sm_out};
    for (int w = wave; w < a.W; w += WALK_WAVES) {
      const int lo = w * cl, hi = lo + cl < a.vocab ? lo + cl : a.vocab;
      const double s = wave_sum_f64(part_sum<PT>(r, lo, hi, lane, 64));
      if (lane == 0) sm_part[w] = s;
    }
    __syncthreads();
  };
  while (sm_want) {                                         // (a rejection each: at most n - 1 times)
    double mass = 0.0;
    for (int w = 0; w < a.W; ++w) mass += sm_part[w];
    const bool none = !(mass > 0.0);                        // nothing left (rounded inputs): what was there stays
    const int cur0 = sm_cur, subs0 = sm_subs;
    __syncthreads();
    if (wave == 0) {
      if (none) --subs; else total = mass;
      const bool more = walk();
      say(more);
    } else __syncthreads();
    if (none || sm_cur != cur0 || sm_subs != subs0) all_parts();
  }

  // the draw: the part, the thread's run of it, the element where the running sum passes u_draw times the whole
  if (t == 0) {
    double sum = 0.0, run = 0.0;
    for (int w = 0; w < a.W; ++w) sum += sm_part[w];
    const double at = (double)a.u_draw[b] * sum;
    int c = -1;
    for (int w = 0; w < a.W && c < 0; ++w) { if (run + sm_part[w] > at) c = w; else run += sm_part[w]; }
    if (c < 0)                                              // rounding at the very end: the last part that has anything
      for (int w = a.W - 1; w >= 0 && c < 0; --w) if (sm_part[w] > 0.0) { c = w; run = -INFINITY; }
    sm_chunk = c; sm_base = at - run; sm_token = -1;
  }
  __syncthreads();
  const int chunk = sm_chunk;
  if (chunk >= 0) {
    const int lo = chunk * cl, hi = lo + cl < a.vocab ? lo + cl : a.vocab, per = (cl + WALK_THREADS - 1) / WALK_THREADS;
    const int x0 = lo + t * per, x1 = x0 + per < hi ? x0 + per : hi;
    double own = 0.0;
    int top = -1;
    for (int x = x0; x < x1; ++x) {
      const double v = r.at(prob<PT>(r.p, x), r.q ? prob<PT>(r.q, x) : 0.0, x);
      own += v;
      if (v > 0.0) top = x;
    }
    double inc = own;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) { const double y = __shfl_up(inc, k); if (lane >= k) inc += y; }
    if (lane == 63) sm_wave[wave] = inc;
    __syncthreads();
    for (int w = 0; w < wave; ++w) inc += sm_wave[w];
    // the lowest thread whose running sum passes: within it the element, at the latest its last one that is not 0
    __shared__ int sm_first, sm_top;
    if (t == 0) { sm_first = WALK_THREADS; sm_top = -1; }
    __syncthreads();
    if (top >= 0) {
      if (inc > sm_base) atomicMin(&sm_first, t);
      atomicMax(&sm_top, top);
    }
    __syncthreads();
    if (t == sm_first) {
      double run = inc - own;
      int token = top;
      for (int x = x0; x <= top; ++x) {
        const double v = r.at(prob<PT>(r.p, x), r.q ? prob<PT>(r.q, x) : 0.0, x);
        run += v;
        if (v > 0.0 && run > sm_base) { token = x; break; }
      }
      sm_token = token;
    }
    __syncthreads();
    if (t == 0 && sm_token < 0) sm_token = sm_top;
    __syncthreads();
  }
  if (t < n) a.path[b * n + t] = sm_path[t];
  if (t == 0) {
    a.n_path[b] = depth;                                    // (thread 0 is of wave 0)
    a.next[b] = sm_token >= 0 ? sm_token : a.vocab - 1;     // no probability anywhere: the last one
  }
}

__global__ void k_walk_init(int* arrived, int B) {
  for (int i = threadIdx.x; i < B; i += blockDim.x) arrived[i] = 0;
}

// ---- the kept path -----------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(TREE_MAX) void k_accept_check(DevView v, int base, int n, const int* path, int n_path, int* info) {
  __shared__ int sm_path[TREE_MAX], sm_tier[TREE_MAX];
  const int b = blockIdx.x, t = threadIdx.x;
  sm_path[t] = t < n_path ? path[(size_t)b * n_path + t] : -1;
  sm_tier[t] = t < n ? v.tier[(size_t)b * v.Nmax + base + t] : 3;
  __syncthreads();
  if (t != 0) return;
  int kept = 0, slots = 0, before = -1;
  bool bad = false;
  for (int j = 0; j < n_path && sm_path[j] != -1; ++j) {
    const int i = sm_path[j];
    if (i <= before || i >= n || sm_tier[i] != 0) { bad = true; break; }   // nodes come after their parents
    before = i;
    ++kept;
  }
  for (int i = 0; i < n; ++i) slots += sm_tier[i] == 0;
  info[2 * b] = bad ? -1 : kept;
  info[2 * b + 1] = slots;
}

__global__ __launch_bounds__(TREE_MAX) void k_accept(DevView v, int base, int n, int keep, const int* path, int n_path, const int* info) {
  __shared__ int sm_path[TREE_MAX], sm_loc[TREE_MAX], sm_free[TREE_MAX];
  __shared__ float sm_score[TREE_MAX];
  const int b = blockIdx.x, t = threadIdx.x, kept = info[2 * b], slots = info[2 * b + 1];
  int* cnt = v.cnt + b * CNT_N;
  const int nfree = cnt[C_FREE0], nF = cnt[C_NF], n0 = cnt[C_N0], n3 = cnt[C_N3];
  const size_t o = (size_t)b * v.Nmax;
  const int p = base + t;
  sm_path[t] = t < kept ? path[(size_t)b * n_path + t] : -1;
  sm_loc[t] = t < n ? v.loc[o + p] : -1;
  sm_score[t] = t < n ? v.score[o + p] : 0.f;
  sm_free[t] = t < n && v.tier[o + p] == 0;
  __syncthreads();
  if (t < kept) sm_free[sm_path[t]] = 0;
  __syncthreads();
  // the others' slots go back on the stack, the last node's first
  if (t < n && sm_free[t]) {
    int rank = 0;
    for (int i = t + 1; i < n; ++i) rank += sm_free[i];
    if (nfree + rank < v.cap0) v.free0[(size_t)b * v.cap0 + nfree + rank] = sm_loc[t];
  }
  if (t < n) {
    const bool live = t < kept;
    const int loc = live ? sm_loc[sm_path[t]] : -1;
    v.tier[o + p] = live || t >= keep ? 0 : 3;
    v.loc[o + p] = loc; v.hloc[o + p] = -1;
    v.score[o + p] = live ? sm_score[sm_path[t]] : 0.f;
    if (live) {
      const int e = nF - slots + t;
      v.f_pos[o + e] = p; v.f_loc[o + e] = loc; v.f_loc_old[o + e] = loc;
      v.idx[o + n0 - slots + t] = p;
    } else if (t < keep) {
      v.idx[((size_t)3 * v.B + b) * v.Nmax + n3 - (n - slots) + (t - kept)] = p;
    }
  }
  if (t == 0) {
    cnt[C_FREE0] = nfree + slots - kept; cnt[C_NF] = nF - slots + kept; cnt[C_N0] = n0 - slots + kept;
    cnt[C_N3] = n3 - (n - slots) + (keep - kept); cnt[C_LEN] = base + keep;
  }
}

// value-row norms go with their rows: grid (kv heads, B, layers)
__global__ __launch_bounds__(TREE_MAX) void k_accept_norms(DevView v, int base, const int* path, int n_path, const int* info) {
  const int kvh = blockIdx.x, b = blockIdx.y, t = threadIdx.x;
  float* row = v.vnorm + (((size_t)blockIdx.z * v.B + b) * v.Hkv + kvh) * v.Nmax + base;
  const bool on = t < info[2 * b];
  const float x = on ? row[path[(size_t)b * n_path + t]] : 0.f;
  __syncthreads();
  if (on) row[t] = x;
}

// Parts of a row: as many as bring a sequence's row in fast, eight at the least (a workgroup alone has a wave for each)
int walk_parts(int B, int vocab, int cus) {
  int w = cus / (B > 0 ? B : 1);
  const int most = vocab / 2048;
  if (w > most) w = most;
  return w < WALK_WAVES ? WALK_WAVES : w > WALK_MAX_PARTS ? WALK_MAX_PARTS : w;
}
hipError_t launch_walk(const WalkArgs& a, int kt, hipStream_t st) {
  if (a.n < 1 || a.n > TREE_MAX || a.W < 1 || a.W > WALK_MAX_PARTS || a.B > 65535) return hipErrorInvalidValue;
  const dim3 grid(a.W, a.B);
  if (kt == KT_F32) hipLaunchKernelGGL((k_walk<KT_F32>), grid, dim3(WALK_THREADS), 0, st, a);
  else if (kt == KT_BF16) hipLaunchKernelGGL((k_walk<KT_BF16>), grid, dim3(WALK_THREADS), 0, st, a);
  else hipLaunchKernelGGL((k_walk<KT_F16>), grid, dim3(WALK_THREADS), 0, st, a);
  return hipGetLastError();
}
hipError_t launch_walk_init(int* arrived, int B, hipStream_t st) {
  hipLaunchKernelGGL(k_walk_init, dim3(1), dim3(256), 0, st, arrived, B);
  return hipGetLastError();
}
hipError_t launch_accept_check(const DevView& v, int base, int n, const int* path, int n_path, int* info, hipStream_t st) {
  hipLaunchKernelGGL(k_accept_check, dim3(v.B), dim3(TREE_MAX), 0, st, v, base, n, path, n_path, info);
  return hipGetLastError();
}
hipError_t launch_accept(const DevView& v, int base, int n, int keep, const int* path, int n_path, const int* info, hipStream_t st) {
  if (v.vnorm && keep > 0) hipLaunchKernelGGL(k_accept_norms, dim3(v.Hkv, v.B, v.L), dim3(TREE_MAX), 0, st, v, base, path, n_path, info);
  hipLaunchKernelGGL(k_accept, dim3(v.B), dim3(TREE_MAX), 0, st, v, base, n, keep, path, n_path, info);
  return hipGetLastError();
}

}  // namespace tkv
