// The host code of drafted trees on a machine without a GPU: the stand-in for the HIP runtime is that of fake_runtime_check.cpp, whose
// scenarios stay out; launches of the tree kernels are compared with the memory alive.
#include <hip/hip_runtime.h>

#define main other_main
#define hipLaunchKernel fake_launch
#include "fake_runtime_check.cpp"
#undef hipLaunchKernel
#undef main

#include "../../paper_2605_09490_amd/csrc/tree.h"

static std::vector<tkv::TreeArgs> g_trees;
static std::vector<tkv::TreeScoreArgs> g_scores;
static std::vector<tkv::WalkArgs> g_walks;
static std::string g_order;                         // a: attention, m: merge, s: scores, g: gain, w: walk, c: check, k: kept path, n: norms

extern "C" hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t st) {
  const std::string& k = g_kernels.at(f);
  const auto is = [&](const char* n) { return k.find(n) != std::string::npos; };
  CHECK(grid.x >= 1 && grid.y >= 1 && grid.y <= 65535 && grid.z >= 1 && grid.z <= 65535);
  if (is("k_tree_attend") || is("k_tree_merge")) {
    const tkv::TreeArgs& a = *(const tkv::TreeArgs*)args[0];
    const size_t D = k.find("ILi128E") != std::string::npos ? 128 : 64, pairs = (size_t)a.B * a.Hkv;
    CHECK(a.C == a.n * a.G && a.S >= 1 && a.groups >= 1);
    if (a.S > 1) CHECK(inside(a.part_ml, pairs * a.S * 2 * a.C * 4) && inside(a.part_o, pairs * a.S * a.C * D * 4));
    CHECK(a.stat_stride >= a.C && inside(a.stat, pairs * a.stat_stride * 8) && inside(a.here, (size_t)a.B * a.n * 4));
    if (is("k_tree_attend")) { CHECK(grid.x >= pairs * a.S * a.groups && grid.x % 8 == 0); g_trees.push_back(a); g_order += 'a'; }
    else { CHECK(a.S > 1 && grid.x * 16 >= (unsigned)a.C && grid.y == pairs); g_order += 'm'; }
    return hipSuccess;
  }
  if (is("k_tree_scores") || is("k_tree_gain")) {
    const tkv::TreeScoreArgs& a = *(const tkv::TreeScoreArgs*)args[0];
    CHECK(a.stride >= a.Nmax + 32 && inside(a.gain, (size_t)a.layers * a.B * a.stride * 4) && inside(a.score, (size_t)a.B * a.Nmax * 4));
    CHECK(inside(a.stat, (size_t)a.layers * a.B * a.Hkv * a.stat_stride * 8) && inside(a.kept, (size_t)a.B * 8));
    if (is("k_tree_scores")) { g_scores.push_back(a); g_order += 's'; } else g_order += 'g';
    return hipSuccess;
  }
  if (is("k_walk_init")) { CHECK(inside(*(int**)args[0], *(int*)args[1] * 4)); return hipSuccess; }
  if (is("k_walk")) {
    const tkv::WalkArgs& a = *(const tkv::WalkArgs*)args[0];
    CHECK((int)grid.x == a.W && (int)grid.y == a.B && a.W >= 1 && a.W <= tkv::WALK_MAX_PARTS);
    CHECK(inside(a.part, (size_t)a.B * tkv::WALK_MAX_PARTS * 8) && inside(a.arrived, (size_t)a.B * 4));
    g_walks.push_back(a); g_order += 'w';
    return hipSuccess;
  }
  if (is("k_accept_check")) g_order += 'c';
  else if (is("k_accept_norms")) g_order += 'n';
  else if (is("k_accept")) g_order += 'k';
  return fake_launch(f, grid, block, args, lds, st);
}

// Pinned memory handed out by the test: the runtime's copies copy nothing, so what the kernels would have counted is put there.
static std::vector<std::pair<void*, size_t>> g_pinned;
static std::vector<int> g_first;                    // the counts of a cache's first accept
static void* take_pinned(size_t n, void*) {
  g_pinned.push_back({std::calloc(n, 1), n});
  if (n == g_first.size() * 4) std::memcpy(g_pinned.back().first, g_first.data(), n);
  return g_pinned.back().first;
}
static void drop_pinned(void* p, void*) { std::free(p); }
static void counts(const tkv_config& cfg, const std::vector<int>& v) {      // {kept, slots} of every sequence
  CHECK(g_pinned.back().second == (size_t)cfg.batch * 8 && v.size() * 4 == g_pinned.back().second);
  std::memcpy(g_pinned.back().first, v.data(), g_pinned.back().second);
}
static const int32_t* const INTS = (const int32_t*)DATA;

static tkv_tree_walk a_walk(int n, int vocab) {
  tkv_tree_walk w;
  std::memset(&w, 0, sizeof w);
  w.parents = w.tokens = INTS; w.p = DATA; w.u_accept = w.u_draw = (const float*)DATA;
  w.path = w.n_path = w.next = (int32_t*)DATA;
  w.n_tree = n; w.vocab = vocab; w.p_stride = w.q_stride = vocab; w.prob_dtype = TKV_F32;
  return w;
}

// Every refusal comes before any launch, and leaves the cache as it was.
static void refusals() {
  tkv_config cfg = config(2, 2, 10, 2, 128, 100);
  tkv_cache* c = nullptr;
  CHECK(tkv_create(&cfg, &c) == TKV_OK);
  g_order.clear();
  int32_t kept = 7;
  const auto refused = [&](tkv_status want, tkv_status got) {
    if (want != got || !g_order.empty()) std::printf("%d, not %d: %s (%s)\n", got, want, c ? tkv_last_error(c) : "", g_order.c_str());
    CHECK(want == got && g_order.empty() && hipGetLastError() == hipSuccess);
  };
  CHECK(tkv_attend_tree(nullptr, 0, DATA, INTS, 1, DATA, STREAM) == TKV_EINVAL && tkv_verify_tree(nullptr, nullptr, STREAM) == TKV_EINVAL);
  CHECK(tkv_accept_tree(nullptr, 1, nullptr, 0, nullptr, &kept, STREAM) == TKV_EINVAL && tkv_commit_tree(nullptr, nullptr, nullptr, &kept, STREAM) == TKV_EINVAL);
  refused(TKV_ESTATE, tkv_attend_tree(c, 0, DATA, INTS, 1, DATA, STREAM));              // an empty cache
  refused(TKV_ESTATE, tkv_accept_tree(c, 1, nullptr, 0, nullptr, &kept, STREAM));
  CHECK(kept == 0);
  fill(c, cfg, 20);
  refused(TKV_EINVAL, tkv_attend_tree(c, -1, DATA, INTS, 1, DATA, STREAM));
  refused(TKV_EINVAL, tkv_attend_tree(c, 2, DATA, INTS, 1, DATA, STREAM));
  refused(TKV_EINVAL, tkv_attend_tree(c, 0, nullptr, INTS, 1, DATA, STREAM));
  refused(TKV_EINVAL, tkv_attend_tree(c, 0, DATA, nullptr, 1, DATA, STREAM));
  refused(TKV_EINVAL, tkv_attend_tree(c, 0, DATA, INTS, 1, nullptr, STREAM));
  refused(TKV_EINVAL, tkv_attend_tree(c, 0, DATA, INTS, 0, DATA, STREAM));
  refused(TKV_EINVAL, tkv_attend_tree(c, 0, DATA, INTS, 129, DATA, STREAM));
  refused(TKV_ESTATE, tkv_attend_tree(c, 0, DATA, INTS, 21, DATA, STREAM));
  refused(TKV_EINVAL, tkv_accept_tree(c, 0, nullptr, 0, nullptr, &kept, STREAM));
  refused(TKV_EINVAL, tkv_accept_tree(c, 129, nullptr, 0, nullptr, &kept, STREAM));
  refused(TKV_EINVAL, tkv_accept_tree(c, 4, nullptr, 2, nullptr, &kept, STREAM));
  refused(TKV_EINVAL, tkv_accept_tree(c, 4, INTS, -1, nullptr, &kept, STREAM));
  refused(TKV_EINVAL, tkv_accept_tree(c, 4, INTS, 129, nullptr, &kept, STREAM));
  refused(TKV_ESTATE, tkv_accept_tree(c, 21, nullptr, 0, nullptr, &kept, STREAM));
  refused(TKV_ESTATE, tkv_accept_tree(c, 4, INTS, 4, DATA, &kept, STREAM));               // no layer has been attended
  OK(tkv_append(c, 0, DATA, DATA, 1, STREAM));
  refused(TKV_ESTATE, tkv_accept_tree(c, 4, INTS, 4, nullptr, &kept, STREAM));             // layers differ
  refused(TKV_ESTATE, tkv_attend_tree(c, 1, DATA, INTS, 1, DATA, STREAM));
  OK(tkv_append(c, 1, DATA, DATA, 1, STREAM));
  const tkv_policy pol{500000, 300000, 200000, 0, 0};
  OK(tkv_classify(c, &pol, STREAM));
  refused(TKV_ESTATE, tkv_accept_tree(c, 4, INTS, 4, nullptr, &kept, STREAM));             // a plan is pending
  CHECK(tkv_layer_length(c, 0) == 21 && tkv_layer_length(c, 1) == 21);
  // the walk's arguments
  tkv_tree_walk w = a_walk(8, 1000);
  refused(TKV_EINVAL, tkv_verify_tree(c, nullptr, STREAM));
  const void** const fields[] = {(const void**)&w.parents, (const void**)&w.tokens, &w.p, (const void**)&w.u_accept, (const void**)&w.u_draw,
                                 (const void**)&w.path, (const void**)&w.n_path, (const void**)&w.next};
  for (auto f : fields) { const void* was = *f; *f = nullptr; refused(TKV_EINVAL, tkv_verify_tree(c, &w, STREAM)); *f = was; }
  const struct { int n, v, t; int64_t ps, qs; bool q; } bad[] = {{0, 9, 0, 9, 9, false}, {129, 9, 0, 9, 9, false}, {4, 0, 0, 9, 9, false}, {4, 9, 3, 9, 9, false}, {4, 9, -1, 9, 9, false},
                                                                {4, 9, 0, 8, 9, false}, {4, 9, 0, 9, 8, true}, {4, (1 << 30) + 1, 0, (int64_t)1 << 31, 0, false}};
  for (auto& b : bad) {
    tkv_tree_walk x = a_walk(b.n, b.v);
    x.prob_dtype = b.t; x.p_stride = b.ps; x.q_stride = b.qs; x.q = b.q ? DATA : nullptr;
    refused(TKV_EINVAL, tkv_verify_tree(c, &x, STREAM));
    refused(TKV_EINVAL, tkv_commit_tree(c, &x, DATA, &kept, STREAM));
  }
  tkv_destroy(c);
  for (int k = 0; k < 3; ++k) {
    tkv_config other = config(2, 2, 10, 2, 128, 100);
    if (k == 0) other.prefetch_mode = TKV_PREFETCH_STREAM;
    else other.scorer = k == 1 ? TKV_SCORE_REDUNDANCY : TKV_SCORE_COMBINED;
    CHECK(tkv_create(&other, &c) == TKV_OK);
    fill(c, other, 20);
    refused(TKV_EINVAL, tkv_attend_tree(c, 0, DATA, INTS, 4, DATA, STREAM));
    refused(TKV_EINVAL, tkv_accept_tree(c, 4, nullptr, 0, nullptr, &kept, STREAM));
    OK(tkv_verify_tree(c, &w, STREAM));                    // (needs none of it)
    g_order.clear();
    tkv_destroy(c);
  }
}

// Shapes and tree sizes: partials, statistics and counts lie in memory that is alive; only the first call, and the first of a larger
// class of sizes, allocates.
static void scratch() {
  const int shapes[][6] = {{3, 1, 28, 4, 128, 1500}, {2, 3, 10, 2, 128, 700}, {4, 8, 40, 8, 128, 4200}, {1, 64, 28, 4, 128, 16500}, {2, 130, 4, 2, 64, 400}, {2, 2, 128, 128, 64, 9000},
                           {1, 1, 8, 1, 64, 70000}};
  for (auto& s : shapes)
    for (int kt : {TKV_F32, TKV_BF16, TKV_F16}) {
      tkv_config cfg = config(s[0], s[1], s[2], s[3], s[4], s[5]);
      cfg.kv_dtype = kt; cfg.scorer = kt == TKV_F16 ? TKV_SCORE_VATP : TKV_SCORE_ATTENTION;
      cfg.pin_alloc = take_pinned; cfg.pin_free = drop_pinned;
      tkv_cache* c = nullptr;
      CHECK(tkv_create(&cfg, &c) == TKV_OK);
      const int first = s[5] < 300 ? s[5] - 140 : s[5] - 300;
      fill(c, cfg, first);
      int cap = 0;
      for (int n : {1, 16, 3, 17, 32, 64, 33, 65, 128, 128, 2}) {
        fill(c, cfg, n);
        g_log.clear(); g_order.clear();
        for (int l = 0; l < s[0]; ++l) OK(tkv_attend_tree(c, l, DATA, INTS, n, DATA, STREAM));
        const bool grows = n > cap;
        while (cap < n) cap = cap ? cap * 2 : 16;
        CHECK((g_log.find('A') != std::string::npos) == grows && g_trees.back().n == n);
        // split or not, every layer is attended, and joined where it is
        CHECK(g_order.size() == (size_t)s[0] * (g_trees.back().S > 1 ? 2 : 1));
        int32_t kept = -1;
        g_log.clear();
        if (n == 1) {                                       // the first accept takes its memory; the counts of the next ones go there
          OK(tkv_accept_tree(c, n, nullptr, 0, nullptr, &kept, STREAM));
          CHECK(kept == 0 && tkv_layer_length(c, 0) == first);
          fill(c, cfg, n);
          for (int l = 0; l < s[0]; ++l) OK(tkv_attend_tree(c, l, DATA, INTS, n, DATA, STREAM));
        }
        std::vector<int> v;
        for (int b = 0; b < s[1]; ++b) { v.push_back(1); v.push_back(n); }
        counts(cfg, v);
        g_scores.clear();
        OK(tkv_accept_tree(c, n, INTS, n, DATA, &kept, STREAM));
        CHECK(kept == 1 && tkv_layer_length(c, 0) == first + 1);
        int layers = 0;
        for (auto& x : g_scores) { CHECK((x.vnorm != nullptr) == (kt == TKV_F16)); layers += x.layers; }
        CHECK(layers == s[0]);
        for (auto& x : v) x = x == 1 ? 0 : 1;               // and that one back
        for (int b = 0; b < s[1]; ++b) { v[2 * b] = 0; v[2 * b + 1] = 1; }
        counts(cfg, v);
        OK(tkv_accept_tree(c, 1, nullptr, 0, nullptr, &kept, STREAM));
        CHECK(kept == 0 && tkv_layer_length(c, 0) == first);
      }
      tkv_tree_walk w = a_walk(64, 50000);
      for (int i = 0; i < 2; ++i) {
        g_log.clear();
        OK(tkv_verify_tree(c, &w, STREAM));
        CHECK((g_log.find('A') != std::string::npos) == (i == 0));
      }
      tkv_destroy(c);
      CHECK(g_mem.size() == 1);
      g_pinned.clear();
    }
}

// A refused allocation is an error without traces; the same call works once there is memory.
static void refused_scratch() {
  tkv_config cfg = config(2, 2, 28, 4, 128, 900);
  tkv_cache* c = nullptr;
  CHECK(tkv_create(&cfg, &c) == TKV_OK);
  fill(c, cfg, 800);
  tkv_tree_walk w = a_walk(20, 5000);
  int32_t kept = 0;
  for (int k = 0; k < 5; ++k) {
    g_allocs = 0; g_fail_at = k;
    const tkv_status s = tkv_attend_tree(c, 1, DATA, INTS, 20, DATA, STREAM);
    g_fail_at = -1;
    CHECK(s == (k < 4 ? TKV_ENOMEM : TKV_OK) && hipGetLastError() == hipSuccess);
  }
  for (int k = 0; k < 3; ++k) {
    g_allocs = 0; g_fail_at = k;
    const tkv_status s = tkv_verify_tree(c, &w, STREAM);
    g_fail_at = -1;
    CHECK(s == (k < 2 ? TKV_ENOMEM : TKV_OK) && hipGetLastError() == hipSuccess);
  }
  OK(tkv_attend_tree(c, 0, DATA, INTS, 20, DATA, STREAM));
  for (int k = 0; k < 4; ++k) {
    g_allocs = 0; g_fail_at = k;
    const tkv_status s = tkv_accept_tree(c, 20, INTS, 20, DATA, &kept, STREAM);
    g_fail_at = -1;
    CHECK(s == (k < 3 ? TKV_ENOMEM : TKV_OK) && hipGetLastError() == hipSuccess);
    CHECK(tkv_layer_length(c, 0) == (k < 3 ? 800 : 780));
  }
  tkv_destroy(c);
  CHECK(g_mem.size() == 1);
}

// Lengths, gaps and what they allow, from the counts that the device would report.
static void lengths_and_gaps() {
  tkv_config cfg = config(2, 2, 10, 2, 128, 60);
  cfg.pin_alloc = take_pinned; cfg.pin_free = drop_pinned;
  tkv_cache* c = nullptr;
  CHECK(tkv_create(&cfg, &c) == TKV_OK);
  fill(c, cfg, 10);
  int32_t kept = 0;
  g_first = {0, 2, 0, 2};
  OK(tkv_accept_tree(c, 2, nullptr, 0, nullptr, &kept, STREAM));   // (takes the counts' memory)
  g_first.clear();
  CHECK(tkv_layer_length(c, 0) == 8);
  fill(c, cfg, 8);
  counts(cfg, {3, 8, 1, 8});
  g_order.clear();
  OK(tkv_accept_tree(c, 8, INTS, 8, nullptr, &kept, STREAM));
  CHECK(kept == 3 && tkv_layer_length(c, 1) == 11 && g_order == "ck");
  // positions 9 and 10 are missing in the second sequence
  CHECK(tkv_attend_tree(c, 0, DATA, INTS, 1, DATA, STREAM) == TKV_ESTATE && tkv_attend_and_score_chunk(c, 0, DATA, DATA, 2, STREAM) == TKV_ESTATE);
  fill(c, cfg, 4);
  CHECK(tkv_attend_tree(c, 0, DATA, INTS, 5, DATA, STREAM) == TKV_ESTATE && tkv_attend_and_score_chunk(c, 0, DATA, DATA, 5, STREAM) == TKV_ESTATE);
  OK(tkv_attend_tree(c, 0, DATA, INTS, 4, DATA, STREAM));
  OK(tkv_attend_and_score_chunk(c, 0, DATA, DATA, 4, STREAM));
  tkv_stats st;
  OK(tkv_get_stats(c, &st));
  CHECK(st.tier_count[0] == 28 && st.tier_count[3] == 2);
  // back to before the gaps: nothing is missing any more
  counts(cfg, {0, 7, 0, 5});
  OK(tkv_accept_tree(c, 7, nullptr, 0, nullptr, &kept, STREAM));
  CHECK(kept == 0 && tkv_layer_length(c, 0) == 8);
  OK(tkv_get_stats(c, &st));
  CHECK(st.tier_count[0] == 16 && st.tier_count[3] == 0);
  fill(c, cfg, 3);
  OK(tkv_attend_tree(c, 0, DATA, INTS, 11, DATA, STREAM));
  // a path that the device finds wrong changes nothing
  counts(cfg, {2, 3, -1, 3});
  g_order.clear();
  CHECK(tkv_accept_tree(c, 3, INTS, 3, nullptr, &kept, STREAM) == TKV_EINVAL && kept == 0 && tkv_layer_length(c, 0) == 11 && g_order == "c");
  // slots: 49 more fit the pool, whatever came and went
  fill(c, cfg, 49);
  CHECK(tkv_append(c, 0, DATA, DATA, 1, STREAM) == TKV_ECAPACITY);
  // statistics belong to one tree at one length
  for (int l = 0; l < 2; ++l) OK(tkv_attend_tree(c, l, DATA, INTS, 4, DATA, STREAM));
  CHECK(tkv_accept_tree(c, 3, INTS, 3, DATA, &kept, STREAM) == TKV_ESTATE);
  OK(tkv_attend_tree(c, 1, DATA, INTS, 3, DATA, STREAM));
  CHECK(tkv_accept_tree(c, 4, INTS, 4, DATA, &kept, STREAM) == TKV_ESTATE);
  OK(tkv_attend_tree(c, 1, DATA, INTS, 4, DATA, STREAM));
  counts(cfg, {4, 4, 4, 4});
  g_order.clear();
  OK(tkv_accept_tree(c, 4, INTS, 4, DATA, &kept, STREAM));
  CHECK(g_order == "cksg" && kept == 4);
  CHECK(tkv_accept_tree(c, 4, INTS, 4, DATA, &kept, STREAM) == TKV_ESTATE);     // once
  tkv_destroy(c);
  g_pinned.clear();
}

int main(int argc, char** argv) {
  const std::string what = argc > 1 ? argv[1] : "";
  if (what == "refusals") refusals();
  else if (what == "scratch") scratch();
  else if (what == "refused_scratch") refused_scratch();
  else if (what == "lengths_and_gaps") lengths_and_gaps();
  else { std::printf("no scenario %s\n", what.c_str()); return 2; }
  std::printf("%s: ok\n", what.c_str());
  return 0;
}
