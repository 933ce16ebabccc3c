// Host-only sanitizer driver of the 4-bit weights and the block residual (test infrastructure): argument checks at the
// ends of their ranges, the choice of kernels over random calls, and what is launched for them: every row once, fewer
// than 2^32 threads a launch, all parts of a workspace inside its size.  Built with ASan/UBSan against w4_stubs.cpp; run
// by tests/test_sanitizers_w4.py.  Exit status 0 = clean.
#include <stdint.h>
#include <stdio.h>

#include <random>

#include "flashnorm.h"
#include "w4_stub_record.h"

bool stub_backward = false;
static int failures = 0;
#define CHECK(cond)                                                                       \
  do {                                                                                    \
    if (!(cond) && ++failures <= 20) fprintf(stderr, "FAIL line %d: %s\n", __LINE__, #cond); \
  } while (0)

static void* P(uintptr_t x) { return reinterpret_cast<void*>(x); }
static float* PF(uintptr_t x) { return reinterpret_cast<float*>(x); }
static const uintptr_t GB = 1u << 30;
static const uintptr_t A = 1 * GB, W = uintptr_t(1) << 50, Y = uintptr_t(1) << 52, X = 8 * GB, R = uintptr_t(1) << 57, S = uintptr_t(1) << 56;

static void fresh() {
  stub_products.clear();
  stub_launches.clear();
}

static void check_threads() {
  for (const auto& l : stub_launches) {
    CHECK((uint64_t)l.grid.x * l.block.x < (uint64_t(1) << 32) && l.grid.x > 0 && l.grid.y > 0 && l.grid.y < 65536);
    CHECK(l.block.x <= 1024);
  }
}

static int log_uniform(std::mt19937_64& rng, double lo, double hi) {
  return (int)std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng));
}

static int product(int kind, int64_t M, int64_t K, int64_t N, int group, bool g, size_t ws_bytes) {
  void* ws = ws_bytes ? P(S) : nullptr;
  const int64_t cols = kind == 1 ? N / 2 : N, ldy = (cols + 7) / 8 * 8;
  const float* gp = g ? PF(X) : nullptr;
  if (kind == 0)
    return flashnorm_linear_w4(P(A), M, K, K, FN_BF16, gp, P(W), N, group, 1e-6f, nullptr, P(Y), ldy, FN_BF16, PF(R), ws, ws_bytes, nullptr);
  if (kind == 1)
    return flashnorm_glu_w4(P(A), M, K, K, FN_BF16, gp, P(W), cols, group, 1e-6f, P(Y), ldy, FN_BF16, ws, ws_bytes, nullptr);
  return rowscale_linear_w4(P(A), M, K, K, FN_BF16, P(W), N, group, PF(R), P(Y), ldy, FN_BF16, ws, ws_bytes, nullptr);
}

static void check_products(int64_t M, int64_t K, int64_t N, int group, int kind, bool g) {
  fresh();
  const int layout = kind == 1 ? FN_LAYOUT_GLU : FN_LAYOUT_LINEAR;
  if (!fold_weights_w4_size(K, N, layout, group)) return;
  const size_t need = flashnorm_w4_workspace_size(M, K, N, layout, group);
  CHECK(product(kind, M, K, N, group, g, need) == FN_OK);
  check_threads();
  const int64_t cols = kind == 1 ? N / 2 : N, ldy = (cols + 7) / 8 * 8;
  int64_t m = 0;
  size_t pass = 0;
  for (const auto& p : stub_products) {
    CHECK(p.y == (const char*)P(Y) + m * ldy * 2);
    CHECK(p.M > 0 && m + p.M <= M);
    if (p.many) {
      const char* ws = (const char*)P(S);
      const int64_t KP = (int64_t)p.KB * 128;
      CHECK((const char*)p.factor >= ws && (const char*)(p.factor + p.M) <= (const char*)p.a);
      CHECK((const char*)p.a + p.M * KP * 2 <= ws + need);
      CHECK(p.splits == 1 || ((const char*)p.partial >= (const char*)p.a + p.M * KP * 2 &&
                              (const char*)(p.partial + (int64_t)p.splits * p.M * p.NP) <= ws + need));
      CHECK(pass < stub_launches.size() && stub_launches[pass].grid.x == (unsigned)p.M);  // a workgroup for each row
      ++pass;
      CHECK(p.row_scale == (kind == 2 ? PF(R) + m : nullptr));
    } else {
      CHECK(p.a == (const char*)P(A) + m * K * 2);
      CHECK(kind == 2 ? p.row_scale == PF(R) + m : kind != 0 || p.inv_rms == PF(R) + m);
    }
    m += p.M;
  }
  CHECK(m == M && pass == stub_launches.size());
  if (need > 0 && !stub_products.empty() && stub_products[0].many) {
    fresh();
    CHECK(product(kind, M, K, N, group, g, 15) == FN_ERR_SIZE && stub_products.empty() && stub_launches.empty());
  }
}

static void check_plan(int64_t M, int64_t K, int64_t N, int group, bool glu, bool g) {
  const int KB = (int)fn::w4_blocks(K);
  const int64_t NP = fn::packed_cols(N, glu);
  const fn::W4Plan p = fn::w4_plan((int)M, (int)K, KB, (int)NP, glu, group, g);
  CHECK(p.splits >= 1 && p.splits <= 16 && (p.many || p.splits == 1));
  CHECK((int64_t)p.splits * p.kb_per_split >= KB && (int64_t)(p.splits - 1) * p.kb_per_split < KB);
  CHECK(!p.many || M > FN_W4_FEW_M);
  CHECK(fn::w4_workspace(p, M, KB, NP) <= fn::w4_workspace(M, K, NP, glu, group));
}

static void check_backward(int64_t M, int64_t K, int64_t T, int dt, bool post, bool pre, bool gate, bool sums) {
  fresh();
  const size_t need = flashnorm_block_residual_bwd_size(M, K, gate ? T : 0, dt);
  CHECK(need > 0);
  stub_backward = true;
  const uintptr_t big = uintptr_t(1) << 44;  // each operand has room of its own
  const int s = flashnorm_block_residual_bwd(
      P(big), K, P(2 * big), K, P(3 * big), K, pre ? P(4 * big) : nullptr, K, M, K, dt, post ? PF(X) : nullptr, 1e-6f,
      gate ? P(5 * big) : nullptr, K, T, 1.0f, 0.5f, pre ? PF(X + GB) : nullptr, 1e-6f, P(6 * big), K, P(7 * big), K,
      gate && sums ? P(8 * big) : nullptr, K, post && sums ? PF(R) : nullptr, pre && sums ? PF(R + GB) : nullptr, P(S), need,
      nullptr);
  stub_backward = false;
  CHECK(s == FN_OK);
  check_threads();
  if (M == 0 || stub_launches.empty()) return;
  // The parts that the units write: outputs themselves, or in the workspace, a row of K for each unit.
  const int64_t units = stub_launches[0].grid.x;
  for (const float* part : stub_launches[0].part) {
    if (!part || part == PF(R) || part == PF(R + GB)) continue;
    CHECK((const char*)part >= (const char*)P(S) && (const char*)(part + units * K) <= (const char*)P(S) + need);
  }
  CHECK(stub_launches.size() <= 2);
}

int main() {
  std::mt19937_64 rng(1);
  auto pick = [&](int n) { return (int)(rng() % n); };
  const int groups[] = {32, 64, 128};
  // Products: random calls, the most rows and columns that there may be, and every piece of theirs.
  for (int i = 0; i < 4000; ++i) {
    const int64_t M = log_uniform(rng, 1, i % 4 ? 4096 : 1 << 30), K = 8 * log_uniform(rng, 1, i % 3 ? 2048 : 1 << 18);
    const int64_t top = std::min<int64_t>(1 << 21, (int64_t(1) << 31) / K), N = log_uniform(rng, 2, (double)std::max<int64_t>(3, top)) / 2 * 2;
    const int group = groups[pick(3)], kind = pick(3);
    const bool g = kind != 2 && pick(2);
    if (!fold_weights_w4_size(K, N, kind == 1, group)) continue;
    check_plan(M, K, N, group, kind == 1, g);
    if ((double)M * (double)N < 1e12 && (double)M * (double)K < 1e12) check_products(M, K, N, group, kind, g);
  }
  for (int64_t M : {(int64_t(1) << 22) - 1, int64_t(1) << 22, (int64_t(1) << 22) + 37, int64_t(1) << 24, int64_t(1) << 30})
    for (int64_t K : {8, 8192, 8200, 40000})
      for (int64_t N : {2, 16, 46, 512})
        for (int kind = 0; kind < 3; ++kind) check_products(M, K, N, 64, kind, false);
  check_products(333, int64_t(1) << 21, 16, 128, 0, true);
  check_products(16, 8, 1 << 21, 128, 0, false);
  check_products(2000, 8, 1 << 21, 128, 0, false);
  fresh();
  CHECK(flashnorm_linear_w4(P(A), int64_t(1) << 30, 8, 8, FN_BF16, nullptr, P(W), 1 << 20, 32, 1e-6f, nullptr, P(Y), 1 << 20,
                            FN_BF16, nullptr, P(uintptr_t(1) << 60), size_t(1) << 59, nullptr) == FN_ERR_SIZE);
  CHECK(stub_products.empty() && stub_launches.empty());
  // Folds, packing and unpacking: the largest strides and weights.
  const int64_t far = (int64_t(1) << 40) - 1, wide = (int64_t(1) << 31) - 1;
  fresh();
  CHECK(fold_weights_w4(P(uintptr_t(1) << 32), far, wide, FN_F32, nullptr, 1 << 21, 1536, 0, 128, 1, P(A), nullptr) == FN_OK);
  CHECK(fold_weights_w4(P(W), 1, 1 << 21, FN_BF16, PF(X), 1 << 21, 1536, 0, 32, 0, P(A), nullptr) == FN_OK);
  CHECK(fold_weights_w4(P(W), 29000000, 1, FN_BF16, nullptr, 8, 29000000, 1, 128, 1, P(A), nullptr) == FN_OK);
  // The last element of the farthest view lies in the packed weight.
  const uintptr_t last = ((uint64_t)((1 << 21) - 1) * far + (uint64_t)1535 * wide) * 4;
  CHECK(fold_weights_w4(P(uintptr_t(1) << 32), far, wide, FN_F32, nullptr, 1 << 21, 1536, 0, 128, 1,
                        P(((uintptr_t(1) << 32) + last) & ~uintptr_t(15)), nullptr) == FN_ERR_ALIAS);
  CHECK(pack_weights_w4((const uint8_t*)P(W), far, PF(Y), far, (const uint8_t*)P(S), far, 1 << 21, 1536, 0, 32, P(A), nullptr) == FN_OK);
  CHECK(unpack_weights_w4(P(A), 1 << 21, 1536, 0, 32, PF(W), far, nullptr) == FN_OK);
  CHECK(stub_launches.size() >= 5);
  check_threads();
  // The block residual: random calls, gates from one per row to one for all, more rows than a card holds.
  for (int i = 0; i < 4000; ++i) {
    const int dt = pick(2) ? FN_BF16 : FN_F32, unit = dt == FN_BF16 ? 8 : 4;
    const int64_t M = i % 50 ? log_uniform(rng, 1, i % 3 ? 5000 : 1 << 24) : pick(2), K = unit * log_uniform(rng, 1, 16384 / unit);
    const int64_t T = pick(4) ? log_uniform(rng, 1, (double)std::max<int64_t>(2, 2 * M)) : pick(2) ? 1 : INT64_MAX;
    const bool gate = pick(2);
    check_backward(M, K, T, dt, pick(3), pick(3), gate, pick(4));
    fresh();
    const uintptr_t big = uintptr_t(1) << 44;
    CHECK(flashnorm_block_residual(P(big), K, P(2 * big), K, M, K, dt, PF(X), 1e-6f, gate ? P(3 * big) : nullptr, K, T, 1.0f, 1.0f,
                                   PF(X + GB), 1e-6f, P(2 * big), K, P(big), K, PF(R), nullptr) == FN_OK);
    check_threads();
    CHECK(stub_launches.size() == (M > 0));
  }
  if (failures) {
    fprintf(stderr, "%d check(s) failed\n", failures);
    return 1;
  }
  printf("4-bit and block residual driver: clean\n");
  return 0;
}
