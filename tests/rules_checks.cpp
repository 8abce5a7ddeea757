// Checks of a trace's rules (csrc/op_checks.cpp) on the CPU, built with
// AddressSanitizer and UndefinedBehaviorSanitizer by tests/test_rules_checks.py.
#include <cstdio>
#include <vector>

#include "op_checks.h"

static int g_fail = 0;
#define CHECK(cond)                                                          \
  do {                                                                       \
    if (!(cond)) {                                                           \
      std::fprintf(stderr, "%s:%d: CHECK failed: %s\n", __FILE__, __LINE__, #cond); \
      ++g_fail;                                                              \
    }                                                                        \
  } while (0)

static jet_trace_rules plain() {
  jet_trace_rules r{};
  r.repetition = 1.0f;
  return r;
}
static bool refused(const jet_trace_rules &r, int32_t n_q, int32_t n_steps, int64_t vocab = 40) {
  const jet::Status s = jet::check_rules(&r, n_q, n_steps, vocab);
  return !s && s.code == JET_E_INVALID;
}

static void check_mask_indices() {
  const uint32_t masks[4] = {1, 0, 0, 1};  // two masks of two words
  std::vector<int32_t> index(6, -1);
  jet_trace_rules r = plain();
  CHECK(!refused(r, 2, 3));
  // none without masks
  r.mask_index = index.data();
  CHECK(!refused(r, 2, 3));
  index[5] = 0;
  CHECK(refused(r, 2, 3));
  CHECK(!refused(r, 1, 5));  // (not its step)
  r.masks = masks;           // an empty list of masks has none either
  CHECK(refused(r, 2, 3));
  r.n_masks = 2;
  CHECK(!refused(r, 2, 3));
  index[0] = 2;
  CHECK(refused(r, 2, 3));
  index[0] = 1;
  CHECK(!refused(r, 2, 3));
  r.mask_index = nullptr;  // masks without an index
  CHECK(refused(r, 2, 3));
}

// Contexts are held in rows as long as the longest: refused before anything is
// allocated for them.
static void check_context_sizes() {
  const int32_t n_q = 1025;
  std::vector<int32_t> tokens((1 << 20) - 1, 3);
  std::vector<int64_t> offsets(n_q + 1, (int64_t)tokens.size());
  offsets[0] = 0;
  jet_trace_rules r = plain();
  r.context_offsets = offsets.data();
  r.context_tokens = tokens.data();
  CHECK(refused(r, n_q, 1));       // 1025 2^20
  CHECK(!refused(r, n_q - 1, 1));  // 2^30
  CHECK(refused(r, n_q - 1, 2));
  for (int64_t &o : offsets) o = o < 1000 ? o : 1000;
  CHECK(!refused(r, n_q, 1));
}

int main() {
  check_mask_indices();
  check_context_sizes();
  std::printf("%d failure(s)\n", g_fail);
  return g_fail != 0;
}
