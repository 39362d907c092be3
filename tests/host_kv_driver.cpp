// Host-side driver for the sanitizer build of the attention block's host code (tests/test_kv_host_sanitized.py links it with
// csrc/mdbf_kv.hip and csrc/mdbf_kv_attn.hip, host parts only, under AddressSanitizer and UndefinedBehaviorSanitizer).  The HIP runtime's
// entry points are stand-ins here: a launch is recorded and goes nowhere, so calls of any size run over placeholder pointers.
// Every call's grid is compared with what its sizes ask for.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>

#include "mdbf.h"

struct Dim3 {
  uint32_t x, y, z;
};
struct Launch {
  Dim3 grid, block;
};
static std::vector<Launch> g_launches;
static Launch g_pushed;

namespace mdbf {
int hip_fail(int e) { return e ? MDBF_EHIP : MDBF_OK; }
}
extern "C" {
int hipGetLastError() { return 0; }
int hipLaunchKernel(const void*, Dim3 grid, Dim3 block, void**, size_t, void*) {
  g_launches.push_back({grid, block});
  return 0;
}
unsigned __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t, void*) {
  g_pushed = {grid, block};
  return 0;
}
int __hipPopCallConfiguration(Dim3* grid, Dim3* block, size_t* shared, void** stream) {
  *grid = g_pushed.grid, *block = g_pushed.block, *shared = 0, *stream = nullptr;
  return 0;
}
void** __hipRegisterFatBinary(const void*) {
  static void* handle;
  return &handle;
}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
void __hipUnregisterFatBinary(void**) {}
}

static void* const P = (void*)(uintptr_t)0x10000000;
static const size_t kHuge = (size_t)1 << 50;
static int g_fail = 0, g_cases = 0;

static void expect(bool ok, const char* what, long long a, long long b, long long c) {
  ++g_cases;
  if (ok) return;
  printf("FAIL %s (%lld, %lld, %lld)\n", what, a, b, c);
  ++g_fail;
}

static void tokens_in_and_out(int T, int heads, int d) {
  const mdbf_kv_t kv = {1000, heads, d, 256, MDBF_BF16};
  const int64_t row = (int64_t)heads * d;
  auto covers = [&](int most_units) {      // four tokens to a workgroup, all tokens and no more; the heads on the second dimension
    if (g_launches.size() != 1) return false;
    const Launch& l = g_launches[0];
    return (int64_t)l.grid.x * 4 >= T && ((int64_t)l.grid.x - 1) * 4 < T && l.grid.y >= 1 && (int)l.grid.y <= most_units && l.grid.z == 1;
  };
  for (int dt : {MDBF_F16, MDBF_BF16, MDBF_F32}) {
    g_launches.clear();
    expect(mdbf_kv_append(&kv, P, kHuge, P, row, P, row, dt, (const int64_t*)P, T, nullptr) == MDBF_OK && covers(2 * heads), "append", T, heads, d);
    g_launches.clear();
    expect(mdbf_kv_read(&kv, P, kHuge, (const int64_t*)P, T, P, row, P, row, dt, nullptr) == MDBF_OK && covers(1), "read", T, heads, d);
    const mdbf_rope_t rope = {heads, heads, d, d, 100, dt, MDBF_BF16, 0, 1e-6f};
    g_launches.clear();
    expect(mdbf_qk_norm_rope(&rope, P, row, P, row, nullptr, nullptr, (const float*)P, (const int32_t*)P, T, P, row, P, row, nullptr, nullptr, 0,
                             nullptr, 0, nullptr, nullptr) == MDBF_OK && covers(2 * heads), "norm and rotation", T, heads, d);
  }
}

static void slots(int requests, int T) {
  int32_t* const i = (int32_t*)P;
  g_launches.clear();
  expect(mdbf_kv_slots(requests, 16, i, i, i, 9, 9, i, 0x7fffffff, i, T, i, i, (int64_t*)P, i, i, i, nullptr) == MDBF_OK, "slots", requests, T, 0);
  int64_t workgroups = g_launches.size() == 2 ? g_launches[1].grid.x : 0;
  expect(g_launches.size() <= 2 && g_launches[0].grid.x == 1 && (workgroups == 0 || (workgroups * 1024 >= T && (workgroups - 1) * 1024 < T)),
         "slots' launches", requests, T, workgroups);
}

static void attention(int requests, int T, int q_heads, int kv_heads, int d, int max_fresh, int max_length, int window, uint32_t flags) {
  const mdbf_kv_t kv = {1000, kv_heads, d, 64, MDBF_F16};
  const mdbf_attn_t at = {q_heads, flags, window, max_fresh, max_length, 0.1f};
  const int64_t row = (int64_t)q_heads * d;
  size_t bytes = 0;
  expect(mdbf_kv_attention_workspace_bytes(&kv, &at, requests, T, &bytes) == MDBF_OK && bytes < (size_t)1 << 31, "workspace", requests, T, bytes);
  expect(*mdbf_kv_attention_kernel(&kv, &at, requests, T) != 0, "kernel", requests, T, max_fresh);
  g_launches.clear();
  const int st = mdbf_kv_attention(&kv, &at, P, kHuge, (const int32_t*)P, 9, 9, (const int32_t*)P, (const int32_t*)P, requests, P, row, T, P, row, P, bytes,
                                   nullptr);
  const bool shares = strstr(mdbf_kv_attention_kernel(&kv, &at, requests, T), "shares");
  expect(requests <= 0x70000000 || st == MDBF_EUNSUPPORTED, "requests that a kernel's loop cannot count", requests, T, st);
  if (st == MDBF_OK)
    expect(g_launches.size() == (shares ? 2u : 1u) && g_launches[0].grid.x >= 1 && g_launches[0].grid.x <= 0x7fffffffu, "attention's launches", requests, T,
           g_launches.size());
  else      // beyond what a launch's index or a row's number holds
    expect(st == MDBF_EUNSUPPORTED && g_launches.empty() && ((int64_t)T * (q_heads / kv_heads) > 0x70000000 || requests > 0x70000000 ||
           (int64_t)requests * kv_heads * ((int64_t)(max_fresh < T ? max_fresh : T) * (q_heads / kv_heads) / 16 + 1) > 0x7fffffff), "attention", requests, T, st);
}

int main() {
  const int sizes[] = {1, 2, 3, 4, 5, 1000, 1 << 20, (1 << 24) + 1, (1 << 30) - 1, 1 << 30, (1 << 30) + 1, 0x70000000, 0x7ffffffc, 0x7ffffffd, 0x7ffffffe, 0x7fffffff};
  for (int T : sizes)
    for (int heads : {1, 5, 65536})
      for (int d : {64, 128, 256}) tokens_in_and_out(T, heads, d);
  for (int n : sizes)
    for (int T : sizes) slots(n, T);
  for (int n : sizes)
    for (int T : sizes)
      for (int fresh : sizes)
        for (int length : {1, 1024, 1025, 200000, 0x7fffffff})
          for (int window : {0, 1, 1000, 0x7fffffff})
            for (uint32_t flags : {(uint32_t)MDBF_ATTN_CAUSAL, (uint32_t)(MDBF_ATTN_CAUSAL | MDBF_ATTN_EXACT_QUERIES)})
              for (int d : {64, 128, 256}) {
                attention(n, T, 8, 2, d, fresh, length, window, flags);
                if (d != 128) continue;
                attention(n, T, 65536, 1, d, fresh, length, window, flags);
                attention(n, T, 1, 1, d, fresh, length, window, flags);
              }
  printf("%d cases, %d failures\n", g_cases, g_fail);
  if (!g_fail) printf("ok\n");
  return g_fail != 0;
}
