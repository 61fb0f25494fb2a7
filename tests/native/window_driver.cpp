// Drives the metadata builder of dlfp_cache.h on seeded random inputs and prints
// every input and output as one JSON line per case, for tests/test_native_window.py
// to check against the definition.  Built with a host compiler and its sanitizers,
// so any out-of-bounds access or undefined operation aborts the run.
//
// usage: window_driver SEED CASES
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "dlfp_cache.h"

namespace {

uint64_t g_state;
uint64_t next_u64() {  // splitmix64
  uint64_t z = (g_state += 0x9E3779B97F4A7C15ull);
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
int64_t uniform(int64_t lo, int64_t hi) {  // inclusive
  return lo + (int64_t)(next_u64() % (uint64_t)(hi - lo + 1));
}

void print_array(const char* name, const std::vector<int32_t>& a) {
  std::printf("\"%s\":[", name);
  for (size_t i = 0; i < a.size(); ++i) std::printf(i ? ",%d" : "%d", a[i]);
  std::printf("],");
}

void one_case() {
  const int gs[] = {1, 2, 4, 8}, hkvs[] = {1, 2, 8};
  const int g = gs[uniform(0, 3)], hkv = hkvs[uniform(0, 2)];
  const dlfp_dims dims = {g * hkv, hkv, 128, 16};
  dlfp_tuning tn = {0, 0, 0, 0, 0, 0};
  if (uniform(0, 2) == 0) {
    tn.decode_split_tokens = (int32_t)(16 * uniform(0, 30));
    tn.prefill_split_tokens = (int32_t)(64 * uniform(0, 8));
    tn.target_units = (int32_t)uniform(0, 3000);
    tn.prefill_tile_tokens = (int32_t)uniform(0, 128 / g);
    tn.prefill_lead_units = (int32_t)uniform(-1, 40);
  }
  const int n = (int)uniform(0, 5);
  std::vector<int32_t> q, kv;
  int most = 1;
  for (int s = 0; s < n; ++s) {
    q.push_back(uniform(0, 1) ? 1 : (int32_t)uniform(1, 200));
    kv.push_back(q.back() + (int32_t)(uniform(0, 3) ? uniform(0, 900) : 0));
    most = kv.back() > 16 * most ? (kv.back() + 15) / 16 : most;
  }
  // A table of exactly the entries that the call may read.
  std::vector<int32_t> table((size_t)n * most);
  const int blocks = n * most + 1;
  for (size_t i = 0; i < table.size(); ++i) table[i] = (int32_t)i;
  const int32_t windows[] = {1, 2, 16, 17, 100, 640, INT32_MAX};
  const dlfp_window w = {windows[uniform(0, 6)], (int32_t)(uniform(0, 1) ? uniform(0, 70) : 0)};
  const bool masked = uniform(0, 2) != 0;
  dlfp_meta probe = {};
  int st = dlfp_build_window_meta(&dims, &tn, masked ? &w : nullptr, n, q.data(), kv.data(),
                                  table.data(), most, blocks, &probe);
  std::vector<int32_t> cu(probe.num_seqs + 1), pos(probe.num_seqs + 1), slots(probe.num_tokens),
      work((size_t)probe.num_units * DLFP_WORK_INTS);
  dlfp_meta m = {};
  m.cu_q = cu.data(), m.q_pos0 = pos.data(), m.slot_mapping = slots.data(), m.work = work.data();
  m.cap_seqs = probe.num_seqs, m.cap_tokens = probe.num_tokens, m.cap_work = probe.num_units;
  const int st2 = dlfp_build_window_meta(&dims, &tn, masked ? &w : nullptr, n, q.data(), kv.data(),
                                         table.data(), most, blocks, &m);
  std::printf("{\"probe\":%d,\"status\":%d,\"hq\":%d,\"hkv\":%d,\"window\":%d,\"sinks\":%d,", st, st2,
              g * hkv, hkv, masked ? w.window : 0, masked ? w.sinks : 0);
  print_array("q_len", q);
  print_array("kv_len", kv);
  print_array("cu_q", cu);
  print_array("slots", slots);
  print_array("work", work);
  std::printf("\"max_blocks\":%d,\"prefill\":%d,\"groups\":%d,\"workspace\":%lld}\n", most,
              m.num_prefill_units, m.num_groups, (long long)m.workspace_bytes);
}

void refusals() {
  const dlfp_dims dims = {8, 8, 128, 16};
  const int32_t q[] = {1}, kv[] = {40};
  const int32_t table[] = {0, 1, 2};
  dlfp_meta m = {};
  auto call = [&](const dlfp_dims* d, const dlfp_window* w, int n, const int32_t* ql, dlfp_meta* out) {
    return dlfp_build_window_meta(d, nullptr, w, n, ql, kv, table, 3, 3, out);
  };
  const dlfp_window bad = {0, 0}, worse = {4, -1};
  const dlfp_dims other = {8, 8, 64, 16};
  std::printf("{\"refused\":[%d,%d,%d,%d,%d,%d,%d]}\n", call(&dims, &bad, 1, q, &m),
              call(&dims, &worse, 1, q, &m), call(&dims, nullptr, -1, q, &m),
              call(&dims, nullptr, 1, nullptr, &m), call(&dims, nullptr, 1, q, nullptr),
              call(nullptr, nullptr, 1, q, &m), call(&other, nullptr, 1, q, &m));
}

}  // namespace

int main(int argc, char** argv) {
  if (argc != 3) return 2;
  g_state = (uint64_t)std::atoll(argv[1]);
  for (int i = std::atoi(argv[2]); i > 0; --i) one_case();
  refusals();
  return 0;
}
