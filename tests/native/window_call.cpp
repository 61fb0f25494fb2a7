// Makes one call of the metadata builder of dlfp_cache.h and prints its result, for
// tests/test_native_window_calls.py.  Built with a host compiler and its sanitizers.
// Pages that a row sees or that hold new tokens are block 0 of the pool, the others -1.
//
// usage: window_call HQ HKV WINDOW SINKS DECODE_SPLIT PREFILL_SPLIT TARGET_UNITS TILE
//                    {Q_LEN KV_LEN}...        (WINDOW 0: none)
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "dlfp_cache.h"

int main(int argc, char** argv) {
  if (argc < 9) return 2;
  auto arg = [&](int i) { return (int32_t)std::atoll(argv[i]); };
  const dlfp_dims dims = {arg(1), arg(2), 128, 16};
  const dlfp_window w = {arg(3), arg(4)};
  const dlfp_tuning tn = {arg(5), arg(6), arg(7), arg(8), 0, 0};
  const int n = (argc - 9) / 2;
  std::vector<int32_t> q, kv;
  int64_t most = 1;
  for (int s = 0; s < n; ++s) {
    q.push_back(arg(9 + 2 * s));
    kv.push_back(arg(10 + 2 * s));
    most = std::max(most, ((int64_t)kv[s] + 15) / 16);
  }
  std::vector<int32_t> table((size_t)(n * most), -1);
  for (int s = 0; s < n; ++s)
    for (int64_t p = 0; 16 * p < kv[s]; ++p) {
      // The page's last key against the window of the first new token; its first
      // against the sinks.
      const int64_t last = std::min<int64_t>(16 * p + 15, kv[s] - 1), pos = (int64_t)kv[s] - q[s];
      if (!w.window || pos - last < w.window || 16 * p < w.sinks) table[(size_t)(s * most + p)] = 0;
    }
  dlfp_meta m = {};
  auto call = [&] {
    return dlfp_build_window_meta(&dims, &tn, w.window ? &w : nullptr, n, q.data(), kv.data(),
                                  table.data(), (int32_t)most, 1, &m);
  };
  int st = call();
  std::vector<int32_t> cu, pos, slots, work;
  if (st == DLFP_ENOSPC) {
    cu.resize(m.num_seqs + 1), pos.resize(m.num_seqs), slots.resize(m.num_tokens);
    work.resize((size_t)m.num_units * DLFP_WORK_INTS);
    m.cu_q = cu.data(), m.q_pos0 = pos.data(), m.slot_mapping = slots.data(), m.work = work.data();
    m.cap_seqs = m.num_seqs, m.cap_tokens = m.num_tokens, m.cap_work = m.num_units;
    st = call();
  }
  std::printf("{\"status\":%d,\"prefill\":%d,\"groups\":%d,\"workspace\":%lld,\"units\":[", st,
              m.num_prefill_units, m.num_groups, (long long)m.workspace_bytes);
  for (int i = 0; st == DLFP_OK && i < m.num_units; ++i) {
    std::printf(i ? ",[" : "[");
    for (int f = 0; f < DLFP_WORK_INTS; ++f)
      std::printf(f ? ",%d" : "%d", work[(size_t)i * DLFP_WORK_INTS + f]);
    std::printf("]");
  }
  std::printf("]}\n");
  return 0;
}
