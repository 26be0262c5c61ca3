// Host-side harness for tests/test_plan_host_kv8.py: plan_harness.cpp's lines for launches over the 8-bit cache,
// whose plans have prices and, with head_dim 256, a workgroup shape of their own.  Input and output as there; the
// input's v_transposed and ws_cap are read and have no meaning here.
#include "attn_bf16.hip"

#include <cstdio>
#include <vector>

namespace nexus {
hipError_t launch_attention_f32(const AttnLaunch &, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_attn_d128_dma(const AttnArgs &, const AttnPlan &, int, bool, hipStream_t) {
  return hipErrorNotSupported;
}
hipError_t launch_attn_d256_vt(const AttnArgs &, const AttnPlan &, int, bool, hipStream_t) {
  return hipErrorNotSupported;
}
}  // namespace nexus

int main() {
  using namespace nexus;
  int hq, hkv, d, vt, n;
  long long cap;
  while (scanf("%d %d %d %d %lld %d", &hq, &hkv, &d, &vt, &cap, &n) == 6) {
    std::vector<AttnSeq> seqs(n);
    int q = 0;
    for (AttnSeq &s : seqs) {
      long long np;
      if (scanf("%d %lld", &s.len, &np) != 2) return 1;
      s.n_past = np;
      s.q_start = q;
      q += s.len;
    }
    AttnLaunch p{};
    p.n_q_heads = hq;
    p.n_kv_heads = hkv;
    p.head_dim = d;
    p.is_bf16 = true;
    p.kv8 = true;
    p.n_seqs = n;
    p.seqs = seqs.data();
    static AttnPlan plan;
    if (!plan_attention(p, plan)) {
      printf("plan none\nend\n");
      continue;
    }
    printf("plan ok %d %d %d %d %zu\n", plan.units_per_head, plan.range_major, plan.qpw, plan.waves, plan.ws_bytes);
    for (int b = 0; b < n; ++b) {
      const SeqPlan &s = plan.seq[b];
      printf("seq %d %d %d %lld %d %d %d\n", b, s.q_start, s.len, (long long)s.n_past, s.n_tg, s.n_tasks,
             s.max_splits);
    }
    for (int u = 0; u < plan.units_per_head; ++u) {
      const UnitLoc l = locate_unit(plan, u);
      printf("unit %d %d %d %d %d %d %d %d\n", u, l.seq, l.w.tgrp, l.w.split, l.w.k_begin, l.w.split_keys,
             l.w.n_splits, group_splits(plan.seq[l.seq], l.w.tgrp));
    }
    printf("end\n");
  }
  return 0;
}
