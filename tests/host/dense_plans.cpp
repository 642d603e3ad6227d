// Launch plans of dense attention calls: "B H H_kv N N_k d dtype left right" per
// line in, "few tiles splits qtiles qsplits ktiles ksplits" per line out.
#include <cstdio>

#include "../../paper_2602_01219_amd/csrc/layer_check.hpp"

int main() {
  mita_dense_cfg_t c{};
  while (scanf("%d %d %d %d %d %d %d %d %d", &c.B, &c.H, &c.H_kv, &c.N, &c.N_k, &c.d, &c.dtype, &c.left, &c.right) == 9) {
    if (mita::check_dense(&c, nullptr) != MITA_OK) return 1;
    const mita::DensePlan p = mita::dense_plan(c);
    const mita::DenseBwdPlan q = mita::dense_bwd_plan(c);
    printf("%d %d %d %d %d %d %d\n", (int)p.few, p.tiles, p.splits, q.qtiles, q.qsplits, q.ktiles, q.ksplits);
  }
  return 0;
}
