// The tiles that attention calls take: reads "heads kv_heads head_dim dtype dim cap queries keys segments" lines,
// prints "forward queries keys paired" for each, F or W for tiles of 32 or 128 rows and the number of their cuts.
#include <stdio.h>
#include "../../paper_2402_15106_amd/csrc/attn_plan.hpp"

int main() {
  dsmp_attention_desc d{};
  long long nq, nk, n_seg;
  while (scanf("%d %d %d %d %d %f %lld %lld %lld", &d.heads, &d.kv_heads, &d.head_dim, &d.dtype, &d.dim, &d.cap, &nq, &nk, &n_seg) == 9) {
    const dsmp_segments qs{nq, n_seg, nullptr}, ks{nk, n_seg, nullptr};
    const dsmp::FwdPlan f = dsmp::fwd_plan(d, qs, ks);
    const dsmp::BwdPlan b = dsmp::bwd_plan(d, qs, ks);
    printf("%c%d %c%d %c%d %d\n", f.few ? 'F' : 'W', f.splits, b.wide_q ? 'W' : 'F', b.splits_q, b.wide_k ? 'W' : 'F', b.splits_k,
           (int)(b.wide_k && dsmp::rows_paired(d)));
  }
  return 0;
}
