// Attention backward, the gradients of the queries, for tiles of 128 rows that fill the card.
#include "attn_bwd.hpp"

using namespace dsmp;

namespace {

template <typename T, int D, typename M>
__global__ __launch_bounds__(BT, sizeof(T) == 4 ? (D == 128 ? 1 : 2) : D == 128 ? 2 : D == 64 ? 3 : 4) void k_attn_dq(AttnArgs a) {
  using C = Bwd<T, D, false, false>;
  DSMP_BWD_LDS(C, lds);
  dq_tile<T, D, false, M>(a, lds, blockIdx.x);
}

}  // namespace

namespace dsmp {

void launch_attention_dq(dsmp_handle* h, const dsmp_attention_desc& d, const AttnArgs& a, int64_t grid) {
  by_attention(d, [&](auto t, auto width, auto mode) {
    hipLaunchKernelGGL((k_attn_dq<decltype(t), decltype(width)::value, decltype(mode)>), dim3((unsigned)grid), dim3(BT), 0,
                       h->stream, a);
  });
}

}  // namespace dsmp
