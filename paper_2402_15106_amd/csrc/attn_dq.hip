// Attention backward, the gradients of the queries, for tiles of 128 rows that fill the card.
#include "attn_bwd.hpp"

using namespace dsmp;

namespace {

template <typename T, int D, typename M>
__global__ __launch_bounds__(BT, D == 128 && (sizeof(T) == 4 || M::DIM > 2) ? 1 : 2) void k_attn_dq(AttnArgs a) {
  __shared__ __align__(16) unsigned char smem[Bwd<T, D, false, false>::LDS];
  dq_tile<T, D, false, M>(a, smem, blockIdx.x);
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
