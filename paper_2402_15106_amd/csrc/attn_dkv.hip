// Attention backward, the gradients of the keys and values, for tiles of 128 keys that fill the
// card.  D_i and lse_i come from the launch for the queries.
#include "attn_bwd.hpp"

using namespace dsmp;

namespace {

// waves to a SIMD that the registers are cut to
template <typename T, int D, typename M>
constexpr int WAVES = D == 128 || (D == 64 && sizeof(T) == 4) ? 1 : sizeof(T) == 4 ? 2 : D == 64 ? 3 - (M::DIM > 0 || M::CAP > 0) : 4 - (M::DIM > 0);

template <typename T, int D, bool PAIRED, typename M>
__global__ __launch_bounds__(BT, (WAVES<T, D, M>)) void k_attn_dkv(AttnArgs a) {
  using C = Bwd<T, D, false, true>;
  DSMP_BWD_LDS(C, lds);
  dkv_tile<T, D, false, PAIRED, M>(a, lds, blockIdx.x);
}

}  // namespace

namespace dsmp {

void launch_attention_dkv(dsmp_handle* h, const dsmp_attention_desc& d, const AttnArgs& a, int64_t grid) {
  by_attention(d, [&](auto t, auto width, auto mode) {
    using T = decltype(t);
    constexpr int D = decltype(width)::value;
    using M = decltype(mode);
    constexpr bool PAIRS = sizeof(T) == 2 && M::DIM > 0;   // something to gain
    if (PAIRS && rows_paired(d)) hipLaunchKernelGGL((k_attn_dkv<T, D, PAIRS, M>), dim3((unsigned)grid), dim3(BT), 0, h->stream, a);
    else hipLaunchKernelGGL((k_attn_dkv<T, D, false, M>), dim3((unsigned)grid), dim3(BT), 0, h->stream, a);
  });
}

}  // namespace dsmp
