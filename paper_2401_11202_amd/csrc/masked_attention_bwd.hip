// Gradients of masked attention: the two passes of cross_attention_bwd_kernels.h
// in their masked forms.  With t = tanh(scale q k / cap), P = 2^(z - lse):
//   dS = P (dP - D) (1 - t^2)   (without a cap the last factor is 1)
// and the rest as there; the bias has no gradient.  D is the rowsum of dO * O.
#include <algorithm>

#include "cross_attention_bwd_kernels.h"

namespace partir {
namespace {

template <int F>
void launch_form(const MaskedBwdParams& p, CrossBwdPass pass, hipStream_t s) {
  const int64_t nbh = (int64_t)p.B * p.Hk;
  if (pass == CROSS_DQ) {
    const int64_t blocks = ((int64_t)p.G * p.Sq + 127) / 128;
    hipLaunchKernelGGL((cross_bwd_dq_kernel<F>), dim3((unsigned)(blocks * nbh * p.q_parts)), dim3(NT), 0, s, p);
  } else {
    const int64_t blocks = ((int64_t)p.Sk + 255) / 256;
    const dim3 grid((unsigned)(blocks * nbh * p.k_parts));
    if (16 % p.G == 0)
      hipLaunchKernelGGL((cross_bwd_dkv_kernel<true, F>), grid, dim3(2 * NT), 0, s, p);
    else
      hipLaunchKernelGGL((cross_bwd_dkv_kernel<false, F>), grid, dim3(2 * NT), 0, s, p);
  }
}

}  // namespace

hipError_t launch_masked_backward(const MaskedBwdParams& p, int form, CrossBwdPass pass, hipStream_t s) {
  switch (form & (kCap | kBias)) {
    case 0: launch_form<kMasked>(p, pass, s); break;
    case kCap: launch_form<kMasked | kCap>(p, pass, s); break;
    case kBias: launch_form<kMasked | kBias>(p, pass, s); break;
    default: launch_form<kMasked | kCap | kBias>(p, pass, s);
  }
  return hipGetLastError();
}

}  // namespace partir
