// The MX4 forms of the MFMA decode kernel (decode_mfma_kernel.h): a latent cache in 4 bits, without a log-sum-exp and with one.
#include "decode_mfma_kernel.h"

namespace mlra {

int launch_decode_mx4(const DecodeArgs& a, const mfma_tile::MfmaParams& p, bool paired, unsigned n_wg) {
  if (a.precise)
    return paired ? launch_form<kStagesPairedMx4, 1, true, true>(a, p, n_wg) : launch_form<kStagesMx4, 0, true, true>(a, p, n_wg);
  return paired ? launch_form<kStagesPairedMx4, 1, true>(a, p, n_wg) : launch_form<kStagesMx4, 0, true>(a, p, n_wg);
}

}  // namespace mlra
