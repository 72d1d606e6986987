// One Muon step over a list of matrices: which kernels take which tensor.  Spectral weights go mode by mode (fno_muon_modes2.hip,
// fno_muon_modes5.hip, fno_muon_modes.hip), small real matrices a block each (fno_muon_small.hip), the others tile by tile
// (fno_muon_dense.hip).
#include "fno_muon.h"

namespace fno {

size_t muon_workspace_bytes(const MuonTensor* t, int count) { return muon_dense_bytes(t, count); }

hipError_t launch_muon(const MuonTensor* t, int count, const MuonStep& st, void* ws, hipStream_t s) {
  const MuonScalars c{(float)st.momentum, (float)st.a, (float)st.b, (float)st.c, (float)st.max_norm, st.nesterov ? 1 : 0,
                      st.iterations, st.eps, st.norm};
  hipError_t e = launch_muon_modes5(t, count, c, st.lr, s);
  if (e == hipSuccess) e = launch_muon_modes2(t, count, c, st.lr, s);
  if (e == hipSuccess) e = launch_muon_modes(t, count, c, st.lr, s);
  if (e == hipSuccess) e = launch_muon_small(t, count, c, st.lr, s);
  if (e == hipSuccess) e = launch_muon_dense(t, count, c, st.lr, ws, s);
  return e;
}

}  // namespace fno
