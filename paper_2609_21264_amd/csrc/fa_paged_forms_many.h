// Launch of the instances of the kernel in fa_paged_many.h with one form (Cfg::FORM). Internal; included by the sources that
// hold the instances of a form each, which the build compiles side by side.
#pragma once

#include "fa_paged_many.h"

namespace fa {
namespace {

template <int DQK, int DV, bool E4M3, int FORM>
hipError_t launch_form_dims(const PagedParams& p, const PagedMany& m, hipStream_t stream) {
  constexpr bool SHORT = !E4M3 && DQK != 192;  // as paged_many has it
  return m.split ? launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, true, FORM>::C>(p, m.blocks, stream)
                 : launch_many<typename PagedInstance<DQK, DV, E4M3, SHORT, false, FORM>::C>(p, m.blocks, stream);
}
template <int FORM>
hipError_t launch_form(PagedParams p, const PagedMany& m, int d_qk, bool e4m3, hipStream_t stream) {
  many_constants(p);
  if (d_qk == 64) return e4m3 ? launch_form_dims<64, 64, true, FORM>(p, m, stream) : launch_form_dims<64, 64, false, FORM>(p, m, stream);
  if (d_qk == 128)
    return e4m3 ? launch_form_dims<128, 128, true, FORM>(p, m, stream) : launch_form_dims<128, 128, false, FORM>(p, m, stream);
  return e4m3 ? launch_form_dims<192, 128, true, FORM>(p, m, stream) : launch_form_dims<192, 128, false, FORM>(p, m, stream);
}

}  // namespace
}  // namespace fa
