// The attention kernel's instances with a sliding window and visible first keys
// (attn_fwd_kernel.h, WINDOW), 16-bit types: eight wavefronts (256 query rows, one
// workgroup per CU) or four (128 rows, two or three per CU; 192-wide keys one), and
// eight in key groups on the smallest grids (64 or 128 rows; see
// attn_fwd_split_gfx950.hip).
#include <hip/hip_runtime.h>

#include "attn_fwd_kernel.h"
#include "attn_fwd_launch.h"

namespace qm {
namespace {

template <int DK, int WAVES>
constexpr int per_cu() {
  return WAVES == 8 || DK == 192 ? 1 : wgs_per_cu<DK, WAVES>();
}

template <int DK, int DV, int DT, int WAVES, int LAYOUTS>
__global__ __launch_bounds__(64 * WAVES, (wgs_per_cu<DK, WAVES>())) void attn_fwd_window_kernel(KParams p) {
  attn_fwd_body<DK, DV, DT, true, WAVES, 1, LAYOUTS, true>(p);
}

template <int DK, int DV, int DT, int WAVES, int LAYOUTS>
hipError_t launch_instance(const AttnArgs& a, const Device& dev, hipStream_t stream) {
  constexpr size_t lds = lds_bytes<DK, DV, DT, WAVES>();
  constexpr int n = per_cu<DK, WAVES>();
  static_assert(lds * n <= 160 * 1024, "the workgroups of a CU fit its LDS");
  return launch_tiles<attn_fwd_window_kernel<DK, DV, DT, WAVES, LAYOUTS>>(
      a, dev, 32 * WAVES, 64 * WAVES, lds, n, stream);
}

template <int DK, int DV, int DT, int G, int LAYOUTS>
__global__ __launch_bounds__(512, 1) void attn_fwd_window_split_kernel(KParams p) {
  attn_fwd_body<DK, DV, DT, true, 8 / G, G, LAYOUTS, true>(p);
}

template <int DK, int DT, int G>
hipError_t launch_groups(const AttnArgs& a, const Device& dev, hipStream_t stream) {
  constexpr size_t lds = lds_bytes<DK, DK, DT, 8 / G, G>();
  static_assert(lds <= 160 * 1024, "a workgroup's rings fit the LDS");
  return a.layout ? launch_tiles<attn_fwd_window_split_kernel<DK, DK, DT, G, kBnhdOnly>>(
                        a, dev, 256 / G, 512, lds, 1, stream)
                  : launch_tiles<attn_fwd_window_split_kernel<DK, DK, DT, G, kBhndOnly>>(
                        a, dev, 256 / G, 512, lds, 1, stream);
}

// Four waves take one layout each, eight either (see the other instances' files).  At
// d = 64 four waves were faster at every window (choose_window_waves): it has no others.
template <int DK, int DT>
hipError_t launch_width(const AttnArgs& a, const Device& dev, int waves, hipStream_t stream) {
  if constexpr (DK == 128) {
    if (waves == 8) return launch_instance<DK, DK, DT, 8, kEitherLayout>(a, dev, stream);
  }
  return a.layout ? launch_instance<DK, DK, DT, 4, kBnhdOnly>(a, dev, stream)
                  : launch_instance<DK, DK, DT, 4, kBhndOnly>(a, dev, stream);
}

template <int DT>
hipError_t launch_type(const AttnArgs& a, const Device& dev, hipStream_t stream) {
  const int groups = window_groups(a, dev.cus);
  if (groups == 4) return launch_groups<64, DT, 4>(a, dev, stream);
  if (groups == 2) {
    return a.d == 64 ? launch_groups<64, DT, 2>(a, dev, stream) : launch_groups<128, DT, 2>(a, dev, stream);
  }
  const int waves = a.tile_rows ? a.tile_rows / 32 : choose_window_waves(a, dev.cus);
  if (a.d == 64) return launch_width<64, DT>(a, dev, waves, stream);
  if (a.d == 128) return launch_width<128, DT>(a, dev, waves, stream);
  return waves == 8 ? launch_instance<192, 128, DT, 8, kBhndOnly>(a, dev, stream)
                    : launch_instance<192, 128, DT, 4, kBhndOnly>(a, dev, stream);
}

}  // namespace

hipError_t launch_attn_fwd_window(const AttnArgs& a, hipStream_t stream) {
  Device dev;
  const hipError_t e = current_device(&dev);
  if (e != hipSuccess) return e;
  return a.dtype == 0 ? launch_type<0>(a, dev, stream) : launch_type<1>(a, dev, stream);
}

}  // namespace qm
