// Equal parts of a row of pages (sfmp_attention.h), also for a host program (tests/parts_driver.cpp).
#pragma once

#include <stdint.h>

#if defined(__HIP__)
#define SFMP_PARTS_FN __host__ __device__ __forceinline__
#else
#define SFMP_PARTS_FN inline
#endif

namespace sfmp {

// Part of a wavefront.
struct Part {
  int begin, end;
};

// `total` pages (0 .. 2^31 - 1) in parts for `waves` wavefronts of each workgroup, of `least` pages or more.  Sums pass 2^31, not 2^32: with 2^8 to
// 2^12 wavefronts and `least` up to 2^15 they stay below 2^31 + 2^28.
struct Parts {
  uint32_t total, of_wave, of_workgroup;
  SFMP_PARTS_FN Parts(const int all, const int workgroups, const int waves, const int least) {
    const uint32_t n = (uint32_t)workgroups * (uint32_t)waves;
    total = (uint32_t)all;
    of_wave = (total + n - 1) / n;
    if (of_wave < (uint32_t)least) of_wave = (uint32_t)least;
    of_workgroup = of_wave * (uint32_t)waves;
  }
  SFMP_PARTS_FN Part part(const int workgroup, const int wave) const {
    const uint32_t from = (uint32_t)workgroup * of_workgroup + (uint32_t)wave * of_wave, to = from + of_wave;
    return Part{(int)(from < total ? from : total), (int)(to < total ? to : total)};
  }
  // ... of all wavefronts of a workgroup
  SFMP_PARTS_FN Part whole(const int workgroup) const {
    const uint32_t from = (uint32_t)workgroup * of_workgroup, to = from + of_workgroup;
    return Part{(int)(from < total ? from : total), (int)(to < total ? to : total)};
  }
  SFMP_PARTS_FN int workgroup_of(const int page) const { return (int)((uint32_t)page / of_workgroup); }
};

}  // namespace sfmp
