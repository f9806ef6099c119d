// What the tensor-core kernels of the cross attention share: K and V as they lie, for TMA.
#pragma once

#include "cross.cuh"
#include "tc_common.cuh"

namespace restkv {
namespace {

// Whether rows can be described by a tensor map: strides that are no smaller than a row, nor past its 40 bits of bytes.
inline bool cross_map_fits(const CrossProblem& c, const RowsView& v) {
  for (long long st : {v.sb, v.sh, v.sn})
    if (st < c.d || st >= 1ll << 38) return false;
  return true;
}

// Boxes of box_rows rows and 64 dims of [sources, Hkv, n_rows, d]; rows past n_rows are filled with zeros.
inline bool make_cross_map(TcState* st, CUtensorMap* map, const CrossProblem& c, const RowsView& v, cuuint32_t box_rows) {
  const cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)c.n_rows, (cuuint64_t)c.Hkv, (cuuint64_t)c.sources};
  const cuuint64_t str[3] = {(cuuint64_t)v.sn * 2, (cuuint64_t)v.sh * 2, (cuuint64_t)v.sb * 2};
  return encode_tiles(st, map, v.data, 4, dims, str, box_rows) == CUDA_SUCCESS;
}

}  // namespace
}  // namespace restkv
