// The 16-byte pieces of memory that rows of logits lie in, apart from the kernel so that it can be checked on the host what is read of them.
#pragma once

#ifndef RESTKV_HOST_DEVICE
#ifdef __CUDACC__
#define RESTKV_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define RESTKV_HOST_DEVICE inline
#endif
#endif

namespace restkv {

// Whether the last of the rows (the first of which begins with a piece) ends inside a piece, whose rest may be nobody's memory.
RESTKV_HOST_DEVICE bool rows_end_inside_a_piece(long long rows, long long stride, int elements, int size) {
  return ((rows - 1) * stride + elements) * size % 16 != 0;
}

// A row that begins `off` bytes into its first piece.  Where the rows end with a piece, all of the row's pieces are loaded: what a piece has beside the
// row is another row's or lies between two.  Where they do not (kRagged), only those with no byte behind the row's end are, and the tokens that have a part in
// the last one are loaded one by one.
template <bool kRagged> struct RowPieces {
  int loaded;   // pieces that are loaded
  int inside;   // 16 bytes of the row from byte 16 i on, i below this, are all the row's and lie in loaded pieces (in i, and in i + 1 if off > 0)
  RESTKV_HOST_DEVICE RowPieces(unsigned int off, int elements, int size) {
    const long long end = (long long)elements * size + off;
    loaded = (int)((kRagged ? end : end + 15) / 16);
    inside = (int)(end / 16) - (off > 0 ? 1 : 0);
  }
};

}  // namespace restkv
