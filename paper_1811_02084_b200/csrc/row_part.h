// Rows of words of 2 or 4 bytes read 16 bytes at a time from wherever they begin: which of a row's pieces may be put together from two whole loads.
#pragma once

#ifdef __CUDACC__
#define MTF_ON_BOTH __host__ __device__ __forceinline__
#else
#define MTF_ON_BOTH inline
#endif

namespace mtf {

// A row of n words begins `at` words into a tensor of `total`, whose address is a multiple of 16 bytes (`words` words).  Piece p is the row's words p words .. (p + 1) words - 1; where rows may begin
// anywhere it is cut out of the 16 bytes that it begins in and the 16 behind those, also in a row that begins on 16 bytes, and both have to lie inside the tensor.
// Returns how many pieces, from the first on, are whole and may be read so.
MTF_ON_BOTH int whole_pieces(long long at, int n, long long total, int words, bool aligned) {
  const int whole = n / words;
  if (aligned) return whole;
  const long long inside = (total - (at - at % words)) / words - 1;
  return (int)(inside < 0 ? 0 : inside < whole ? inside : whole);
}

}  // namespace mtf
