// Where the rows of a paged cache of the caller's lie: plain host arithmetic, so that it can be worked through without a GPU.
#pragma once
#include <algorithm>

namespace confkv {

// Pages, tokens of a page, heads of a token: how many, and how many values apart.
struct PagesDim {
  long long size, stride;
};

// Sorts the dimensions by their strides.  Values from the first to the last of the rows of D values; 0 where rows overlap or a size or stride
// is out of bounds.
inline long long pages_extent(PagesDim (&d)[3], int D) {
  constexpr long long kMostStride = 1ll << 40;
  std::sort(d, d + 3, [](const PagesDim &x, const PagesDim &y) { return x.stride < y.stride || (x.stride == y.stride && x.size < y.size); });
  long long extent = D;
  for (const PagesDim &x : d) {
    if (x.stride < 0 || x.stride > kMostStride || x.stride % 8) return 0;
    if (x.size == 1) continue;
    if (x.stride < extent || x.size > (1ll << 56) / x.stride) return 0;
    extent += (x.size - 1) * x.stride;
  }
  return extent;
}

// Whether a row of one plane and a row of another one like it, `apart` values behind, share a value.  d as pages_extent leaves them: what the
// dimensions below one reach is no longer than its stride, so that two steps of it can bring the rows together.
inline bool planes_meet(const PagesDim (&d)[3], int D, long long apart, int dim = 2) {
  if (dim < 0) return apart > -D && apart < D;
  if (d[dim].size == 1) return planes_meet(d, D, apart, dim - 1);
  const long long s = d[dim].stride, most = d[dim].size - 1;
  const long long down = apart >= 0 ? apart / s : -((-apart + s - 1) / s);
  for (long long n : {down, down + 1})
    if (n >= -most && n <= most && planes_meet(d, D, apart - n * s, dim - 1)) return true;
  return false;
}

}  // namespace confkv
