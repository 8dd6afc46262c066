// Which cached tokens a query sees.  Without HIP, so that it also compiles for the host.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define WFKV_BOTH __host__ __device__ __forceinline__
#else
#define WFKV_BOTH inline
#endif

namespace wfkv {

struct Sight {
  int lo, hi;
};

// The tokens [lo, hi) of a row of len cached ones (0 .. 2^30) that a query at position p
// sees, none where lo >= hi.  p is what a device array holds, so any number: lo stops at len, so that a
// unit of tokens counted from it, and those asked ahead of it, stay within 32 bits.
WFKV_BOTH Sight sight_of(int p, int len, int window) {
  const int hi = p < 0 ? 0 : p < len ? p + 1 : len;
  const int lo = window && p >= window ? p - window + 1 : 0;
  return Sight{lo < len ? lo : len, hi};
}

}  // namespace wfkv
