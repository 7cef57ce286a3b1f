// The rows of a group of a grouped product, as every CTA takes them from the ranges in device memory; the function also runs on the
// host, where a test gives it the corners of 32-bit numbers.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace regione {

// [b, e) cut to [0, cap]: its first row and how many.  Both ends are cut before they are subtracted, since the difference of two
// 32-bit numbers need not be one.  False: the range as given is not within the buffer.
__host__ __device__ __forceinline__ bool cut_range(int b, int e, int cap, int& begin, int& rows) {
    begin = b < 0 ? 0 : b < cap ? b : cap;
    const int end = e < 0 ? 0 : e < cap ? e : cap;
    rows = end > begin ? end - begin : 0;
    return b >= 0 && e <= cap && b <= e;
}

}  // namespace regione
