// Which keys a row of a packed document sees.  Plain C++, so that a test can ask it without a GPU.
#pragma once

#if defined(__HIPCC__)
#define MP_MASK_HOST_DEVICE __host__ __device__ __forceinline__
#else
#define MP_MASK_HOST_DEVICE inline
#endif

namespace mp {

// Row r of a document with rows [start, end), start <= r < end: keys [lo, hi).  has_prefix: the first `prefix` rows are seen by all of it
// (a negative number: none).  Rows may number nearly 2^31, and a window or a prefix anything, so nothing is added that could pass that.
MP_MASK_HOST_DEVICE void seen_in_document(int r, int start, int end, int causal, bool has_prefix, int prefix, int window, int& lo, int& hi) {
    lo = start;
    hi = causal ? r + 1 : end;
    if (has_prefix) {
        const int first = prefix <= 0 ? start : prefix < end - start ? start + prefix : end;
        if (first > hi) hi = first;
    }
    if (window) {
        if (window <= r - start) lo = r - window + 1;
        if (window < hi - r) hi = r + window;
    }
}

}  // namespace mp
