// Index arithmetic of the norm join's rings, in a form that a host compiler
// takes too: tests run it at the limits of its types.
#pragma once

#ifdef __CUDACC__
#define IFVS_HD __host__ __device__ __forceinline__
#else
#define IFVS_HD inline
#endif

namespace ifvs {

// A team's tokens end at `end`; a place holds up to `per` of them and one place
// begins with token t <= end.  Tokens of the place `ahead` places later (none:
// 0), which begins with t + ahead * per.  end may be 2^31 - 1: what is left is
// compared, since t + ahead * per may lie beyond an int.
IFVS_HD int place_count(int t, int end, int per, int ahead) {
    const int left = end - t - ahead * per;
    return left <= 0 ? 0 : (left < per ? left : per);
}
// whether token t is the last of the place that begins with `first`
IFVS_HD bool ends_place(int t, int first, int end, int per) { return t - first == per - 1 || t == end - 1; }

}  // namespace ifvs
