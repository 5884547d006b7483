// api_util.h -- host helpers shared by the translation units of the C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <vector>

namespace attn {

inline bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

// Do the D-element rows of an output with these sizes and strides stay
// disjoint? Ordered by stride, every dimension must step past the whole extent
// of the ones inside it (sufficient, and what every ordinary layout meets);
// dimensions of size one are ignored. Overlapping output rows would make the
// result depend on which workgroup writes last.
inline bool rows_disjoint(int64_t d, int n, const int64_t* size, const int64_t* stride)
{
    int64_t sz[3], st[3];
    int m = 0;
    for (int i = 0; i < n; ++i)
        if (size[i] > 1) {
            sz[m] = size[i];
            st[m] = stride[i];
            ++m;
        }
    for (int a = 0; a < m; ++a)  // insertion sort by stride
        for (int b = a; b > 0 && st[b] < st[b - 1]; --b) {
            int64_t t = st[b]; st[b] = st[b - 1]; st[b - 1] = t;
            t = sz[b]; sz[b] = sz[b - 1]; sz[b - 1] = t;
        }
    int64_t extent = d;  // elements covered by one row
    for (int a = 0; a < m; ++a) {
        if (st[a] < extent) return false;
        extent = st[a] * (sz[a] - 1) + extent;
    }
    return true;
}

// Host copy of a device array, on `stream` (ATTN_FLAG_VALIDATE only).
template <class T>
bool fetch(const T* dev, int64_t n, hipStream_t stream, std::vector<T>* out)
{
    out->assign((size_t)n, 0);
    if (n == 0) return true;
    if (hipMemcpyAsync(out->data(), dev, (size_t)n * sizeof(T), hipMemcpyDeviceToHost,
                       stream) != hipSuccess)
        return false;
    return hipStreamSynchronize(stream) == hipSuccess;
}

}  // namespace attn
