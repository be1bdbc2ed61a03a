// Whether two tensors have an element's memory in common: host arithmetic.
#pragma once

#include <algorithm>

#include "runtime.h"

namespace ms {
namespace rt {

enum class Shared { kNo, kYes, kUnknown };

// Of one type, with non-negative strides.  Where the dims that vary in both have the same strides this
// is exact: an element of each lies at one address if the pointers' difference is a sum of k_i stride_i,
// -(extents of b) < k_i < (extents of a).  Else it is known only where the ranges that they span do not meet
// or begin together.
inline Shared shared(const ms_tensor *a, const ms_tensor *b) {
    if (!a || !b || !a->data || !b->data || numel(a) == 0 || numel(b) == 0) return Shared::kNo;
    const int64_t e = (int64_t)elt_size(a->dtype);
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a->data), pb = reinterpret_cast<uintptr_t>(b->data);
    auto bytes = [&](const ms_tensor *t) {   // of its span
        int64_t n = 1;
        for (int i = 0; i < t->ndim; ++i) n += (t->shape[i] - 1) * t->stride[i];
        return (uintptr_t)(n * e);
    };
    if (pa + bytes(a) <= pb || pb + bytes(b) <= pa) return Shared::kNo;
    if (pa == pb) return Shared::kYes;
    const int64_t apart = (int64_t)(pb - pa);
    if (a->dtype != b->dtype || a->ndim != b->ndim || apart % e) return Shared::kUnknown;
    struct Dim {
        int64_t stride, na, nb;   // steps that a, b can take
    } d[5];
    int n = 0;
    for (int i = 0; i < a->ndim; ++i) {
        const int64_t na = a->shape[i] - 1, nb = b->shape[i] - 1;
        if (na > 0 && nb > 0 && a->stride[i] != b->stride[i]) return Shared::kUnknown;
        const int64_t s = na > 0 ? a->stride[i] : b->stride[i];
        if ((na > 0 || nb > 0) && s > 0) d[n++] = Dim{s, na, nb};
    }
    std::sort(d, d + n, [](const Dim &x, const Dim &y) { return x.stride > y.stride; });
    int64_t most[6] = {0}, least[6] = {0};   // of the sums over the dims from i on
    for (int i = n - 1; i >= 0; --i) {
        most[i] = most[i + 1] + d[i].na * d[i].stride;
        least[i] = least[i + 1] - d[i].nb * d[i].stride;
    }
    // The differences that are left after i dims: few where strides nest.
    constexpr int kMany = 64;
    int64_t left[kMany], next[kMany];
    int count = 1;
    left[0] = apart / e;
    for (int i = 0; i < n; ++i) {
        int m = 0;
        for (int j = 0; j < count; ++j) {
            const int64_t s = d[i].stride, v = left[j];
            // least <= v - k s <= most of the other dims
            int64_t k = std::max(-d[i].nb, (v - most[i + 1]) / s - 1);
            for (; k <= d[i].na && v - k * s >= least[i + 1]; ++k) {
                if (v - k * s > most[i + 1]) continue;
                if (m == kMany) return Shared::kUnknown;
                next[m++] = v - k * s;
            }
        }
        count = m;
        std::copy(next, next + m, left);
    }
    for (int j = 0; j < count; ++j)
        if (left[j] == 0) return Shared::kYes;
    return Shared::kNo;
}

// The same elements in the same places.
inline bool same_places(const ms_tensor *a, const ms_tensor *b) {
    if (a->data != b->data || !same_shape(a, b)) return false;
    for (int i = 0; i < a->ndim; ++i)
        if (a->shape[i] > 1 && a->stride[i] != b->stride[i]) return false;
    return true;
}

}  // namespace rt
}  // namespace ms
