// Whether two tensors have an element's memory in common: host arithmetic.
#pragma once

#include <algorithm>

#include "runtime.h"

namespace ms {
namespace rt {

enum class Shared { kNo, kYes, kUnknown };

// Of one type, with non-negative strides.  An element of each lies at one address if the pointers'
// difference is a sum of i stride over a's dims less one over b's; tried from the largest stride down, which
// leaves few possibilities where strides nest, as those of slices do (kUnknown where it leaves many).
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
    const int64_t difference = (int64_t)(pb - pa);
    if (a->dtype != b->dtype || difference % e) return Shared::kUnknown;
    struct Dim {
        int64_t stride, up, down;   // steps that a, b can take
    } d[10];
    int n = 0;
    for (const ms_tensor *t : {a, b}) {
        Dim own[5];
        int m = 0;
        for (int i = 0; i < t->ndim; ++i)
            if (t->shape[i] > 1 && t->stride[i] > 0) own[m++] = Dim{t->stride[i], t->shape[i] - 1, 0};
        std::sort(own, own + m, [](const Dim &x, const Dim &y) { return x.stride < y.stride; });
        int last = -1;   // dims without a gap between them are one
        for (int i = 0; i < m; ++i) {
            if (last >= 0 && own[i].stride == own[last].stride * (own[last].up + 1)) own[last].up = (own[last].up + 1) * (own[i].up + 1) - 1;
            else own[++last] = own[i];
        }
        for (int i = 0; i <= last; ++i) d[n++] = t == a ? own[i] : Dim{own[i].stride, 0, own[i].up};
    }
    std::sort(d, d + n, [](const Dim &x, const Dim &y) { return x.stride > y.stride; });
    // Of the sums over the dims from i on: the largest, the least, whether all between them are sums.
    int64_t most[11], least[11];
    bool every[11];
    most[n] = least[n] = 0;
    every[n] = true;
    for (int i = n - 1; i >= 0; --i) {
        most[i] = most[i + 1] + d[i].up * d[i].stride;
        least[i] = least[i + 1] - d[i].down * d[i].stride;
        every[i] = every[i + 1] && d[i].stride <= most[i + 1] - least[i + 1] + 1;
    }
    constexpr int kMany = 64;
    int64_t left[kMany], next[kMany];   // what is left of the difference after i dims
    int count = 1;
    left[0] = difference / e;
    for (int i = 0; i < n; ++i) {
        int m = 0;
        for (int j = 0; j < count; ++j) {
            if (every[i] && left[j] >= least[i] && left[j] <= most[i]) return Shared::kYes;
            for (int64_t k = std::max(-d[i].down, (left[j] - most[i + 1]) / d[i].stride - 1); k <= d[i].up; ++k) {
                const int64_t v = left[j] - k * d[i].stride;
                if (v < least[i + 1]) break;
                if (v > most[i + 1]) continue;
                if (every[i + 1]) return Shared::kYes;
                if (m == kMany) return Shared::kUnknown;
                next[m++] = v;
            }
        }
        count = m;
        std::copy(next, next + m, left);
    }
    for (int j = 0; j < count; ++j)
        if (left[j] == 0) return Shared::kYes;
    return Shared::kNo;
}

// Whether y's elements lie where x's of the same index do.
inline bool same_places(const ms_tensor *x, const ms_tensor *y) {
    if (x->data != y->data) return false;
    for (int i = 0; i < y->ndim; ++i)
        if (y->shape[i] > 1 && x->stride[i] != y->stride[i]) return false;
    return true;
}

}  // namespace rt
}  // namespace ms
