// Size limit of the fp32 contractions, host-side only (plain C++): as limits.h's, the
// byte count of every operand and output, copies made for them among them, lies below
// the offset that stands for "past the end", by a load.
#pragma once

#include "limits.h"

namespace ms {
namespace g2 {

constexpr int64_t kMostFloats = ((int64_t)kOOB - 16) / 4;

}  // namespace g2
}  // namespace ms
