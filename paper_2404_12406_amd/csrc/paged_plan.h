// How the keys of a paged attention's sequences are divided over blocks: host arithmetic,
// no HIP.
#pragma once

#include <algorithm>
#include <cstdint>

#include "device.h"

namespace ms {
namespace att {

struct PagedPlan {
    int splits, per;   // blocks of a sequence at most, keys of each
};

constexpr int kPagedBlocks = 8192;

// Keys a block: some 8192 blocks if every sequence filled its table, whole steps of a
// block's four waves.  How full the tables are is known on the device alone, so blocks past a sequence's end
// return at once, and there have to be enough of the others.  At most the whole table (below 2^31, as the kernel
// counts), and splits by what is left: every place has a block.
inline PagedPlan paged_plan(const PagedArgs &a) {
    const int64_t room = (int64_t)a.width * a.page, work = (int64_t)a.n * a.Hk * ((a.Hq / a.Hk + 31) / 32);
    auto whole = [](int64_t keys) { return std::max<int64_t>(128, (keys + 127) / 128 * 128); };
    const int64_t per = std::min(whole(room), whole(room * work / kPagedBlocks));
    return {(int)std::max<int64_t>(1, (room + per - 1) / per), (int)per};
}

}  // namespace att
}  // namespace ms
