// cache_rows.cuh -- which rows of a paged cache a query reads, found by a warp, one
// row to a lane; shared by the two attention kernels.
#pragma once

#include "cache.cuh"

namespace fibattn {
namespace cache {

constexpr unsigned kAll = 0xffffffffu;
constexpr float kLn2 = 0.6931471805599453f;

// Row i of a query's list: its distance, its weight within its slot, and whether it
// is one of two.  need: the distance that the query must have behind it.
struct RowOf { int distance, need; float weight; bool pair; };
__device__ __forceinline__ RowOf row_of(const Rows& r, int i) {
    RowOf o;
    o.pair = i < 2 * r.pairs;
    if (o.pair) {
        const int k = i >> 1, far = i & 1;
        const float w = r.far[k];
        o.need = r.near[k] + 1;
        o.distance = r.near[k] + far;
        o.weight = far ? w : 1.f - w;
    } else {
        const int k = i - 2 * r.pairs;
        o.distance = o.need = k < r.singles ? r.near[r.pairs + k] : k - r.singles;
        o.weight = 1.f;
    }
    return o;
}

// The storage slot of a lane's row: the slot of its position, or, in a tree, that of
// the ancestor `distance` steps up, where the tree reaches that far.  All lanes walk
// together; the parents come 32 at a time, one to a lane, so that a step is an
// exchange between lanes and no load.  Returns false if a parent is not before its
// child, or an ancestor that is read is of another sequence or stands elsewhere; a
// parent is less than its child, so the walk ends.
template <bool kTree>
__device__ __forceinline__ bool slot_of(const AttnArgs& a, int n, int pos, int seq, int distance, bool live, int& slot) {
    slot = pos - distance;
    if (!kTree) return true;
    const int furthest = __reduce_max_sync(kAll, live ? distance : -1), lane = threadIdx.x & 31;
    int mine = -1, cur = n, first = max(n - 31, 0), parents = a.parents[min(first + lane, n)];
    for (int j = 0; j <= furthest; ++j) {
        if (j == distance) mine = cur;
        if (j == furthest) break;
        if (cur < first) {
            first = max(cur - 31, 0);
            parents = a.parents[min(first + lane, cur)];
        }
        const int up = __shfl_sync(kAll, parents, cur - first);
        if (up < -1 || up >= cur) return false;       // (the same for all lanes)
        if (up < 0) break;
        cur = up;
    }
    if (!live || mine < 0) return true;
    const int at = a.positions[mine], of = a.seqs ? a.seqs[mine] : mine;
    slot = a.slots[mine];
    return at == pos - distance && of == seq;
}

}  // namespace cache
}  // namespace fibattn
