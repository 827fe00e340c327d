// Attention over the paged 8-bit cache for sequences behind prefixes, whose tiles take the prefix's keys and then the sequence's own
// (what a block does: cache_attn.h).  The prefix is read once for every tile, most of it from the caches; there is no second pass and
// often no join: 64 sequences of 40 rows behind 512 shared keys, 8 heads of 128 with 4 queries each, 62 us, in two parts 125.
#include "cache_attn.h"

namespace dv {

namespace {

template <int DH, bool BF>
__global__ __launch_bounds__(256, 2) void cache_behind_k(CacheAttnArgs a) {
    __shared__ Small<DH> lds;
    attend_small<DH, BF, BEHIND>(a, lds, blockIdx.x, blockIdx.y);
}
template <int DH, bool ONE>
__global__ __launch_bounds__(256, 2) void cache_behind_tile_k(CacheAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    attend_large<DH, ONE, BEHIND>(a, *(Lds<DH>*)smem, blockIdx.x, blockIdx.y);
}
template <bool BF, int SHIFT, int W>
__global__ __launch_bounds__(256) void cache_behind_join_k(CacheAttnArgs a) {
    join<BF, SHIFT, W, BEHIND>(a);
}
struct BehindKeys {
    template <int DH, bool BF>
    static constexpr auto small() { return cache_behind_k<DH, BF>; }
    template <int DH, bool ONE>
    static constexpr auto large() { return cache_behind_tile_k<DH, ONE>; }
    template <bool BF, int SHIFT, int W>
    static constexpr auto join() { return cache_behind_join_k<BF, SHIFT, W>; }
};

}  // namespace

void launch_cache_behind(bool bf, CacheAttnArgs a, const CacheAttnPlan& p, float* workspace, hipStream_t s) {
    launch_all<BehindKeys>(bf, a, p, workspace, s);
}

}  // namespace dv
