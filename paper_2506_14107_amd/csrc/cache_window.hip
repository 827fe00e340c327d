// Attention over the paged 8-bit cache with a window and first keys that stay visible (what a block does: cache_attn.h).
// The keys of a tile are the steps of 64 that some row of it sees: the first ones, then those from its first row's window
// on; splits are cut from these.  Single tokens are bound by what they see: 64 streams of up to 12,000 keys, windows of 2048 behind 257
// first ones, 8 heads of 128: 54 us (277 MB, 5.1 TB/s).  Prompts take large tiles: 2 x 2048 rows behind up to 6144 keys, windows of 1024,
// 99 us (742 TFLOP/s on what rows see; 17 of a tile's 19 steps are that, and blocks are short).
#include "cache_attn.h"

namespace dv {

namespace {

template <int DH, bool BF>
__global__ __launch_bounds__(256, 2) void cache_window_k(CacheAttnArgs a) {
    __shared__ Small<DH> lds;
    attend_small<DH, BF, WINDOW>(a, lds, blockIdx.x, blockIdx.y);
}
template <int DH, bool ONE>
__global__ __launch_bounds__(256, 2) void cache_window_tile_k(CacheAttnArgs a) {
    extern __shared__ __attribute__((aligned(16))) uint8_t smem[];
    attend_large<DH, ONE, WINDOW>(a, *(Lds<DH>*)smem, blockIdx.x, blockIdx.y);
}
template <bool BF, int SHIFT, int W>
__global__ __launch_bounds__(256) void cache_window_join_k(CacheAttnArgs a) {
    join<BF, SHIFT, W, WINDOW>(a);
}
struct WindowKeys {
    template <int DH, bool BF>
    static constexpr auto small() { return cache_window_k<DH, BF>; }
    template <int DH, bool ONE>
    static constexpr auto large() { return cache_window_tile_k<DH, ONE>; }
    template <bool BF, int SHIFT, int W>
    static constexpr auto join() { return cache_window_join_k<BF, SHIFT, W>; }
};

}  // namespace

void launch_cache_window(bool bf, CacheAttnArgs a, const CacheAttnPlan& p, float* workspace, hipStream_t s) {
    launch_all<WindowKeys>(bf, a, p, workspace, s);
}

}  // namespace dv
