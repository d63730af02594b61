// The ring of tiles that the K loader and the V loader of the shared-prefix kernel fill in turn, as arithmetic that a plain
// C++ compiler takes too.
//
// K tile x has number 2 x, V tile x number 2 x + 1; tile `number` lands in slot number % slots and completes phase
// number / slots of that slot's barrier.  A loader requests a tile only when the slot's last one has been consumed.
#pragma once

#ifdef __CUDACC__
#define HG_RING_FN __host__ __device__ __forceinline__
#else
#define HG_RING_FN inline
#endif

namespace hg {

// Number of the last tile requested into `slot` when the loaders have requested k_tiles and v_tiles, or -1: of a slot's tiles
// the only one that can still be on its way.  (Waiting for an earlier one would not do: the slot may have gone through
// two phases since, and the parity of its phase is the awaited one's again.)
HG_RING_FN int ring_last_tile(int slot, int slots, int k_tiles, int v_tiles) {
    int last = -1;
    for (int which = 0; which < 2; ++which)
        for (int i = 0, n = 2 * (which ? v_tiles : k_tiles) - 2 + which; i < slots && n > last; ++i, n -= 2)
            if (n % slots == slot) { last = n; break; }
    return last;
}

}  // namespace hg
