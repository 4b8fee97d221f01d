// Which of a warp's two result buffers its next chunk takes, and which of its
// stores have to have read theirs before (mxf4_pair.cu). On its own, so that the
// order can be walked through without a GPU.
#pragma once

#ifndef SVL_DEVINL
#define SVL_DEVINL inline
#endif

namespace svl {

// Until a CTA's last tile there is buffer 0 alone; in the last one buffers 1 and
// 0, in turn. The first chunk there goes into buffer 1, while the store of the tile
// before may still be reading buffer 0; with a residual it goes into
// buffer 0, where its part of the residual is already on its way.
struct ResultSlots {
  int slot = 0;
  bool both = false;
  SVL_DEVINL void enter_last(bool residual) {
    both = true;
    if (!residual) slot = 1;
  }
  // How many stores, the most recent ones, may be unread when a chunk is written to `slot`.
  SVL_DEVINL int unread() const { return both ? 1 : 0; }
  SVL_DEVINL void stored() {
    if (both) slot ^= 1;
  }
};

}  // namespace svl
