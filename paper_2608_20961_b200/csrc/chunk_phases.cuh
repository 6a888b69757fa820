// The hand-over of outputs in the tensor-core kernel of treewy_attn_chunk: who says that an output in tensor memory has been read.
// Plain C++, so that a model of the roles can be checked with the kernel's own rule on a CPU.
//
// Each output has a barrier.  A phase of it is a USE of the output: an item in which it has products.  The thread that issues
// them waits for the phase of the use before, ahead of the first one of its own, and the warps that read the output last arrive: those
// of its own stream, or, where a stream's outputs are joined with the other's (an item with one row tile), those of the first stream
// alone.  So every arrival lies behind the wait for the phase before it, whichever stream is ahead.  (Were a phase an item, streams
// that take no part in one could complete two phases ahead of the thread that waits for the first: a parity does not tell it that
// they are over, and it would wait for good.)
#pragma once

#include "attn_phases.cuh"

namespace treewy {

// arrivals of a use: the warps of one stream
constexpr int O_FREE_ARRIVALS = 4;

// Whether a warp of stream `strm` arrives for output `which` at an item's end.  apart: each stream has rows of its own (one row tile: the
// first stream joins both outputs); used: the item has products in that output.
TREEWY_PHASE_FN bool frees_output(bool apart, int strm, int which, bool used) { return used && strm == (apart ? which : 0); }

}  // namespace treewy
