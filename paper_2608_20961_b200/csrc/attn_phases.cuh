// Barriers of the tensor-core attention kernel whose events can run ahead of their waiter: which one carries an
// event, and the parity of its phase.  Plain C++, so that a model of the roles can be checked with the kernel's own
// arithmetic on a CPU.
#pragma once

#ifdef __CUDACC__
#define TREEWY_PHASE_FN __host__ __device__ constexpr
#else
#define TREEWY_PHASE_FN constexpr
#endif

namespace treewy {

struct Phase {
    unsigned barrier, parity;
};

// Q buffers for heads of d: what 512 columns of tensor memory leave beside O and S.
TREEWY_PHASE_FN int q_buffers(int d) { return d == 256 ? 1 : 2; }

// "The queries of item `item` are in tensor memory."  One barrier to a buffer.  The softmax warps take item i + 1 before
// their last tiles of item i; with two buffers and an item of one or two tiles that is before any product of item i,
// so i and i + 1 can both be announced before Q K^T looks at the first.  On one barrier that would be two phases, and a
// parity does not tell the second from none.  Item i + 2 is not taken before all of item i is done.
TREEWY_PHASE_FN Phase q_phase(unsigned item, int buffers)
{
    return {item % (unsigned)buffers, (item / (unsigned)buffers) & 1u};
}

}  // namespace treewy
