// peer_round.h — rounds of posts between the blocks of a cluster, plain arithmetic for the device and
// the host.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define SIMX_PEER_HD __host__ __device__ __forceinline__
#else
#define SIMX_PEER_HD inline
#endif

namespace simx {

// A thread's view of the rounds.  Every block posts to every block once a round, into one of two slots
// by turns, and waits until its slot of the round has all posts; waits are bounded.  A block may post a
// round while another still reads the one before, but not the one before that: what keeps it from doing
// so is its own wait for the other's post of the round between.  So a thread that gave up waiting
// posts nothing any more: its next posts could land on a slot that a slow block has yet to read, and be
// counted there in another's place.  The blocks that are still waiting then give up as well, and what
// any of them has read until then was complete.
struct PeerRound {
  uint32_t state;  // the round modulo 4, and 4 once a wait has run out
  SIMX_PEER_HD uint32_t slot() const { return state & 1u; }
  SIMX_PEER_HD uint32_t parity() const { return (state >> 1) & 1u; }  // of the slot's phase
  SIMX_PEER_HD bool lost() const { return (state & 4u) != 0u; }
  SIMX_PEER_HD bool posts() const { return !lost(); }
  SIMX_PEER_HD void end(bool came) { state = ((state + 1u) & 3u) | (state & 4u) | (came ? 0u : 4u); }
};

}  // namespace simx
