// Trees of drafted tokens on the device: a wave holds a tree, lane i its node i.
#pragma once

#include "en_device.h"

struct EnTreeLane {
    unsigned long long way;      // bit m: node m lies on the way from the root to this node, itself included; 0: absent
    int depth;                   // nodes of the way before this one
    __device__ __forceinline__ bool present() const { return way != 0; }
};

// The whole wave calls. room: new tokens that the plan has left, done to N_q (nodes of depth >= room are absent).
// Pointer doubling: after a round a lane knows twice as much of its way, so seven rounds of exchanges see the longest chain to
// its end, and a tree of depth 6 takes four.
__device__ __forceinline__ EnTreeLane tree_lane(int p, int n, int room)          // p: the parent of node `lane`
{
    const int lane = threadIdx.x % 64;
    bool whole = p >= -1 && p < lane;            // every link looked at so far is one
    int up = whole && p >= 0 ? p : lane;         // the node that the way is known down from (a root: itself)
    unsigned long long way = (1ull << lane) | (1ull << up);      // .. with all nodes on the way there
    while (true) {
        const int next = __shfl(up | (whole ? 0 : 64), up, 64);
        whole = whole && next < 64;
        if (!__any((next & 63) != up))           // all ways are known up to their ends
            break;
        way |= __shfl(way, up, 64);
        up = next & 63;
    }
    EnTreeLane t;
    t.depth = (int)__popcll(way) - 1;
    t.way = whole && t.depth < room ? way : 0ull;
    return t;
}

__device__ __forceinline__ int tree_parent(const int32_t *parent, int n)
{
    const int lane = threadIdx.x % 64;
    return lane < n ? parent[lane] : -2;
}

// New tokens left to an agent that has used `done` of N_q; 0 where done is no count (an idle agent).
__device__ __forceinline__ int tree_room(int done, int Nq)
{
    return done >= 0 && done <= Nq ? Nq - done : 0;
}
