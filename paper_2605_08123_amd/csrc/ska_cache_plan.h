// How the attention on caches is launched: arithmetic on sizes, without anything of the GPU.
#pragma once

// Launches of the join of a call's parts: d / 4 threads a row for each slice of the parts, as many slices as there are parts, or threads.
struct CaJoin {
    static constexpr int THREADS = 256;   // of a workgroup
    int slices;
    long per;                             // rows of a workgroup
    CaJoin(int parts, int d) : slices(1)
    {
        while (slices * 2 <= parts && slices * 2 * (d / 4) <= THREADS) slices *= 2;
        per = THREADS / (d / 4) / slices;
    }
    // Rows of a launch, which has 2^31 threads at most: one of 2^32 would be accepted, and run their number modulo 2^32
    long most() const { return per << 23; }
};
