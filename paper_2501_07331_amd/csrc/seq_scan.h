// What the scan's forward and backward kernels share.
#pragma once

#include "seq_device.h"

namespace {

template <int S>
struct ScanShape {
    static constexpr int NP = 4 * S;                            // states of a channel, padded
    static constexpr int CB = S <= 4 ? 64 : S == 8 ? 32 : 16;   // channels of a workgroup
    static constexpr int NT = CB * S;                           // threads
};

// Staging of B and C (BOTH, or B alone) of a tile: [TT][1 or 2][NP] fp32 in
// LDS, zero past the sample's steps and the states.  A thread takes E groups
// of four neighbouring states.
template <class T, int S, int TT, bool BOTH>
struct GroupTile {
    static constexpr int NP = ScanShape<S>::NP, NT = ScanShape<S>::NT;
    static constexpr int W = BOTH ? 2 * NP : NP, V = TT * W / 4, E = (V + NT - 1) / NT;
    Raw<T, 4, false> raw[E];
    RowIn<T, 4, false> p[E];
    __device__ __forceinline__ void init(const ScanArgs& a, int b, int g, int tid) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = e * NT + tid, k = i % (W / 4) * 4;
            p[e].init(k < NP ? a.B : a.C, b, i / (W / 4), a.T, g * a.state + k % NP);
        }
    }
    // end: the steps that are read
    __device__ __forceinline__ void load(const ScanArgs& a, int t0, int end, int tid) {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = e * NT + tid, k = i % (W / 4) * 4;
            const bool in = (V % NT == 0 || i < V) && t0 + i / (W / 4) < end;
            // a row's stride is the tensor's, which differs between a wave's lanes
            const long long row = k < NP ? a.B.row : a.C.row;
            raw_dense(raw[e], reinterpret_cast<const T*>(p[e].p) + t0 * row, in ? a.state - k % NP : 0);
        }
    }
    __device__ __forceinline__ void store(float* bc, int tid) const {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int i = e * NT + tid;
            if (V % NT == 0 || i < V)
                *reinterpret_cast<float4*>(&bc[4 * i]) = make_float4((float)raw[e].e[0], (float)raw[e].e[1],
                                                                     (float)raw[e].e[2], (float)raw[e].e[3]);
        }
    }
};

}  // namespace
