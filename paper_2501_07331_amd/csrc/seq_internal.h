// Internal types shared by the host side and the kernels of the sequence
// operators (include/snn_seq.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "snn_seq.h"

// A sequence as a kernel takes it: strides in elements.  packed: bytes with
// scales, blocks scales a row.
struct SeqT {
    char* p;
    const float* scale;
    long long row, sample;
    int packed, blocks;
};

// Steps of a forward tile of the scan; a backward tile is one segment between
// saved states.
constexpr int kScanTile = 32;
constexpr int kScanSeg = SNN_SEQ_SEGMENT;

struct ScanArgs {
    SeqT u, delta, B, C, z, y;             // forward
    SeqT dy, du, ddelta, dz;               // backward
    const float* A;
    const float* D;
    const float* delta_bias;
    const float* h0;
    float* hT;
    float* saved;                          // [batch][segments][channels][NP]
    const int* lengths;
    int batch, T, channels, state, groups, softplus;
    int per;                               // channels a group
    int gblocks;                           // channel blocks a group
    int chunks, chunk_len;                 // parts of the time axis; steps a part (whole tiles)
    int joined;                            // a launch of its own joins them
    int segs;                              // saved states a sample
    float* carry;                          // [batch][chunks][channels][NP] states / adjoints between parts
    float* dsum;                           // [batch][chunks][channels] sums of delta' of a part
    // backward pass that computes the states again, in parts: their first states, and the sums of
    // delta' from a part's start to each saved state; NULL otherwise
    float* hcarry;                         // [batch][chunks][channels][NP]
    float* csum;                           // [batch][segs][channels]
    // backward
    const float* dhT;
    float* dh0;
    float* bcpart;                         // [batch][T][groups * gblocks][2 NP] shares of dB, dC
    float* apart;                          // [batch * chunks][channels][NP] shares of dA
    float* dpart;                          // [batch * chunks][2][channels] shares of dD, ddelta_bias
    SeqT dB, dC;
    float* dA;
    float* dD;
    float* ddelta_bias;
};

struct ConvArgs {
    SeqT x, y, dy, dx;
    const float* w;
    const float* bias;
    const int* lengths;
    const char* state;
    char* state_out;
    const char* dstate_out;
    char* dstate;
    float* part;                           // [batch * time tiles][channels][taps + 1] shares of dw, dbias
    float* dw;
    float* dbias;
    int batch, T, channels, taps, silu, tiles;
};

struct PackArgs {
    SeqT x;
    unsigned char* q;
    float* scale;
    int batch, T, n;
};

struct BinArgs {
    const int* offsets;                    // spike lists: [batch + 1]; NULL: records
    const int* count;
    const int* step;
    const int* neuron;
    int nnz, capacity;
    SeqT y;
    int batch, T, n, factor, rows, tile;   // rows of the output, rows of a workgroup
    int past;                              // the output goes past the caches
};

// states of a channel, padded to what the lanes of a channel hold (4 each)
inline int scan_np(int state) { return state <= 4 ? 4 : state <= 8 ? 8 : state <= 16 ? 16 : state <= 32 ? 32 : 64; }
// channels of a workgroup of the scan
inline int scan_cb(int np) { return np <= 16 ? 64 : np == 32 ? 32 : 16; }

// time tiles of the convolution's backward (one share of dw each)
int conv_tiles(int T, int channels, int taps);

hipError_t launch_scan_forward(const ScanArgs& a, int dtype, hipStream_t s);
hipError_t launch_scan_states(const ScanArgs& a, int dtype, hipStream_t s);   // only a.saved
hipError_t launch_scan_backward(const ScanArgs& a, int dtype, hipStream_t s);
hipError_t launch_scan_step(const ScanArgs& a, int dtype, hipStream_t s);
hipError_t launch_conv_forward(const ConvArgs& a, int dtype, hipStream_t s);
hipError_t launch_conv_backward(const ConvArgs& a, int dtype, hipStream_t s);
hipError_t launch_conv_step(const ConvArgs& a, int dtype, hipStream_t s);
hipError_t launch_pack(const PackArgs& a, int dtype, hipStream_t s);
hipError_t launch_unpack(const PackArgs& a, int dtype, hipStream_t s);
hipError_t launch_bin(const BinArgs& a, int dtype, hipStream_t s);
