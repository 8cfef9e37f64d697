// Short causal convolution of each channel with its own taps, and SiLU.
//
// Bound by memory: a thread takes VW neighbouring channels (a 16-byte vector)
// over kConvRun steps and keeps the window of inputs in registers, so that
// every input is read once but for the window at a run's start.  The backward
// pass goes over the same run in the same order: the pre-activation is made
// again from x, and dx[t] leaves when the last output that read x[t] is done,
// taps - 1 steps later.
#include "seq_device.h"

namespace {

constexpr int kConvRun = 16;      // steps of a thread
constexpr int kConvLanes = 16;    // threads side by side along the channels
constexpr int kConvRows = 16;     // threads along the time axis

// channels of a thread: 8, or 4 where many taps' windows fill the registers
template <int K>
constexpr int conv_vw() { return K <= 4 ? 8 : 4; }

__device__ __forceinline__ void dsilu(float x, float& y, float& dy) {
    const float p = sigmoid(x);
    y = x * p;
    dy = p * fmaf(x, 1.0f - p, 1.0f);
}

// x[t] of the sample: from the state before the first step, zero past len.
template <class T, int VW, bool PK>
__device__ __forceinline__ void conv_in(const ConvArgs& a, int b, int t, int len, int c, int n, float (&o)[VW]) {
    if (t >= 0) {
        Raw<T, VW, PK> r;
        raw_load(r, a.x, b, t, a.T, c, t < len ? n : 0);
        raw_get(r, a.x, c, o);
        return;
    }
    const SeqT s{const_cast<char*>(a.state), nullptr, a.channels, (long long)(a.taps - 1) * a.channels, 0, 0};
    Raw<T, VW, false> r;
    raw_load(r, s, b, a.taps - 1 + t, a.T, c, a.state ? n : 0);
    raw_get(r, s, c, o);
}

template <class T, int K>
__global__ void __launch_bounds__(kConvLanes * kConvRows) conv_forward_kernel(ConvArgs a) {
    constexpr int VW = conv_vw<K>();
    const int c = (blockIdx.x * kConvLanes + threadIdx.x % kConvLanes) * VW, n = a.channels - c;
    const int b = blockIdx.z;
    const int t0 = (blockIdx.y * kConvRows + threadIdx.x / kConvLanes) * kConvRun;
    if (n <= 0 || t0 >= a.T) return;
    const int len = clamp_len(a.lengths, b, a.T);
    float w[K][VW], bias[VW], x[K][VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) {
        bias[i] = a.bias && i < n ? a.bias[c + i] : 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) w[k][i] = i < n ? a.w[(long long)(c + i) * K + k] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < K - 1; ++k) conv_in<T, VW, false>(a, b, t0 - (K - 1) + k, len, c, n, x[k]);
#pragma unroll
    for (int j = 0; j < kConvRun; ++j) {
        const int t = t0 + j;
        if (t >= a.T) break;
        conv_in<T, VW, false>(a, b, t, len, c, n, x[K - 1]);
        float o[VW];
#pragma unroll
        for (int i = 0; i < VW; ++i) {
            float p = bias[i];
#pragma unroll
            for (int k = 0; k < K; ++k) p = fmaf(w[k][i], x[k][i], p);
            if (a.silu) p *= sigmoid(p);
            o[i] = t < len ? p : 0.0f;
        }
        store_vec<T, VW>(a.y, b, t, c, n, o);
#pragma unroll
        for (int k = 0; k < K - 1; ++k)
#pragma unroll
            for (int i = 0; i < VW; ++i) x[k][i] = x[k + 1][i];
    }
}

// The last taps - 1 inputs of each sample, oldest first.
template <class T>
__global__ void __launch_bounds__(256) conv_state_kernel(ConvArgs a) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(i % a.channels), k = (int)(i / a.channels % (a.taps - 1));
    const long long b = i / a.channels / (a.taps - 1);
    if (b >= a.batch) return;
    const int t = clamp_len(a.lengths, (int)b, a.T) - (a.taps - 1) + k;
    T v = T(0.0f);
    if (t >= 0)
        v = reinterpret_cast<const T*>(a.x.p)[b * a.x.sample + t * a.x.row + c];
    else if (a.state)
        v = reinterpret_cast<const T*>(a.state)[(b * (a.taps - 1) + a.taps - 1 + t) * a.channels + c];
    reinterpret_cast<T*>(a.state_out)[i] = v;
}

template <class T, int K>
__global__ void __launch_bounds__(kConvLanes * kConvRows) conv_backward_kernel(ConvArgs a) {
    constexpr int VW = conv_vw<K>();
    __shared__ float part[kConvRows][kConvLanes * VW + 1];
    const int lane = threadIdx.x % kConvLanes, row = threadIdx.x / kConvLanes;
    const int c = (blockIdx.x * kConvLanes + lane) * VW, n = a.channels - c;
    const int b = blockIdx.z;
    const int t0 = (blockIdx.y * kConvRows + row) * kConvRun;
    const int len = clamp_len(a.lengths, b, a.T);
    // g[k]: dy act'(pre) of steps t - (K - 1) + k
    float w[K][VW], dw[K][VW], x[K][VW], g[K][VW], bias[VW], db[VW];
#pragma unroll
    for (int i = 0; i < VW; ++i) {
        bias[i] = a.bias && i < n ? a.bias[c + i] : 0.0f;
        db[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            w[k][i] = i < n ? a.w[(long long)(c + i) * K + k] : 0.0f;
            dw[k][i] = x[k][i] = g[k][i] = 0.0f;
        }
    }
    if (n > 0 && t0 < a.T) {
#pragma unroll
        for (int k = 0; k < K - 1; ++k) conv_in<T, VW, true>(a, b, t0 - (K - 1) + k, len, c, n, x[k]);
        const int t_end = min(a.T, t0 + kConvRun);
        for (int t = t0; t < t_end + K - 1; ++t) {
            // past the run the outputs only give their share of its dx
            conv_in<T, VW, true>(a, b, t, t < a.T ? len : 0, c, n, x[K - 1]);
            float dy[VW];
            Raw<T, VW, false> r;
            raw_load(r, a.dy, b, t, a.T, c, t < len ? n : 0);
            raw_get(r, a.dy, c, dy);
#pragma unroll
            for (int i = 0; i < VW; ++i) {
                float d = dy[i];
                if (a.silu) {
                    float p = bias[i], y, ds;
#pragma unroll
                    for (int k = 0; k < K; ++k) p = fmaf(w[k][i], x[k][i], p);
                    dsilu(p, y, ds);
                    d *= ds;
                }
                d = t < len ? d : 0.0f;
                g[K - 1][i] = d;
                if (t < t_end) {
                    db[i] += d;
#pragma unroll
                    for (int k = 0; k < K; ++k) dw[k][i] = fmaf(d, x[k][i], dw[k][i]);
                }
            }
            // x[s] was read by outputs s .. s + K - 1: output s + j with tap K - 1 - j
            const int s = t - (K - 1);
            if (s >= t0) {
                float o[VW];
#pragma unroll
                for (int i = 0; i < VW; ++i) {
                    float v = 0.0f;
#pragma unroll
                    for (int j = 0; j < K; ++j) v = fmaf(w[K - 1 - j][i], g[j][i], v);
                    o[i] = v;
                }
                if (a.dstate_out && s < len) {
                    // x[s] is entry s - (len - (K - 1)) of the state after the last step
                    const int e = s - (len - (K - 1));
                    if (e >= 0)
#pragma unroll
                        for (int i = 0; i < VW; ++i)
                            if (i < n)
                                o[i] += (float)reinterpret_cast<const T*>(
                                    a.dstate_out)[((long long)b * (K - 1) + e) * a.channels + c + i];
                }
#pragma unroll
                for (int i = 0; i < VW; ++i) o[i] = s < len ? o[i] : 0.0f;
                store_vec<T, VW>(a.dx, b, s, c, n, o);
            }
#pragma unroll
            for (int k = 0; k < K - 1; ++k)
#pragma unroll
                for (int i = 0; i < VW; ++i) x[k][i] = x[k + 1][i], g[k][i] = g[k + 1][i];
        }
    }
    // the workgroup's share of dw and dbias: its runs in order
#pragma unroll
    for (int k = 0; k <= K; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VW; ++i) part[row][lane * VW + i] = k < K ? dw[k < K ? k : 0][i] : db[i];
        __syncthreads();
        if (threadIdx.x < kConvLanes * VW) {
            const int cc = blockIdx.x * kConvLanes * VW + threadIdx.x;
            float v = 0.0f;
#pragma unroll
            for (int r = 0; r < kConvRows; ++r) v += part[r][threadIdx.x];
            if (cc < a.channels)
                a.part[(((long long)b * a.tiles + blockIdx.y) * (K + 1) + k) * a.channels + cc] = v;
        }
    }
}

// Gradient of the state before the first step: entry e is x[e - (K - 1)],
// read by the outputs up to its K-th step, or kept as an entry of the state
// after a sample shorter than the window.
template <class T>
__global__ void __launch_bounds__(256) conv_dstate_kernel(ConvArgs a) {
    const int K = a.taps;
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(i % a.channels), e = (int)(i / a.channels % (K - 1));
    const int b = (int)(i / a.channels / (K - 1));
    if (b >= a.batch) return;
    const int len = clamp_len(a.lengths, b, a.T);
    const int s = e - (K - 1);
    float v = 0.0f;
    for (int t = 0; t <= s + K - 1 && t < len; ++t) {
        float p = a.bias ? a.bias[c] : 0.0f;
        for (int k = 0; k < K; ++k) {
            float x[1];
            conv_in<T, 1, true>(a, b, t - (K - 1) + k, len, c, 1, x);
            p = fmaf(a.w[(long long)c * K + k], x[0], p);
        }
        float y, ds = 1.0f;
        if (a.silu) dsilu(p, y, ds);
        const float dy = (float)reinterpret_cast<const T*>(a.dy.p)[b * a.dy.sample + t * a.dy.row + c];
        v = fmaf(a.w[(long long)c * K + K - 1 - (t - s)], dy * ds, v);
    }
    const int o = s - (len - (K - 1));
    if (a.dstate_out && o >= 0)
        v += (float)reinterpret_cast<const T*>(a.dstate_out)[((long long)b * (K - 1) + o) * a.channels + c];
    reinterpret_cast<T*>(a.dstate)[i] = (T)v;
}

// dw and dbias from the workgroups' shares: 32 channels of one tap a
// workgroup, the shares in 8 interleaved runs that are added up in order.
__global__ void __launch_bounds__(256) conv_sums_kernel(ConvArgs a) {
    __shared__ float part[8][32];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, k = blockIdx.y, run = threadIdx.x / 32;
    const int rows = a.batch * a.tiles;
    float v = 0.0f;
    if (c < a.channels)
        for (int r = run; r < rows; r += 8) v += a.part[((long long)r * (a.taps + 1) + k) * a.channels + c];
    part[run][threadIdx.x % 32] = v;
    __syncthreads();
    if (run || c >= a.channels) return;
#pragma unroll
    for (int r = 1; r < 8; ++r) v += part[r][threadIdx.x];
    if (k < a.taps)
        a.dw[(long long)c * a.taps + k] = v;
    else if (a.dbias)
        a.dbias[c] = v;
}

// One step.  A thread reads all of a channel's window before it writes, so
// the new state may take the old one's place.
template <class T>
__global__ void __launch_bounds__(256) conv_step_kernel(ConvArgs a) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    const int c = (int)(i % a.channels);
    const long long b = i / a.channels;
    if (b >= a.batch) return;
    const int K = a.taps;
    T old[SNN_SEQ_MAX_TAPS];
    float p = a.bias ? a.bias[c] : 0.0f;
#pragma unroll
    for (int k = 0; k < SNN_SEQ_MAX_TAPS; ++k) {
        if (k >= K) break;
        old[k] = k == K - 1 ? reinterpret_cast<const T*>(a.x.p)[b * a.x.sample + c]
                 : a.state  ? reinterpret_cast<const T*>(a.state)[(b * (K - 1) + k) * a.channels + c]
                            : T(0.0f);
        p = fmaf(a.w[(long long)c * K + k], (float)old[k], p);
    }
    if (a.silu) p *= sigmoid(p);
    reinterpret_cast<T*>(a.y.p)[b * a.y.sample + c] = (T)p;
#pragma unroll
    for (int k = 1; k < SNN_SEQ_MAX_TAPS; ++k) {
        if (k >= K) break;
        if (a.state_out) reinterpret_cast<T*>(a.state_out)[(b * (K - 1) + k - 1) * a.channels + c] = old[k];
    }
}

template <class T, int K>
hipError_t conv_pass(const ConvArgs& a, bool back, hipStream_t s) {
    constexpr int VW = conv_vw<K>();
    const dim3 grid((a.channels + kConvLanes * VW - 1) / (kConvLanes * VW), a.tiles, a.batch);
    if (back)
        conv_backward_kernel<T, K><<<grid, kConvLanes * kConvRows, 0, s>>>(a);
    else
        conv_forward_kernel<T, K><<<grid, kConvLanes * kConvRows, 0, s>>>(a);
    return hipGetLastError();
}

template <class T>
hipError_t conv_by_taps(const ConvArgs& a, bool back, hipStream_t s) {
    switch (a.taps) {
        case 1: return conv_pass<T, 1>(a, back, s);
        case 2: return conv_pass<T, 2>(a, back, s);
        case 3: return conv_pass<T, 3>(a, back, s);
        case 4: return conv_pass<T, 4>(a, back, s);
        case 5: return conv_pass<T, 5>(a, back, s);
        case 6: return conv_pass<T, 6>(a, back, s);
        case 7: return conv_pass<T, 7>(a, back, s);
        default: return conv_pass<T, 8>(a, back, s);
    }
}

unsigned blocks(long long n) { return (unsigned)((n + 255) / 256); }

}  // namespace

int conv_tiles(int T) { return (T + kConvRun * kConvRows - 1) / (kConvRun * kConvRows); }

hipError_t launch_conv_forward(const ConvArgs& a, int dtype, hipStream_t s) {
    SEQ_BY_TYPE(dtype, T, {
        hipError_t e = conv_by_taps<T>(a, false, s);
        if (e != hipSuccess) return e;
        if (a.state_out && a.taps > 1) {
            conv_state_kernel<T><<<blocks((long long)a.batch * (a.taps - 1) * a.channels), 256, 0, s>>>(a);
            e = hipGetLastError();
        }
        return e;
    });
}

hipError_t launch_conv_backward(const ConvArgs& a, int dtype, hipStream_t s) {
    SEQ_BY_TYPE(dtype, T, {
        hipError_t e = conv_by_taps<T>(a, true, s);
        if (e != hipSuccess) return e;
        conv_sums_kernel<<<dim3((a.channels + 31) / 32, a.taps + 1), 256, 0, s>>>(a);
        if (a.dstate && a.taps > 1)
            conv_dstate_kernel<T><<<blocks((long long)a.batch * (a.taps - 1) * a.channels), 256, 0, s>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_conv_step(const ConvArgs& a, int dtype, hipStream_t s) {
    SEQ_BY_TYPE(dtype, T, {
        conv_step_kernel<T><<<blocks((long long)a.batch * a.channels), 256, 0, s>>>(a);
        return hipGetLastError();
    });
}
