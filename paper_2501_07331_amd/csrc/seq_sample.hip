// A class drawn from each row of scores by a given random number, after
// temperature, top-k, top-p and min-p (include/snn_seq.h).
//
// Weights are whole numbers, exp((z - m) / temperature) in fp64 times 2^s,
// rounded, with s so large that a row's sum just fits 63 bits.  Their sums are
// exact in any order, so histograms may be filled by atomics, and a border is
// the same however the row is divided.
//
// What top-k, top-p and min-p keep is a beginning of the row in falling
// order, which ends at a key (the score's bits, made to order as unsigned)
// and a number of elements that have that key, the first ones by index.  The
// end is found without a sort: a histogram of counts and weights over kBins
// intervals of (m - z) / temperature, the interval in which the first of the
// limits is passed, and again inside that interval over equal parts of its
// keys, until a part is a single key.  The draw then goes over the row once
// in index order.
#include "seq_device.h"
#include "seq_sample.h"

namespace {

typedef unsigned long long u64;
constexpr int kBins = 2048;

// NaN orders below everything, as -inf.
__device__ __forceinline__ unsigned key_of(float z) {
    if (!(z == z)) z = -INFINITY;
    if (z == 0.0f) z = 0.0f;                       // -0 and 0 are one score
    const unsigned u = __float_as_uint(z);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float score_of(unsigned key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr unsigned kNegInf = 0x007fffffu;          // key_of(-inf)

// a * b / 2^shift, rounded down (up: ceil), of a 64-bit and a 24-bit number.
__device__ u64 scaled(u64 a, unsigned b, int shift, bool up) {
    const u64 lo = a * b, hi = __umul64hi(a, b);
    if (shift >= 128) return up && (lo | hi) ? 1 : 0;
    u64 v, rest;
    if (shift >= 64) {
        v = shift == 64 ? hi : hi >> (shift - 64);
        rest = lo | (shift == 64 ? 0 : hi & ((1ull << (shift - 64)) - 1));
    } else {
        v = shift ? (hi << (64 - shift)) | (lo >> shift) : lo;
        rest = lo & ((1ull << shift) - 1);
    }
    return v + (up && rest ? 1 : 0);
}
// a f, rounded down or up, for 0 <= f < 1
__device__ u64 share(u64 a, float f, bool up) {
    int e;
    const float m = frexpf(f, &e);                 // f = m 2^e, m a 24-bit fraction, e <= 0
    return scaled(a, (unsigned)ldexpf(m, 24), 24 - e, up);
}

// A row's parameters, with their defaults and limits.
struct RowArgs {
    float temperature, min_p, u;
    float top_p;
    int top_k;
};
__device__ __forceinline__ RowArgs row_args(const SampleArgs& a, int row) {
    RowArgs r;
    const float t = a.temperature ? a.temperature[row] : 1.0f;
    r.temperature = t == t ? t : 1.0f;
    const float q = a.min_p ? a.min_p[row] : 0.0f;
    r.min_p = q > 0.0f ? fminf(q, 1.0f) : 0.0f;
    const float p = a.top_p ? a.top_p[row] : 1.0f;
    r.top_p = p == p ? p : 1.0f;
    const int k = a.top_k ? a.top_k[row] : 0;
    r.top_k = k > 0 ? k : 0x7fffffff;
    const float u = a.u[row];
    r.u = u >= 0.0f ? fminf(u, 1.0f - 0x1p-24f) : 0.0f;
    return r;
}

// (m - z) / temperature: 0 for the largest scores, infinite ones among them.
__device__ __forceinline__ double depth64(float m, float z, float temperature) {
    if (z == m) return 0.0;
    return m == INFINITY ? (double)INFINITY : ((double)m - (double)z) / (double)temperature;
}
// its interval: a function that never falls as z falls
__device__ __forceinline__ int bin_of(float m, float z, float temperature) {
    const float x = z == m ? 0.0f : (m - z) / temperature * 64.0f;
    return (int)fminf(x, (float)(kBins - 1));
}

template <class T, int VW>
__device__ __forceinline__ void load_scores(const SampleArgs& a, int row, int i, float (&z)[VW]) {
    const T* p = reinterpret_cast<const T*>(a.scores) + (long long)row * a.row + i;
    if (i + VW <= a.n) {
        const typename Vec<T, VW>::type v = *reinterpret_cast<const typename Vec<T, VW>::type*>(p);
#pragma unroll
        for (int j = 0; j < VW; ++j) z[j] = (float)v[j];
    } else {
#pragma unroll
        for (int j = 0; j < VW; ++j) z[j] = i + j < a.n ? (float)p[j] : -INFINITY;
    }
}

// Inclusive sums over the wave's lanes.
template <class V>
__device__ __forceinline__ V wave_scan(V x) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const V y = __shfl_up(x, d);
        if ((int)(threadIdx.x & 63) >= d) x += y;
    }
    return x;
}
template <class V>
__device__ __forceinline__ V wave_sum(V x) {
#pragma unroll
    for (int d = 32; d; d /= 2) x += __shfl_xor(x, d);
    return x;
}

template <class T, int NT>
__global__ void __launch_bounds__(NT) sample_row_kernel(SampleArgs a) {
    constexpr int VW = sizeof(T) == 4 ? 4 : 8, W = NT / 64, PB = kBins / NT;
    __shared__ u64 mass[kBins];
    __shared__ unsigned count[kBins];
    __shared__ u64 wmass[W];
    __shared__ unsigned wcount[W];
    __shared__ struct {
        u64 mass, below;           // weight above the cut; that of the cut interval
        unsigned count, inside;    // elements above the cut; in the cut interval
        unsigned lo, hi;           // keys of the cut interval
        int bin, token;
    } cut;
    const int row = blockIdx.x, tid = threadIdx.x, wave = tid / 64, lane = tid % 64;
    const RowArgs r = row_args(a, row);

    // the largest score, as its key
    unsigned top = 0;
    for (int i = tid * VW; i < a.n; i += NT * VW) {
        float z[VW];
        load_scores<T, VW>(a, row, i, z);
#pragma unroll
        for (int j = 0; j < VW; ++j) top = max(top, i + j < a.n ? key_of(z[j]) : 0u);
    }
#pragma unroll
    for (int d = 32; d; d /= 2) top = max(top, (unsigned)__shfl_xor((int)top, d));
    if (lane == 0) wcount[wave] = top;
    if (tid == 0) cut.token = a.n;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w) top = max(top, wcount[w]);
    const float m = score_of(top);
    if (top <= kNegInf) {
        if (tid == 0) {
            a.token[row] = -1;
            if (a.logprob) a.logprob[row] = -INFINITY;
        }
        return;
    }
    if (!(r.temperature > 0.0f)) {
        int first = a.n;
        for (int i = tid * VW; i < a.n && first == a.n; i += NT * VW) {
            float z[VW];
            load_scores<T, VW>(a, row, i, z);
#pragma unroll
            for (int j = VW - 1; j >= 0; --j)
                if (i + j < a.n && key_of(z[j]) == top) first = i + j;
        }
        atomicMin(&cut.token, first);
        __syncthreads();
        if (tid == 0) {
            a.token[row] = cut.token;
            if (a.logprob) a.logprob[row] = 0.0f;
        }
        return;
    }

    const double unit = ldexp(1.0, a.shift);
    // the weight of a score that is kept by min-p; total gets every weight
    auto weigh = [&](float z, u64* total) {
        const double w = exp(-depth64(m, z, r.temperature));
        const u64 v = (u64)rint(w * unit);
        if (total) *total += v;
        return w >= (double)r.min_p ? v : ~0ull;
    };

    u64 all = 0, limit = 0;
    u64 above = 0;                 // weight and number of the elements above the interval
    unsigned n_above = 0;
    unsigned lo = kNegInf + 1, hi = top;   // the interval's keys
    unsigned end_key = 0, end_count = 0;   // where the kept ones end
    u64 kept = 0;                  // their weight
    for (int level = 0;; ++level) {
        int sh = 0;
        while ((hi - lo) >> sh >= (unsigned)kBins) ++sh;
        for (int i = tid; i < kBins; i += NT) mass[i] = 0, count[i] = 0;
        __syncthreads();
        u64 sum = 0;
        for (int i = tid * VW; i < a.n; i += NT * VW) {
            float z[VW];
            load_scores<T, VW>(a, row, i, z);
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                const unsigned key = key_of(z[j]);
                if (key < lo || key > hi) continue;
                const u64 w = weigh(z[j], &sum);
                if (w == ~0ull) continue;
                const int b = level ? (int)((hi - key) >> sh) : bin_of(m, z[j], r.temperature);
                atomicAdd(&mass[b], w);
                atomicAdd(&count[b], 1u);
            }
        }
        if (level == 0) {
            sum = wave_sum(sum);
            if (lane == 0) wmass[wave] = sum;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) all += wmass[w];
            limit = r.top_p >= 1.0f ? ~0ull : r.top_p > 0.0f ? max((u64)1, share(all, r.top_p, true)) : 1;
        }
        if (tid == 0) cut.bin = kBins;
        __syncthreads();
        // running sums over the intervals, PB a thread
        u64 tm = 0;
        unsigned tc = 0;
#pragma unroll
        for (int j = 0; j < PB; ++j) tm += mass[tid * PB + j], tc += count[tid * PB + j];
        const u64 sm = wave_scan(tm);
        const unsigned sc = wave_scan(tc);
        if (lane == 63) wmass[wave] = sm, wcount[wave] = sc;
        __syncthreads();
        u64 bm = above + sm - tm;
        unsigned bc = n_above + sc - tc;
        for (int w = 0; w < wave; ++w) bm += wmass[w], bc += wcount[w];
#pragma unroll
        for (int j = 0; j < PB; ++j) {
            const int b = tid * PB + j;
            const u64 em = bm + mass[b];
            const unsigned ec = bc + count[b];
            // the first interval at whose end a limit is reached or passed
            if (count[b] && (ec > (unsigned)r.top_k || em >= limit)) atomicMin(&cut.bin, b);
            bm = em, bc = ec;
        }
        __syncthreads();
        const int cb = cut.bin;
        if (cb / PB == tid || (cb == kBins && tid == NT - 1)) {
            // bm, bc are the sums at the end of this thread's intervals: back to the cut's start
            u64 x = bm;
            unsigned y = bc;
            if (cb < kBins)
                for (int b = (tid + 1) * PB - 1; b >= cb; --b) x -= mass[b], y -= count[b];
            cut.mass = x, cut.count = y;
            cut.below = cb < kBins ? mass[cb] : 0;
            cut.inside = cb < kBins ? count[cb] : 0;
        }
        if (tid == 0 && cb < kBins) {
            if (level) {
                cut.hi = hi - ((unsigned)cb << sh);
                cut.lo = max(lo, cut.hi - ((1u << sh) - 1));
            } else {
                // the keys of an interval of depth: its ends by bisection
                unsigned x = lo, y = hi;           // the least key with bin <= cb
                while (x < y) {
                    const unsigned k = x + (y - x) / 2;
                    if (bin_of(m, score_of(k), r.temperature) <= cb) y = k; else x = k + 1;
                }
                cut.lo = x;
                y = hi;                            // the largest with bin >= cb
                while (x < y) {
                    const unsigned k = y - (y - x) / 2;
                    if (bin_of(m, score_of(k), r.temperature) >= cb) x = k; else y = k - 1;
                }
                cut.hi = x;
            }
        }
        __syncthreads();
        above = cut.mass, n_above = cut.count;
        if (cb == kBins) {                         // nothing is cut off
            end_key = 0;
            kept = above;
            break;
        }
        lo = cut.lo, hi = cut.hi;
        if (lo == hi) {
            // a single key: as many as the limits leave
            end_key = lo;
            end_count = min(cut.inside, (unsigned)r.top_k - n_above);
            const u64 w = cut.below / cut.inside;
            if (above >= limit) end_count = 0;
            else if (w) end_count = (unsigned)min((u64)end_count, (limit - above - 1) / w + 1);
            kept = above + w * end_count;
            break;
        }
        __syncthreads();                           // cut is written again
    }

    // the draw: the first index whose running sum is above u times the total
    const u64 goal = share(kept, r.u, false);
    u64 run = 0;
    unsigned ties = 0;
    for (int base = 0; base < a.n; base += NT * VW) {
        const int i = base + tid * VW;
        float z[VW];
        u64 w[VW], tm = 0;
        unsigned tc = 0;
        if (i < a.n) load_scores<T, VW>(a, row, i, z);
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            w[j] = 0;
            const unsigned key = i + j < a.n ? key_of(z[j]) : 0;
            if (key <= kNegInf || key < end_key) continue;
            const u64 v = weigh(z[j], nullptr);
            if (v == ~0ull) continue;
            w[j] = v;
            if (key == end_key) tc += 1; else tm += v;
        }
        const unsigned sc = wave_scan(tc);
        __syncthreads();
        if (lane == 63) wcount[wave] = sc;
        __syncthreads();
        unsigned before = ties + sc - tc;
        for (int k = 0; k < wave; ++k) before += wcount[k];
        for (int k = 0; k < W; ++k) ties += wcount[k];
        // of the elements with the last key the first end_count by index
#pragma unroll
        for (int j = 0; j < VW; ++j) {
            const unsigned key = i + j < a.n ? key_of(z[j]) : 0;
            if (end_key && key == end_key && w[j]) {
                if (before >= end_count) w[j] = 0;
                ++before;
                tm += w[j];
            }
        }
        const u64 sm = wave_scan(tm);
        if (lane == 63) wmass[wave] = sm;
        __syncthreads();
        u64 at = run + sm - tm;
        for (int k = 0; k < wave; ++k) at += wmass[k];
        for (int k = 0; k < W; ++k) run += wmass[k];
        if (at <= goal && at + tm > goal) {        // one thread of the row
            int token = 0;
#pragma unroll
            for (int j = 0; j < VW; ++j) {
                if (at <= goal && at + w[j] > goal) token = j;
                at += w[j];
            }
            a.token[row] = i + token;
            float zt = z[0];
#pragma unroll
            for (int j = 1; j < VW; ++j) zt = token == j ? z[j] : zt;
            if (a.logprob) a.logprob[row] = (float)(-depth64(m, zt, r.temperature) - log((double)kept / unit));
        }
        if (run > goal) break;
    }
}

template <class T>
hipError_t sample(const SampleArgs& a, hipStream_t s) {
    if (a.n <= 4096)
        sample_row_kernel<T, 256><<<a.rows, 256, 0, s>>>(a);
    else
        sample_row_kernel<T, 1024><<<a.rows, 1024, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_sample(const SampleArgs& a, int dtype, hipStream_t s) {
    SEQ_BY_TYPE(dtype, T, return sample<T>(a, s));
}
