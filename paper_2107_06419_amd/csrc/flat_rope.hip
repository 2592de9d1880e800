// Rotary positions of Q and K (and their gradient: the same with the opposite angle).
//
// The work is one read and one write of every element, so what matters beside wide accesses is that the angle costs nothing: a thread
// has VP pairs of one position, finds their sines and cosines once, and applies them to every head it is given (all of them in long calls;
// in short ones the heads are spread over threads instead, since there latency counts).
//
// Angles.  p * freq is needed modulo a turn, and p may be far: in fp32 the angle at position 10^6 would be off by 0.06.  p * (freq / 2 pi)
// is formed in fp64, its nearest integer is taken off, and only the fraction of a turn that remains becomes fp32 (off by 2^-26 of a turn at most).
#include "flat_cache8.hpp"
#include "flat_common.hpp"

namespace flat {

namespace {

constexpr int kThreads = 256;
constexpr int kAhead = 4;  // heads whose loads are issued together

struct RopeArgs {
    const void* in[2];
    void* out[2];
    int heads0, heads_all;
    int N, d, rot;
    const double* freqs;
    const int* positions;
    float magnitude, sign;
    int rows;             // B * N
    int chunks;           // work items of a row: rot / 2 / VP to turn, then those that are copied
    int turn_chunks;
    int copy_elems;       // elements of a copied item
    int heads_per_block;  // heads of one thread
    Divisor by_chunks, by_N;
};

template <typename T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T>
struct Vec<T, 1> {
    typedef T type;
};
template <typename V, int N>
__device__ __forceinline__ float get(const V& v, int i) {
    if constexpr (N == 1) return (float)v;
    else return (float)v[i];
}
template <typename T, typename V, int N>
__device__ __forceinline__ void set(V& v, int i, float x) {
    if constexpr (N == 1) v = (T)x;
    else v[i] = (T)x;
}

template <typename T, int VP, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rope_kernel(const RopeArgs a) {
    typedef typename Vec<T, VP>::type half_t;
    typedef typename Vec<T, 2 * VP>::type pair_t;
    const unsigned item = blockIdx.x * (unsigned)kThreads + threadIdx.x;
    if (item >= (unsigned)a.rows * (unsigned)a.chunks) return;
    const int row = a.by_chunks.quotient((int)item), chunk = (int)item - row * a.chunks;
    const int b = a.by_N.quotient(row), n = row - b * a.N;
    const int h0 = blockIdx.y * a.heads_per_block, h1 = min(h0 + a.heads_per_block, a.heads_all);
    auto at = [&](int h) __attribute__((always_inline)) {  // element offset of row n of head h
        const int second = h >= a.heads0, hh = h - (second ? a.heads0 : 0), H = second ? a.heads_all - a.heads0 : a.heads0;
        return ((size_t)((long long)b * H + hh) * a.N + n) * a.d;
    };
    if (chunk >= a.turn_chunks) {  // channels that do not turn
        const int c = a.rot + (chunk - a.turn_chunks) * a.copy_elems;
        for (int h = h0; h < h1; ++h) {
            const int s = h >= a.heads0;
            if (a.in[s] == a.out[s]) continue;
            const T* x = (const T*)a.in[s] + at(h) + c;
            T* y = (T*)a.out[s] + at(h) + c;
            if (a.copy_elems > 1) *(uint4v*)y = *(const uint4v*)x;
            else *y = *x;
        }
        return;
    }
    const int i0 = chunk * VP, c0 = INTERLEAVED ? 2 * i0 : i0, c1 = i0 + a.rot / 2;
    const double p = a.positions ? (double)a.positions[row] : (double)n;
    float cs[VP], sn[VP];
#pragma unroll
    for (int i = 0; i < VP; ++i) {
        double turns = p * (a.freqs[i0 + i] * 0.15915494309189533577);
        turns -= __builtin_rint(turns);
        float s, c;
        sincospif(2.0f * (float)turns, &s, &c);
        cs[i] = c * a.magnitude;
        sn[i] = s * a.sign;
    }
    for (int h = h0; h < h1; h += kAhead) {
        pair_t x[kAhead];
        half_t u[kAhead], v[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (h + k < h1) {
                const T* src = (const T*)a.in[h + k >= a.heads0] + at(h + k);
                if constexpr (INTERLEAVED) x[k] = *(const pair_t*)(src + c0);
                else u[k] = *(const half_t*)(src + c0), v[k] = *(const half_t*)(src + c1);
            }
        }
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
            if (h + k < h1) {
                T* dst = (T*)a.out[h + k >= a.heads0] + at(h + k);
                if constexpr (INTERLEAVED) {
                    pair_t y;
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        const float f = (float)x[k][2 * i], g = (float)x[k][2 * i + 1];
                        y[2 * i] = (T)(f * cs[i] - g * sn[i]);
                        y[2 * i + 1] = (T)(f * sn[i] + g * cs[i]);
                    }
                    *(pair_t*)(dst + c0) = y;
                } else {
                    half_t y, z;
#pragma unroll
                    for (int i = 0; i < VP; ++i) {
                        const float f = get<half_t, VP>(u[k], i), g = get<half_t, VP>(v[k], i);
                        set<T, half_t, VP>(y, i, f * cs[i] - g * sn[i]);
                        set<T, half_t, VP>(z, i, f * sn[i] + g * cs[i]);
                    }
                    *(half_t*)(dst + c0) = y;
                    *(half_t*)(dst + c1) = z;
                }
            }
        }
    }
}

template <typename T, int VP, bool INTERLEAVED>
hipError_t launch(RopeArgs& a, hipStream_t stream) {
    a.turn_chunks = a.rot / 2 / VP;
    constexpr int kWide = 16 / (int)sizeof(T);
    a.copy_elems = a.rot % kWide == 0 ? kWide : 1;  // d is a multiple of kWide, so the rest of a row then starts and ends on 16 bytes
    a.chunks = a.turn_chunks + (a.d - a.rot) / a.copy_elems;
    const long long blocks = ((long long)a.rows * a.chunks + kThreads - 1) / kThreads;  // rows * chunks < 2^31: rows * d is
    a.by_chunks = Divisor(a.chunks);
    // heads of a thread: all once the items alone fill the chip (2048 blocks of 256), else as few as bring that many blocks
    const long long want = 2048;
    a.heads_per_block = (int)((long long)a.heads_all * blocks / want);
    a.heads_per_block = a.heads_per_block < 1 ? 1 : a.heads_per_block > a.heads_all ? a.heads_all : a.heads_per_block;
    if ((a.heads_all + a.heads_per_block - 1) / a.heads_per_block > 65535) a.heads_per_block = (a.heads_all + 65534) / 65535;
    const unsigned y = (unsigned)((a.heads_all + a.heads_per_block - 1) / a.heads_per_block);
    hipLaunchKernelGGL((rope_kernel<T, VP, INTERLEAVED>), dim3((unsigned)blocks, y), dim3(kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeProblem& p, hipStream_t stream) {
    RopeArgs a{{p.in[0], p.in[1]}, {p.out[0], p.out[1]}, p.heads[0], p.heads[0] + p.heads[1], p.N, p.d, p.rot, p.freqs, p.positions, p.magnitude,
               p.transpose ? -p.magnitude : p.magnitude, p.B * p.N, 0, 0, 0, 0, Divisor(1), Divisor(p.N)};
    const int half = p.rot / 2;
    // 16 bytes an access where the pairs come out even, else pair by pair
    if (p.f32) {
        if (p.interleaved) return half % 2 == 0 ? launch<float, 2, true>(a, stream) : launch<float, 1, true>(a, stream);
        return half % 4 == 0 ? launch<float, 4, false>(a, stream) : launch<float, 1, false>(a, stream);
    }
    if (p.interleaved) return half % 4 == 0 ? launch<bf16, 4, true>(a, stream) : launch<bf16, 1, true>(a, stream);
    return half % 8 == 0 ? launch<bf16, 8, false>(a, stream) : launch<bf16, 1, false>(a, stream);
}

}  // namespace flat
