// Rotary positions (sm_103a): feature pair i of a token at position p turns by
// the angle p f_i,
//   (u, v) -> A (u cos - v sin, u sin + v cos),
// pairs (i, i + r/2) ("half") or (2i, 2i + 1) ("interleaved"), i < r/2; the
// features behind r are copied.  The inverse turns by -p f_i: its result on an
// output's gradient is the input's gradient.
//
// Angles: in fp32 the product p f_i of a far position (10^6) is off by 0.06
// rad, and fp64 is slow here.  A frequency is kept as a 64-bit fixed-point
// fraction of a turn per token, F = 2^64 frac(f / 2 pi), and p F mod 2^64 is
// the angle's fraction of a turn: an integer product that wraps where the
// angle does, exact but for F's rounding (that of f / 2 pi in fp64, and 2^-65 of a turn).
//
// Bound by memory: each value is read and written once.  A thread keeps the
// sines of its pairs for several heads, which all turn alike.  2 x 8192 tokens of
// 32 + 8 heads of 128 in bf16, token-major: 53 us (6.3 TB/s); with four heads'
// loads in flight and two CTAs an SM instead of two heads' and four CTAs, 64.
#include "common.cuh"
#include "layer.cuh"
#include "pack.cuh"

namespace nystra {

constexpr int kRotThreads = 256;

struct RotArgs {
    nystra_host::RotaryTensor q, k;
    const double* inv_freq;
    const void* positions;
    long long positions_stride;
    float amplitude;
    int N, d, r, layout, inverse, positions32;
    int slots, turning;   // packs of a head's row that one thread each takes: slots, of which `turning` turn
    int heads_per_thread;
    long long tokens;     // n * N
};

template <typename T, int P, int LAYOUT>
__global__ void __launch_bounds__(kRotThreads, 4) rotary_kernel(const RotArgs a) {
    __shared__ unsigned long long turns[128];
    const int half = a.r / 2;
    for (int i = threadIdx.x; i < half; i += blockDim.x) {
        // of a negative frequency's size, then negated: 1 - f would cut a small one off at 2^-54
        const double f = fabs(a.inv_freq[i]) * 0.15915494309189533577;  // 1 / (2 pi)
        const unsigned long long t = __double2ull_rn((f - floor(f)) * 18446744073709551616.0);
        turns[i] = a.inv_freq[i] < 0 ? 0 - t : t;
    }
    __syncthreads();
    const int slot = threadIdx.x % a.slots;
    const int per_block = blockDim.x / a.slots;
    const bool turn = slot < a.turning;
    // offsets of the slot's two packs in a row
    const int i0 = slot * P;
    const int at0 = turn ? (LAYOUT == 0 ? i0 : 2 * i0) : a.r + (slot - a.turning) * 2 * P;
    const int at1 = turn && LAYOUT == 0 ? i0 + half : at0 + P;
    const bool two = at1 < a.d;
    const int h0 = blockIdx.y * a.heads_per_thread;
    const int h1 = min(h0 + a.heads_per_thread, a.q.heads + a.k.heads);
    for (long long tok = (long long)blockIdx.x * per_block + threadIdx.x / a.slots; tok < a.tokens;
         tok += (long long)gridDim.x * per_block) {
        const long long w = tok / a.N, t = tok - w * a.N;
        float cs[P], sn[P];
        if (turn) {
            long long p = t;
            if (a.positions)
                p = a.positions32 ? (long long)static_cast<const int*>(a.positions)[w * a.positions_stride + t]
                                  : static_cast<const long long*>(a.positions)[w * a.positions_stride + t];
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const long long f = (long long)(turns[i0 + e] * (unsigned long long)p);  // 2^-63 half turns
                sincospif(__ll2float_rn(f) * 1.0842021724855044e-19f, &sn[e], &cs[e]);
                cs[e] *= a.amplitude;
                sn[e] *= a.inverse ? -a.amplitude : a.amplitude;
            }
        }
        // Loads of two heads before the first store: out may be x itself, so the
        // compiler cannot move a later head's load over an earlier head's store.
        constexpr int HB = 2;
        for (int hb = h0; hb < h1; hb += HB) {
            Pack<T, P> u[HB], v[HB];
            T* py[HB];
#pragma unroll
            for (int j = 0; j < HB; ++j) {
                const int h = hb + j;
                if (h >= h1) break;
                const bool isk = h >= a.q.heads;
                const nystra_host::RotaryTensor& x = isk ? a.k : a.q;
                const int hh = isk ? h - a.q.heads : h;
                const T* px = static_cast<const T*>(x.x) + w * x.sx.n + hh * x.sx.head + t * x.sx.token;
                py[j] = static_cast<T*>(x.y) + w * x.sy.n + hh * x.sy.head + t * x.sy.token;
                u[j].load(px + at0);
                if (two) v[j].load(px + at1);
            }
#pragma unroll
            for (int j = 0; j < HB; ++j) {
                if (hb + j >= h1) break;
                if (turn) {
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        // half: element e of either pack; interleaved: elements 2e, 2e + 1 of the two packs in a row
                        const int e0 = 2 * e, e1 = 2 * e + 1;
                        T& y0 = LAYOUT == 0 ? u[j].v[e] : e0 < P ? u[j].v[e0 % P] : v[j].v[e0 % P];
                        T& y1 = LAYOUT == 0 ? v[j].v[e] : e1 < P ? u[j].v[e1 % P] : v[j].v[e1 % P];
                        const float x0 = to_f32(y0), x1 = to_f32(y1);
                        y0 = from_f32<T>(fmaf(x0, cs[e], -x1 * sn[e]));
                        y1 = from_f32<T>(fmaf(x0, sn[e], x1 * cs[e]));
                    }
                }
                u[j].store(py[j] + at0);
                if (two) v[j].store(py[j] + at1);
            }
        }
    }
}

}  // namespace nystra

namespace nystra_host {
using namespace nystra;

namespace {

template <typename T, int P>
cudaError_t run_rotary(RotArgs a, cudaStream_t st) {
    const bool in_place = (a.q.heads == 0 || a.q.x == a.q.y) && (a.k.heads == 0 || a.k.x == a.k.y);
    a.turning = a.r / 2 / P;
    a.slots = a.turning + (in_place ? 0 : (a.d - a.r + 2 * P - 1) / (2 * P));
    if (a.slots == 0) return cudaSuccess;  // in place and nothing turns
    const int per_block = kRotThreads / a.slots, heads = a.q.heads + a.k.heads;
    const long long blocks = (a.tokens + per_block - 1) / per_block;
    // Sines are worth sharing between heads once there are tokens enough to fill the GPU (152 SMs x 8 CTAs) without.
    int hpt = 8;
    while (hpt > 1 && blocks * ((heads + hpt - 1) / hpt) < 152 * 8) hpt /= 2;
    a.heads_per_thread = hpt;
    const int groups = (heads + hpt - 1) / hpt;
    if (groups > 65535) return cudaErrorInvalidConfiguration;
    const long long most = 152 * 16;
    const dim3 grid((unsigned)(blocks < most ? blocks : most), groups);
    if (a.layout == 0)
        rotary_kernel<T, P, 0><<<grid, per_block * a.slots, 0, st>>>(a);
    else
        rotary_kernel<T, P, 1><<<grid, per_block * a.slots, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t pick_rotary(const RotArgs& a, cudaStream_t st) {
    long long strides = 0;
    uintptr_t pointers = 0;
    for (const RotaryTensor* x : {&a.q, &a.k}) {
        if (x->heads == 0) continue;
        strides |= x->sx.n | x->sx.head | x->sx.token | x->sy.n | x->sy.head | x->sy.token;
        pointers |= (uintptr_t)x->x | (uintptr_t)x->y;
    }
    int v = 16 / (int)sizeof(T);
    for (; v > 1; v /= 2)
        if ((a.r / 2) % v == 0 && a.d % v == 0 && strides % v == 0 && pointers % (v * sizeof(T)) == 0) break;
    if constexpr (sizeof(T) == 2)
        if (v == 8) return run_rotary<T, 8>(a, st);
    if (v == 4) return run_rotary<T, 4>(a, st);
    if (v == 2) return run_rotary<T, 2>(a, st);
    return run_rotary<T, 1>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotaryTensor& q, const RotaryTensor& k, const double* inv_freq, int rotary,
                          const void* positions, bool positions32, long long positions_stride, float amplitude, int n,
                          int N, int d, int layout, bool inverse, int dtype, cudaStream_t st) {
    RotArgs a{};
    a.q = q;
    a.k = k;
    a.inv_freq = inv_freq;
    a.positions = positions;
    a.positions_stride = positions_stride;
    a.amplitude = amplitude;
    a.N = N;
    a.d = d;
    a.r = rotary;
    a.layout = layout;
    a.inverse = inverse;
    a.positions32 = positions32;
    a.tokens = (long long)n * N;
    return dtype == 0   ? pick_rotary<float>(a, st)
           : dtype == 1 ? pick_rotary<__nv_bfloat16>(a, st)
                        : pick_rotary<__half>(a, st);
}

}  // namespace nystra_host
