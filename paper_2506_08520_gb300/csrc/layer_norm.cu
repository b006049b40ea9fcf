// Layer norm over the last axis, forward and backward (sm_103a).
//
// Forward, per row of C values: mean = sum x / C, var = sum (x - mean)^2 / C,
// rstd = (var + eps)^-1/2, y = (x - mean) rstd w + b.  The row stays in
// registers between the two sums, so the variance is that of the centred
// values (no cancellation) and x is read once.
// Backward, xh = (x - mean) rstd, g = dy w:
//   dx = rstd (g - mean_C(g) - xh mean_C(g xh)),  dw = sum_rows dy xh,  db = sum_rows dy.
// Each thread owns the same columns of every row its CTA takes, sums dw and
// db for them in registers, and writes one partial row per CTA; a second
// kernel adds the partial rows in a fixed order (no atomics: the same bits
// every time).
// Both directions are bound by memory: 2 (forward) and 3 (backward) elements
// moved per element, about 8 and 14 operations.  Measured: forward of 262144 rows of
// 180 in bf16 35 us (5.4 TB/s; loads without copies ahead 46 at 64 registers, 38 at 88),
// backward of 16384 x 4096 in bf16 88 us + 6 for the sums (4.3 TB/s).  The backward
// pass issues 350 instructions a thread and row at 15 warps an SM (114 registers): 44% of
// the issue slots, waiting for its shuffles and shared memory.  xh, formed once a row,
// takes the registers of x (formed again for dx: 6 us more); weights in shared memory
// instead of registers give three CTAs an SM and were slower all the same (115 us).
// Rows that do not fit the registers (forward above 8192 values in fp32 and 16384 in 16
// bits, backward above 8192, less where rows are not aligned) go value by value.
#include "common.cuh"
#include "layer.cuh"
#include "pack.cuh"
#include "ptx.cuh"

namespace nystra {

// VEC weight or bias values, fp32 or of the type of x.  `wide`: they start on the
// boundaries of one load.
template <typename T, int VEC>
__device__ __forceinline__ void load_param(float (&f)[VEC], const void* p, int at, bool p32, bool wide, float none) {
    if (p == nullptr) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = none;
    } else if (p32) {
        const float* q = static_cast<const float*>(p) + at;
        if (VEC % 4 == 0 && wide) {
#pragma unroll
            for (int e = 0; e < VEC; e += 4)
                *reinterpret_cast<float4*>(f + (VEC % 4 == 0 ? e : 0)) = __ldg(reinterpret_cast<const float4*>(q + e));
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = __ldg(q + e);
        }
    } else {
        const T* q = static_cast<const T*>(p) + at;
        if (wide) {
            Pack<T, VEC> x;
            x.load(q);
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = to_f32(x.v[e]);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = to_f32(q[e]);
        }
    }
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Sums of K values over the TPR threads of a row, the same bits in each of
// them.  Up to 32 threads: lanes of a warp.  Wider rows own the CTA; `scratch`
// is written alternately in two halves, so one barrier per sum is enough.
template <int TPR, int K>
__device__ __forceinline__ void row_sum(float (&x)[K], float (*scratch)[32 * 2], int& half) {
    static_assert(K <= 2, "");
#pragma unroll
    for (int o = TPR < 32 ? TPR / 2 : 16; o; o >>= 1)
#pragma unroll
        for (int k = 0; k < K; ++k) x[k] += __shfl_xor_sync(0xffffffffu, x[k], o);
    if constexpr (TPR > 32) {
        constexpr int W = TPR / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) {
#pragma unroll
            for (int k = 0; k < K; ++k) scratch[half][warp * 2 + k] = x[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {  // W is a power of two up to 16: every half warp adds all of them
            float s = scratch[half][(lane & (W - 1)) * 2 + k];
#pragma unroll
            for (int o = W / 2; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            x[k] = s;
        }
        half ^= 1;
    }
}

// The shape of a row in registers: TPR threads, NV packs of VEC columns each.
constexpr int cta_threads(int tpr) { return tpr <= 32 ? 128 : tpr; }

struct NormFwd {
    const void* x;
    const void* w;
    const void* b;
    void* y;
    float* mean;
    float* rstd;
    long long xs, ys, rows;
    int C;
    float eps;
    bool w32, wide;  // wide: weight and bias can be read in packs
};

// The next rows' values are copied ahead into shared memory.  Each thread
// copies what it will read itself, so a wait for its own copies is all it takes.
constexpr int kAhead = 3;  // rows in flight, the current one among them

template <int BYTES>
__device__ __forceinline__ void copy_ahead(void* dst, const void* src) {
    const uint32_t d = static_cast<uint32_t>(__cvta_generic_to_shared(dst));
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(d), "l"(src) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(d), "l"(src), "n"(BYTES) : "memory");
}

// TPR threads per row (lanes of a warp, or the whole CTA), NV packs of VEC columns
// per thread, R rows at a time.
template <typename T, int VEC, int NV, int TPR, int R>
__global__ void __launch_bounds__(cta_threads(TPR)) layer_norm_kernel(const NormFwd a) {
    constexpr int GROUPS = cta_threads(TPR) / TPR;
    constexpr bool HOLD = R > 1 && NV * VEC <= 12;  // weight and bias stay in registers over the rows
    constexpr bool AHEAD = VEC * sizeof(T) >= 4;    // cp.async moves 4 bytes at least
    constexpr int THREADS = cta_threads(TPR);
    using P = Pack<T, VEC>;
    __shared__ float scratch[2][32 * 2];
    extern __shared__ __align__(16) unsigned char ring[];  // [kAhead][R][NV][THREADS] packs
    int half = 0;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const float invC = 1.f / (float)a.C;
    float w[HOLD ? NV : 1][VEC], b[HOLD ? NV : 1][VEC];
    if constexpr (HOLD) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * VEC;
            if (c < a.C) {
                load_param<T, VEC>(w[i], a.w, c, a.w32, a.wide, 1.f);
                load_param<T, VEC>(b[i], a.b, c, a.w32, a.wide, 0.f);
            }
        }
    }
    // every lane of a warp takes part in its sums, so the rows of a warp end together
    const long long step = (long long)gridDim.x * GROUPS * R, first = (long long)blockIdx.x * GROUPS * R;
    const auto slot = [&](int d, int r, int i) {
        return reinterpret_cast<P*>(ring) + (((d * R + r) * NV + i) * THREADS + threadIdx.x);
    };
    const auto fetch = [&](long long row0, int d) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row0 + r >= a.rows) break;
            const T* p = static_cast<const T*>(a.x) + (row0 + r) * a.xs;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * VEC;
                if (c < a.C) copy_ahead<VEC * sizeof(T)>(slot(d, r, i), p + c);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if constexpr (AHEAD) {
#pragma unroll
        for (int d = 0; d < kAhead - 1; ++d) fetch(first + group * R + d * step, d);
    }
    int d = 0;
    for (long long base = first; base < a.rows; base += step) {
        const long long row0 = base + group * R;
        P x[R][NV];
        if constexpr (AHEAD) {
            fetch(row0 + (kAhead - 1) * step, d == 0 ? kAhead - 1 : d - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * VEC;
                if (c < a.C && row0 + r < a.rows) {
                    if constexpr (AHEAD)
                        x[r][i] = *slot(d, r, i);
                    else
                        x[r][i].load(static_cast<const T*>(a.x) + (row0 + r) * a.xs + c);
                } else {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) x[r][i].v[e] = from_f32<T>(0.f);
                }
            }
        }
        d = d == kAhead - 1 ? 0 : d + 1;
        float mean[R], rstd[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[0] += to_f32(x[r][i].v[e]);
            row_sum<TPR>(s, scratch, half);
            mean[r] = s[0] * invC;
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s[1] = {0.f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if ((t + i * TPR) * VEC < a.C) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const float d = to_f32(x[r][i].v[e]) - mean[r];
                        s[0] = fmaf(d, d, s[0]);
                    }
                }
            }
            row_sum<TPR>(s, scratch, half);
            rstd[r] = rsqrtf(fmaf(s[0], invC, a.eps));
            if (t == 0 && row0 + r < a.rows) {
                if (a.mean) a.mean[row0 + r] = mean[r];
                if (a.rstd) a.rstd[row0 + r] = rstd[r];
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * VEC;
            if (c >= a.C) continue;
            float wi[VEC], bi[VEC];
            if constexpr (HOLD) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    wi[e] = w[i][e];
                    bi[e] = b[i][e];
                }
            } else {
                load_param<T, VEC>(wi, a.w, c, a.w32, a.wide, 1.f);
                load_param<T, VEC>(bi, a.b, c, a.w32, a.wide, 0.f);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                if (row0 + r >= a.rows) continue;
                P y;
#pragma unroll
                for (int e = 0; e < VEC; ++e)
                    y.v[e] = from_f32<T>(fmaf((to_f32(x[r][i].v[e]) - mean[r]) * rstd[r], wi[e], bi[e]));
                y.store(static_cast<T*>(a.y) + (row0 + r) * a.ys + c);
            }
        }
    }
    if constexpr (AHEAD) asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// Rows that do not fit the registers: a CTA per row that reads it three times
// (the second and third time from the caches), any C and alignment.
template <typename T>
__global__ void __launch_bounds__(512) layer_norm_long_kernel(const NormFwd a) {
    __shared__ float scratch[2][32 * 2];
    int half = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* p = static_cast<const T*>(a.x) + row * a.xs;
        float s[1] = {0.f};
        for (int c = threadIdx.x; c < a.C; c += 512) s[0] += to_f32(p[c]);
        row_sum<512>(s, scratch, half);
        const float mean = s[0] / (float)a.C;
        s[0] = 0.f;
        for (int c = threadIdx.x; c < a.C; c += 512) {
            const float d = to_f32(p[c]) - mean;
            s[0] = fmaf(d, d, s[0]);
        }
        row_sum<512>(s, scratch, half);
        const float rstd = rsqrtf(s[0] / (float)a.C + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (int c = threadIdx.x; c < a.C; c += 512) {
            float w[1], b[1];
            load_param<T, 1>(w, a.w, c, a.w32, false, 1.f);
            load_param<T, 1>(b, a.b, c, a.w32, false, 0.f);
            static_cast<T*>(a.y)[row * a.ys + c] = from_f32<T>(fmaf((to_f32(p[c]) - mean) * rstd, w[0], b[0]));
        }
    }
}

struct NormBwd {
    const void* dy;
    const void* x;
    const float* mean;
    const float* rstd;
    const void* w;
    void* dx;
    float* part;  // [grid][2][C]: this CTA's sums of dy xh and dy; null: none wanted
    long long dys, xs, dxs, rows;
    int C;
    bool w32, wide;  // wide: the weight can be read in packs
};

template <typename T, int VEC, int NV, int TPR>
__global__ void __launch_bounds__(cta_threads(TPR)) layer_norm_backward_kernel(const NormBwd a) {
    constexpr int THREADS = cta_threads(TPR), GROUPS = THREADS / TPR;
    constexpr bool AHEAD = VEC * sizeof(T) >= 4;  // cp.async moves 4 bytes at least
    using P = Pack<T, VEC>;
    __shared__ float scratch[2][32 * 2];
    // [kAhead][x, dy][NV][THREADS] packs and [kAhead][mean, rstd][THREADS]; at the end the groups' sums
    extern __shared__ __align__(16) unsigned char ring[];
    int half = 0;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const float invC = 1.f / (float)a.C;
    // Columns go in pairs of fp32 (the second of a lone column is 0): half the instructions.
    constexpr int H = (VEC + 1) / 2;
    uint64_t w[NV][H], dw[NV][H], db[NV][H];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * VEC;
        float f[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) f[e] = 0.f;
        if (c < a.C) load_param<T, VEC>(f, a.w, c, a.w32, a.wide, 1.f);
#pragma unroll
        for (int e = 0; e < H; ++e) {
            w[i][e] = pack_x2(f[2 * e], 2 * e + 1 < VEC ? f[2 * e + 1 < VEC ? 2 * e + 1 : 0] : 0.f);
            dw[i][e] = db[i][e] = 0ull;
        }
    }
    const auto pair = [](const Pack<T, VEC>& p, int e) {
        return pack_x2(to_f32(p.v[2 * e]), 2 * e + 1 < VEC ? to_f32(p.v[2 * e + 1 < VEC ? 2 * e + 1 : 0]) : 0.f);
    };
    const long long step = (long long)gridDim.x * GROUPS;
    const auto slot = [&](int d, int which, int i) {
        return reinterpret_cast<P*>(ring) + (((d * 2 + which) * NV + i) * THREADS + threadIdx.x);
    };
    const auto stat = [&](int d, int which) {
        return reinterpret_cast<float*>(ring + kAhead * 2 * NV * THREADS * sizeof(P)) + (d * 2 + which) * THREADS +
               threadIdx.x;
    };
    const auto fetch = [&](long long row, int d) {
        if (row < a.rows) {
            const T* px = static_cast<const T*>(a.x) + row * a.xs;
            const T* pd = static_cast<const T*>(a.dy) + row * a.dys;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int c = (t + i * TPR) * VEC;
                if (c < a.C) {
                    copy_ahead<VEC * sizeof(T)>(slot(d, 0, i), px + c);
                    copy_ahead<VEC * sizeof(T)>(slot(d, 1, i), pd + c);
                }
            }
            copy_ahead<4>(stat(d, 0), a.mean + row);
            copy_ahead<4>(stat(d, 1), a.rstd + row);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const long long first = (long long)blockIdx.x * GROUPS;
    if constexpr (AHEAD) {
#pragma unroll
        for (int d = 0; d < kAhead - 1; ++d) fetch(first + group + d * step, d);
    }
    int d = 0;
    // every lane of a warp takes part in its sums, so the rows of a warp end together
    for (long long base = first; base < a.rows; base += step) {
        const long long row = base + group;
        const bool live = row < a.rows;
        P x[NV], dy[NV];
        if constexpr (AHEAD) {
            fetch(row + (kAhead - 1) * step, d == 0 ? kAhead - 1 : d - 1);
            asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
        }
        float mean = 0.f, rstd = 0.f;
        if (live) {
            mean = AHEAD ? *stat(d, 0) : __ldg(a.mean + row);
            rstd = AHEAD ? *stat(d, 1) : __ldg(a.rstd + row);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * VEC;
            if (live && c < a.C) {
                if constexpr (AHEAD) {
                    x[i] = *slot(d, 0, i);
                    dy[i] = *slot(d, 1, i);
                } else {
                    x[i].load(static_cast<const T*>(a.x) + row * a.xs + c);
                    dy[i].load(static_cast<const T*>(a.dy) + row * a.dys + c);
                }
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    x[i].v[e] = from_f32<T>(0.f);
                    dy[i].v[e] = from_f32<T>(0.f);
                }
            }
        }
        d = d == kAhead - 1 ? 0 : d + 1;
        // xh = (x - mean) rstd: x rstd - mean rstd would be off by a rounding of the mean's size.  The
        // second of a lone column stays 0, however large the mean.
        const uint64_t scale = pack_x2(rstd, rstd), shift = pack_x2(-mean, VEC > 1 ? -mean : 0.f);
        uint64_t s0 = 0ull, s1 = 0ull, xh[NV][H];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            // columns behind C must not meet a mean or rstd that is not finite
            if ((t + i * TPR) * VEC < a.C) {
#pragma unroll
                for (int e = 0; e < H; ++e) {
                    const uint64_t f = pair(dy[i], e), g = mul_x2(f, w[i][e]);
                    xh[i][e] = mul_x2(add_x2(pair(x[i], e), shift), scale);
                    s0 = add_x2(s0, g);
                    s1 = fma_x2(g, xh[i][e], s1);
                    dw[i][e] = fma_x2(f, xh[i][e], dw[i][e]);
                    db[i][e] = add_x2(db[i][e], f);
                }
            }
        }
        const float2 t0 = unpack_x2(s0), t1 = unpack_x2(s1);
        float s[2] = {t0.x + t0.y, t1.x + t1.y};
        row_sum<TPR>(s, scratch, half);
        // dx = rstd g - (rstd c1 + rstd c2 xh)
        const float c1 = -s[0] * invC * rstd, c2 = -s[1] * invC * rstd;
        const uint64_t k1 = pack_x2(c1, c1), k2 = pack_x2(c2, c2);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (t + i * TPR) * VEC;
            if (!live || c >= a.C) continue;
            P o;
#pragma unroll
            for (int e = 0; e < H; ++e) {
                const uint64_t g = mul_x2(pair(dy[i], e), w[i][e]);
                const float2 y = unpack_x2(fma_x2(g, scale, fma_x2(xh[i][e], k2, k1)));
                o.v[2 * e] = from_f32<T>(y.x);
                if (2 * e + 1 < VEC) o.v[2 * e + 1 < VEC ? 2 * e + 1 : 0] = from_f32<T>(y.y);
            }
            o.store(static_cast<T*>(a.dx) + row * a.dxs + c);
        }
    }
    if constexpr (AHEAD) asm volatile("cp.async.wait_group 0;" ::: "memory");
    if (a.part == nullptr) return;
    if constexpr (GROUPS > 1) {  // the CTA's groups, added in their order
        uint64_t* fold = reinterpret_cast<uint64_t*>(ring);  // [GROUPS - 1][NV * H][2][TPR]
        __syncthreads();
        const auto at = [&](int gr, int i, int e, int k) { return ((gr * NV * H + i * H + e) * 2 + k) * TPR + t; };
        if (group > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < H; ++e) {
                    fold[at(group - 1, i, e, 0)] = dw[i][e];
                    fold[at(group - 1, i, e, 1)] = db[i][e];
                }
        }
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < H; ++e)
                for (int gr = 0; gr < GROUPS - 1; ++gr) {
                    dw[i][e] = add_x2(dw[i][e], fold[at(gr, i, e, 0)]);
                    db[i][e] = add_x2(db[i][e], fold[at(gr, i, e, 1)]);
                }
    }
    float* part = a.part + (long long)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (t + i * TPR) * VEC;
        if (c >= a.C) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const float2 fw = unpack_x2(dw[i][e / 2]), fb = unpack_x2(db[i][e / 2]);
            part[c + e] = e % 2 ? fw.y : fw.x;
            part[a.C + c + e] = e % 2 ? fb.y : fb.x;
        }
    }
}

// Shared memory of the kernel above: the ring, or the sums that take its place.
template <typename T, int VEC, int NV, int TPR>
constexpr int backward_smem() {
    const int ahead = VEC * (int)sizeof(T) >= 4 ? kAhead * 2 * cta_threads(TPR) * (NV * VEC * (int)sizeof(T) + 4) : 0;
    const int fold = (cta_threads(TPR) / TPR - 1) * NV * ((VEC + 1) / 2) * 2 * TPR * 8;
    return ahead > fold ? ahead : fold;
}

// Rows that do not fit the registers: the CTA's partial row lies in the
// workspace and is added to there, by the thread that owns the column.
template <typename T>
__global__ void __launch_bounds__(512) layer_norm_backward_long_kernel(const NormBwd a) {
    __shared__ float scratch[2][32 * 2];
    int half = 0;
    const float invC = 1.f / (float)a.C;
    float* part = a.part ? a.part + (long long)blockIdx.x * 2 * a.C : nullptr;
    if (part)
        for (int c = threadIdx.x; c < a.C; c += 512) part[c] = part[a.C + c] = 0.f;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* px = static_cast<const T*>(a.x) + row * a.xs;
        const T* pd = static_cast<const T*>(a.dy) + row * a.dys;
        const float mean = __ldg(a.mean + row), rstd = __ldg(a.rstd + row);
        float s[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < a.C; c += 512) {
            float w[1];
            load_param<T, 1>(w, a.w, c, a.w32, false, 1.f);
            const float d = to_f32(pd[c]), xh = (to_f32(px[c]) - mean) * rstd, g = d * w[0];
            s[0] += g;
            s[1] = fmaf(g, xh, s[1]);
            if (part) {
                part[c] = fmaf(d, xh, part[c]);
                part[a.C + c] += d;
            }
        }
        row_sum<512>(s, scratch, half);
        const float c1 = s[0] * invC, c2 = s[1] * invC;
        for (int c = threadIdx.x; c < a.C; c += 512) {
            float w[1];
            load_param<T, 1>(w, a.w, c, a.w32, false, 1.f);
            const float xh = (to_f32(px[c]) - mean) * rstd, g = to_f32(pd[c]) * w[0];
            static_cast<T*>(a.dx)[row * a.dxs + c] = from_f32<T>(rstd * (g - c1 - xh * c2));
        }
    }
}

// dw and db: the sum of `parts` partial rows.  A CTA takes 32 columns of one
// of the two; its 32 warps each add every 32nd partial row, then one warp
// adds the warps' sums.
template <typename W>
__global__ void __launch_bounds__(1024) layer_norm_fold_kernel(const float* part, int parts, int C, W* dw, W* db) {
    __shared__ float sums[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + lane;
    W* out = blockIdx.y == 0 ? dw : db;
    float s = 0.f;
    if (c < C)
        for (int p = warp; p < parts; p += 32) s += part[((long long)p * 2 + blockIdx.y) * C + c];
    sums[warp][lane] = s;
    __syncthreads();
    s = warp_sum(sums[lane][warp]);  // column `warp` of this CTA
    const int o = blockIdx.x * 32 + warp;
    if (lane == 0 && o < C && out) out[o] = from_f32<W>(s);
}

}  // namespace nystra

namespace nystra_host {
using namespace nystra;

namespace {

int sm_count(cudaError_t* e) {
    int dev = 0, sms = 0;
    if ((*e = cudaGetDevice(&dev)) == cudaSuccess)
        *e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    return sms;
}

// The widest pack that every row start allows.
template <typename T>
int pack_of(int C, long long strides, uintptr_t pointers) {
    for (int v = 16 / (int)sizeof(T); v > 1; v /= 2)
        if (C % v == 0 && strides % v == 0 && pointers % (v * sizeof(T)) == 0) return v;
    return 1;
}

// Shapes of the register kernels: threads per row and packs per thread for a
// row of `packs` packs; threads = 0: the row does not fit.  The fewest threads that
// `most` packs each cover (more work per sum over the lanes), then the fewest packs.
struct RowShape {
    int threads, nv;
};
constexpr RowShape row_shape(int packs, int most) {
    for (int threads : {8, 16, 32, 128, 256, 512})
        for (int nv = 1; nv <= most; ++nv)
            if (packs <= threads * nv && (nv < 4 || threads >= 32)) return {threads, nv};
    return {0, 0};
}
// Whether a row takes this shape: if any does, the longest that it covers.
constexpr bool row_taken(int threads, int nv, int most) {
    const RowShape s = row_shape(threads * nv, most);
    return s.threads == threads && s.nv == nv;
}
// The shapes that rows take with two packs at most or with four: no kernel is built that no call reaches.
#define NYSTRA_ROWS(ROW)                                                       \
    ROW(8, 1) ROW(8, 2) ROW(8, 3) ROW(16, 2) ROW(16, 3) ROW(32, 2) ROW(32, 3)  \
    ROW(32, 4) ROW(128, 1) ROW(128, 2) ROW(128, 3) ROW(128, 4) ROW(256, 2)     \
    ROW(256, 3) ROW(256, 4) ROW(512, 2) ROW(512, 3) ROW(512, 4)
#define NYSTRA_ROW(TPR, NV) static_assert(row_taken(TPR, NV, 2) || row_taken(TPR, NV, 4), "no row takes this shape");
NYSTRA_ROWS(NYSTRA_ROW)
#undef NYSTRA_ROW
// ... and no row goes without: every shape that is taken has a kernel.
#define NYSTRA_ROW(TPR, NV) +(row_taken(TPR, NV, MOST) ? 1 : 0)
template <int MOST> constexpr bool rows_complete() {
    int taken = 0;
    for (int threads : {8, 16, 32, 128, 256, 512})
        for (int nv = 1; nv <= MOST; ++nv) taken += row_taken(threads, nv, MOST);
    return taken == 0 NYSTRA_ROWS(NYSTRA_ROW);
}
#undef NYSTRA_ROW
static_assert(rows_complete<2>() && rows_complete<4>(), "a row's shape has no kernel");

template <typename T, int VEC, int NV, int TPR>
cudaError_t run_fwd(const NormFwd& a, int sms, cudaStream_t st) {
    constexpr int R = TPR > 32 ? 1 : NV == 1 ? 4 : NV <= 3 ? 2 : 1, PER = cta_threads(TPR) / TPR * R;
    constexpr int smem = VEC * sizeof(T) >= 4 ? kAhead * R * NV * cta_threads(TPR) * VEC * (int)sizeof(T) : 0;
    auto k = layer_norm_kernel<T, VEC, NV, TPR, R>;
    static std::atomic<int> cache[kMaxDevices];
    int most = 0;
    const cudaError_t e = persistent_grid(k, cta_threads(TPR), smem, cache, &most);
    if (e != cudaSuccess) return e;
    const long long want = (a.rows + PER - 1) / PER;
    k<<<(unsigned)(want < most ? want : most), cta_threads(TPR), smem, st>>>(a);
    return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t pick_fwd(const NormFwd& a, int sms, cudaStream_t st) {
    const RowShape s = row_shape(a.C / VEC, 4);
#define NYSTRA_ROW(TPR, NV)                    \
    if constexpr (row_taken(TPR, NV, 4))       \
        if (s.threads == TPR && s.nv == NV) return run_fwd<T, VEC, NV, TPR>(a, sms, st);
    NYSTRA_ROWS(NYSTRA_ROW)
#undef NYSTRA_ROW
    const long long most = (long long)sms * 4;
    layer_norm_long_kernel<T><<<(unsigned)(a.rows < most ? a.rows : most), 512, 0, st>>>(a);
    return cudaGetLastError();
}

// Whether weight and bias can be read in packs of v: 16 bytes of fp32 at most at once.
bool params_wide(const void* w, const void* b, int v, size_t es) {
    const size_t to = es == 4 ? (v < 4 ? v * 4 : 16) : v * es;
    return (((uintptr_t)w | (uintptr_t)b) & (to - 1)) == 0;
}

template <typename T>
cudaError_t fwd(NormFwd a, int sms, cudaStream_t st) {
    const int v = pack_of<T>(a.C, a.xs | a.ys, (uintptr_t)a.x | (uintptr_t)a.y);
    a.wide = params_wide(a.w, a.b, v, a.w32 ? 4 : sizeof(T));
    if constexpr (sizeof(T) == 2)
        if (v == 8) return pick_fwd<T, 8>(a, sms, st);
    if (v == 4) return pick_fwd<T, 4>(a, sms, st);
    if (v == 2) return pick_fwd<T, 2>(a, sms, st);
    return pick_fwd<T, 1>(a, sms, st);
}

// Each launches at most *grid CTAs, and leaves in *grid how many: the partial rows there are.
template <typename T, int VEC, int NV, int TPR>
cudaError_t run_bwd(const NormBwd& a, int* grid, cudaStream_t st) {
    constexpr int smem = backward_smem<T, VEC, NV, TPR>();
    auto k = layer_norm_backward_kernel<T, VEC, NV, TPR>;
    static std::atomic<int> cache[kMaxDevices];
    int most = 0;
    const cudaError_t e = persistent_grid(k, cta_threads(TPR), smem, cache, &most);
    if (e != cudaSuccess) return e;
    if (most < *grid) *grid = most;
    k<<<*grid, cta_threads(TPR), smem, st>>>(a);
    return cudaGetLastError();
}

template <typename T, int VEC>
cudaError_t pick_bwd(const NormBwd& a, int* grid, cudaStream_t st) {
    // Sums, weights and values of 16 columns at most: more leave too few registers for two CTAs on an SM.
    constexpr int MOST = VEC == 8 ? 2 : 4;
    const RowShape s = row_shape(a.C / VEC, MOST);
#define NYSTRA_ROW(TPR, NV)                    \
    if constexpr (row_taken(TPR, NV, MOST))    \
        if (s.threads == TPR && s.nv == NV) return run_bwd<T, VEC, NV, TPR>(a, grid, st);
    NYSTRA_ROWS(NYSTRA_ROW)
#undef NYSTRA_ROW
    if (*grid > 152 * 4) *grid = 152 * 4;
    layer_norm_backward_long_kernel<T><<<*grid, 512, 0, st>>>(a);
    return cudaGetLastError();
}

template <typename T>
cudaError_t bwd(NormBwd a, int* grid, cudaStream_t st) {
    const int v = pack_of<T>(a.C, a.xs | a.dys | a.dxs, (uintptr_t)a.x | (uintptr_t)a.dy | (uintptr_t)a.dx);
    a.wide = params_wide(a.w, nullptr, v, a.w32 ? 4 : sizeof(T));
    if constexpr (sizeof(T) == 2)
        if (v == 8) return pick_bwd<T, 8>(a, grid, st);
    if (v == 4) return pick_bwd<T, 4>(a, grid, st);
    if (v == 2) return pick_bwd<T, 2>(a, grid, st);
    return pick_bwd<T, 1>(a, grid, st);
}

template <typename W>
cudaError_t fold(const float* part, int parts, int C, void* dw, void* db, cudaStream_t st) {
    layer_norm_fold_kernel<W><<<dim3((C + 31) / 32, 2), 1024, 0, st>>>(part, parts, C, static_cast<W*>(dw),
                                                                      static_cast<W*>(db));
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_layer_norm(const void* x, long long xs, const void* w, const void* b, void* y, long long ys,
                              float* mean, float* rstd, long long rows, int C, float eps, int dtype, bool w32,
                              cudaStream_t st) {
    cudaError_t e;
    const int sms = sm_count(&e);
    if (e != cudaSuccess) return e;
    const NormFwd a{x, w, b, y, mean, rstd, xs, ys, rows, C, eps, w32, false};
    return dtype == 0 ? fwd<float>(a, sms, st) : dtype == 1 ? fwd<__nv_bfloat16>(a, sms, st) : fwd<__half>(a, sms, st);
}

int layer_norm_parts(long long rows, int C) {
    // One partial row per CTA, of which at most so many run at once (128 threads
    // take rows of up to 512 values, more threads longer ones).
    const long long most = 152 * (C <= 512 ? 16 : C <= 2048 ? 8 : 4);
    const long long want = (rows + 3) / 4;
    return (int)(want < 1 ? 1 : want < most ? want : most);
}

cudaError_t launch_layer_norm_backward(const void* dy, long long dys, const void* x, long long xs, const float* mean,
                                       const float* rstd, const void* w, void* dx, long long dxs, void* dw, void* db,
                                       long long rows, int C, int dtype, bool w32, float* part, cudaStream_t st) {
    int parts = layer_norm_parts(rows, C);
    const bool wanted = dw || db;
    const NormBwd a{dy, x, mean, rstd, w, dx, wanted ? part : nullptr, dys, xs, dxs, rows, C, w32, false};
    cudaError_t e = cudaSuccess;
    if (rows > 0)
        e = dtype == 0   ? bwd<float>(a, &parts, st)
            : dtype == 1 ? bwd<__nv_bfloat16>(a, &parts, st)
                         : bwd<__half>(a, &parts, st);
    if (e != cudaSuccess || !wanted) return e;
    const int n = rows > 0 ? parts : 0;
    if (w32 || dtype == 0) return fold<float>(part, n, C, dw, db, st);
    return dtype == 1 ? fold<__nv_bfloat16>(part, n, C, dw, db, st) : fold<__half>(part, n, C, dw, db, st);
}

}  // namespace nystra_host
