// Linear attention with a decay per head, 64 tokens at a time on the tensor
// cores (LinRole in layer.cuh; sm_103a).  With u counting the
// chunk's tokens, S the state that enters it and e0 = 1 (0 backward in time,
// where S has its first decay already), a chunk is
//   P_us = o_scale s_scale gamma^(u-s) a_u . b_s  (s <= u, else 0)
//   out_u = o_scale gamma^(u+e0) a_u S + sum_s P_us c_s
//   S <- gamma^64 S + sum_s w_s b_s c_s^T,   w_s = s_scale gamma^(64-e0-s).
//
// Each warp owns 16 rows of S^T (features of c) in registers, where they are the
// accumulator of the state's product and, packed in pairs, the A operand of
// S^T a^T: the state never leaves the registers.  So the output is formed as
// out^T = S^T a^T + c^T P^T, with P made by all warps together in shared memory.
//
// 16-bit types.  Roundings to 16 bits, each by half a step: P (but two parts of it in
// the first chunk that a sequence visits, if no state enters it or it is the only one:
// results of few terms would show the rounding as it is, not averaged over many); S as
// an operand (never the S that is carried); the result.  w_s c_s, the A operand of the state's
// product, is split into 16-bit parts: two where the state is only read again as
// such an operand, and in bf16 three, which carry all of fp32, where it is returned.
// fp16: P, S and w c are scaled by powers of two that put the largest of them
// at 2^14, so that 28 octaves below it stay normal numbers; their products
// accumulate in fp32 and are scaled back there.
//
// fp32.  Every operand is three bf16 parts, hi + mid + lo, which carry all of it,
// and a product takes the six MMAs of parts i + j <= 2: what is left out is 2^-24 of
// it.  The five small ones have accumulators of their own, since the tensor cores cut an
// accumulator off at every MMA (24 of them into one cost 9e-7 where 4 cost 3e-7).  Six
// times the MMAs are still fewer cycles than the same products on the fp32 units.  No rounding but fp32's own.
// Bound by issue and latency: a chunk of 64-feature heads is about 6000 warp
// instructions and 544 MMAs (650 of the 1400 cycles that its bytes take at the memory's
// rate, on one SM).  Measured (d = 64, fp16, 8 heads x 65536 tokens in 74 segments each):
// 87 us for the outputs with four CTAs an SM (with three a fifth more), 38 for the segments'
// states, 11 to combine them; 50% of issue slots, tensor pipe 41%.
#pragma once

#include <type_traits>

#include "common.cuh"
#include "layer.cuh"
#include "linear.cuh"
#include "pack.cuh"
#include "ptx.cuh"

namespace nystra {

constexpr int kChunk = 64;

// ------------------------------------------------------------ operands
// How values of type T lie in shared memory: kParts tiles of type E that add up to them.
template <typename T> struct ChunkIo {
    using E = T;
    static constexpr int kParts = 1, kStages = 2;
};
template <> struct ChunkIo<float> {
    using E = __nv_bfloat16;
    static constexpr int kParts = 3, kStages = 1;
};

// A tile of 64 rows of DP 16-bit values, in 16-byte pieces permuted within a row so
// that eight rows' pieces of one column (an ldmatrix block) lie in distinct banks.
// DP = 128: two panels of 64 columns.  A panel of 64 is the 128-byte swizzle that the
// tensor-core descriptors know (linear_umma.cu).
constexpr int kPanel = kChunk * 64;
template <int DP>
__device__ __forceinline__ int tile_at(int row, int col) {
    if constexpr (DP == 32) return row * 32 + (((col >> 3) ^ ((row >> 1) & 3)) << 3) + (col & 7);
    return (DP == 128 ? (col >> 6) * kPanel : 0) + row * 64 + ((((col >> 3) & 7) ^ (row & 7)) << 3) + (col & 7);
}
// From the shared-memory address of an element, the one `ks` blocks of 16 columns and
// `rb` blocks of 16 rows on: the pieces' permutation only depends on row mod 8.
template <int DP>
__device__ __forceinline__ uint32_t tile_step(uint32_t at, int ks, int rb) {
    return (at ^ ((ks & 3) << 5)) + (ks >> 2) * (kPanel * 2) + rb * (16 * (DP < 64 ? DP : 64) * 2);
}

// P: its ten blocks of 16 x 16 on and under the diagonal, row by row of blocks.  A
// row's two 16-byte pieces are swapped in every second group of four rows, for the banks.
constexpr int kBlocks = 10, kBlock = 256;
__device__ __forceinline__ constexpr int block_at(int bi, int bj) { return (bi * (bi + 1) / 2 + bj) * kBlock; }
__device__ __forceinline__ int in_block(int row, int piece) { return row * 16 + ((piece ^ ((row >> 2) & 1)) << 3); }

// ldmatrix row addresses of a 16 x 16 block of a tile: lane l gives the row
// (l & 7) + 8 (l >> 3 & 1) and column 8 (l >> 4) ("by rows": A operands stored
// row by row, and transposed B operands), or with the two bits swapped.
template <int DP, typename E>
__device__ __forceinline__ const E* by_rows(const E* tile, int row, int col, int lane) {
    return tile + tile_at<DP>(row + (lane & 15), col + (lane >> 4) * 8);
}
template <int DP, typename E>
__device__ __forceinline__ const E* by_cols(const E* tile, int row, int col, int lane) {
    return tile + tile_at<DP>(row + (lane & 7) + (lane >> 4) * 8, col + ((lane >> 3) & 1) * 8);
}
template <bool TRANS>
__device__ __forceinline__ void ldsm_at(uint32_t (&r)[4], uint32_t at) {
    if constexpr (TRANS)
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(at)
                     : "memory");
    else
        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                     : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                     : "r"(at)
                     : "memory");
}
// Four 8x8 blocks transposed on the way to shared memory: block i's column j
// becomes the eight values at the address of lane 8i + j.
__device__ __forceinline__ void stsm_x4_t(void* p, uint32_t r0, uint32_t r1, uint32_t r2, uint32_t r3) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(smem_addr(p)), "r"(r0),
                 "r"(r1), "r"(r2), "r"(r3)
                 : "memory");
}

// The 16 x 16 block's fragments of PARTS tiles TILE values apart.
template <int PARTS, int TILE, bool TRANS>
__device__ __forceinline__ void load_parts(uint32_t (&r)[PARTS][4], uint32_t at) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) ldsm_at<TRANS>(r[p], at + p * TILE * 2);
}
// Two 16 x 8 accumulators += a b over the parts that matter, the small products first.
template <typename E, int PA, int PB>
__device__ __forceinline__ void mma_parts(float (&c0)[4], float (&c1)[4], const uint32_t (&a)[PA][4],
                                          const uint32_t (&b)[PB][4]) {
    constexpr int MOST = (PA > PB ? PA : PB) - 1;
#pragma unroll
    for (int sum = MOST; sum >= 0; --sum)
#pragma unroll
        for (int i = 0; i <= sum; ++i) {
            const int j = sum - i;
            if (i < PA && j < PB) {
                Mma16<E>::k16(c0, a[i], b[j][0], b[j][1]);
                Mma16<E>::k16(c1, a[i], b[j][2], b[j][3]);
            }
        }
}
// The same with the small products in accumulators of their own (SMALL: there are
// any), so that the large ones' is cut off by its own products only.
template <typename E, int PA, int PB, bool SMALL>
__device__ __forceinline__ void mma_parts(float (&c0)[4], float (&c1)[4], float (&s0)[4], float (&s1)[4],
                                          const uint32_t (&a)[PA][4], const uint32_t (&b)[PB][4]) {
    if constexpr (!SMALL) {
        mma_parts<E, PA, PB>(c0, c1, a, b);
    } else {
#pragma unroll
        for (int sum = PA - 1; sum >= 0; --sum)
#pragma unroll
            for (int i = 0; i <= sum; ++i) {
                Mma16<E>::k16(sum ? s0 : c0, a[i], b[sum - i][0], b[sum - i][1]);
                Mma16<E>::k16(sum ? s1 : c1, a[i], b[sum - i][2], b[sum - i][3]);
            }
    }
}
// N accumulators set to zero, and the small products' added to them.
template <int N>
__device__ __forceinline__ void clear(float (&c)[N][4]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[i][e] = 0.f;
}
template <int N>
__device__ __forceinline__ void join(float (&c)[N][4], const float (&small)[N][4]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) c[i][e] += small[i][e];
}
// PARTS 16-bit values that add up to each of a pair of fp32 values.
template <typename E, int PARTS>
__device__ __forceinline__ void split_pair(uint32_t (&out)[PARTS], float x0, float x1) {
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        out[p] = Mma16<E>::pack(x0, x1);
        if (p + 1 < PARTS) {
            const float2 f = Mma16<E>::unpack(out[p]);
            x0 -= f.x;
            x1 -= f.y;
        }
    }
}
template <typename E, int PARTS>
__device__ __forceinline__ float2 join_pair(const uint32_t (&part)[PARTS]) {
    float2 f = Mma16<E>::unpack(part[PARTS - 1]);
#pragma unroll
    for (int p = PARTS - 2; p >= 0; --p) {
        const float2 h = Mma16<E>::unpack(part[p]);
        f.x += h.x;
        f.y += h.y;
    }
    return f;
}

// 2^e, e in -126..127.
__device__ __forceinline__ float pow2i(int e) { return __int_as_float((e + 127) << 23); }
// The exponent e with which x 2^e lies in [2^14, 2^15), held to -100..60; 0 for x = 0.
__device__ __forceinline__ int to_2_14(float x) {
    return x == 0.f ? 0 : min(max(14 + 127 - (int)(__float_as_uint(x) >> 23), -100), 60);
}

// ------------------------------------------------------------ global memory
template <int BYTES>
__device__ __forceinline__ void cp_async(uint32_t dst, const void* src, bool in) {
    const int n = in ? BYTES : 0;
    if constexpr (BYTES == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
    else
        asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(n)
                     : "memory");
}

// Rows 0..63 of a tile from global rows first, first + step, ...: `cnt` rows of d
// values, zeros elsewhere.  A thread takes one column piece of every RP-th row.
template <typename T, int DP, int THREADS, int BYTES>
__device__ __forceinline__ void load_rows(typename ChunkIo<T>::E* tile, const T* first, long long step, int d,
                                          int cnt) {
    using E = typename ChunkIo<T>::E;
    constexpr int V = BYTES / (int)sizeof(T), PER = DP / V, RP = THREADS / PER;
    static_assert(THREADS % PER == 0 && kChunk % RP == 0, "");
    const int row0 = threadIdx.x / PER, col = threadIdx.x % PER * V;
    const T* src = first + row0 * step + col;
    if constexpr (sizeof(T) == 2 && BYTES >= 4) {
        const uint32_t at = smem_addr(tile + tile_at<DP>(row0, col));
#pragma unroll
        for (int k = 0; k < kChunk / RP; ++k) {
            const bool in = row0 + k * RP < cnt && col < d;
            const uint32_t dst = RP % 8 == 0 ? at + k * RP * (DP < 64 ? DP : 64) * 2
                                             : smem_addr(tile + tile_at<DP>(row0 + k * RP, col));
            cp_async<BYTES>(dst, in ? src : first, in);
            src += RP * step;
        }
    } else {
        constexpr int U = kChunk / RP < 8 ? kChunk / RP : 8;  // rows in flight
#pragma unroll 1
        for (int k0 = 0; k0 < kChunk / RP; k0 += U) {
            Pack<T, V> x[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (row0 + (k0 + k) * RP < cnt && col < d) {
                    x[k].load(src);
                } else {
#pragma unroll
                    for (int e = 0; e < V; ++e) x[k].v[e] = from_f32<T>(0.f);
                }
                src += RP * step;
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                E* dst = tile + tile_at<DP>(row0 + (k0 + k) * RP, col);
                if constexpr (sizeof(T) == 2) {
                    *dst = x[k].v[0];
                } else {
#pragma unroll
                    for (int p = 0; p < ChunkIo<T>::kParts; ++p) {
                        Pack<E, V> y;
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            y.v[e] = from_f32<E>(x[k].v[e]);
                            x[k].v[e] -= to_f32(y.v[e]);
                        }
                        y.store(dst + p * kChunk * DP);
                    }
                }
            }
        }
    }
}
template <typename T, int DP, int THREADS>
__device__ __forceinline__ void load_tile(typename ChunkIo<T>::E* tile, const T* first, long long step, int d, int cnt,
                                          int bytes) {
    if (bytes == 16)
        load_rows<T, DP, THREADS, 16>(tile, first, step, d, cnt);
    else if (bytes == 8)
        load_rows<T, DP, THREADS, 8>(tile, first, step, d, cnt);
    else if (sizeof(T) == 4 || bytes == 4)
        load_rows<T, DP, THREADS, 4>(tile, first, step, d, cnt);
    else if constexpr (sizeof(T) == 2)
        load_rows<T, DP, THREADS, 2>(tile, first, step, d, cnt);
}

// The output tile: 16-bit values as in the tiles above, fp32 row by row with the groups
// of eight columns permuted by the row, so that an accumulator's lanes meet distinct banks.
template <typename T, int DP>
__device__ __forceinline__ int out_at(int row, int col) {
    if constexpr (sizeof(T) == 2) return tile_at<DP>(row, col);
    return row * DP + (col ^ (((row >> 1) & 3) << 3));
}
template <typename T, int DP, int THREADS, int BYTES>
__device__ __forceinline__ void store_rows(const T* tile, T* first, long long step, int d, int cnt) {
    constexpr int V = BYTES / (int)sizeof(T), PER = DP / V, RP = THREADS / PER;
    const int row0 = threadIdx.x / PER, col = threadIdx.x % PER * V;
    if (col >= d) return;
    T* to = first + row0 * step + col;
#pragma unroll 4
    for (int row = row0; row < cnt; row += RP) {
        Pack<T, V> x;
        x.load(tile + out_at<T, DP>(row, col));
        x.store(to);
        to += RP * step;
    }
}
template <typename T, int DP, int THREADS>
__device__ __forceinline__ void store_tile(const T* tile, T* first, long long step, int d, int cnt, int bytes) {
    if (bytes == 16)
        store_rows<T, DP, THREADS, 16>(tile, first, step, d, cnt);
    else if (bytes == 8)
        store_rows<T, DP, THREADS, 8>(tile, first, step, d, cnt);
    else if (sizeof(T) == 4 || bytes == 4)
        store_rows<T, DP, THREADS, 4>(tile, first, step, d, cnt);
    else if constexpr (sizeof(T) == 2)
        store_rows<T, DP, THREADS, 2>(tile, first, step, d, cnt);
}

// Rows behind a sequence: `rows` rows of d zeros, a thread a column piece of every RP-th row.
template <int THREADS, int BYTES>
__device__ __forceinline__ void zero_rows(unsigned char* first, long long step, int row_bytes, int rows) {
    const int per = row_bytes / BYTES, rp = THREADS / per;
    const int row0 = threadIdx.x / per, piece = threadIdx.x % per;
    if (row0 >= rp) return;
    using Raw = typename RawWord<BYTES>::type;
    unsigned char* to = first + row0 * step + piece * BYTES;
#pragma unroll 4
    for (int row = row0; row < rows; row += rp) {
        *reinterpret_cast<Raw*>(to) = Raw{};
        to += rp * step;
    }
}
template <typename T, int THREADS>
__device__ __forceinline__ void zero_tile(T* first, long long step, int d, int rows, int bytes) {
    unsigned char* const p = reinterpret_cast<unsigned char*>(first);
    const long long s = step * (long long)sizeof(T);
    const int n = d * (int)sizeof(T);
    if (bytes == 16)
        zero_rows<THREADS, 16>(p, s, n, rows);
    else if (bytes == 8)
        zero_rows<THREADS, 8>(p, s, n, rows);
    else if (sizeof(T) == 4 || bytes == 4)
        zero_rows<THREADS, 4>(p, s, n, rows);
    else if constexpr (sizeof(T) == 2)
        zero_rows<THREADS, 2>(p, s, n, rows);
}

// ------------------------------------------------------------ the kernel
// Powers of gamma with their factors, by what they multiply.
struct ChunkTables {
    float score[16 + kChunk];    // [16 + lag]: s_scale o_scale gamma^lag, 0 for lag < 0
    float inter[kChunk];         // [u]: o_scale gamma^(u + e0)
    float weight[2 * kChunk];    // [kChunk - cnt + s]: s_scale gamma^(cnt - e0 - s) for s < cnt, whatever cnt is
    unsigned int top[4];         // fp16: the chunk's largest score
};

template <typename T, int DP>
struct ChunkShape {
    using Io = ChunkIo<T>;
    static constexpr int kWarps = DP / 16, kThreads = kWarps * 32;
    static constexpr int kTile = kChunk * DP;  // values of one part of a tile
    static constexpr int kTiles = Io::kStages * 3 * Io::kParts * kTile;
    static constexpr int kScores = Io::kParts * kBlocks * kBlock;
    // In front of the tiles: room for what the first chunk's low part of P has more than its tile of a
    static constexpr int kPad = Io::kParts == 1 && kTile < kScores ? kScores - kTile : 0;
    static constexpr size_t kSmem = (kPad + kTiles + kScores) * 2 + sizeof(ChunkTables);
    // CTAs per SM that registers are cut for: 16 warps of 128, or what the fp32 tiles leave room for
    static constexpr int kResident = Io::kParts == 1 ? 16 / kWarps : 128 / DP;
};

// S^T <- gamma^cnt S^T + sum over the chunk's tokens of (w c)^T b.  The chunk's
// sum has accumulators of its own (32 registers, in two passes over the columns
// where there are more): the tensor cores cut an accumulator off where fp32
// rounds, and in thousands of additions to S itself that would show.
template <typename T, int DP, int PARTS>
__device__ __forceinline__ void update_state(float (&s)[DP / 8][4], uint32_t b_rows, uint32_t c_cols,
                                             const float* weight, const LinPower& g, int cnt, int db, int lane) {
    using E = typename ChunkIo<T>::E;
    using Op = Mma16<E>;
    constexpr bool SCALED = Op::kNarrowRange, SMALL = ChunkIo<T>::kParts > 1;
    constexpr int IN = ChunkIo<T>::kParts, TILE = kChunk * DP;
    const float* wt = weight + (kChunk - cnt) + (lane & 3) * 2;
    int ew = 0;
    if constexpr (SCALED) {
        float m = 0.f;
#pragma unroll
        for (int ks = 0; ks < kChunk / 16; ++ks) {
            uint32_t v[4];
            ldsm_at<true>(v, tile_step<DP>(c_cols, 0, ks));
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = Op::unpack(v[i]);
                m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
            }
        }
        // the last token's weight is the largest
        ew = to_2_14(warp_max_nonneg(m) * fabsf(weight[kChunk - 1]));
    }
    const float up = SCALED ? pow2i(ew) : 1.f, down = SCALED ? pow2i(-ew) : 1.f;
    constexpr int PASSES = DP > 64 ? 2 : 1, NP = DP / 16 / PASSES;  // pairs of column tiles of a pass
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        if (pass * NP * 16 >= db) break;
        float d[2 * NP][4], ds[SMALL ? 2 * NP : 2][4];
        clear(d);
        clear(ds);
#pragma unroll
        for (int ks = 0; ks < kChunk / 16; ++ks) {
            if (ks * 16 >= cnt) break;
            uint32_t v[IN][4], a[PARTS][4];
            load_parts<IN, TILE, true>(v, tile_step<DP>(c_cols, 0, ks));
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // rows g, g + 8 at tokens 2c, then at 2c + 8
                uint32_t in[IN], part[PARTS];
#pragma unroll
                for (int p = 0; p < IN; ++p) in[p] = v[p][i];
                const float2 f = join_pair<E, IN>(in);
                const float w0 = wt[ks * 16 + (i >> 1) * 8] * up, w1 = wt[ks * 16 + (i >> 1) * 8 + 1] * up;
                split_pair<E, PARTS>(part, f.x * w0, f.y * w1);
#pragma unroll
                for (int p = 0; p < PARTS; ++p) a[p][i] = part[p];
            }
#pragma unroll
            for (int np = 0; np < NP; ++np) {
                uint32_t b[IN][4];
                load_parts<IN, TILE, true>(b, tile_step<DP>(b_rows, pass * NP + np, ks));
                mma_parts<E, PARTS, IN, SMALL>(d[2 * np], d[2 * np + 1], ds[SMALL ? 2 * np : 0],
                                               ds[SMALL ? 2 * np + 1 : 1], a, b);
            }
        }
        if constexpr (SMALL) join(d, ds);
#pragma unroll
        for (int nt = 0; nt < 2 * NP; ++nt)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                float(&x)[4] = s[pass * 2 * NP + nt];
                if (SCALED) mul_x2(d[nt][e], d[nt][e + 1], down);
                g.decay2(x[e], x[e + 1], d[nt][e], d[nt][e + 1]);
            }
    }
}

// MAIN: outputs, from the state that enters the segment.  Otherwise the
// segment's own contribution to the state, from zero, into the workspace.
template <typename T, int DP, bool MAIN>
__global__ void __launch_bounds__(ChunkShape<T, DP>::kThreads, ChunkShape<T, DP>::kResident)
linear_chunk_kernel(const __grid_constant__ LinArgs args) {
    using Shape = ChunkShape<T, DP>;
    using Io = ChunkIo<T>;
    using E = typename Io::E;
    using Op = Mma16<E>;
    constexpr bool SCALED = Op::kNarrowRange, SMALL = Io::kParts > 1;
    constexpr int THREADS = Shape::kThreads, NW = Shape::kWarps, IN = Io::kParts, TILE = Shape::kTile;
    extern __shared__ __align__(1024) unsigned char smem[];
    E* const tiles = reinterpret_cast<E*>(smem) + Shape::kPad;  // stages of a, b, c
    E* const tp = tiles + Shape::kTiles;
    ChunkTables& tab = *reinterpret_cast<ChunkTables*>(tp + Shape::kScores);

    const LinRole& r = args.role[blockIdx.y];
    const int unit = blockIdx.x / args.segs, seg = blockIdx.x % args.segs;
    const int w = unit / args.heads, h = unit % args.heads;
    const int len = lin_length(args, w);
    const int u0 = seg * args.seg_len, u1 = min(u0 + args.seg_len, args.N);
    const int live = min(u1, len);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, c2 = (lane & 3) * 2;
    const int row0 = warp * 16;
    const LinDecay decay(args.log_decay[h]);
    const LinPower whole = decay.pair(kChunk);
    const int e0 = r.backward ? 0 : 1;
    // rows in the order of the visits
    const long long first = r.backward ? len - 1 - u0 : u0;
    const long long da = r.backward ? -r.sa.token : r.sa.token, dbs = r.backward ? -r.sb.token : r.sb.token,
                    dcs = r.backward ? -r.sc.token : r.sc.token, dos = r.backward ? -r.so.token : r.so.token;
    const T* pa = static_cast<const T*>(r.a) + w * r.sa.n + h * r.sa.head + first * r.sa.token;
    const T* pb = static_cast<const T*>(r.b) + w * r.sb.n + h * r.sb.head + first * r.sb.token;
    const T* pc = static_cast<const T*>(r.c) + w * r.sc.n + h * r.sc.head + first * r.sc.token;
    T* const out = static_cast<T*>(r.out) + w * r.so.n + h * r.so.head;
    T* po = out + first * r.so.token;

    const auto stage = [&](int i) { return tiles + (i % Io::kStages) * 3 * IN * TILE; };
    const auto load = [&](int i) {
        const long long at = (long long)i * kChunk;
        const int cnt = min(live - u0 - i * kChunk, kChunk);
        E* const st = stage(i);
        if (MAIN) load_tile<T, DP, THREADS>(st, pa + at * da, da, r.db, cnt, r.wa);
        load_tile<T, DP, THREADS>(st + IN * TILE, pb + at * dbs, dbs, r.db, cnt, r.wb);
        load_tile<T, DP, THREADS>(st + 2 * IN * TILE, pc + at * dcs, dcs, r.dc, cnt, r.wc);
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const int chunks = live > u0 ? (live - u0 + kChunk - 1) / kChunk : 0;
    // The second part that P has in the first chunk: in the stage that a single chunk leaves free, or
    // in the place of a, which nobody reads any more once the scores are made and no state meets it.
    E* const tp_low = chunks == 1 ? tiles + 3 * IN * TILE : tiles - Shape::kPad;
    if (Io::kStages == 2 && chunks > 0) load(0);
    for (int i = threadIdx.x; i < 2 * kChunk; i += THREADS) {
        const float p = decay.power(max(i - 16, 0));
        if (i < 16 + kChunk) tab.score[i] = i < 16 ? 0.f : r.s_scale * r.o_scale * p;
        if (i < kChunk) tab.inter[i] = r.o_scale * decay.power(i + e0);
        tab.weight[i] = i < kChunk ? r.s_scale * decay.power(kChunk - e0 - i) : 0.f;
    }
    if (MAIN) {  // rows behind the sequence (here, so that nothing of it stays in registers over the chunks)
        const int z0 = max(u0, len);
        zero_tile<T, THREADS>(out + z0 * r.so.token, r.so.token, r.dc, u1 - z0, r.wo);
    }

    // the state: rows row0 + g (+ 8), columns 8 nt + c2 (+ 1)
    float s[DP / 8][4];
    const float* s_in = nullptr;
    bool t_in = false;
    if (MAIN) {
        s_in = seg > 0 || (args.segs > 1 && r.s_in) ? lin_ws(args, blockIdx.y, unit, seg)
               : r.s_in ? r.s_in + (long long)unit * r.db * r.dc : nullptr;
        t_in = args.segs == 1 && r.transposed;
    }
#pragma unroll
    for (int nt = 0; nt < DP / 8; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = row0 + g + (e >> 1) * 8, b = nt * 8 + c2 + (e & 1);
            s[nt][e] = s_in && c < r.dc && b < r.db ? s_in[t_in ? c * r.db + b : b * r.dc + c] : 0.f;
        }
    bool has_state = s_in != nullptr;
    const bool keep = MAIN ? args.segs == 1 && r.s_out : true;  // whether the state behind the last chunk is wanted
    const bool exact = r.s_out && (!MAIN || args.segs == 1);    // ... as a result

    for (int i = 0; i < chunks; ++i) {
        const int cnt = min(live - u0 - i * kChunk, kChunk);
        // whether P has two parts: in the first chunk that the sequence visits
        [[maybe_unused]] const bool fine = IN == 1 && u0 == 0 && i == 0 && (chunks == 1 || !has_state);
        E *ta = stage(i), *tb = ta + IN * TILE, *tc = ta + 2 * IN * TILE;
        if constexpr (Io::kStages == 1) {
            __syncthreads();  // the last chunk's readers are done
            load(i);
        }
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (MAIN && SCALED && threadIdx.x == 0) tab.top[0] = 0u;
        __syncthreads();  // the stage has landed, and the other one is free
        if (Io::kStages == 2 && i + 1 < chunks) load(i + 1);
        const uint32_t c_cols = smem_addr(by_cols<DP>(tc, 0, row0, lane));

        if constexpr (MAIN) {
            const uint32_t a_rows = smem_addr(by_rows<DP>(ta, 0, 0, lane)),
                           a_cols = smem_addr(by_cols<DP>(ta, 0, 0, lane)),
                           b_cols = smem_addr(by_cols<DP>(tb, 0, 0, lane));
            // P, a 16 x 16 block at a time
            constexpr int PER = (kBlocks + NW - 1) / NW;
            float p[PER][2][4];
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int blk = warp + j * NW;
                const int bi = blk < 1 ? 0 : blk < 3 ? 1 : blk < 6 ? 2 : 3, bj = blk - bi * (bi + 1) / 2;
                if (blk >= kBlocks || bi * 16 >= cnt) break;
                float ps[2][4];
                clear(p[j]);
                clear(ps);
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks) {
                    uint32_t a[IN][4], b[IN][4];
                    load_parts<IN, TILE, false>(a, tile_step<DP>(a_rows, ks, bi));
                    load_parts<IN, TILE, false>(b, tile_step<DP>(b_cols, ks, bj));
                    mma_parts<E, IN, IN, SMALL>(p[j][0], p[j][1], ps[0], ps[1], a, b);
                }
                if constexpr (SMALL) join(p[j], ps);
                const float* f = tab.score + 16 + (bi - bj) * 16 + g - c2;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        // on the diagonal lags go down to -15
                        const float x = p[j][nt][e] * f[(e >> 1) * 8 - nt * 8 - (e & 1)];
                        p[j][nt][e] = bi == bj && g + (e >> 1) * 8 < nt * 8 + c2 + (e & 1) ? 0.f : x;
                        if (SCALED) most = fmaxf(most, fabsf(p[j][nt][e]));
                    }
            }
            int ep = 0;
            if constexpr (SCALED) {
                most = warp_max_nonneg(most);
                if (lane == 0) atomicMax(tab.top, __float_as_uint(most));
                __syncthreads();
                ep = to_2_14(__uint_as_float(tab.top[0]));
            } else if (fine && chunks > 1) {
                __syncthreads();  // a has been read
            }
            const float up = SCALED ? pow2i(ep) : 1.f;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const int blk = warp + j * NW;
                const int bi = blk < 1 ? 0 : blk < 3 ? 1 : blk < 6 ? 2 : 3;
                if (blk >= kBlocks || bi * 16 >= cnt) break;
#pragma unroll
                for (int nt = 0; nt < 2; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const float x0 = p[j][nt][e] * up, x1 = p[j][nt][e + 1] * up;
                        const int at = blk * kBlock + in_block(g + e * 4, nt) + c2;
                        uint32_t part[IN];
                        split_pair<E, IN>(part, x0, x1);
                        E* to = tp + at;
                        if (fine) {
                            uint32_t two[2];
                            split_pair<E, 2>(two, x0, x1);
                            *reinterpret_cast<uint32_t*>(tp_low + at) = two[1];
                        }
#pragma unroll
                        for (int q = 0; q < IN; ++q)
                            *reinterpret_cast<uint32_t*>(to + q * kBlocks * kBlock) = part[q];
                    }
            }
            // S^T a^T
            float o[kChunk / 8][4], os[SMALL ? kChunk / 8 : 2][4];
            clear(o);
            clear(os);
            if (has_state) {
                int es = 0;
                if constexpr (SCALED) {
                    float m = 0.f;
#pragma unroll
                    for (int nt = 0; nt < DP / 8; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(s[nt][e]));
                    es = to_2_14(warp_max_nonneg(m));
                }
                const float su = SCALED ? pow2i(es) : 1.f;
#pragma unroll
                for (int ks = 0; ks < DP / 16; ++ks) {
                    uint32_t a[IN][4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float* x = &s[2 * ks + (e >> 1)][(e & 1) * 2];
                        uint32_t part[IN];
                        float x0 = x[0], x1 = x[1];
                        if (SCALED) mul_x2(x0, x1, su);
                        split_pair<E, IN>(part, x0, x1);
#pragma unroll
                        for (int q = 0; q < IN; ++q) a[q][e] = part[q];
                    }
#pragma unroll
                    for (int np = 0; np < kChunk / 16; ++np) {
                        uint32_t b[IN][4];
                        load_parts<IN, TILE, false>(b, tile_step<DP>(a_cols, ks, np));
                        mma_parts<E, IN, IN, SMALL>(o[2 * np], o[2 * np + 1], os[SMALL ? 2 * np : 0],
                                                    os[SMALL ? 2 * np + 1 : 1], a, b);
                    }
                }
                if constexpr (SMALL) {
                    join(o, os);
                    clear(os);
                }
                // o_scale gamma^(u+e0) S a, in P's units
                const float f = SCALED ? pow2i(ep) * pow2i(-es) : 1.f;
#pragma unroll
                for (int nt = 0; nt < kChunk / 8; ++nt) {
                    float2 t = *reinterpret_cast<const float2*>(tab.inter + nt * 8 + c2);
                    if (SCALED) mul_x2(t.x, t.y, f);
                    fma_x2(o[nt][0], o[nt][1], o[nt][0], o[nt][1], t.x, t.y, 0.f, 0.f);
                    fma_x2(o[nt][2], o[nt][3], o[nt][2], o[nt][3], t.x, t.y, 0.f, 0.f);
                }
            }
            __syncthreads();  // P is there, and nobody reads a any more
            // + c^T P^T
            const int p_lane = in_block((lane & 7) + (lane >> 4) * 8, (lane >> 3) & 1);
            const uint32_t p_cols = smem_addr(tp + p_lane), p_low = smem_addr(tp_low + p_lane);
#pragma unroll
            for (int ks = 0; ks < kChunk / 16; ++ks) {
                if (ks * 16 >= cnt) break;
                uint32_t a[IN][4];
                load_parts<IN, TILE, true>(a, tile_step<DP>(c_cols, 0, ks));
#pragma unroll
                for (int np = ks; np < kChunk / 16; ++np) {
                    uint32_t b[IN][4];
                    load_parts<IN, kBlocks * kBlock, false>(b, p_cols + block_at(np, ks) * 2);
                    mma_parts<E, IN, IN, SMALL>(o[2 * np], o[2 * np + 1], os[SMALL ? 2 * np : 0],
                                                os[SMALL ? 2 * np + 1 : 1], a, b);
                    if (fine) {
                        ldsm_at<false>(b[0], p_low + block_at(np, ks) * 2);
                        Op::k16(o[2 * np], a[0], b[0][0], b[0][1]);
                        Op::k16(o[2 * np + 1], a[0], b[0][2], b[0][3]);
                    }
                }
            }
            if constexpr (SMALL) join(o, os);
            if (fine && chunks > 1) __syncthreads();  // P's second part has been read
            [[maybe_unused]] const float down = SCALED ? pow2i(-ep) : 1.f;
            T* const to = reinterpret_cast<T*>(ta);
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int np = 0; np < kChunk / 16; ++np) {
                    uint32_t x[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int nt = 2 * np + (e >> 1), k = (e & 1) * 2;
                        if (SCALED) mul_x2(o[nt][k], o[nt][k + 1], down);
                        x[e] = Op::pack(o[nt][k], o[nt][k + 1]);
                    }
                    stsm_x4_t(to + tile_at<DP>(np * 16 + (lane & 7) + (lane >> 4) * 8, row0 + ((lane >> 3) & 1) * 8),
                              x[0], x[1], x[2], x[3]);
                }
            } else {
#pragma unroll
                for (int nt = 0; nt < kChunk / 8; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        to[out_at<T, DP>(nt * 8 + c2 + (e & 1), row0 + g + (e >> 1) * 8)] = o[nt][e];
            }
        }
        if (i + 1 < chunks || keep) {
            const LinPower gc = cnt == kChunk ? whole : decay.pair(cnt);
            const uint32_t b_rows = smem_addr(by_rows<DP>(tb, 0, 0, lane));
            if constexpr (IN == 3) {
                update_state<T, DP, 3>(s, b_rows, c_cols, tab.weight, gc, cnt, r.db, lane);
            } else if (!SCALED && exact) {
                update_state<T, DP, 3>(s, b_rows, c_cols, tab.weight, gc, cnt, r.db, lane);
            } else {
                update_state<T, DP, 2>(s, b_rows, c_cols, tab.weight, gc, cnt, r.db, lane);
            }
            has_state = true;
        }
        if constexpr (MAIN) {
            __syncthreads();  // the output tile is whole
            store_tile<T, DP, THREADS>(reinterpret_cast<const T*>(ta), po + (long long)i * kChunk * dos, dos, r.dc, cnt,
                                       r.wo);
        }
    }
    if (!keep) return;
    float* e_out = MAIN ? r.s_out + (long long)unit * r.db * r.dc : lin_ws(args, blockIdx.y, unit, seg);
    const bool t_out = MAIN && r.transposed;
#pragma unroll
    for (int nt = 0; nt < DP / 8; ++nt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int c = row0 + g + (e >> 1) * 8, b = nt * 8 + c2 + (e & 1);
            if (c < r.dc && b < r.db) e_out[t_out ? c * r.db + b : b * r.dc + c] = s[nt][e];
        }
}

}  // namespace nystra

namespace nystra_host {

// Opts `k` in to `smem` bytes of dynamic shared memory, once per device (`done`: a zero-initialised static).
template <typename K>
cudaError_t opt_in_smem(K k, size_t smem, std::atomic<int> (&done)[nystra::kMaxDevices]) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 0 || dev >= nystra::kMaxDevices) return cudaErrorInvalidDevice;
    if (!done[dev].load(std::memory_order_relaxed)) {
        e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e == cudaSuccess) done[dev].store(1, std::memory_order_relaxed);
    }
    return e;
}

template <typename T, int DP>
cudaError_t run_linear_chunk(const nystra::LinArgs& a, cudaStream_t st) {
    using Shape = nystra::ChunkShape<T, DP>;
    static std::atomic<int> s_local[nystra::kMaxDevices], s_main[nystra::kMaxDevices];
    const dim3 grid((unsigned)(a.n * a.heads * a.segs), a.roles);
    cudaError_t e;
    if (a.segs > 1) {
        auto local = nystra::linear_chunk_kernel<T, DP, false>;
        if ((e = opt_in_smem(local, Shape::kSmem, s_local)) != cudaSuccess) return e;
        local<<<grid, Shape::kThreads, Shape::kSmem, st>>>(a);
        if ((e = cudaGetLastError()) != cudaSuccess) return e;
        if ((e = launch_linear_combine(a, st)) != cudaSuccess) return e;
    }
    auto main = nystra::linear_chunk_kernel<T, DP, true>;
    if ((e = opt_in_smem(main, Shape::kSmem, s_main)) != cudaSuccess) return e;
    main<<<grid, Shape::kThreads, Shape::kSmem, st>>>(a);
    return cudaGetLastError();
}

// Bytes of the widest access (16 at most) that d features in rows of these strides allow.
template <typename T>
int row_access(const void* p, const nystra::Strided& s, int d) {
    const unsigned long long all = (unsigned long long)(uintptr_t)p | (unsigned long long)s.n * sizeof(T) |
                                   (unsigned long long)s.head * sizeof(T) | (unsigned long long)s.token * sizeof(T) |
                                   (unsigned long long)d * sizeof(T);
    return all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : 2;
}

template <typename T>
void set_row_access(nystra::LinArgs& a) {
    for (int i = 0; i < a.roles; ++i) {
        nystra::LinRole& r = a.role[i];
        r.wa = row_access<T>(r.a, r.sa, r.db);
        r.wb = row_access<T>(r.b, r.sb, r.db);
        r.wc = row_access<T>(r.c, r.sc, r.dc);
        r.wo = row_access<T>(r.out, r.so, r.dc);
    }
}

template <typename T>
cudaError_t linear_chunk(const nystra::LinArgs& args, cudaStream_t st) {
    nystra::LinArgs a = args;
    set_row_access<T>(a);
    const int d = lin_widest(a);
    if (d <= 32) return run_linear_chunk<T, 32>(a, st);
    if (d <= 64) return run_linear_chunk<T, 64>(a, st);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) {
        cudaError_t e;
        if (launch_linear_umma(a, st, &e)) return e;
    }
    return run_linear_chunk<T, 128>(a, st);
}

}  // namespace nystra_host
