// Softmax cross entropy over a large vocabulary with its gradient, without keeping the logits.
//
//   l = h w^T,  lse_i = log sum_v exp(l_iv),  loss_i = lse_i - l_i,target(i)
//   P_iv = exp(l_iv - lse_i),  D_iv = dloss_i (P_iv - [v = target(i)]),  dh = D w,  dw = D^T h
//
// Three uses of one tcgen05 matrix-product kernel, which differ in what happens to a tile of accumulators:
//   kLoss  a tile of logits is reduced, row by row, to (maximum, sum of exp) and discarded; a small kernel
//          joins the tiles of a row.  Nothing of size tokens x vocab is ever written.
//   kSoft  a tile of logits becomes a tile of D for one piece of the vocabulary (as many columns as the
//          workspace holds), written in 16 bits by TMA stores.
//   kGrad  the two products of that piece: rows of dw, complete, and dh, added up over the pieces in fp32.
// The logits are therefore computed twice: 8 instead of 6 flops per (token, vocabulary entry, dim), in exchange for
// tokens x vocab values of memory.
//
// Operands are bf16.  An fp32 operand is held as three bf16 parts, hi + mid + lo, which represent it
// exactly, and a product takes the part pairs of order up to 2^-16 (six of nine; three when the other
// operand is bf16): what is left out is below fp32's own rounding.  D is one part when the gradients are
// bf16 (a rounding of 2^-9 of each coefficient, as in any 16-bit training step) and three when they are fp32.
//
// One CTA (CG 1) or pair (CG 2) per SM (pair) is persistent over tiles of 128 CG x 256: one thread issues TMA
// loads into a ring of stages of 64 of K, one issues the matrix instructions into one of two accumulators
// of 256 columns of tensor memory, four warps take the other accumulator to its destination meanwhile.
// Both gradient products read D or w or h along the dimension that is not contiguous; the matrix
// instructions take such operands ("MN-major") directly, so nothing is transposed in memory.
#pragma once

#include "tcgen05.cuh"

namespace tk {

enum { kXentLoss = 0, kXentSoft = 1, kXentGrad = 2 };

constexpr int kTileM = 128, kTileN = 256, kTileK = 64;
constexpr int kXentThreads = 256;   // warps: TMA, matrix instructions, tensor memory, -, 4 x epilogue
constexpr int kXentEpiWarp = 4;
constexpr int kBoxBytes = 64 * 64 * 2;                        // an MN-major box: 64 values x 64 of K
constexpr int kABytes = kTileM * kTileK * 2;
template <int CG> struct XentShape {
    static constexpr int kBRows = kTileN / CG;                // rows of the right operand this CTA holds
    static constexpr int kStageBytes = kABytes + kBRows * kTileK * 2;
    static constexpr int kStages = CG == 1 ? 4 : 6;           // 192 KB either way
    static constexpr int kStaging = 8192;                     // per epilogue warp
    static constexpr int kSmem = kStages * kStageBytes + 4 * kStaging + 512 + 1024;
};

struct alignas(64) XentProblem {
    CUtensorMap a, b;
    int tiles_m, tiles_n, kblocks;
    int cols;                 // columns of the result
    int a_mn, b_mn;           // operand is MN-major
    int a_off, b_off;         // first row (M, N) within the operand's map
    int a_koff, b_koff;       // first K within the operand's map
    int nseg;                 // part pairs, smallest products first
    unsigned char sa[6], sb[6];
    // kGrad: where the tile goes
    void* out;                // null: only into acc
    float* acc;               // fp32 [rows][cols], or null
    int64_t ld, rows;
    int out_bf16, acc_read, acc_write;
};

struct XentArgs {
    XentProblem p[2];
    CUtensorMap store;        // kSoft: D, [parts][tokens][piece]
    u32 tiles0, tiles;        // tiles of the first problem, and of both
    int tokens, vocab;
    int v0;                   // kSoft: first vocabulary entry of the piece
    const int* target;
    const float* lse;
    const float* dloss;
    float2* partial;          // kLoss: [tile of the vocabulary][tokens] (maximum, sum)
    float* picked;            // kLoss: [tokens] logit of the target
    int* status;
};

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Keeps results below the smallest normal number
__device__ __forceinline__ float exp2_gradual(float x) {
    float y;
    asm("ex2.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// D of a 16-bit gradient takes 2^24 exp(l - lse) times 2^-24 dloss: the fast exponential flushes results
// below 2^-126 to zero, and so nothing that bf16 can hold is lost.  (The rounding of an exponent near 24 is
// 2^-20 of the result, far below bf16's; the three-part form subtracts lse first instead.)
constexpr float kSoftLift = 24.0f, kSoftDrop = 5.9604644775390625e-8f;

struct XentTile {
    int problem, m, n;
};
template <int MODE> __device__ __forceinline__ XentTile xent_tile(const XentArgs& A, u32 id) {
    XentTile t;
    t.problem = id >= A.tiles0;
    const XentProblem& P = A.p[t.problem];
    if (t.problem) id -= A.tiles0;
    if (MODE == kXentGrad) {   // the tiles of a row of the result share the long operand: side by side
        t.m = (int)(id / (u32)P.tiles_n);
        t.n = (int)(id % (u32)P.tiles_n);
    } else {                   // all tokens meet the same part of w before the next
        t.m = (int)(id % (u32)P.tiles_m);
        t.n = (int)(id / (u32)P.tiles_m);
    }
    return t;
}
template <int MODE, int CG> __device__ __forceinline__ int xent_columns(const XentProblem& P, int n) {
    if (MODE != kXentGrad) return kTileN;
    const int left = P.cols - n * kTileN, unit = 16 * CG;
    return left >= kTileN ? kTileN : (left + unit - 1) / unit * unit;
}

// One row's 32 logits into the running (maximum, sum of exp2((l - maximum) log2 e)).
__device__ __forceinline__ void loss_chunk(const float (&v)[32], float& top, float& sum) {
    float t = fmaxf(v[0], v[1]);
#pragma unroll
    for (int i = 2; i < 32; ++i) t = fmaxf(t, v[i]);
    if (t > top) {
        sum *= exp2_approx((top - t) * kLog2e);
        top = t;
    }
    const float shift = top * kLog2e;
    float s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int i = 0; i < 32; i += 2) {
        s0 += exp2_approx(fmaf(v[i], kLog2e, -shift));
        s1 += exp2_approx(fmaf(v[i + 1], kLog2e, -shift));
    }
    sum += s0 + s1;
}

// Two values' part `p` as a word of two bf16, leaving in a, b what the parts so far do not hold
__device__ __forceinline__ u32 take_part(float& a, float& b, bool last) {
    __nv_bfloat162 q = __floats2bfloat162_rn(a, b);
    if (!last) {
        a -= __bfloat162float(q.x);
        b -= __bfloat162float(q.y);
    }
    return *(u32*)&q;
}

template <int MODE, int CG, int PARTS>
__global__ void __launch_bounds__(kXentThreads, 1) xent_kernel(const __grid_constant__ XentArgs A) {
    using S = XentShape<CG>;
    extern __shared__ unsigned char raw[];
    const u32 base = (smem_addr(raw) + 1023u) & ~1023u;
    unsigned char* sm = raw + (base - smem_addr(raw));
    const u32 staging = base + S::kStages * S::kStageBytes;
    const u32 bars = staging + 4 * S::kStaging;
    const u32 full = bars, empty = bars + 8 * S::kStages, done = bars + 16 * S::kStages, freed = done + 16, drain = done + 32;
    const u32 tmem_slot = done + 48;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const u32 rank = CG == 2 ? cluster_rank() : 0;
    const u32 worker = blockIdx.x / CG, workers = gridDim.x / CG;

    if (threadIdx.x == 0) {
        for (int i = 0; i < S::kStages; ++i) {
            mbar_init(full + 8 * i, 1);
            mbar_init(empty + 8 * i, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(done + 8 * i, 1);
            mbar_init(freed + 8 * i, 4 * CG);
        }
        mbar_init(drain, 1);
        mbar_init_fence();
    }
    if (warp == 2) tmem_alloc<CG>(tmem_slot, 512);
    tcgen05_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    tcgen05_fence_after();
    const u32 tmem = *(volatile u32*)(sm + (tmem_slot - base));

    if (warp == 0 && lane == 0) {
        // ---- loads ----
        const u32 full0 = CG == 2 ? mapped_addr(full, 0) : full;   // both CTAs' copies report to the leader
        u32 it = 0;
        bool ok = true;
        for (u32 id = worker; ok && id < A.tiles; id += workers) {
            const XentTile t = xent_tile<MODE>(A, id);
            const XentProblem& P = A.p[t.problem];
            const int mine = xent_columns<MODE, CG>(P, t.n) / CG;
            const int a0 = P.a_off + (t.m * CG + (int)rank) * kTileM, b0 = P.b_off + t.n * kTileN + (int)rank * mine;
            const int boxes = P.b_mn ? (mine + 63) / 64 : 0;
            const u32 bytes = kABytes + (P.b_mn ? boxes * kBoxBytes : S::kBRows * kTileK * 2);
            for (int s = 0; ok && s < P.nseg; ++s) {
                const int pa = P.sa[s], pb = P.sb[s];
                for (int k = 0; k < P.kblocks; ++k, ++it) {
                    const u32 stage = it % S::kStages, phase = (it / S::kStages) & 1;
                    if (!(ok = mbar_wait(empty + 8 * stage, phase ^ 1))) break;
                    const u32 a = base + stage * S::kStageBytes, b = a + kABytes, bar = full0 + 8 * stage;
                    if (rank == 0) mbar_expect(full + 8 * stage, bytes * CG);
                    const int ka = P.a_koff + k * kTileK, kb = P.b_koff + k * kTileK;
                    if (P.a_mn) {
                        tma_load<CG>(a, &P.a, bar, a0, ka, pa);
                        tma_load<CG>(a + kBoxBytes, &P.a, bar, a0 + 64, ka, pa);
                    } else {
                        tma_load<CG>(a, &P.a, bar, ka, a0, pa);
                    }
                    if (P.b_mn)
                        for (int j = 0; j < boxes; ++j) tma_load<CG>(b + j * kBoxBytes, &P.b, bar, b0 + 64 * j, kb, pb);
                    else
                        tma_load<CG>(b, &P.b, bar, kb, b0, pb);
                }
            }
        }
        // nothing of this CTA is in flight when it ends: every stage that was filled has been consumed
        for (u32 i = it > (u32)S::kStages ? it - S::kStages : 0; i < it; ++i)
            if (!mbar_wait(empty + 8 * (i % S::kStages), (i / S::kStages) & 1)) ok = false;
        if (!ok) atomicExch(A.status, 1);
    } else if (warp == 1 && lane == 0 && rank == 0) {
        // ---- matrix instructions ----
        u32 it = 0, turn = 0;
        bool ok = true;
        for (u32 id = worker; ok && id < A.tiles; id += workers, ++turn) {
            const XentTile t = xent_tile<MODE>(A, id);
            const XentProblem& P = A.p[t.problem];
            const u32 desc = mma_desc(kTileM * CG, xent_columns<MODE, CG>(P, t.n), P.a_mn, P.b_mn);
            const u32 slot = turn & 1, acc = tmem + slot * kTileN;
            if (!(ok = mbar_wait(freed + 8 * slot, ((turn >> 1) & 1) ^ 1))) break;
            tcgen05_fence_after();
            const u64 step_a = P.a_mn ? 2048 >> 4 : 32 >> 4, step_b = P.b_mn ? 2048 >> 4 : 32 >> 4;
            const int rounds = P.nseg * P.kblocks;
            for (int k = 0; k < rounds; ++k, ++it) {
                const u32 stage = it % S::kStages, phase = (it / S::kStages) & 1;
                if (!(ok = mbar_wait(full + 8 * stage, phase))) break;
                tcgen05_fence_after();
                const u32 a = base + stage * S::kStageBytes, b = a + kABytes;
                u64 da = smem_desc(a, P.a_mn ? kBoxBytes : 0, 1024), db = smem_desc(b, P.b_mn ? kBoxBytes : 0, 1024);
#pragma unroll
                for (int i = 0; i < kTileK / 16; ++i) mma_bf16<CG>(acc, da + i * step_a, db + i * step_b, desc, k > 0 || i > 0);
                mma_commit<CG>(empty + 8 * stage);
            }
            if (ok) mma_commit<CG>(done + 8 * slot);
        }
        if (!ok) {
            mma_commit<CG>(drain);
            mbar_wait(drain, 0);
            atomicExch(A.status, 1);
        }
    } else if (warp >= kXentEpiWarp) {
        // ---- accumulators to their destination ----
        const int w = warp - kXentEpiWarp;
        const u32 stage_smem = staging + w * S::kStaging;
        float* stage_ptr = (float*)(sm + (stage_smem - base));
        const u32 freed0 = CG == 2 ? mapped_addr(freed, 0) : mapped_addr(freed, cluster_rank());
        u32 turn = 0;
        for (u32 id = worker; id < A.tiles; id += workers, ++turn) {
            const XentTile t = xent_tile<MODE>(A, id);
            const XentProblem& P = A.p[t.problem];
            const u32 slot = turn & 1;
            const int m0 = (t.m * CG + (int)rank) * kTileM + 32 * w;   // first row of this warp
            const int row = m0 + lane, n0 = t.n * kTileN;
            int target = -1;
            float scale = 0.0f, lse = 0.0f;
            if (MODE != kXentGrad && row < A.tokens) {
                target = A.target[row];
                if (MODE == kXentSoft) {
                    lse = A.lse[row];
                    scale = target >= 0 && target < A.vocab ? A.dloss[row] : 0.0f;
                }
            }
            if (!mbar_wait(done + 8 * slot, (turn >> 1) & 1)) {
                if (lane == 0) atomicExch(A.status, 1);
                break;
            }
            tcgen05_fence_after();
            const u32 acc = tmem + slot * kTileN + ((u32)(32 * w) << 16);
            if (MODE == kXentLoss) {
                const int valid = min(kTileN, A.vocab - n0);
                const int hit = target >= 0 ? target - n0 : -1;   // column of the target, if it is in this tile
                float top = -3.0e38f, sum = 0.0f;
#pragma unroll 1
                for (int c = 0; c < valid; c += 32) {
                    float v[32];
                    tmem_load32(acc + c, v);
                    tmem_load_wait();
                    if (c + 32 > valid) {
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c + i >= valid) v[i] = -INFINITY;
                    }
                    const bool here = (u32)(hit - c) < 32u && hit < valid;
                    if (__any_sync(0xffffffffu, here)) {
                        float x = 0.0f;
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c + i == hit) x = v[i];
                        if (here) A.picked[row] = x;
                    }
                    loss_chunk(v, top, sum);
                }
                if (row < A.tokens) A.partial[(int64_t)t.n * A.tokens + row] = make_float2(top, sum);
            } else if (MODE == kXentSoft) {
                const int valid = min(kTileN, A.vocab - A.v0 - n0);
                const int hit = target >= 0 ? target - A.v0 - n0 : -1;
                const float shift = kSoftLift - lse * kLog2e, drop = scale * kSoftDrop;
#pragma unroll 1
                for (int c = 0; c < kTileN; c += 64) {
                    float v[64];
                    tmem_load32(acc + c, *(float(*)[32])v);
                    tmem_load32(acc + c + 32, *(float(*)[32])(v + 32));
                    tmem_load_wait();
                    if (PARTS == 1) {
#pragma unroll
                        for (int i = 0; i < 64; ++i) v[i] = drop * exp2_approx(fmaf(v[i], kLog2e, shift));
                    } else {
#pragma unroll
                        for (int i = 0; i < 64; ++i) v[i] = scale * exp2_gradual((v[i] - lse) * kLog2e);
                    }
                    if (c + 64 > valid) {   // past the end of the vocabulary: exact zeros
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (c + i >= valid) v[i] = 0.0f;
                    }
                    if (__any_sync(0xffffffffu, (u32)(hit - c) < 64u)) {
#pragma unroll
                        for (int i = 0; i < 64; ++i)
                            if (c + i == hit) v[i] -= scale;
                    }
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) {
                        // the buffer's previous store has been read (two buffers, one store each in flight)
                        const u32 buf = ((c >> 6) * PARTS + p) & 1;
                        if (lane == 0) tma_store_wait_read<1>();
                        __syncwarp();
                        u32* to = (u32*)stage_ptr + buf * 1024 + lane * 32;
#pragma unroll
                        for (int j = 0; j < 8; ++j) {
                            uint4 q;
                            q.x = take_part(v[8 * j], v[8 * j + 1], p == PARTS - 1);
                            q.y = take_part(v[8 * j + 2], v[8 * j + 3], p == PARTS - 1);
                            q.z = take_part(v[8 * j + 4], v[8 * j + 5], p == PARTS - 1);
                            q.w = take_part(v[8 * j + 6], v[8 * j + 7], p == PARTS - 1);
                            *(uint4*)(to + ((j ^ (lane & 7)) << 2)) = q;
                        }
                        smem_to_async_fence();
                        __syncwarp();
                        if (lane == 0) {
                            if (m0 < A.tokens) tma_store(&A.store, stage_smem + buf * 4096, n0 + c, m0, p);
                            tma_store_commit();
                        }
                    }
                }
            } else {
                const int cols = min(kTileN, P.cols - n0);
#pragma unroll 1
                for (int c = 0; c < cols; c += 32) {
                    float v[32];
                    tmem_load32(acc + c, v);
                    tmem_load_wait();
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 32; ++i) stage_ptr[lane * 33 + i] = v[i];
                    __syncwarp();
                    if (c + lane < cols) {
                        const int64_t col = n0 + c + lane;
                        for (int r = 0; r < 32 && m0 + r < P.rows; ++r) {
                            float x = stage_ptr[r * 33 + lane];
                            float* sum = P.acc + (int64_t)(m0 + r) * P.cols + col;
                            if (P.acc_read) x += *sum;
                            if (P.acc_write) *sum = x;
                            if (P.out) store_any(P.out, (int64_t)(m0 + r) * P.ld + col, x, P.out_bf16);
                        }
                    }
                }
            }
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(freed0 + 8 * slot);
        }
        if (MODE == kXentSoft && lane == 0) tma_store_wait_all();
    }
    tcgen05_fence_before();
    __syncthreads();
    if (CG == 2) cluster_sync();
    if (warp == 2) tmem_free<CG>(tmem, 512);
}

// Joins the tiles of each row: lse and loss.  `lanes` (a power of two up to 32) threads per row.
__global__ void __launch_bounds__(256) xent_join_kernel(const float2* partial, const float* picked, const int* target, int tokens,
                                                        int vocab, int tiles, int lanes, float* loss, float* lse) {
    // lanes of a warp lie side by side along the rows, so that a warp's loads are whole lines when lanes is 1
    const int rows = 32 / lanes;
    const int warp = (int)((blockIdx.x * 256 + threadIdx.x) >> 5), lane = threadIdx.x & 31;
    const int row = warp * rows + lane % rows;
    float top = -3.0e38f, sum = 0.0f;
    if (row < tokens)
        for (int i = lane / rows; i < tiles; i += lanes) {
            const float2 q = partial[(int64_t)i * tokens + row];
            const float t = fmaxf(top, q.x);
            sum = sum * exp2_approx((top - t) * kLog2e) + q.y * exp2_approx((q.x - t) * kLog2e);
            top = t;
        }
    for (int o = rows; o < 32; o <<= 1) {
        const float t2 = __shfl_xor_sync(0xffffffffu, top, o), s2 = __shfl_xor_sync(0xffffffffu, sum, o);
        const float t = fmaxf(top, t2);
        sum = sum * exp2_approx((top - t) * kLog2e) + s2 * exp2_approx((t2 - t) * kLog2e);
        top = t;
    }
    if (row < tokens && lane < rows) {
        const float l = top + logf(sum);
        const int t = target[row];
        lse[row] = l;
        loss[row] = t < 0 ? 0.0f : (t < vocab ? l - picked[row] : NAN);
    }
}

// An operand [rows][dim] as PARTS bf16 matrices [rows][ld] (zeros beyond dim).
template <typename T, int PARTS>
__global__ void __launch_bounds__(256) xent_pack_kernel(const T* x, int64_t stride, int64_t rows, int dim, int ld, bf16* out) {
    const int64_t n = rows * ld, step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += step) {
        const int64_t r = i / ld;
        const int c = (int)(i - r * ld);
        float v = c < dim ? to_float(x[r * stride + c]) : 0.0f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            bf16 q = from_float<bf16>(v);
            out[p * n + i] = q;
            v -= to_float(q);
        }
    }
}

}  // namespace tk
