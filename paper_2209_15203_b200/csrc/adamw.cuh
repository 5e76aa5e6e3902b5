// AdamW over many tensors in one launch, states in 32 or in 8 bits.
//
//   m <- b1 m + (1 - b1) g          v <- b2 v + (1 - b2) g^2
//   p <- p - lr wd p - lr / (1 - b1^t) * m / (sqrt(v) / sqrt(1 - b2^t) + eps)
//
// One rounding per multiply and add in m and v (no fused multiply-add), so that the 8-bit codes do not
// depend on how an expression is contracted.
//
// States in 8 bits.  256 consecutive values of a tensor (a block) share one fp32 scale s per state.
//   first moment   m = +-c^2 s,  c = 0 .. 127,  s = max|m| / 127^2
//   second moment  r = sqrt(v) = c^2 s,  c = 0 .. 255,  s = max r / 255^2   (v = r^2)
// with c the code of the nearest value.  A square law spaces codes by 1.6 % (m) and 0.8 % (r) near the
// block's maximum and still reaches 6e-5 and 1.5e-5 of it; the scale is a full fp32 number, so a block
// that only decays does so exactly although no code changes.  The root is held, not v: it halves the
// range to cover, and the update needs it anyway.  A positive r never gets code 0 (the update would
// divide by eps alone).  A block whose s would fall below the smallest normal number holds zeros.
//
// Work split: one warp per block of 256 values; lane t takes values t, t+32, ... t+224, so every access
// to p and g is one coalesced line whatever their alignment (layer blocks of a flat vector start
// anywhere), and the codes of a lane's eight values lie together as one 8-byte word in the state.
#pragma once

#include "train.cuh"

namespace tk {

constexpr int kAdamBlock = 256;     // values that share a scale
constexpr int kAdamPerLane = kAdamBlock / 32;
constexpr int kAdamThreads = 256;
constexpr int kAdamWarps = kAdamThreads / 32;
constexpr int kAdamChunk = 2 * kAdamWarps;   // blocks of 256 values per CTA

struct AdamEntry {
    char* p;
    const char* g;
    char* m;
    char* v;
    float2* scales;   // 8-bit states: (scale of m, scale of r) per block
    bf16* copy16;     // 16-bit copy of the updated parameters, or null
    int64_t n;
    u32 first;        // first chunk of this tensor in the launch's grid
    float decay;      // lr * weight decay
};

struct AdamHyper {
    float b1, c1, b2, c2;   // beta and 1 - beta, each rounded once from the caller's double
    float eps, lr1, rbc2;   // lr / (1 - b1^t), 1 / sqrt(1 - b2^t)
    float gscale;           // multiplies the gradient (1: left out)
};

// The tensors of one launch travel in its parameters: no table to copy, nothing to keep alive.
// Kernel parameters hold 32,764 bytes; the small form keeps ordinary launches under the 4 KB that
// every launch carries cheaply.
template <int CAP>
struct AdamGroup {
    AdamHyper h;
    int count;
    int scaled;   // gscale != 1
    AdamEntry e[CAP];
};
constexpr int kAdamSmallCap = 62, kAdamLargeCap = 500;

template <int CAP>
__device__ __forceinline__ int adam_find(const AdamGroup<CAP>& G, u32 chunk) {
    int lo = 0, hi = G.count - 1;   // the last entry whose first chunk is <= chunk
    while (lo < hi) {
        int mid = (lo + hi + 1) >> 1;
        if (G.e[mid].first <= chunk)
            lo = mid;
        else
            hi = mid - 1;
    }
    return lo;
}

constexpr float kMagic = 8388608.0f;   // 2^23: adding it leaves an integer 0 .. 2^23 in the low mantissa bits
constexpr float kLevelsM = 127.0f, kLevelsR = 255.0f;

// byte j of a word as a float
__device__ __forceinline__ float byte_float(u32 word, int j) {
    return __uint_as_float(__byte_perm(word, 0x4b000000u, 0x7440 | j)) - kMagic;
}

// The code c of y = a / s: the number of thresholds k^2 + k + 1/2 (k = 0, 1, ..), the midpoints between k^2 and
// (k+1)^2, that lie below y.  c is near round(sqrt(y - 1/4)); an approximate root gives it up to one, and
// comparing with the two thresholds around it, which are exact in fp32, settles it.
__device__ __forceinline__ float square_code(float y) {
    float root;
    asm("sqrt.approx.f32 %0, %1;" : "=f"(root) : "f"(fmaxf(y - 0.25f, 0.0f)));
    float c = (root + kMagic) - kMagic;
    float t = fmaf(c, c, c) + 0.5f;
    float down = fmaf(-2.0f, c, t);
    if (y > t)
        c += 1.0f;
    else if (y <= down)
        c -= 1.0f;
    return fmaxf(c, 0.0f);
}

// (scale, 1 / scale) of a block whose largest magnitude is `top`
__device__ __forceinline__ float2 block_scale(float top, float inv_levels2) {
    float s = __fmul_rn(top, inv_levels2);
    if (!(s >= 1.17549435e-38f)) return make_float2(0.0f, 0.0f);
    return make_float2(s, __frcp_rn(s));
}

__device__ __forceinline__ float block_max(float v) {   // v >= 0: its bits order as integers
    return __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(v)));
}

__device__ __forceinline__ void decode_m(uint2 w, float s, float (&m)[kAdamPerLane]) {
#pragma unroll
    for (int k = 0; k < kAdamPerLane; ++k) {
        u32 word = k < 4 ? w.x : w.y;
        float c = byte_float(word & 0x7f7f7f7fu, k & 3);
        u32 sign = (word << (24 - 8 * (k & 3))) & 0x80000000u;
        m[k] = __uint_as_float(__float_as_uint(__fmul_rn(__fmul_rn(c, c), s)) | sign);
    }
}
__device__ __forceinline__ void decode_r(uint2 w, float s, float (&r)[kAdamPerLane]) {
#pragma unroll
    for (int k = 0; k < kAdamPerLane; ++k) {
        float c = byte_float(k < 4 ? w.x : w.y, k & 3);
        r[k] = __fmul_rn(__fmul_rn(c, c), s);
    }
}
__device__ __forceinline__ u32 pack4(u32 a, u32 b, u32 c, u32 d) {
    return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}

// Codes and scales of the block's new m and r (0 in lanes past the end of the tensor), held as
// lane-major bytes: byte 8 t + k is value t + 32 k.
__device__ __forceinline__ void encode_block(const float (&m)[kAdamPerLane], const float (&r)[kAdamPerLane], uint2& wm,
                                             uint2& wr, float2& scales) {
    float tm = 0.0f, tr = 0.0f;
#pragma unroll
    for (int k = 0; k < kAdamPerLane; ++k) {
        tm = fmaxf(tm, fabsf(m[k]));
        tr = fmaxf(tr, r[k]);
    }
    float2 sm = block_scale(block_max(tm), 1.0f / (kLevelsM * kLevelsM));
    float2 sr = block_scale(block_max(tr), 1.0f / (kLevelsR * kLevelsR));
    u32 bm[kAdamPerLane], br[kAdamPerLane];
#pragma unroll
    for (int k = 0; k < kAdamPerLane; ++k) {
        float c = square_code(__fmul_rn(fabsf(m[k]), sm.y));
        bm[k] = (__float_as_uint(c + kMagic) & 0x7fu) | ((__float_as_uint(m[k]) >> 24) & 0x80u);
        c = square_code(__fmul_rn(r[k], sr.y));
        c = fmaxf(c, r[k] > 0.0f && sr.x > 0.0f ? 1.0f : 0.0f);
        br[k] = __float_as_uint(c + kMagic) & 0xffu;
    }
    wm = make_uint2(pack4(bm[0], bm[1], bm[2], bm[3]), pack4(bm[4], bm[5], bm[6], bm[7]));
    wr = make_uint2(pack4(br[0], br[1], br[2], br[3]), pack4(br[4], br[5], br[6], br[7]));
    scales = make_float2(sm.x, sr.x);
}

template <typename P, typename G, int BITS, int CAP>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamGroup<CAP> A) {
    const int at = adam_find(A, blockIdx.x);
    const AdamEntry& e = A.e[at];
    const AdamHyper& h = A.h;
    const int lane = threadIdx.x & 31;
    const int64_t blocks = (e.n + kAdamBlock - 1) / kAdamBlock;
    const int64_t b0 = (int64_t)(blockIdx.x - e.first) * kAdamChunk + (threadIdx.x >> 5);
    for (int64_t b = b0; b < b0 + kAdamChunk && b < blocks; b += kAdamWarps) {
        const int64_t base = b * kAdamBlock + lane;
        const int left = (int)min((int64_t)kAdamBlock, e.n - b * kAdamBlock) - lane;   // value k is there if 32 k < left
        P* pp = (P*)e.p + base;
        const G* gp = (const G*)e.g + base;
        float p[kAdamPerLane], g[kAdamPerLane], m[kAdamPerLane], v[kAdamPerLane];
        uint2 wm, wr;
        float2 sc;
        if (BITS == 8) {
            wm = *(const uint2*)(e.m + b * kAdamBlock + lane * kAdamPerLane);
            wr = *(const uint2*)(e.v + b * kAdamBlock + lane * kAdamPerLane);
            sc = e.scales[b];
        }
#pragma unroll
        for (int k = 0; k < kAdamPerLane; ++k) {
            bool in = 32 * k < left;
            p[k] = in ? to_float(pp[32 * k]) : 0.0f;
            g[k] = in ? to_float(gp[32 * k]) : 0.0f;
            if (BITS == 32) {
                m[k] = in ? ((const float*)e.m)[base + 32 * k] : 0.0f;
                v[k] = in ? ((const float*)e.v)[base + 32 * k] : 0.0f;
            }
        }
        if (BITS == 8) {
            decode_m(wm, sc.x, m);
            decode_r(wr, sc.y, v);
#pragma unroll
            for (int k = 0; k < kAdamPerLane; ++k) v[k] = __fmul_rn(v[k], v[k]);
        }
#pragma unroll
        for (int k = 0; k < kAdamPerLane; ++k) {
            float gk = A.scaled ? __fmul_rn(g[k], h.gscale) : g[k];
            m[k] = __fadd_rn(__fmul_rn(m[k], h.b1), __fmul_rn(gk, h.c1));
            v[k] = __fadd_rn(__fmul_rn(v[k], h.b2), __fmul_rn(__fmul_rn(gk, h.c2), gk));
            float r = __fsqrt_rn(v[k]);
            float step = m[k] / (r * h.rbc2 + h.eps);
            p[k] = (p[k] - e.decay * p[k]) - h.lr1 * step;
            if (BITS == 32) {
                if (32 * k < left) {
                    ((float*)e.m)[base + 32 * k] = m[k];
                    ((float*)e.v)[base + 32 * k] = v[k];
                }
            } else {
                v[k] = r;
            }
            if (32 * k < left) {
                P out = from_float<P>(p[k]);
                pp[32 * k] = out;
                if (e.copy16) e.copy16[base + 32 * k] = from_float<bf16>(to_float(out));
            }
        }
        if (BITS == 8) {
            // lanes past the end carry code 0 and gradient 0, so their m and r are 0 and stay 0
            encode_block(m, v, wm, wr, sc);
            *(uint2*)(e.m + b * kAdamBlock + lane * kAdamPerLane) = wm;
            *(uint2*)(e.v + b * kAdamBlock + lane * kAdamPerLane) = wr;
            if (lane == 0) e.scales[b] = sc;
        }
    }
}

// 8-bit states from and to fp32 values (a checkpoint's): p holds m's values, g holds v's.
template <bool LOAD, int CAP>
__global__ void __launch_bounds__(kAdamThreads) adamw_state_kernel(const __grid_constant__ AdamGroup<CAP> A) {
    const int at = adam_find(A, blockIdx.x);
    const AdamEntry& e = A.e[at];
    const int lane = threadIdx.x & 31;
    const int64_t blocks = (e.n + kAdamBlock - 1) / kAdamBlock;
    const int64_t b0 = (int64_t)(blockIdx.x - e.first) * kAdamChunk + (threadIdx.x >> 5);
    for (int64_t b = b0; b < b0 + kAdamChunk && b < blocks; b += kAdamWarps) {
        const int64_t base = b * kAdamBlock + lane;
        const int left = (int)min((int64_t)kAdamBlock, e.n - b * kAdamBlock) - lane;
        float* mp = (float*)e.p + base;
        float* vp = (float*)const_cast<char*>(e.g) + base;
        uint2* wmp = (uint2*)(e.m + b * kAdamBlock + lane * kAdamPerLane);
        uint2* wrp = (uint2*)(e.v + b * kAdamBlock + lane * kAdamPerLane);
        float m[kAdamPerLane], r[kAdamPerLane];
        if (LOAD) {
#pragma unroll
            for (int k = 0; k < kAdamPerLane; ++k) {
                bool in = 32 * k < left;
                m[k] = in ? mp[32 * k] : 0.0f;
                r[k] = in ? __fsqrt_rn(vp[32 * k]) : 0.0f;
            }
            uint2 wm, wr;
            float2 sc;
            encode_block(m, r, wm, wr, sc);
            *wmp = wm;
            *wrp = wr;
            if (lane == 0) e.scales[b] = sc;
        } else {
            float2 sc = e.scales[b];
            decode_m(*wmp, sc.x, m);
            decode_r(*wrp, sc.y, r);
#pragma unroll
            for (int k = 0; k < kAdamPerLane; ++k)
                if (32 * k < left) {
                    mp[32 * k] = m[k];
                    vp[32 * k] = __fmul_rn(r[k], r[k]);
                }
        }
    }
}

}  // namespace tk
