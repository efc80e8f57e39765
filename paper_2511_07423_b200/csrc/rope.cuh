// Per-head RMSNorm and rotary positions of queries and keys in one pass, dense or on the way into the paged cache.
//
//   y = R(pos) n,   n = x / sqrt(mean x^2 + eps) * gain  (n = x without a gain)
//   R turns the pair (a, b) of a head by pos * f_p: (a cos - b sin, b cos + a sin); pair p is (n[p], n[p + d/2]) in the layout
//   of halves, (n[2p], n[2p + 1]) in the interleaved one, d the components that rotate; the others pass through.
//
// HBM bounds it: every value is read once and written once.  A head is one group of lanes of a warp, four pairs to a lane,
// so the norm's sum is a few shuffles and a rotation stays in its lane.
// A warp takes some heads of one token: it requests their values, computes the token's cosines and sines meanwhile, and
// keeps a lane's four of each for all its heads; no barrier between warps.
// Angles: the frequencies are turns per position in 64 bits, the product and its fraction of a turn are taken in 64 bits, and
// the rest of the fraction beyond 24 bits is folded in to first order, so a position of 2^20 has as exact a cosine as position 1.
// Measured (8192 tokens of 32 + 8 heads of 128, norms): bf16 34 us = 4.9 TB/s read and written (0.75 of the copy rate), interleaved 37; 4096
// tokens in fp32 30.6 us = 5.5 TB/s.  In 16 bits instruction issue is as near its bound as HBM: the arithmetic runs on pairs of values
// (with single ones 52 us), gains are multiplied into the cosines and sines (integer divisions, a barrier per token and a table
// for several tokens had it at 71).  A half that is no multiple of 4 components (54 of 128: 81 us) is read one by one.
// The launch bounds hold an instance to 64 registers (40 with one access in flight), and each spills: in bf16 40 bytes of stores in halves, 80
// in pairs, 400 one by one.
#pragma once
#include "ptx.cuh"

namespace syn {

constexpr int ROPE_MAX_DIM = 256;      // components of a head
constexpr int ROPE_WARPS = 2;          // of a block, at most
constexpr int ROPE_UNROLL = 4;         // accesses in flight of a warp that has several

// What syn_rope holds: no device memory, so a handle serves every device and stream.
struct RopeTable {
    double turns[ROPE_MAX_DIM / 2];    // f_p / 2 pi
    float amplitude;                   // of cosine and sine
    int half;                          // pairs: d / 2; 0: no rotation
    int interleaved;
};

// Heads that are handled alike.
struct RopeSeg {
    const void* x;
    int64_t x_stride;                  // elements between tokens
    void* y;                           // dense output; the cache's segments have none
    int64_t y_stride;
    const __nv_bfloat16* gain;         // [head_dim] or NULL: no norm
    int n_heads;
    int end;                           // one past the segment's last chunk of heads, counted through all segments
    int turn;                          // 1: rotates
    int plane;                         // -1: dense, 0: K of the cache, 1: V
};

struct RopeParams {
    RopeTable rope;
    RopeSeg seg[3];
    const int* pos;                    // [T]
    const int* slot;                   // [T] page * 16 + row, for the cache's segments
    op16* pool;                        // the layer's pages
    int T, heads_per_warp, head_dim, n_kv_heads;
    int lane_bits;                     // log2 of the lanes of a head
    float eps, inv_hd;
};

__device__ __forceinline__ float rope_f32(float v) { return v; }
__device__ __forceinline__ float rope_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float rope_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T rope_to(float v);   // one rounding, to nearest
template <> __device__ __forceinline__ float rope_to<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 rope_to<__nv_bfloat16>(float v) { return __float2bfloat16(v); }
template <> __device__ __forceinline__ __half rope_to<__half>(float v) { return to_op(v); }   // saturates, as everywhere in this library

// Four neighbouring components, in one access.
template <typename T>
__device__ __forceinline__ void rope_load4(const T* p, float (&v)[4]) {
    struct alignas(4 * sizeof(T)) Raw { T e[4]; };
    const Raw r = *reinterpret_cast<const Raw*>(p);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = rope_f32(r.e[j]);
}
__device__ __forceinline__ void rope_store4(__half* p, const float (&v)[4]) {
    *reinterpret_cast<uint2*>(p) = make_uint2(pack_op(v[0], v[1]), pack_op(v[2], v[3]));
}
__device__ __forceinline__ void rope_store4(__nv_bfloat16* p, const float (&v)[4]) {
    uint32_t w[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[j]) : "f"(v[2 * j + 1]), "f"(v[2 * j]));
    *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
}
__device__ __forceinline__ void rope_store4(float* p, const float (&v)[4]) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }

// How a head's components lie in its lanes.  A lane holds four pairs (a[j], b[j]); those beyond the rotating ones are any two others.
// ROPE_VEC_HALVES: pairs 4 l ..: components 4 l .. and half + 4 l .., two accesses of four components (half a multiple of 4, rows on
// 16-byte boundaries; lanes behind the rotating ones hold eight neighbours).  ROPE_VEC_PAIRS: the eight neighbours 8 l .., paired.
// ROPE_SCALAR: pairs l, l + lanes, ...: any half and any alignment, one component an access.
enum { ROPE_VEC_HALVES = 0, ROPE_VEC_PAIRS = 1, ROPE_SCALAR = 2 };

template <int MODE>
struct RopeLane {
    int e1, e2;              // vector modes: components of a[0] and of b[0] (halves), of the first and the second four (pairs)
    int ia[4], ib[4];        // scalar mode: components of a[j] and b[j]; ia[j] < 0: none
    int l, lph;
    __device__ __forceinline__ RopeLane(int l_, int lph_, int half, int hd, int interleaved) : l(l_), lph(lph_) {
        const bool halves = MODE == ROPE_VEC_HALVES && 4 * l < half;
        e1 = halves ? 4 * l : 8 * l;
        e2 = halves ? half + 4 * l : 8 * l + 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = pair(j);
            const bool apart = c < half && !interleaved;
            ia[j] = 2 * c >= hd ? -1 : apart ? c : 2 * c;
            ib[j] = apart ? c + half : 2 * c + 1;
        }
    }
    __device__ __forceinline__ int pair(int j) const { return MODE == ROPE_SCALAR ? l + lph * j : 4 * l + j; }
    template <typename T>
    __device__ __forceinline__ void load(const T* x, float (&a)[4], float (&b)[4]) const {
        if constexpr (MODE == ROPE_SCALAR) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool none = ia[j] < 0;   // reads the head's first component and counts for nothing
                const float u = rope_f32(x[none ? 0 : ia[j]]), v = rope_f32(x[none ? 0 : ib[j]]);
                a[j] = none ? 0.f : u;
                b[j] = none ? 0.f : v;
            }
        } else {
            float u[4], v[4];
            if constexpr (MODE == ROPE_VEC_PAIRS && sizeof(T) == 2) {
                struct alignas(16) Raw { T e[8]; };
                const Raw r = *reinterpret_cast<const Raw*>(x + e1);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    u[j] = rope_f32(r.e[j]);
                    v[j] = rope_f32(r.e[j + 4]);
                }
            } else {
                rope_load4(x + e1, u);
                rope_load4(x + e2, v);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a[j] = MODE == ROPE_VEC_HALVES ? u[j] : j < 2 ? u[2 * j] : v[2 * j - 4];
                b[j] = MODE == ROPE_VEC_HALVES ? v[j] : j < 2 ? u[2 * j + 1] : v[2 * j - 3];
            }
        }
    }
    template <typename T>
    __device__ __forceinline__ void store(T* y, const float (&a)[4], const float (&b)[4]) const {
        if constexpr (MODE == ROPE_SCALAR) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (ia[j] < 0) continue;
                y[ia[j]] = rope_to<T>(a[j]);
                y[ib[j]] = rope_to<T>(b[j]);
            }
        } else if constexpr (MODE == ROPE_VEC_HALVES) {
            rope_store4(y + e1, a);
            rope_store4(y + e2, b);
        } else {
            const float u[4] = {a[0], b[0], a[1], b[1]}, v[4] = {a[2], b[2], a[3], b[3]};
            rope_store4(y + e1, u);
            rope_store4(y + e2, v);
        }
    }
};

// A warp takes one token and some heads of one segment (blockIdx.y: which), U accesses' worth of heads at a time.
// Gains and angles are the same for all heads of a token, so they are multiplied into four factors a pair once:
// y_a = r (x_a gain_a cos - x_b gain_b sin), y_b = r (x_b gain_b cos + x_a gain_a sin), r = 1 / sqrt(mean x^2 + eps).
template <typename TIN, typename TOUT, int MODE, int U>
__global__ void __launch_bounds__(ROPE_WARPS * 32, U == 1 ? 24 : 16)
rope_kernel(const __grid_constant__ RopeParams p) {
    __shared__ alignas(16) float table[ROPE_WARPS][2][ROPE_MAX_DIM / 2];
    const int t = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (t >= p.T) return;
    const int hd = p.head_dim, half = p.rope.half;
    const int lane = threadIdx.x & 31, lane_of_head = lane & ((1 << p.lane_bits) - 1);
    const bool lane_live = lane_of_head * (MODE == ROPE_SCALAR ? 2 : 8) < hd;
    const int l = lane_live ? lane_of_head : 0;              // (idle lanes read what lane 0 reads, and store nothing)
    float* tc = table[threadIdx.x >> 5][0];
    float* ts = table[threadIdx.x >> 5][1];
    const int si = (int)blockIdx.y < p.seg[0].end ? 0 : (int)blockIdx.y < p.seg[1].end ? 1 : 2;
    const RopeSeg& sg = p.seg[si];
    const int h_begin = ((int)blockIdx.y - (si ? p.seg[si - 1].end : 0)) * p.heads_per_warp, h_end = min(h_begin + p.heads_per_warp, sg.n_heads);
    const int per = 32 >> p.lane_bits, sub = lane >> p.lane_bits;   // heads of a warp at a time, and which of them is this lane's
    const RopeLane<MODE> ln(l, 1 << p.lane_bits, half, hd, p.rope.interleaved);
    const TIN* x = reinterpret_cast<const TIN*>(sg.x) + t * sg.x_stride;
    const bool norm = sg.gain != nullptr, turns = sg.turn && half > 0;
    float a[U][4], b[U][4];
    auto load = [&](int h0) {                                // heads beyond the last: the last again
#pragma unroll
        for (int i = 0; i < U; ++i) ln.load(x + min(h0 + i * per + sub, h_end - 1) * hd, a[i], b[i]);
    };
    load(h_begin);
    float ga[4], gb[4], c[4], s[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) ga[j] = gb[j] = 1.f;
    if (norm) ln.load(sg.gain, ga, gb);
    const bool dense = sg.plane < 0;
    const int slot = dense ? 0 : p.slot[t];
    if (turns) {
        const double pos = (double)p.pos[t];
        for (int c = lane; c < half; c += 32) {
            double u = pos * p.rope.turns[c];
            u = 2.0 * (u - rint(u));                         // half turns in [-1, 1]
            const float hi = (float)u, lo = (float)(u - (double)hi) * 3.14159265358979f;
            const float cs = cospif(hi), sn = sinpif(hi);
            tc[c] = (cs - sn * lo) * p.rope.amplitude;
            ts[c] = (sn + cs * lo) * p.rope.amplitude;
        }
        __syncwarp();
    }
    Two aa[2], ab[2], bb[2], ba[2];                          // y_a = aa x_a + ab x_b, y_b = bb x_b + ba x_a
    const bool some = turns && ln.pair(0) < half;            // some pair of the lane turns
    const bool mixed = some && ln.pair(3) >= half;           // and some passes through: those are not multiplied by a sine of 0, which is no 0 times infinity
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bool in = turns && ln.pair(j) < half;
        c[j] = in ? tc[ln.pair(j)] : 1.f;
        s[j] = in ? ts[ln.pair(j)] : 0.f;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        aa[j] = two_of(ga[2 * j] * c[2 * j], ga[2 * j + 1] * c[2 * j + 1]);
        ab[j] = two_of(-gb[2 * j] * s[2 * j], -gb[2 * j + 1] * s[2 * j + 1]);
        bb[j] = two_of(gb[2 * j] * c[2 * j], gb[2 * j + 1] * c[2 * j + 1]);
        ba[j] = two_of(ga[2 * j] * s[2 * j], ga[2 * j + 1] * s[2 * j + 1]);
    }
    TOUT* y = reinterpret_cast<TOUT*>(sg.y) + t * sg.y_stride;
    op16* row = p.pool + ((int64_t)(slot >> 4) * p.n_kv_heads * 2 + sg.plane) * 16 * hd + (slot & 15) * hd;
    for (int h0 = h_begin;;) {
#pragma unroll
        for (int i = 0; i < U; ++i) {
            Two xa[2], xb[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                xa[j] = two_of(a[i][2 * j], a[i][2 * j + 1]);
                xb[j] = two_of(b[i][2 * j], b[i][2 * j + 1]);
            }
            if (norm) {
                const Two sq = fma2(xb[1], xb[1], fma2(xa[1], xa[1], fma2(xb[0], xb[0], mul2(xa[0], xa[0]))));
                float s0, s1;
                untwo(sq, s0, s1);
                float ss = lane_live ? s0 + s1 : 0.f;
#pragma unroll
                for (int k = 4; k >= 0; --k)
                    if (k < p.lane_bits) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, 1 << k);
                const float r = rsqrtf(fmaf(ss, p.inv_hd, p.eps));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    xa[j] = mul2(xa[j], two_of(r, r));
                    xb[j] = mul2(xb[j], two_of(r, r));
                }
            }
            Two ya[2], yb[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                ya[j] = mul2(xa[j], aa[j]);
                yb[j] = mul2(xb[j], bb[j]);
            }
            if (MODE == ROPE_VEC_HALVES ? some : some && !mixed) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    ya[j] = fma2(xb[j], ab[j], ya[j]);
                    yb[j] = fma2(xa[j], ba[j], yb[j]);
                }
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                untwo(ya[j], a[i][2 * j], a[i][2 * j + 1]);
                untwo(yb[j], b[i][2 * j], b[i][2 * j + 1]);
            }
            if (MODE != ROPE_VEC_HALVES && mixed) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const Two za = mul2(xb[j], ab[j]), zb = mul2(xa[j], ba[j]);
                    float a0, a1, b0, b1;
                    untwo(za, a0, a1);
                    untwo(zb, b0, b1);
                    if (ln.pair(2 * j) < half) { a[i][2 * j] += a0; b[i][2 * j] += b0; }
                    if (ln.pair(2 * j + 1) < half) { a[i][2 * j + 1] += a1; b[i][2 * j + 1] += b1; }
                }
            }
            const int h = h0 + i * per + sub;
            if (lane_live && h < h_end) {
                if (dense) ln.store(y + h * hd, a[i], b[i]);
                else ln.store(row + (int64_t)h * 32 * hd, a[i], b[i]);
            }
        }
        h0 += U * per;
        if (h0 >= h_end) break;
        load(h0);
    }
}

}  // namespace syn
