// Per-head RMSNorm and rotary positions of queries and keys in one pass, dense or on the way into the paged cache.
//
//   y = R(pos) n,   n = x / sqrt(mean x^2 + eps) * gain  (n = x without a gain)
//   R turns the pair (a, b) of a head by pos * f_p: (a cos - b sin, b cos + a sin); pair p is (n[p], n[p + d/2]) in the layout
//   of halves, (n[2p], n[2p + 1]) in the interleaved one, d the components that rotate; the others pass through.
//
// HBM bounds it: every value is read once and written once.  A head is one group of lanes of a warp, eight components to a
// lane (16 bytes of a 16-bit type), so the norm's sum is a few shuffles and a pair's other half is in the same lane
// (interleaved), one shuffle away (halves of a multiple of eight components), or read again, from L1 (other halves).
// A block holds some heads of NV tokens: its threads request their values, compute the tokens' cosines and sines
// meanwhile (64 angles serve all heads of a token), and meet once.
// Angles: the frequencies are turns per position in 64 bits, the product and its fraction of a turn are taken in 64 bits, and
// the rest of the fraction beyond 24 bits is folded in to first order, so a position of 2^20 has as exact a cosine as position 1.
#pragma once
#include "ptx.cuh"

namespace syn {

constexpr int ROPE_MAX_DIM = 256;      // components of a head
constexpr int ROPE_THREADS = 256;

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
    int end;                           // one past the segment's last head, counted through all segments
    int turn;                          // 1: rotates
    int plane;                         // -1: dense, 0: K of the cache, 1: V
};

struct RopeParams {
    RopeTable rope;
    RopeSeg seg[3];
    const int* pos;                    // [T]
    const int* slot;                   // [T] page * 16 + row, for the cache's segments
    op16* pool;                        // the layer's pages
    int T, n_heads, heads_per_block, head_dim, n_kv_heads;
    float eps;
};

__device__ __forceinline__ float rope_f32(float v) { return v; }
__device__ __forceinline__ float rope_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float rope_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T, bool VEC>
__device__ __forceinline__ void rope_load8(const T* p, float (&v)[8]) {
    if constexpr (VEC) {
        struct alignas(16) Raw { T e[16 / sizeof(T)]; };
        constexpr int N = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < 8 / N; ++i) {
            const Raw r = *reinterpret_cast<const Raw*>(p + i * N);
#pragma unroll
            for (int j = 0; j < N; ++j) v[i * N + j] = rope_f32(r.e[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = rope_f32(p[j]);
    }
}

// One rounding, to nearest; half precision saturates as everywhere in this library.
__device__ __forceinline__ void rope_pack8(const float (&v)[8], __half* to) {
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<uint32_t*>(to + 2 * j) = pack_op(v[2 * j], v[2 * j + 1]);
}
__device__ __forceinline__ void rope_pack8(const float (&v)[8], __nv_bfloat16* to) {
#pragma unroll
    for (int j = 0; j < 4; ++j) *reinterpret_cast<__nv_bfloat162*>(to + 2 * j) = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
}
__device__ __forceinline__ void rope_pack8(const float (&v)[8], float* to) {
#pragma unroll
    for (int j = 0; j < 8; ++j) to[j] = v[j];
}
template <typename T, bool VEC>
__device__ __forceinline__ void rope_store8(T* p, const float (&v)[8]) {
    alignas(16) T out[8];
    rope_pack8(v, out);
    if constexpr (VEC) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) reinterpret_cast<uint4*>(p)[i] = reinterpret_cast<const uint4*>(out)[i];
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = out[j];
    }
}

// VEC: every row of every segment starts on a 16-byte boundary.  NV: tokens of a block.  blockDim.x = heads_per_block * LPH.
template <typename TIN, typename TOUT, bool VEC, int NV>
__global__ void __launch_bounds__(ROPE_THREADS)
rope_kernel(const __grid_constant__ RopeParams p) {
    __shared__ float2 table[NV][ROPE_MAX_DIM / 2];
    const int hd = p.head_dim, half = p.rope.half;
    const int lph = blockDim.x / p.heads_per_block;          // lanes of a head: a power of two, at most 32
    const int l = threadIdx.x % lph, e0 = l * 8;
    const int head = blockIdx.y * p.heads_per_block + threadIdx.x / lph;
    const int t0 = blockIdx.x * NV;
    const int nt = min(NV, p.T - t0);
    const bool live = head < p.n_heads && e0 < hd;
    const int si = head < p.seg[0].end ? 0 : head < p.seg[1].end ? 1 : 2;
    const RopeSeg& sg = p.seg[si];
    const int h = head - (si ? p.seg[si - 1].end : 0);       // head of the segment
    const TIN* x = reinterpret_cast<const TIN*>(sg.x) + (int64_t)t0 * sg.x_stride + (int64_t)h * hd;
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (live && i < nt) rope_load8<TIN, VEC>(x + i * sg.x_stride + e0, v[i]);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        }
    }
    for (int k = threadIdx.x; k < nt * half; k += blockDim.x) {
        const int i = k / half, c = k - i * half;
        double u = (double)p.pos[t0 + i] * p.rope.turns[c];
        u = 2.0 * (u - rint(u));                             // half turns in [-1, 1]
        const float hi = (float)u, lo = (float)(u - (double)hi) * 3.14159265358979f;
        float sn, cs;
        sincospif(hi, &sn, &cs);
        table[i][c] = make_float2((cs - sn * lo) * p.rope.amplitude, (sn + cs * lo) * p.rope.amplitude);
    }
    float g[8];
    const bool norm = live && sg.gain != nullptr;
#pragma unroll
    for (int j = 0; j < 8; ++j) g[j] = norm ? __bfloat162float(sg.gain[e0 + j]) : 1.f;
    __syncthreads();
    const bool turns = sg.turn && half > 0;
    const bool lanes = (half & 7) == 0;                      // halves: a pair's other component sits at the same place of another lane
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        // (i < nt is uniform over the block, live is not: every lane takes part in the shuffles)
        if (i >= nt) break;
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fmaf(v[i][j], v[i][j], ss);
        for (int o = lph >> 1; o > 0; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
        const float r = norm ? rsqrtf(ss / (float)hd + p.eps) : 1.f;
        float w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = v[i][j] * r * g[j];
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = w[j];
        if (p.rope.interleaved) {
            if (turns)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int c = e0 / 2 + j;
                    if (c < half) {
                        const float2 cs = table[i][c];
                        y[2 * j] = w[2 * j] * cs.x - w[2 * j + 1] * cs.y;
                        y[2 * j + 1] = w[2 * j + 1] * cs.x + w[2 * j] * cs.y;
                    }
                }
        } else if (lanes) {
            const bool first = e0 < half;
            const int from = (threadIdx.x & 31) + (first ? half >> 3 : -(half >> 3));
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float o = __shfl_sync(0xFFFFFFFFu, w[j], from & 31);
                if (turns && e0 < 2 * half) {
                    const float2 cs = table[i][first ? e0 + j : e0 + j - half];
                    y[j] = first ? w[j] * cs.x - o * cs.y : w[j] * cs.x + o * cs.y;
                }
            }
        } else if (live && turns) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int e = e0 + j;
                if (e < 2 * half) {
                    const int other = e < half ? e + half : e - half;
                    const float o = rope_f32(x[i * sg.x_stride + other]) * r * (norm ? __bfloat162float(sg.gain[other]) : 1.f);
                    const float2 cs = table[i][min(e, other)];
                    y[j] = e < half ? w[j] * cs.x - o * cs.y : w[j] * cs.x + o * cs.y;
                }
            }
        }
        __syncwarp();                                        // in place: a head's lanes have read what is overwritten now
        if (!live) continue;
        const int t = t0 + i;
        if (sg.plane < 0) rope_store8<TOUT, VEC>(reinterpret_cast<TOUT*>(sg.y) + (int64_t)t * sg.y_stride + (int64_t)h * hd + e0, y);
        else {
            const int s = p.slot[t];
            op16* row = p.pool + (((int64_t)(s >> 4) * p.n_kv_heads + h) * 2 + sg.plane) * 16 * hd + (s & 15) * hd;
            rope_store8<op16, true>(row + e0, y);
        }
    }
}

}  // namespace syn
