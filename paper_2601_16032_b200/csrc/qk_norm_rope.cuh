// RMS norm of every query and key head with the position rotation, the append to the paged cache, and the gradients.
//
// All of it is one pass over memory (per row of d values some 100 instructions against 4 d bytes), so the kernels are laid
// out for wide loads in flight: a row is held by kD / 8 lanes with 16 bytes each; its sum of squares is reduced by
// shuffles; the partner of a rotated pair is in the same lane (adjacent pairs) or rot_dim / 16 lanes away (halves).
// A token's angles are the same for all of its heads: a CTA takes a few tokens, computes their sines and cosines once into shared
// memory while the first rows are on their way, and then walks the tokens' rows.  Angles are formed and reduced to a part of a
// turn in 64 bits (position * inv_freq loses its fraction in 32 bits when positions are far); the sine and cosine of the part, and
// everything else, are 32-bit.
#pragma once
#include "paged_common.cuh"

namespace sawtooth {

struct RopeTensor {      // rows of d elements
    const uint16_t* p;
    long long token, head;
};
struct RopeOut {
    uint16_t* p;
    long long token, head;
};

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxTokens = 4;    // tokens a CTA takes at a time

struct RopeParams {
    RopeTensor q, k, v;          // the projections
    RopeTensor dq_out, dk_out;   // backward pass
    RopeOut q_out, k_out;        // forward: results (k_out.p may be null); backward: dq and dk
    const void* q_weight;        // null: no norm
    const void* k_weight;
    const int* position;
    const double* inv_freq;
    const long long* slot;       // null: no cache
    CacheView cache;
    float* partial;              // backward pass: [CTA][2][d] sums for the weights
    int* status;
    float eps;
    int T, H, kv_heads, rot, weight_f32, tokens_per_cta;
    FastDiv rows;                // rows.d = rows of a token: H + kv_heads, or with a cache H + 2 kv_heads
};

template <int kD>
struct RopeShared {
    float cosine[kRopeMaxTokens][kD / 2];
    float sine[kRopeMaxTokens][kD / 2];
    long long cache_at[kRopeMaxTokens];   // element offset of the token's first cache row; -1: none, -2: leave the token alone
};

// Angles of tokens t0 .. t0 + n - 1 into shared memory, and where their cache rows are.
template <int kD>
__device__ __forceinline__ void rope_prepare(const RopeParams& p, RopeShared<kD>& s, int t0, int n, bool backward)
{
    const int half = p.rot >> 1;
    for (int i = threadIdx.x; i < n * (kD / 2); i += kRopeThreads) {
        const int t = i / (kD / 2), j = i % (kD / 2);
        if (j >= half) continue;
        const double turns = (double)p.position[t0 + t] * p.inv_freq[j] * 0.15915494309189535;   // / 2 pi
        float sn, cs;
        sincospif(2.f * (float)(turns - rint(turns)), &sn, &cs);
        s.cosine[t][j] = cs;
        s.sine[t][j] = backward ? -sn : sn;
    }
    if (!backward && threadIdx.x < n) {
        long long at = -1;
        if (p.slot) {
            const long long slot = p.slot[t0 + threadIdx.x];
            if (slot < 0) {
                at = -2;
            } else {
                const long long page = slot < 2147483648ll ? (long long)p.cache.page.div((uint32_t)slot) : slot / p.cache.page.d;
                if (page >= p.cache.num_pages) note_index(p.status, kIndexSlot);
                else at = page * p.cache.page_stride + (slot - page * p.cache.page.d) * p.cache.token_stride;
            }
        }
        s.cache_at[threadIdx.x] = at;
    }
}

__device__ __forceinline__ void load_weight(const void* w, int f32, int bf16, int e0, float (&out)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) out[i] = 1.f;
    if (!w) return;
    if (f32) {
        const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(w) + e0);
        const float4 a = f[0], b = f[1];
        out[0] = a.x; out[1] = a.y; out[2] = a.z; out[3] = a.w; out[4] = b.x; out[5] = b.y; out[6] = b.z; out[7] = b.w;
    } else {
        const uint4 u = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(w) + e0);
        if (bf16) unpack8<1>(u, out); else unpack8<0>(u, out);
    }
}

template <int kLanes>
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// Rotates a row (this lane's eight values y, columns 8 * part ..) by the angles of cs / sn.  Whole warps.
template <int kD, int kAdjacent>
__device__ __forceinline__ void rotate_row(float (&y)[8], const float* cs, const float* sn, int rot, int part)
{
    if (kAdjacent) {
        if (8 * part < rot) {
            const float4 c = *reinterpret_cast<const float4*>(cs + 4 * part), s = *reinterpret_cast<const float4*>(sn + 4 * part);
            const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = y[2 * i], b = y[2 * i + 1];
                y[2 * i] = a * cc[i] - b * ss[i];
                y[2 * i + 1] = b * cc[i] + a * ss[i];
            }
        }
    } else {
        const int half = rot >> 4;               // lanes that hold the first halves of the pairs
        const bool turns = part < 2 * half, lower = part < half;
        const int partner = (int)ptx::lane_id() + (!turns ? 0 : lower ? half : -half);
        float other[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) other[i] = __shfl_sync(0xffffffffu, y[i], partner);
        if (turns) {
            const int at = 8 * (lower ? part : part - half);
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const float4 c = *reinterpret_cast<const float4*>(cs + at + 4 * q), s = *reinterpret_cast<const float4*>(sn + at + 4 * q);
                const float cc[4] = {c.x, c.y, c.z, c.w}, ss[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float sg = lower ? -ss[i] : ss[i];
                    y[4 * q + i] = y[4 * q + i] * cc[i] + other[4 * q + i] * sg;
                }
            }
        }
    }
}

// Forward.  Rows of a token in the order queries, keys, values; group g of kD / 8 lanes takes rows g, g + groups, ...
template <int kD, int kBf16, int kAdjacent>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_kernel(const RopeParams p)
{
    constexpr int kLanes = kD / 8, kGroups = kRopeThreads / kLanes, kAhead = 4;
    __shared__ __align__(16) RopeShared<kD> s;
    const int group = threadIdx.x / kLanes, part = threadIdx.x % kLanes;
    const int t0 = blockIdx.x * p.tokens_per_cta;
    const int n = p.T - t0 < p.tokens_per_cta ? p.T - t0 : p.tokens_per_cta;
    const int rows = n * (int)p.rows.d;
    float wq[8], wk[8];
    bool ready = false;
    for (int r0 = 0; r0 < rows; r0 += kAhead * kGroups) {
        uint4 in[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int r = r0 + a * kGroups + group;
            in[a] = make_uint4(0, 0, 0, 0);
            if (r < rows) {
                const int t = (int)p.rows.div((uint32_t)r), h = r - t * (int)p.rows.d;
                const RopeTensor& x = h < p.H ? p.q : h < p.H + p.kv_heads ? p.k : p.v;
                const int head = h < p.H ? h : h < p.H + p.kv_heads ? h - p.H : h - p.H - p.kv_heads;
                in[a] = *reinterpret_cast<const uint4*>(x.p + (long long)(t0 + t) * x.token + (long long)head * x.head + 8 * part);
            }
        }
        if (!ready) {
            ready = true;
            load_weight(p.q_weight, p.weight_f32, kBf16, 8 * part, wq);
            load_weight(p.k_weight, p.weight_f32, kBf16, 8 * part, wk);
            rope_prepare<kD>(p, s, t0, n, false);
            __syncthreads();
        }
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            // The whole warp stays in step for the shuffles; groups beyond the rows compute on zeros and store nothing.
            const int r = r0 + a * kGroups + group;
            if (!__any_sync(0xffffffffu, r < rows)) break;
            const int rr = r < rows ? r : rows - 1;
            const int t = (int)p.rows.div((uint32_t)rr), h = rr - t * (int)p.rows.d;
            const bool is_q = h < p.H, is_v = h >= p.H + p.kv_heads;
            const long long at = s.cache_at[t];
            uint4 out = in[a];
            float x[8];
            unpack8<kBf16>(in[a], x);
            float sq = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], sq);
            sq = row_sum<kLanes>(sq);
            const float scale = (is_q ? p.q_weight : p.k_weight) ? rsqrtf(sq * (1.f / kD) + p.eps) : 1.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = x[i] * scale * (is_q ? wq[i] : wk[i]);
            rotate_row<kD, kAdjacent>(x, s.cosine[t], s.sine[t], p.rot, part);
            if (!is_v) out = pack8<kBf16>(x);
            if (r < rows && at != -2) {
                const int head = is_q ? h : is_v ? h - p.H - p.kv_heads : h - p.H;
                if (is_q) {
                    *reinterpret_cast<uint4*>(p.q_out.p + (long long)(t0 + t) * p.q_out.token + (long long)head * p.q_out.head + 8 * part) = out;
                } else {
                    if (!is_v && p.k_out.p)
                        *reinterpret_cast<uint4*>(p.k_out.p + (long long)(t0 + t) * p.k_out.token + (long long)head * p.k_out.head + 8 * part) = out;
                    if (at >= 0) {
                        uint16_t* base = const_cast<uint16_t*>(is_v ? p.cache.v : p.cache.k);
                        *reinterpret_cast<uint4*>(base + at + (long long)head * p.cache.head_stride + 8 * part) = out;
                    }
                }
            }
        }
    }
}

// Backward.  A grid of resident CTAs walks the tokens; each lane keeps the weight sums of its eight columns over all of its
// rows in registers (a few dozen rows), a CTA adds its groups' in a fixed order and leaves the sum in `partial`.
template <int kD, int kBf16, int kAdjacent>
__global__ void __launch_bounds__(kRopeThreads) qk_norm_rope_bwd_kernel(const RopeParams p)
{
    constexpr int kLanes = kD / 8, kGroups = kRopeThreads / kLanes, kAhead = 2;
    __shared__ __align__(16) RopeShared<kD> s;
    __shared__ float sums[kGroups][kD];
    const int group = threadIdx.x / kLanes, part = threadIdx.x % kLanes;
    float wq[8], wk[8], aq[8] = {}, ak[8] = {};
    load_weight(p.q_weight, p.weight_f32, kBf16, 8 * part, wq);
    load_weight(p.k_weight, p.weight_f32, kBf16, 8 * part, wk);
    for (long long t0l = (long long)blockIdx.x * p.tokens_per_cta; t0l < p.T; t0l += (long long)gridDim.x * p.tokens_per_cta) {
        const int t0 = (int)t0l;
        const int n = p.T - t0 < p.tokens_per_cta ? p.T - t0 : p.tokens_per_cta;
        const int rows = n * (int)p.rows.d;
        bool ready = false;
        for (int r0 = 0; r0 < rows; r0 += kAhead * kGroups) {
            uint4 in[kAhead], grad[kAhead];
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int r = r0 + a * kGroups + group;
                in[a] = grad[a] = make_uint4(0, 0, 0, 0);
                if (r < rows) {
                    const int t = (int)p.rows.div((uint32_t)r), h = r - t * (int)p.rows.d;
                    const RopeTensor& x = h < p.H ? p.q : p.k;
                    const RopeTensor& g = h < p.H ? p.dq_out : p.dk_out;
                    const int head = h < p.H ? h : h - p.H;
                    in[a] = *reinterpret_cast<const uint4*>(x.p + (long long)(t0 + t) * x.token + (long long)head * x.head + 8 * part);
                    grad[a] = *reinterpret_cast<const uint4*>(g.p + (long long)(t0 + t) * g.token + (long long)head * g.head + 8 * part);
                }
            }
            if (!ready) {
                ready = true;
                __syncthreads();     // the last tokens' angles have been used
                rope_prepare<kD>(p, s, t0, n, true);
                __syncthreads();
            }
#pragma unroll
            for (int a = 0; a < kAhead; ++a) {
                const int r = r0 + a * kGroups + group;
                if (!__any_sync(0xffffffffu, r < rows)) break;
                const int rr = r < rows ? r : rows - 1;
                const int t = (int)p.rows.div((uint32_t)rr), h = rr - t * (int)p.rows.d;
                const bool is_q = h < p.H;
                float x[8], y[8];
                unpack8<kBf16>(in[a], x);
                unpack8<kBf16>(grad[a], y);
                rotate_row<kD, kAdjacent>(y, s.cosine[t], s.sine[t], p.rot, part);   // the sines are negated: R^T
                // The sums are taken by whole warps, whether or not this lane's row has a weight.
                const bool normed = (is_q ? p.q_weight : p.k_weight) != nullptr;
                float sq = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], sq);
                sq = row_sum<kLanes>(sq);
                const float rs = rsqrtf(sq * (1.f / kD) + p.eps);
                float dot = 0.f, g[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] *= rs;                             // x r
                    g[i] = y[i] * (is_q ? wq[i] : wk[i]);
                    dot = fmaf(g[i], x[i], dot);
                }
                dot = row_sum<kLanes>(dot) * (1.f / kD);
                if (normed && r < rows) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float term = y[i] * x[i];     // dn x r
                        if (is_q) aq[i] += term; else ak[i] += term;
                        y[i] = rs * (g[i] - x[i] * dot);
                    }
                }
                if (r < rows) {
                    const RopeOut& o = is_q ? p.q_out : p.k_out;
                    *reinterpret_cast<uint4*>(o.p + (long long)(t0 + t) * o.token + (long long)(is_q ? h : h - p.H) * o.head + 8 * part) = pack8<kBf16>(y);
                }
            }
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[group][8 * part + i] = which ? ak[i] : aq[i];
        __syncthreads();
        if (threadIdx.x < kD) {
            float a = 0.f;
            for (int g = 0; g < kGroups; ++g) a += sums[g][threadIdx.x];
            p.partial[((long long)blockIdx.x * 2 + which) * kD + threadIdx.x] = a;
        }
    }
}

// dq_weight[c] and dk_weight[c] = the sum of the CTAs' partial sums, in their order: 32 columns a CTA, 32 threads a column.
__global__ void __launch_bounds__(1024) rope_weight_sum_kernel(const float* partial, int ctas, int d, float* dq_weight, float* dk_weight)
{
    __shared__ float sums[32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int col = threadIdx.x & 31, row = threadIdx.x >> 5, column = blockIdx.x * 32 + col;   // of 2 d
    float a = 0.f;
    for (int c = row; c < ctas; c += 32) a += partial[(long long)c * 2 * d + column];
    sums[row][col] = a;
    __syncthreads();
    if (row == 0) {
        float t = 0.f;
        for (int r = 0; r < 32; ++r) t += sums[r][col];
        float* out = column < d ? dq_weight : dk_weight;
        if (out) out[column < d ? column : column - d] = t;
    }
}

}  // namespace sawtooth
