// Attention of one new token per request over a paged cache: one pass over K and V with a running maximum and sum, the work
// split evenly over the CTAs along the lengths (decode_schedule.h), and a second, short kernel that joins what the split cut.
//
// What bounds it is reading K and V once: per K/V head and token 4 d bytes against 4 d multiply-adds per query head.  So
// the layout serves the loads.  Each warp streams its own 16 tokens of every 64-token tile through a ring of its own in shared
// memory with 16-byte asynchronous copies (any page size and any strides; no barrier between warps in the loop), page numbers
// are looked up one tile ahead, and the loads run across the borders of requests.  The products have as many rows as query heads
// share a K/V head, 16 at most: a warp's mma.sync tile (m16n8k16), with the queries in registers.  A 128-row tcgen05 tile would be
// mostly padding, and its trips through tensor memory would add to the latency of short calls, where the kernel is bound by the
// chain of one tile.
//
// Probabilities enter the second product as the sum of two 16-bit numbers, p = hi + lo, so that rounding them adds nothing to the one
// rounding of the result (a single bf16 would add as much again); they are taken relative to the running maximum, for fp16
// times 2^kBias, so that small ones keep clear of its subnormal numbers.
#pragma once
#include "decode_schedule.h"
#include "paged_common.cuh"

namespace sawtooth {

struct DecodeParams {
    const uint16_t* q;
    uint16_t* o;
    float* lse;              // [B, H] or nullptr
    long long q_request, q_head, o_request, o_head;
    CacheView cache;
    const int* table;
    long long table_stride;
    const int* seq_len;
    int* status;
    int4* join;              // [grid] {parts, request, head block index, 0} of the request cut in that CTA's share
    float2* part_ml;         // [2 grid][16] running maximum (log2 units) and sum
    float* part_o;           // [2 grid][16][d] sums
    float scale_log2;
    int B, H, kv_heads, group, head_blocks, max_len;
};

constexpr int kDecodeThreads = 128;
constexpr int kDecodeWarps = 4;
constexpr int kDecodeWarpTokens = kDecodeTile / kDecodeWarps;   // 16

template <int kD>
struct DecodeGeometry {
    static constexpr int kRowBytes = kD * 2;
    static constexpr int kStageBytes = 2 * kDecodeWarpTokens * kRowBytes;      // K and V of a warp's tokens; also 16 fp32 rows of d
    static constexpr int kStages = kD == 128 ? 3 : 6;
    static constexpr int kSmem = kDecodeWarps * kStages * kStageBytes;          // 96 KiB: two CTAs an SM
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes)   // copies `bytes` (16 or 0), zero-fills the rest
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <int kBf16>
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (kBf16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A request's length, cut to what its table row can hold.
__device__ __forceinline__ int decode_len(const DecodeParams& p, int b)
{
    const int len = p.seq_len[b];
    return len < 0 ? 0 : len > p.max_len ? p.max_len : len;
}

// A place in the line of tiles: tile `tile` of n of the head block `block` of request b.
struct DecodeCursor {
    int b, block, tile, n, len, next_len;   // next_len: the length of request b + 1, read ahead
    __device__ __forceinline__ void advance(const DecodeParams& p, int blocks)
    {
        if (++tile < n) return;
        tile = 0;
        if (++block < blocks) return;
        block = 0;
        do {
            ++b;
            len = next_len;
            next_len = b + 1 < p.B ? decode_len(p, b + 1) : 0;
        } while (len == 0 && b < p.B);
        n = decode_tiles(len);
    }
};

template <int kD, int kBf16>
__global__ void __launch_bounds__(kDecodeThreads, 2) decode_paged_kernel(const DecodeParams p)
{
    using G = DecodeGeometry<kD>;
    constexpr int kStages = G::kStages, kPieces = kD / 8;            // 16-byte pieces of a row
    constexpr float kBias = kBf16 ? 0.f : 15.f;                      // log2 of the factor on the probabilities
    extern __shared__ __align__(128) uint8_t decode_smem[];
    __shared__ float2 warp_ml[kDecodeWarps][kDecodeRows];
    __shared__ uint64_t scan[kDecodeWarps];
    __shared__ int start_at[2];
    __shared__ uint64_t start_off;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int blocks = p.kv_heads * p.head_blocks;

    // ---- this CTA's share: sum of all requests' tiles, then the request and tile the share begins with
    const int chunk = (p.B + kDecodeThreads - 1) / kDecodeThreads, b_lo = tid * chunk, b_hi = min(p.B, b_lo + chunk);
    uint64_t mine = 0;
    bool bad = false;
    for (int b = b_lo; b < b_hi; ++b) {
        const int raw = p.seq_len[b];
        bad |= raw < 0 || raw > p.max_len;
        mine += (uint64_t)decode_tiles(raw < 0 ? 0 : raw > p.max_len ? p.max_len : raw) * blocks;
    }
    if (bad && blockIdx.x == 0) note_index(p.status, kIndexLength);
    uint64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t u = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += u;
    }
    if (lane == 31) scan[warp] = upto;
    __syncthreads();
    uint64_t total = 0;
#pragma unroll
    for (int w = 0; w < kDecodeWarps; ++w) {
        if (w < warp) upto += scan[w];
        total += scan[w];
    }
    const int ctas = decode_ctas(total, gridDim.x), cta = blockIdx.x;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    int4 join = make_int4(0, 0, 0, 0);
    if (cta < ctas) {
        const uint64_t begin = decode_share_begin(total, ctas, cta);
        int left = (int)(decode_share_begin(total, ctas, cta + 1) - begin);
        if (begin >= upto - mine && begin < upto) {
            uint64_t at = begin - (upto - mine);
            int b = b_lo;
            for (;; ++b) {
                const uint64_t t = (uint64_t)decode_tiles(decode_len(p, b)) * blocks;
                if (at < t) break;
                at -= t;
            }
            start_at[0] = b;
            start_off = at;
        }
        __syncthreads();
        DecodeCursor ld;
        ld.b = start_at[0];
        ld.len = decode_len(p, ld.b);
        ld.next_len = ld.b + 1 < p.B ? decode_len(p, ld.b + 1) : 0;
        ld.n = decode_tiles(ld.len);
        ld.block = (int)(start_off / (uint64_t)ld.n);
        ld.tile = (int)(start_off % (uint64_t)ld.n);
        DecodeCursor cp = ld;
        int to_load = left;

        const uint32_t ring = ptx::smem_u32(decode_smem) + warp * kStages * G::kStageBytes;
        // The page of the token that lane l < 16 looks after, in the tile the load cursor is at.
        auto look_up = [&]() -> int {
            const int token = ld.tile * kDecodeTile + warp * kDecodeWarpTokens + (lane & 15);
            return to_load > 0 && token < ld.len ? p.table[(long long)ld.b * p.table_stride + p.cache.page.div((uint32_t)token)] : -1;
        };
        int page = look_up();
        auto issue = [&](int stage) {
            if (to_load > 0) {
                const int token = ld.tile * kDecodeTile + warp * kDecodeWarpTokens + (lane & 15);
                const bool there = token < ld.len;
                long long at = -1;
                if (there) {
                    if (page >= 0 && page < p.cache.num_pages)
                        at = page * p.cache.page_stride + (long long)(token - (int)p.cache.page.div((uint32_t)token) * (int)p.cache.page.d) * p.cache.token_stride +
                             (long long)(ld.block / p.head_blocks) * p.cache.head_stride;
                    else
                        note_index(p.status, kIndexPage);
                }
                constexpr int kRowsAtOnce = 32 / kPieces;
                const uint32_t k_dst = ring + stage * G::kStageBytes, v_dst = k_dst + kDecodeWarpTokens * G::kRowBytes;
                const int piece = lane % kPieces;
#pragma unroll
                for (int i = 0; i < kDecodeWarpTokens / kRowsAtOnce; ++i) {
                    const int row = i * kRowsAtOnce + lane / kPieces;
                    const long long off = __shfl_sync(0xffffffffu, at, row);
                    const uint32_t d = row * G::kRowBytes + ((piece ^ (row & 7)) << 4);
                    const long long from = (off < 0 ? 0 : off) + piece * 8;
                    cp_async16(k_dst + d, p.cache.k + from, off < 0 ? 0 : 16);
                    cp_async16(v_dst + d, p.cache.v + from, off < 0 ? 0 : 16);
                }
                --to_load;
                if (to_load > 0) ld.advance(p, blocks);
                page = look_up();
            }
            cp_async_commit();
        };

        uint32_t qf[kD / 16][4];
        auto load_q = [&]() {
            const int kvh = cp.block / p.head_blocks, first = (cp.block % p.head_blocks) * kDecodeRows;
            const int rows = min(kDecodeRows, p.group - first);
            const uint16_t* base = p.q + (long long)cp.b * p.q_request + (long long)(kvh * p.group + first) * p.q_head + 2 * (lane & 3);
            const int r0 = lane >> 2, r1 = r0 + 8;
#pragma unroll
            for (int kk = 0; kk < kD / 16; ++kk) {
                qf[kk][0] = r0 < rows ? *reinterpret_cast<const uint32_t*>(base + r0 * p.q_head + kk * 16) : 0u;
                qf[kk][1] = r1 < rows ? *reinterpret_cast<const uint32_t*>(base + r1 * p.q_head + kk * 16) : 0u;
                qf[kk][2] = r0 < rows ? *reinterpret_cast<const uint32_t*>(base + r0 * p.q_head + kk * 16 + 8) : 0u;
                qf[kk][3] = r1 < rows ? *reinterpret_cast<const uint32_t*>(base + r1 * p.q_head + kk * 16 + 8) : 0u;
            }
        };

#pragma unroll
        for (int s = 0; s < kStages - 1; ++s) issue(s);
        load_q();
        float acc[kD / 8][4] = {};
        float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
        int stage = 0, first_tile = cp.tile;
        // ldmatrix: the row and piece that this lane gives the address of, for K (tokens are columns of B) and V (tokens are its rows)
        const int k_row = (lane & 7) + ((lane >> 4) << 3), k_half = (lane >> 3) & 1;
        const int v_row = (lane & 7) + (((lane >> 3) & 1) << 3), v_half = lane >> 4;

        for (; left > 0; --left) {
            cp_async_wait<kStages - 2>();
            __syncwarp();
            issue(stage == 0 ? kStages - 1 : stage - 1);
            const uint32_t k_base = ring + stage * G::kStageBytes, v_base = k_base + kDecodeWarpTokens * G::kRowBytes;
            const int valid = cp.len - cp.tile * kDecodeTile - warp * kDecodeWarpTokens;
            if (valid > 0) {
                float s[2][4] = {};
#pragma unroll
                for (int kk = 0; kk < kD / 16; ++kk) {
                    uint32_t b[4];
                    ldmatrix4(b, k_base + k_row * G::kRowBytes + (((2 * kk + k_half) ^ (k_row & 7)) << 4));
                    mma16816<kBf16>(s[0], qf[kk], b[0], b[1]);
                    mma16816<kBf16>(s[1], qf[kk], b[2], b[3]);
                }
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int token = n * 8 + 2 * (lane & 3) + (i & 1);
                        s[n][i] = token < valid ? s[n][i] * p.scale_log2 : -INFINITY;
                    }
                float top[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float t = fmaxf(fmaxf(s[0][2 * r], s[0][2 * r + 1]), fmaxf(s[1][2 * r], s[1][2 * r + 1]));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
                    t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
                    top[r] = fmaxf(m[r], t);
                }
                if (__any_sync(0xffffffffu, top[0] > m[0] || top[1] > m[1])) {
                    const float f0 = top[0] > m[0] ? ptx::ex2(m[0] - top[0]) : 1.f, f1 = top[1] > m[1] ? ptx::ex2(m[1] - top[1]) : 1.f;
                    m[0] = top[0];
                    m[1] = top[1];
                    l[0] *= f0;
                    l[1] *= f1;
#pragma unroll
                    for (int j = 0; j < kD / 8; ++j) { acc[j][0] *= f0; acc[j][1] *= f0; acc[j][2] *= f1; acc[j][3] *= f1; }
                }
                // A row whose scores are all -infinity so far has no reference: its probabilities are 0.
                const float ref0 = m[0] == -INFINITY ? 0.f : m[0] - kBias, ref1 = m[1] == -INFINITY ? 0.f : m[1] - kBias;
                uint32_t hi[4], lo[4];
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float p0 = ptx::ex2(s[n][2 * r] - (r ? ref1 : ref0)), p1 = ptx::ex2(s[n][2 * r + 1] - (r ? ref1 : ref0));
                        l[r] += p0 + p1;
                        const uint32_t h = ptx::pack2<kBf16>(p0, p1);
                        float h0, h1;
                        unpack2<kBf16>(h, h0, h1);
                        hi[2 * n + r] = h;
                        lo[2 * n + r] = ptx::pack2<kBf16>(p0 - h0, p1 - h1);
                    }
#pragma unroll
                for (int j = 0; j < kD / 16; ++j) {
                    uint32_t b[4];
                    ldmatrix4_trans(b, v_base + v_row * G::kRowBytes + (((2 * j + v_half) ^ (v_row & 7)) << 4));
                    mma16816<kBf16>(acc[2 * j], hi, b[0], b[1]);
                    mma16816<kBf16>(acc[2 * j + 1], hi, b[2], b[3]);
                    mma16816<kBf16>(acc[2 * j], lo, b[0], b[1]);
                    mma16816<kBf16>(acc[2 * j + 1], lo, b[2], b[3]);
                }
            }
            const bool ends = cp.tile == cp.n - 1;
            if (ends || left == 1) {
                // ---- the four warps' sums meet in shared memory, each in the stage that its warp has just emptied
                const int r0 = lane >> 2;
                __syncwarp();
                float* mine_o = reinterpret_cast<float*>(decode_smem + (size_t)(warp * kStages + stage) * G::kStageBytes);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
                    l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
                    const int row = r0 + 8 * r;
                    if ((lane & 3) == 0) warp_ml[warp][row] = make_float2(m[r], l[r]);
#pragma unroll
                    for (int j = 0; j < kD / 8; ++j) {
                        const int piece = 2 * j + ((lane & 3) >> 1);     // 16-byte piece of the fp32 row, moved against bank conflicts
                        *reinterpret_cast<float2*>(mine_o + row * kD + ((piece ^ (row & 7)) << 2) + ((lane & 1) << 1)) = make_float2(acc[j][2 * r], acc[j][2 * r + 1]);
                    }
                }
                __syncthreads();
                const int kvh = cp.block / p.head_blocks, first = (cp.block % p.head_blocks) * kDecodeRows;
                const int rows = min(kDecodeRows, p.group - first);
                const bool starts = first_tile == 0, whole = starts && ends;
                const int part = 2 * cta + (starts ? 1 : 0);
                for (int i = tid; i < rows * (kD / 4); i += kDecodeThreads) {
                    const int row = i / (kD / 4), piece = i % (kD / 4);
                    float big = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kDecodeWarps; ++w) big = fmaxf(big, warp_ml[w][row].x);
                    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
                    float total_l = 0.f;
#pragma unroll
                    for (int w = 0; w < kDecodeWarps; ++w) {
                        const float2 ml = warp_ml[w][row];
                        // A warp without a finite score has sums of 0 (or NaN, which is to stay): its weight is 1.
                        const float f = ml.x == -INFINITY ? 1.f : ptx::ex2(ml.x - big);
                        const float* from = reinterpret_cast<const float*>(decode_smem + (size_t)(w * kStages + stage) * G::kStageBytes);
                        const float4 x = *reinterpret_cast<const float4*>(from + row * kD + ((piece ^ (row & 7)) << 2));
                        sum.x += f * x.x; sum.y += f * x.y; sum.z += f * x.z; sum.w += f * x.w;
                        total_l += f * ml.y;
                    }
                    const int head = kvh * p.group + first + row;
                    if (whole) {
                        const float inv = 1.f / total_l;
                        *reinterpret_cast<uint2*>(p.o + (long long)cp.b * p.o_request + (long long)head * p.o_head + 4 * piece) =
                            make_uint2(ptx::pack2<kBf16>(sum.x * inv, sum.y * inv), ptx::pack2<kBf16>(sum.z * inv, sum.w * inv));
                        if (p.lse && piece == 0) p.lse[(long long)cp.b * p.H + head] = (big - kBias + log2f(total_l)) * 0.6931471805599453f;
                    } else {
                        *reinterpret_cast<float4*>(p.part_o + ((size_t)part * kDecodeRows + row) * kD + 4 * piece) = sum;
                        if (piece == 0) p.part_ml[(size_t)part * kDecodeRows + row] = make_float2(big, total_l);
                    }
                }
                if (starts && !ends) {
                    // Cut by the end of this share: the join of the parts is this CTA's to describe.
                    const uint64_t last = begin + (uint64_t)(decode_share_begin(total, ctas, cta + 1) - begin) - 1 + (uint64_t)(cp.n - 1 - cp.tile);
                    join = make_int4(decode_cta_of(total, ctas, last) - cta + 1, cp.b, cp.block, 0);
                }
                __syncthreads();   // the stages may be filled again
                m[0] = m[1] = -INFINITY;
                l[0] = l[1] = 0.f;
#pragma unroll
                for (int j = 0; j < kD / 8; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;
                if (left > 1) {
                    cp.advance(p, blocks);
                    first_tile = 0;
                    load_q();
                }
            } else {
                ++cp.tile;
            }
            stage = stage + 1 == kStages ? 0 : stage + 1;
        }
        cp_async_wait<0>();
    }
    if (tid == 0) p.join[cta] = join;
    // ---- requests without tokens
    for (int b = cta; b < p.B; b += gridDim.x) {
        if (decode_len(p, b) != 0) continue;
        for (int i = tid; i < p.H * (kD / 8); i += kDecodeThreads)
            *reinterpret_cast<uint4*>(p.o + (long long)b * p.o_request + (long long)(i / (kD / 8)) * p.o_head + (i % (kD / 8)) * 8) = make_uint4(0, 0, 0, 0);
        if (p.lse)
            for (int h = tid; h < p.H; h += kDecodeThreads) p.lse[(long long)b * p.H + h] = -INFINITY;
    }
}

// Joins the parts of the request that CTA blockIdx.x began and did not finish, row blockIdx.y of its 16: o = sum_i f_i o_i / sum_i f_i l_i,
// f_i = 2^(m_i - max m).  The eight warps take the parts in turn, each over all columns; their sums are added in a fixed order.
constexpr int kJoinThreads = 256;
template <int kD, int kBf16>
__global__ void __launch_bounds__(kJoinThreads) decode_join_kernel(const DecodeParams p)
{
    constexpr int kWarps = kJoinThreads / 32, kCols = kD / 32;     // columns a lane sums
    constexpr float kBias = kBf16 ? 0.f : 15.f;
    __shared__ float sums[kWarps][kD];
    __shared__ float sums_l[kWarps];
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int4 join = p.join[blockIdx.x];
    if (join.x == 0) return;
    const int n = join.x, row = blockIdx.y, c0 = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int kvh = join.z / p.head_blocks, first = (join.z % p.head_blocks) * kDecodeRows;
    if (first + row >= p.group) return;
    auto entry = [&](int i) { return (size_t)(i == 0 ? 2 * c0 + 1 : 2 * (c0 + i)) * kDecodeRows + row; };
    float big = -INFINITY;
    for (int i = lane; i < n; i += 32) big = fmaxf(big, p.part_ml[entry(i)].x);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    float acc[kCols] = {}, l = 0.f;
#pragma unroll 4
    for (int i = warp; i < n; i += kWarps) {
        const float2 ml = p.part_ml[entry(i)];
        const float f = ml.x == -INFINITY ? 1.f : ptx::ex2(ml.x - big);
        const float* from = p.part_o + entry(i) * kD + lane * kCols;
        float x[kCols];
        if (kCols == 4) {
            const float4 v = *reinterpret_cast<const float4*>(from);
            x[0] = v.x; x[1] = v.y; x[kCols - 2] = v.z; x[kCols - 1] = v.w;
        } else {
            const float2 v = *reinterpret_cast<const float2*>(from);
            x[0] = v.x; x[1] = v.y;
        }
#pragma unroll
        for (int c = 0; c < kCols; ++c) acc[c] += f * x[c];
        l += f * ml.y;
    }
#pragma unroll
    for (int c = 0; c < kCols; ++c) sums[warp][lane * kCols + c] = acc[c];
    if (lane == 0) sums_l[warp] = l;
    __syncthreads();
    if (threadIdx.x < kD / 2) {
        float a = 0.f, b = 0.f, t = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) { a += sums[w][2 * threadIdx.x]; b += sums[w][2 * threadIdx.x + 1]; t += sums_l[w]; }
        const float inv = 1.f / t;
        const int head = kvh * p.group + first + row;
        *reinterpret_cast<uint32_t*>(p.o + (long long)join.y * p.o_request + (long long)head * p.o_head + 2 * threadIdx.x) = ptx::pack2<kBf16>(a * inv, b * inv);
        if (p.lse && threadIdx.x == 0) p.lse[(long long)join.y * p.H + head] = (big - kBias + log2f(t)) * 0.6931471805599453f;
    }
}

}  // namespace sawtooth
