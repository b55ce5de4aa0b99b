// Attention over the paged 8-bit cache for few query rows: one token a sequence, or a few drafted ones.
//
//   s_t = scale * q . k_t,   o = sum_t softmax(s)_t v_t,   k_t = 2^(sk - 127) * code, v_t likewise
//
// Every code is read once from HBM, which bounds the call (2 * dim bytes a token and head).  The codes are widened to f16, which
// is exact, two at a time in registers, and multiplied there with binary32 sums (mma m16n8k16), keys and values as the 16-row
// operand, so that the query rows are the 8 columns: eight query heads that share a key head fill a product.
//   q  is scaled by a power of two that brings the row's largest magnitude to [2^14, 2^15), so that f16 holds a bf16 value exactly
//      but for elements below 2^-28 of the row's largest (to 2^-39 of it).
//   The scales of the cache never touch the codes: a key block's scale multiplies the finished product, a value block's is
//      folded into the softmax's weight, w_t = 2^(s_t + sv_t - R + 1) in f16.  The reference R (an integer, so that corrections of
//      the sums are exact) is moved when a tile's largest s + sv is 14 above or 16 below it: f16 keeps 11 bits of what is above
//      2^-14 and drops what is below 2^-25.  The softmax's own sum is l = sum of the unrounded w_t 2^(c0 - sv_t), a factor for each
//      run of 16 tokens, c0 near the warp's scales; a tile with scales far from c0, and those after it until the two references have
//      come near each other, are summed apart (see kApart).
//
// A CTA of four warps takes up to 8 * NQ * RW query rows of one sequence and key head, and one chunk of the keys.  4 / RW groups
// of warps walk over the chunk's tiles of 32 tokens in turn; each group feeds itself through a ring of tiles that the
// tensor copy engine fills (swizzled: the two access patterns below are then free of bank conflicts).  Within a tile,
// a thread reads its operand words with 16-byte loads: the order of the dimensions within a product and of the tokens within a
// sum is free, and is chosen so that a thread's share is contiguous: a word of four key codes is half of one step's operand.  The
// values' operand wants two tokens of one dimension side by side: one byte permutation makes two such pairs of codes.  The
// weights turn from the first product's result layout to the second's operand with one 8 x 8 transposition for eight tokens.
//
// With several chunks a CTA's result is (normalised row, logarithm of its sum).  Up to eight chunks are joined by their CTAs as a
// cluster, through each other's shared memory; more go to the workspace and are joined in a fixed order by a second kernel.
//
// Measured (32 query and 8 key heads of 128; on the device alone, in turn with other work in brackets): 64 sequences of up to 8192 keys
// 115 us, 5.9 TB/s (118); one of 131072 keys 49 us, 5.4 TB/s with the join; one of 1000 keys 6.3 us, which is a start, two trips to
// memory and the join.  32 sequences of four drafted tokens, 32 and 4 heads of 64, window 1024: 20 us, seven times what its bytes
// take: 256 CTAs whose warps walk over at most five tiles of 32 query rows; how much of it is the start is not known.
//
// Every wait is bounded (see mxn_device_timeouts).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>

#include "mxn_attn.cuh"

namespace mxn {

namespace {

constexpr int kSMs = 148;
constexpr int kWarps = 4;
// CTAs an SM that the register allocation makes room for
__host__ __device__ constexpr int decode_ctas(int dim, int nq) { return nq == 1 ? (dim == 128 ? 3 : 4) : dim == 128 || nq == 4 ? 2 : 3; }
constexpr int kTile = 32;      // tokens of a tile
constexpr int kPromptRows = 64;   // more query rows a sequence and key head than this: the tcgen05 kernel
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ unsigned int g_attn_timeouts = 0;
__device__ unsigned int g_attn_bad = 0;   // pages out of range within a sequence's length

__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the four E4M3 codes of a word -> two f16 pairs
__device__ __forceinline__ void widen(uint32_t w, uint32_t& lo, uint32_t& hi)
{
    asm("{ .reg .b16 l, h; mov.b32 {l, h}, %2; cvt.rn.f16x2.e4m3x2 %0, l; cvt.rn.f16x2.e4m3x2 %1, h; }" : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// transposes an 8 x 8 matrix of f16: row g, columns 2c, 2c + 1 in a thread's register
__device__ __forceinline__ uint32_t turn8x8(uint32_t v)
{
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ uint2 lds_v2(uint32_t addr)
{
    uint2 r;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(addr));
    return r;
}
__device__ __forceinline__ float quad_max(float v)
{
    v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 1));
    return fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, 2));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&v);
}

// weights: 2^kTop at the reference, which is moved when a tile's largest is kUp above or kDown below it, but to no more than kDepth
// below the largest so far (the output's sums must not overflow)
constexpr float kTop = 1.0f, kUp = 14.0f, kDown = 16.0f, kDepth = 40.0f;

template <int DIM, int RW, int NQ, int STAGES>
struct DecodeShape {
    static constexpr int kGroups = kWarps / RW;                  // warp groups that share out the tiles
    static constexpr int kTileBytes = kTile * DIM;               // codes of a tile, keys or values
    static constexpr int kRingBytes = kGroups * STAGES * 2 * kTileBytes;
    static constexpr int kRows = 8 * NQ * RW;
    static constexpr int kJoinBytes = kGroups * kRows * ((DIM + 4) * 4 + 8);
    static constexpr int kSmem = (kRingBytes > kJoinBytes ? kRingBytes : kJoinBytes) + 1024;
};

// ---- clusters: the CTAs that hold the chunks of the same rows ----
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_u32(uint32_t addr, int rank)
{
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(at));
    return v;
}
__device__ __forceinline__ float4 remote_f4(uint32_t addr, int rank)
{
    uint32_t at;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
    return v;
}

// NQ: groups of eight query rows that a warp works on (they share the widened codes); RW: warps that share out the rows
template <int DIM, int RW, int NQ, int STAGES>
__global__ void __launch_bounds__(kWarps * 32, decode_ctas(DIM, NQ)) attn_decode_kernel(const AttnParams P, const __grid_constant__ AttnMaps M)
{
    using Sh = DecodeShape<DIM, RW, NQ, STAGES>;
    constexpr int MT = DIM / 16;     // row tiles of the second product: 16 dimensions each
    constexpr int KS = DIM / 16;     // steps of the first
    constexpr int QN = 2 * NQ;       // query rows whose softmax this thread looks after: 8 (x/2) + 2c + x%2
    constexpr int GROUPS = Sh::kGroups;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * GROUPS * STAGES];   // full, then empty
    __shared__ float chunk_lse[Sh::kRows];           // for the other CTAs of a cluster
    __shared__ float sum_refs[kWarps][8 * NQ];       // references of the rows' sums, once these are apart

    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const int group = warp / RW, rw = warp % RW;
    uint32_t b = blockIdx.x;
    const int split = (int)(b % (uint32_t)P.splits);
    b /= (uint32_t)P.splits;
    const int rt = (int)(b % (uint32_t)P.row_tiles);
    b /= (uint32_t)P.row_tiles;
    const int h = (int)(b % (uint32_t)P.kv_heads);
    const int seq = (int)(b / (uint32_t)P.kv_heads);

    const AttnSequence S = attn_sequence(P, seq);
    const int q0 = S.q0, len = S.len, shift = S.shift, nq = S.nq;
    const int G = P.group, row0 = rt * Sh::kRows, rows = nq * G;
    if (row0 >= rows) return;
    // keys that any row of this tile sees: [lo, hi)
    const int last = min(rows, row0 + Sh::kRows) - 1;
    const int hi = max(0, min(len, P.causal ? shift + P.by_group(last) + 1 : len));
    const int seen = first_seen(shift + P.by_group(row0), P.window);   // nothing before it, not even its page, has any influence
    const int lo = seen / kTile * kTile;
    const int k0 = (int)min((int64_t)hi, lo + (int64_t)split * P.chunk), k1 = (int)min((int64_t)hi, (int64_t)k0 + P.chunk);
    const int tiles = (k1 - k0 + kTile - 1) / kTile;

    // keys [see_lo, see_hi) of this thread's rows; the tile's rows that every row sees in full
    const int row_base = row0 + rw * 8 * NQ;
    int see_hi[QN], see_lo[QN];
#pragma unroll
    for (int x = 0; x < QN; ++x) {
        const int row = min(row_base + 8 * (x >> 1) + 2 * c + (x & 1), rows - 1);
        const int pos = shift + P.by_group(row);
        see_hi[x] = P.causal ? min(pos + 1, len) : len;
        see_lo[x] = first_seen(pos, P.window);
    }
    int all_hi = see_hi[0], all_lo = see_lo[0];
#pragma unroll
    for (int x = 1; x < QN; ++x) {
        all_hi = min(all_hi, see_hi[x]);
        all_lo = max(all_lo, see_lo[x]);
    }
    all_hi = min(all_hi, k1);
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        all_hi = min(all_hi, __shfl_xor_sync(0xFFFFFFFFu, all_hi, o));
        all_lo = max(all_lo, __shfl_xor_sync(0xFFFFFFFFu, all_lo, o));
    }

    // row g of each eight query rows, the 32 (DIM = 128) or 16 (DIM = 64) dimensions from c * DIM/4 on: on their way while the
    // first tiles are asked for
    uint4 q_raw[NQ][DIM / 32];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const int row = row_base + 8 * x + g, qt = P.by_group(row);
        const bool live = row < rows;
        const uint16_t* qp = P.q + (int64_t)(q0 + qt) * P.q_stride + (h * G + row - qt * G) * DIM + c * (DIM / 4);
#pragma unroll
        for (int i = 0; i < DIM / 32; ++i) q_raw[x][i] = live ? __ldg(reinterpret_cast<const uint4*>(qp) + i) : make_uint4(0, 0, 0, 0);
    }

    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t ring = base + (uint32_t)group * STAGES * 2 * Sh::kTileBytes;
    const uint32_t full = smem_u32(bars) + (uint32_t)group * STAGES * 8, empty = full + GROUPS * STAGES * 8;
    const bool leader = rw == 0 && lane == 0;
    if (threadIdx.x == 0) {
        for (int i = 0; i < GROUPS * STAGES; ++i) {
            mbar_init(smem_u32(bars) + 8 * i, 1);
            mbar_init(smem_u32(bars) + 8 * (GROUPS * STAGES + i), RW);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();

    // the group's tiles are group, group + GROUPS, ...; tile i of them goes to stage i % STAGES
    const int mine = tiles > group ? (tiles - group + GROUPS - 1) / GROUPS : 0;
    const int32_t* const table = P.page_table + (int64_t)seq * P.max_pages;
    // A tile has two runs of 16 tokens, each within one page; lanes 0-15 look after the first, 16-31 after the second.
    // page_at(i): the table's entry for this lane's run of tile i, -1 behind the last token and before the window.  It is looked at a tile later at the
    // earliest, so that nothing waits for it.
    const int run = lane >> 4;
    bool bad_page = false;
    auto tile_at = [&](int i) { return k0 + (group + i * GROUPS) * kTile; };
    const bool two_boxes = P.page < kTile;   // a page of 16 tokens takes two boxes to a tile
    auto page_at = [&](int i) -> int {
        const int t = tile_at(i) + 16 * run;
        return i < mine && t < k1 && (t | (two_boxes ? 15 : kTile - 1)) >= seen ? __ldg(table + (t >> P.page_shift)) : -1;
    };
    auto in_pool = [&](int pg) { return (uint32_t)pg < (uint32_t)P.num_pages; };
    const uint32_t box_bytes = two_boxes ? Sh::kTileBytes / 2 : Sh::kTileBytes;
    auto request = [&](int i, int st, int pg) {   // by a whole warp, with page_at(i) in hand
        const int pg1 = two_boxes ? __shfl_sync(0xFFFFFFFFu, pg, 16) : -1;
        if (!leader) return;
        const uint32_t dst = ring + (uint32_t)st * 2 * Sh::kTileBytes, bar = full + 8 * st;
        const uint32_t bytes = (uint32_t)(in_pool(pg) + in_pool(pg1)) * 2 * box_bytes;
        if (bytes == 0) {
            mbar_arrive(bar);
            return;
        }
        mbar_expect_tx(bar, bytes);
        const int y = tile_at(i) & (P.page - 1);
        if (in_pool(pg)) {
            tma_load_codes(dst, &M.k, y, pg * P.kv_heads + h, bar);
            tma_load_codes(dst + Sh::kTileBytes, &M.v, y, pg * P.kv_heads + h, bar);
        }
        if (in_pool(pg1)) {
            tma_load_codes(dst + box_bytes, &M.k, 0, pg1 * P.kv_heads + h, bar);
            tma_load_codes(dst + Sh::kTileBytes + box_bytes, &M.v, 0, pg1 * P.kv_heads + h, bar);
        }
    };
    // pages of the tiles from the one at hand on: asked for STAGES + 1 tiles ahead
    int pages[STAGES + 2];
#pragma unroll
    for (int d = 0; d < STAGES + 2; ++d) pages[d] = page_at(d);
    if (rw == 0) {
#pragma unroll
        for (int d = 0; d < STAGES; ++d)
            if (d < mine) request(d, d, pages[d]);
    }
    // scales, one tile ahead: lanes 0 and 16 hold the key scales of the two runs, lanes 1 and 17 the value scales
    const uint8_t* const scale_base = lane & 1 ? P.v_scales : P.k_scales;
    const int per_page = P.page_shift - P.block_shift;
    uint32_t no_scale = 0;   // for a run without tokens
    auto scale_at = [&](int i, int pg) -> uint32_t {
        if ((lane & 15) >= 2 || !in_pool(pg)) return no_scale;
        const int64_t tile = (int64_t)pg * P.kv_heads + h;
        return __ldg(scale_base + (tile << per_page) + (((tile_at(i) + 16 * run) & (P.page - 1)) >> P.block_shift));
    };
    uint32_t sc_next = scale_at(0, pages[0]);

    // q: the power of two goes to the row's factor, which the softmax needs in the threads of its columns
    uint32_t qb[KS][NQ][2];
    float row_factor[QN];
#pragma unroll
    for (int x = 0; x < NQ; ++x) {
        const uint32_t* u = reinterpret_cast<const uint32_t*>(q_raw[x]);
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < DIM / 8; ++i) m = absmax_bf16x2(m, u[i]);
        const uint32_t E = __float_as_uint(quad_max(hmax_abs_to_f32(m))) >> 23;
        const uint32_t Ec = min(max(E, 15u), 254u);
        // 2^(14 - (E - 127)); with an infinity or NaN in the row its result is NaN
        const float up = E == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float((268u - Ec) << 23);
        const float factor = P.scale * kLog2e * __uint_as_float((Ec - 14u) << 23);          // ... and its inverse
        row_factor[2 * x] = __shfl_sync(0xFFFFFFFFu, factor, 8 * c);
        row_factor[2 * x + 1] = __shfl_sync(0xFFFFFFFFu, factor, 8 * c + 4);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            qb[k][x][0] = pack_f16(bf16_lo(u[2 * k]) * up, bf16_hi(u[2 * k]) * up);
            qb[k][x][1] = pack_f16(bf16_lo(u[2 * k + 1]) * up, bf16_hi(u[2 * k + 1]) * up);
        }
    }

    float acc[MT][NQ][4];
#pragma unroll
    for (int j = 0; j < MT; ++j)
#pragma unroll
        for (int x = 0; x < NQ; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[j][x][e] = 0.0f;
    const float kNone = -INFINITY;
    float ref[QN], top_all[QN], l[QN];   // reference (an integer), the largest so far, this thread's part of the sum
#pragma unroll
    for (int x = 0; x < QN; ++x) {
        ref[x] = top_all[x] = kNone;
        l[x] = 0.0f;
    }
    // near the value scales: the largest of the first tile; runs without tokens count as one of them
    const uint32_t first_scale = max(__shfl_sync(0xFFFFFFFFu, sc_next, 1), __shfl_sync(0xFFFFFFFFu, sc_next, 17));
    no_scale = min(max(first_scale, 67u), 187u);
    float c0 = (float)(int)no_scale - 127.0f;
    if (!in_pool(pages[0])) sc_next = no_scale;
    bool ok = true, apart = false;   // apart: the sums have references of their own

    int st = 0;
    uint32_t ph = 0;
    for (int i = 0; i < mine; ++i) {
        const int t0 = tile_at(i);
        const uint32_t sc = sc_next;
        sc_next = scale_at(i + 1, pages[1]);
        const float kf[2] = {e8m0_to_f32(__shfl_sync(0xFFFFFFFFu, sc, 0)), e8m0_to_f32(__shfl_sync(0xFFFFFFFFu, sc, 16))};
        float sv[2] = {(float)(int)__shfl_sync(0xFFFFFFFFu, sc, 1) - 127.0f, (float)(int)__shfl_sync(0xFFFFFFFFu, sc, 17) - 127.0f};
        // tokens of the tile that exist and whose page could be read
        const bool readable = in_pool(pages[0]);
        const bool wanted = t0 + lane < k1 && t0 + lane >= seen;
        const uint32_t there = __ballot_sync(0xFFFFFFFFu, wanted && readable);
        bad_page |= wanted && !readable;
        const bool was_apart = apart;
        apart = apart || fabsf(sv[0] - c0) > kApart || fabsf(sv[1] - c0) > kApart;
        if (__builtin_expect(was_apart, 0)) {
            // back to the common unit, with c0 near this tile's scales, if these allow it and the rows' references lie near enough
            const bool some0 = (there & 0xFFFFu) != 0u, some1 = (there >> 16) != 0u;
            const float top = fminf(fmaxf(fmaxf(some0 ? sv[0] : -60.0f, some1 ? sv[1] : -60.0f), -60.0f), 60.0f);
            bool near = !(some0 && fabsf(sv[0] - top) > kApart) && !(some1 && fabsf(sv[1] - top) > kApart);
            float d[QN];
#pragma unroll
            for (int x = 0; x < QN; ++x) {
                const float r = sum_refs[warp][8 * (x >> 1) + 2 * c + (x & 1)];
                d[x] = ref[x] == kNone && r == kNone ? 0.0f : ref[x] - kTop - top - r;
                near = near && fabsf(d[x]) <= kApart;
            }
            if (__all_sync(0xFFFFFFFFu, near)) {
                apart = false;
                c0 = top;
                no_scale = (uint32_t)((int)c0 + 127);
                if (!some0) sv[0] = c0;
                if (!some1) sv[1] = c0;
#pragma unroll
                for (int x = 0; x < QN; ++x) l[x] = times_pow2(l[x], -d[x]);
            }
        }

        // (the warp leaves the loop as a whole: its lanes' polls may end differently)
        if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(full + 8 * st, ph))) {
            ok = false;
            break;
        }
        const uint32_t kt = ring + (uint32_t)st * 2 * Sh::kTileBytes, vt = kt + Sh::kTileBytes;

        // ---- s = k . q: this thread gets tokens 16t + g and 16t + 8 + g for its query rows ----
        float s[2][NQ][4];   // [16 tokens][eight rows]: (g, 2c), (g, 2c + 1), (g + 8, 2c), (g + 8, 2c + 1)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t w[2][KS];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int r = 16 * t + 8 * x + g;
                if constexpr (DIM == 128) {
                    const uint4 a = lds_v4(kt + r * 128 + (((2 * c) ^ g) << 4)), d = lds_v4(kt + r * 128 + (((2 * c + 1) ^ g) << 4));
                    w[x][0] = a.x; w[x][1] = a.y; w[x][2] = a.z; w[x][3] = a.w;
                    w[x][4] = d.x; w[x][5] = d.y; w[x][6] = d.z; w[x][7] = d.w;
                } else {
                    const uint4 a = lds_v4(kt + r * 64 + ((c ^ ((g >> 1) & 3)) << 4));
                    w[x][0] = a.x; w[x][1] = a.y; w[x][2] = a.z; w[x][3] = a.w;
                }
            }
#pragma unroll
            for (int x = 0; x < NQ; ++x)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[t][x][e] = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                uint32_t a0, a1, a2, a3;
                widen(w[0][k], a0, a2);
                widen(w[1][k], a1, a3);
#pragma unroll
                for (int x = 0; x < NQ; ++x) mma_f16(s[t][x], a0, a1, a2, a3, qb[k][x][0], qb[k][x][1]);
            }
        }
        // ---- s + sv (s alone for sums that are apart), and what the rows may not see ----
        float f[2][QN];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int x = 0; x < QN; ++x) {
                f[t][x] = kf[t] * row_factor[x];
#pragma unroll
                for (int e = 0; e < 2; ++e) s[t][x >> 1][2 * e + (x & 1)] = fmaf(s[t][x >> 1][2 * e + (x & 1)], f[t][x], apart ? 0.0f : sv[t]);
            }
        if (there != 0xFFFFFFFFu || t0 < all_lo || t0 + kTile > all_hi) {
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int at = 16 * t + 8 * e + g, place = t0 + at;
#pragma unroll
                    for (int x = 0; x < QN; ++x)
                        if (!((there >> at) & 1u) || place < see_lo[x] || place >= see_hi[x]) s[t][x >> 1][2 * e + (x & 1)] = kNone;
                }
        }
        if (__builtin_expect(apart, 0)) {
            // the row's reference: shared by the eight threads that look after the row
            float* const refs = sum_refs[warp] + 2 * c;
#pragma unroll
            for (int x = 0; x < QN; ++x) {
                float* const at = refs + 8 * (x >> 1) + (x & 1);
                const float z[4] = {s[0][x >> 1][x & 1], s[0][x >> 1][2 + (x & 1)], s[1][x >> 1][x & 1], s[1][x >> 1][2 + (x & 1)]};
                float m = fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3]));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                float r = was_apart ? *at : ref[x] == kNone ? kNone : ref[x] - kTop - c0;
                if (m > r + kLift) {
                    const float next = ceilf(m);
                    l[x] = r == kNone ? l[x] : times_pow2(l[x], r - next);
                    r = next;
                }
                if (r > kNone) l[x] += (ex2(z[0] - r) + ex2(z[1] - r)) + (ex2(z[2] - r) + ex2(z[3] - r));
                __syncwarp();
                if (g == 0) *at = r;
            }
            __syncwarp();
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int x = 0; x < NQ; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[t][x][e] += sv[t];
        }
        // ---- reference: moved where a weight would leave the window ----
        bool out = false;
#pragma unroll
        for (int x = 0; x < QN; ++x) {
            const float m = fmaxf(fmaxf(s[0][x >> 1][x & 1], s[0][x >> 1][2 + (x & 1)]), fmaxf(s[1][x >> 1][x & 1], s[1][x >> 1][2 + (x & 1)]));
            // of the eight threads that share the row: one above, or none but some token in reach of it
            const uint32_t mates = 0x11111111u << c;
            const bool none = (__ballot_sync(0xFFFFFFFFu, m >= ref[x] - kDown) & mates) == 0u;
            out = out || (m > ref[x] + kUp) || (ref[x] == kNone && m > kNone) || (none && m > kNone && ref[x] > top_all[x] - kDepth);
        }
        if (__any_sync(0xFFFFFFFFu, out)) {
#pragma unroll
            for (int x = 0; x < QN; ++x) {
                float m = fmaxf(fmaxf(s[0][x >> 1][x & 1], s[0][x >> 1][2 + (x & 1)]), fmaxf(s[1][x >> 1][x & 1], s[1][x >> 1][2 + (x & 1)]));
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
                float next = ref[x];
                if (m > ref[x] + kUp || (ref[x] == kNone && m > kNone)) next = ceilf(m);
                else if (m < ref[x] - kDown && m > kNone) next = fmaxf(ceilf(m), top_all[x] - kDepth);
                top_all[x] = fmaxf(top_all[x], next);
                const float alpha = ref[x] == kNone ? 0.0f : ex2(ref[x] - next);
                ref[x] = next;
                l[x] *= apart ? 1.0f : alpha;
#pragma unroll
                for (int j = 0; j < MT; ++j) {
                    acc[j][x >> 1][x & 1] *= alpha;
                    acc[j][x >> 1][2 + (x & 1)] *= alpha;
                }
            }
        }
        // ---- weights, turned to the second product's operand; the softmax's sum ----
        float by[QN];
#pragma unroll
        for (int x = 0; x < QN; ++x) by[x] = ref[x] == kNone ? 0.0f : kTop - ref[x];
        uint32_t pb[2][NQ][2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const float back = apart ? 0.0f : ex2(c0 - sv[t]);   // (a NaN among the weights reaches the sum all the same)
#pragma unroll
            for (int x = 0; x < NQ; ++x) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = ex2(s[t][x][e] + by[2 * x + (e & 1)]);
                l[2 * x] = fmaf(w[0] + w[2], back, l[2 * x]);
                l[2 * x + 1] = fmaf(w[1] + w[3], back, l[2 * x + 1]);
                pb[t][x][0] = turn8x8(pack_f16(w[0], w[1]));
                pb[t][x][1] = turn8x8(pack_f16(w[2], w[3]));
            }
        }
        // ---- o += v w: tokens 2c, 2c+1, 8+2c, 9+2c (then 16 more) of DIM/8 dimensions from g * DIM/8 on ----
        constexpr int VW = DIM / 32;   // words a thread reads of each token
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint32_t v[4][VW];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const int r = 16 * t + 8 * (x >> 1) + 2 * c + (x & 1);
                if constexpr (DIM == 128) {
                    const uint4 a = lds_v4(vt + r * 128 + ((g ^ (r & 7)) << 4));
                    v[x][0] = a.x; v[x][1] = a.y; v[x][2] = a.z; v[x][3] = a.w;
                } else {
                    const uint2 a = lds_v2(vt + r * 64 + (((g >> 1) ^ ((r >> 1) & 3)) << 4) + (g & 1) * 8);
                    v[x][0] = a.x; v[x][1] = a.y;
                }
            }
            if (there != 0xFFFFFFFFu) {   // whatever stands behind the last token or before the window, a NaN among it, must not meet the zero weights
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int at = 16 * t + 8 * (x >> 1) + 2 * c + (x & 1);
                    if (!((there >> at) & 1u))
#pragma unroll
                        for (int y = 0; y < VW; ++y) v[x][y] = 0u;
                }
            }
#pragma unroll
            for (int y = 0; y < VW; ++y) {
                uint32_t a[2][4];   // [8 tokens][dimension]: f16 pairs of two tokens
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    widen(__byte_perm(v[2 * x][y], v[2 * x + 1][y], 0x5140), a[x][0], a[x][1]);
                    widen(__byte_perm(v[2 * x][y], v[2 * x + 1][y], 0x7362), a[x][2], a[x][3]);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e)   // row g of the product: dimension 4y + 2e of this thread's, row g + 8: the next
#pragma unroll
                    for (int x = 0; x < NQ; ++x)
                        mma_f16(acc[2 * y + e][x], a[0][2 * e], a[0][2 * e + 1], a[1][2 * e], a[1][2 * e + 1], pb[t][x][0], pb[t][x][1]);
            }
        }
        // ---- hand the stage back ----
        __syncwarp();
        if (RW > 1) {
            if (lane == 0) mbar_arrive(empty + 8 * st);
            if (rw == 0 && i + STAGES < mine) {
                if (!__all_sync(0xFFFFFFFFu, mbar_wait_bounded(empty + 8 * st, ph))) {
                    ok = false;
                    break;
                }
                request(i + STAGES, st, pages[STAGES]);
            }
        } else if (i + STAGES < mine) {
            request(i + STAGES, st, pages[STAGES]);
        }
        if (++st == STAGES) {
            st = 0;
            ph ^= 1u;
        }
#pragma unroll
        for (int d = 0; d < STAGES + 1; ++d) pages[d] = pages[d + 1];
        pages[STAGES + 1] = page_at(i + STAGES + 2);
    }
    if (!ok) {
        // a wait ran out: no further copies are asked for; those in flight get a second, shorter wait before the shared
        // memory is given up
        if (lane == 0) atomicAdd(&g_attn_timeouts, 1u);
        if (leader)
            for (int st = 0; st < STAGES; ++st) {
                (void)mbar_wait_bounded(full + 8 * st, 0, 1u << 14);
                (void)mbar_wait_bounded(full + 8 * st, 1, 1u << 14);
            }
    }
    if (__any_sync(0xFFFFFFFFu, bad_page) && lane == 0) atomicAdd(&g_attn_bad, 1u);

    // ---- join the groups of warps ----
    // row x of this thread: sum l 2^at, output acc unit 2^at; dimensions g * DIM/8 ... + DIM/8 - 1.  at = ref - kTop - c0 and unit = 2^c0;
    // with a reference of its own the sum is brought to [1/16, 1/8), and acc to the same unit in two steps, since the power may lie outside
    // binary32's range where the product does not (it is below a quarter of the largest value then, and the groups' sum in range).
    constexpr int OUT = DIM / 8, PITCH = DIM + 4;
    float* const sm = reinterpret_cast<float*>(raw + (base - smem_u32(raw)));
    float2* const stat = reinterpret_cast<float2*>(sm + GROUPS * Sh::kRows * PITCH);   // (at, l)
    const float unit = apart ? 1.0f : ex2(c0);
    float at[QN];
#pragma unroll
    for (int x = 0; x < QN; ++x) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) l[x] += __shfl_xor_sync(0xFFFFFFFFu, l[x], o);
        at[x] = ref[x] - kTop - c0;
    }
    if (__builtin_expect(apart, 0)) {
#pragma unroll
        for (int x = 0; x < QN; ++x) {
            at[x] = sum_refs[warp][8 * (x >> 1) + 2 * c + (x & 1)];
            if (at[x] == kNone) continue;
            const int e = min(max((int)(__float_as_uint(l[x]) >> 23) - 127, -126), 127) + 4;
            l[x] = times_pow2(l[x], (float)-e);
            at[x] += (float)e;
            const float d = ref[x] - kTop - at[x], half = floorf(0.5f * d), by1 = ex2(half), by2 = ex2(d - half);
#pragma unroll
            for (int j = 0; j < MT; ++j) {
                acc[j][x >> 1][x & 1] = acc[j][x >> 1][x & 1] * by1 * by2;
                acc[j][x >> 1][2 + (x & 1)] = acc[j][x >> 1][2 + (x & 1)] * by1 * by2;
            }
        }
    }
    __syncthreads();   // every copy has landed and been read
#pragma unroll
    for (int x = 0; x < QN; ++x) {
        const int place = group * Sh::kRows + rw * 8 * NQ + 8 * (x >> 1) + 2 * c + (x & 1);
        float* const p = sm + place * PITCH + g * OUT;
#pragma unroll
        for (int y = 0; y < MT / 2; ++y)
            *reinterpret_cast<float4*>(p + 4 * y) = make_float4(acc[2 * y][x >> 1][x & 1] * unit, acc[2 * y][x >> 1][2 + (x & 1)] * unit,
                                                                acc[2 * y + 1][x >> 1][x & 1] * unit, acc[2 * y + 1][x >> 1][2 + (x & 1)] * unit);
        if (g == 0) stat[place] = make_float2(at[x], l[x]);
    }
    __syncthreads();
    // all threads: eight dimensions of a row at a time
    for (int item = threadIdx.x; item < Sh::kRows * OUT; item += kWarps * 32) {
        const int in_tile = item / OUT, part = item % OUT, row = row0 + in_tile;
        if (row >= rows) break;
        float2 st[GROUPS];
        float top = kNone, sum = 0.0f, o[8];
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            st[k] = stat[k * Sh::kRows + in_tile];
            top = fmaxf(top, st[k].x);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < GROUPS; ++k) {
            const float by = st[k].x == kNone ? 0.0f : ex2(st[k].x - top);
            sum = fmaf(st[k].y, by, sum);
            const float* const p = sm + (k * Sh::kRows + in_tile) * PITCH + 8 * part;
            const float4 u = *reinterpret_cast<const float4*>(p), v = *reinterpret_cast<const float4*>(p + 4);
            o[0] = fmaf(u.x, by, o[0]); o[1] = fmaf(u.y, by, o[1]); o[2] = fmaf(u.z, by, o[2]); o[3] = fmaf(u.w, by, o[3]);
            o[4] = fmaf(v.x, by, o[4]); o[5] = fmaf(v.y, by, o[5]); o[6] = fmaf(v.z, by, o[6]); o[7] = fmaf(v.w, by, o[7]);
        }
        const bool some = sum != 0.0f;                                    // a row that sees nothing: zeros (NaN scores: NaN)
        const float inv = some ? __fdiv_rn(1.0f, sum) : 0.0f;
        const int qt = P.by_group(row), head = h * G + row - qt * G;
        const int64_t tok = q0 + qt, out_row = tok * P.q_heads + head;
        if (P.splits == 1) {
            const uint32_t r[4] = {pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv), pack_bf16(o[4] * inv, o[5] * inv),
                                   pack_bf16(o[6] * inv, o[7] * inv)};
            st_v4(P.out + tok * P.out_stride + head * DIM + 8 * part, r);
            if (P.lse != nullptr && part == 0) P.lse[out_row] = some ? (top + log2f(sum)) * kLn2 : kNone;
        } else if (P.cluster) {   // over the first group's part, which no other thread reads
            if (part == 0) chunk_lse[in_tile] = some ? top + log2f(sum) : kNone;
            float* const y = sm + in_tile * PITCH + 8 * part;
            *reinterpret_cast<float4*>(y) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
            *reinterpret_cast<float4*>(y + 4) = make_float4(o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv);
        } else {
            const int64_t to = out_row * P.splits + split;
            if (part == 0) P.part_lse[to] = some ? top + log2f(sum) : kNone;
            if (some) {
                float* const y = P.part_out + to * DIM + 8 * part;
                *reinterpret_cast<float4*>(y) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
                *reinterpret_cast<float4*>(y + 4) = make_float4(o[4] * inv, o[5] * inv, o[6] * inv, o[7] * inv);
            }
        }
    }
    if (!P.cluster) return;
    // ---- join the chunks: the CTAs of a cluster hold a chunk each, and share out the rows' pieces ----
    cluster_sync();
    const uint32_t parts_at = base, lse_at = smem_u32(chunk_lse);
    for (int item = threadIdx.x + split * kWarps * 32; item < Sh::kRows * OUT; item += P.splits * kWarps * 32) {
        const int in_tile = item / OUT, part = item % OUT, row = row0 + in_tile;
        if (row >= rows) break;
        float lse[8], top = kNone, sum = 0.0f, o[8];
        float4 u[8], v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            lse[k] = kNone;
            u[k] = v[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (k < P.splits) {
                lse[k] = __uint_as_float(remote_u32(lse_at + 4 * in_tile, k));
                u[k] = remote_f4(parts_at + (in_tile * PITCH + 8 * part) * 4, k);
                v[k] = remote_f4(parts_at + (in_tile * PITCH + 8 * part) * 4 + 16, k);
            }
            top = fmaxf(top, lse[k]);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const float by = lse[k] == kNone ? 0.0f : ex2(lse[k] - top);
            sum += by;
            o[0] = fmaf(u[k].x, by, o[0]); o[1] = fmaf(u[k].y, by, o[1]); o[2] = fmaf(u[k].z, by, o[2]); o[3] = fmaf(u[k].w, by, o[3]);
            o[4] = fmaf(v[k].x, by, o[4]); o[5] = fmaf(v[k].y, by, o[5]); o[6] = fmaf(v[k].z, by, o[6]); o[7] = fmaf(v[k].w, by, o[7]);
        }
        const bool some = sum != 0.0f;
        const float inv = some ? __fdiv_rn(1.0f, sum) : 0.0f;
        const int qt = P.by_group(row), head = h * G + row - qt * G;
        const int64_t tok = q0 + qt;
        const uint32_t r[4] = {pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv), pack_bf16(o[4] * inv, o[5] * inv),
                               pack_bf16(o[6] * inv, o[7] * inv)};
        st_v4(P.out + tok * P.out_stride + head * DIM + 8 * part, r);
        if (P.lse != nullptr && part == 0) P.lse[tok * P.q_heads + head] = some ? (top + log2f(sum)) * kLn2 : kNone;
    }
    cluster_sync();   // nobody leaves while its shared memory is read
}

// joins the chunks of each row.  A CTA takes a row: each of its eight warps adds every eighth chunk, eight at a time in flight, and
// the warps' sums are added in order.
constexpr int kJoinWarps = 8;
template <int DIM>
__global__ void __launch_bounds__(kJoinWarps * 32) attn_join_kernel(const AttnParams P)
{
    constexpr int E = DIM / 32;   // dimensions of a thread
    __shared__ float sums[kJoinWarps][DIM + 1];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t row = blockIdx.x, tok = blockIdx.x / (uint32_t)P.q_heads;
    const int first = __ldg(P.cu_q), end = __ldg(P.cu_q + P.seqs);
    const float* const part = P.part_lse + row * P.splits;
    // a warp's chunks, eight at a time, asked for before anything is known about them
    float li[8], v[8][E];
    auto ask = [&](int from) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int i = from + kJoinWarps * k + warp;
            li[k] = -INFINITY;
            if (i < P.splits) {
                li[k] = part[i];
                const float* const p = P.part_out + (row * P.splits + i) * DIM + lane * E;
                if constexpr (E == 4) *reinterpret_cast<float4*>(v[k]) = *reinterpret_cast<const float4*>(p);
                else *reinterpret_cast<float2*>(v[k]) = *reinterpret_cast<const float2*>(p);
            }
        }
    };
    ask(0);
    float top = -INFINITY;
    for (int i = lane; i < P.splits; i += 32) top = fmaxf(top, part[i]);
    if (tok >= end || tok < first) return;   // rows of no sequence are left as they were
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    float sum = 0.0f, acc[E] = {};
    for (int from = 0; from < P.splits; from += 8 * kJoinWarps) {
        if (from > 0) ask(from);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (li[k] == -INFINITY) continue;   // an empty chunk wrote no row
            const float f = ex2(li[k] - top);
            sum += f;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = fmaf(v[k][e], f, acc[e]);
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sums[warp][lane * E + e] = acc[e];
    if (lane == 0) sums[warp][DIM] = sum;
    __syncthreads();
    float all = 0.0f;
#pragma unroll
    for (int k = 0; k < kJoinWarps; ++k) all += sums[k][DIM];
    const bool none = all == 0.0f;
    const float inv = none ? 0.0f : __fdiv_rn(1.0f, all);
    if (threadIdx.x < DIM / 2) {
        float a = 0.0f, b = 0.0f;
#pragma unroll
        for (int k = 0; k < kJoinWarps; ++k) {
            a += sums[k][2 * threadIdx.x];
            b += sums[k][2 * threadIdx.x + 1];
        }
        reinterpret_cast<uint32_t*>(P.out + tok * P.out_stride + (row - tok * P.q_heads) * DIM)[threadIdx.x] = pack_bf16(a * inv, b * inv);
    }
    if (P.lse != nullptr && threadIdx.x == 0) P.lse[row] = none ? -INFINITY : (top + log2f(all)) * kLn2;
}

// the same for up to eight chunks: a warp takes a row, with all of its loads at once
template <int DIM>
__global__ void __launch_bounds__(kJoinWarps * 32) attn_join_few_kernel(const AttnParams P)
{
    constexpr int E = DIM / 32;
    pdl_prologue();
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kJoinWarps + (threadIdx.x >> 5);
    if (row >= P.n * P.q_heads) return;
    const int64_t tok = (uint32_t)row / (uint32_t)P.q_heads;
    const int first = __ldg(P.cu_q), end = __ldg(P.cu_q + P.seqs);
    float lse[8], v[8][E];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        lse[k] = -INFINITY;
        if (k < P.splits) {
            lse[k] = P.part_lse[row * P.splits + k];
            const float* const p = P.part_out + (row * P.splits + k) * DIM + lane * E;
            if constexpr (E == 4) *reinterpret_cast<float4*>(v[k]) = *reinterpret_cast<const float4*>(p);
            else *reinterpret_cast<float2*>(v[k]) = *reinterpret_cast<const float2*>(p);
        }
    }
    if (tok >= end || tok < first) return;   // rows of no sequence are left as they were
    float top = lse[0], sum = 0.0f, acc[E] = {};
#pragma unroll
    for (int k = 1; k < 8; ++k) top = fmaxf(top, lse[k]);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (lse[k] == -INFINITY) continue;   // an empty chunk wrote no row
        const float f = ex2(lse[k] - top);
        sum += f;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = fmaf(v[k][e], f, acc[e]);
    }
    const bool none = sum == 0.0f;
    const float inv = none ? 0.0f : __fdiv_rn(1.0f, sum);
    uint32_t* const y = reinterpret_cast<uint32_t*>(P.out + tok * P.out_stride + (row - tok * P.q_heads) * DIM + lane * E);
#pragma unroll
    for (int e = 0; e < E; e += 2) y[e / 2] = pack_bf16(acc[e] * inv, acc[e + 1] * inv);
    if (P.lse != nullptr && lane == 0) P.lse[row] = none ? -INFINITY : (top + log2f(sum)) * kLn2;
}

template <class K, class... Args>
cudaError_t launch(K kernel, int64_t ctas, int cluster, int threads, int smem, cudaStream_t stream, const Args&... args)
{
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)cluster, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// the driver's encoder, looked up once per process (nothing of it depends on the device)
EncodeTiled encoder()
{
    static const EncodeTiled fn = [] {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<EncodeTiled>(p);
    }();
    return fn;
}

bool make_map(CUtensorMap* map, const uint8_t* codes, const AttnParams& P, int box_rows)
{
    const EncodeTiled enc = encoder();
    if (enc == nullptr) return false;
    const cuuint64_t dims[3] = {(cuuint64_t)P.dim, (cuuint64_t)P.page, (cuuint64_t)P.num_pages * (cuuint64_t)P.kv_heads};
    const cuuint64_t strides[2] = {(cuuint64_t)P.dim, (cuuint64_t)P.dim * (cuuint64_t)P.page};
    const cuuint32_t box[3] = {(cuuint32_t)P.dim, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
    return enc(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 3, const_cast<uint8_t*>(codes), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               P.dim == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int DIM, int RW, int NQ, int STAGES>
cudaError_t launch_decode(const AttnParams& P, const AttnMaps& M, int64_t ctas, cudaStream_t stream)
{
    return launch(attn_decode_kernel<DIM, RW, NQ, STAGES>, ctas, P.cluster ? P.splits : 1, kWarps * 32, DecodeShape<DIM, RW, NQ, STAGES>::kSmem, stream, P, M);
}
cudaError_t launch_rows(const AttnParams& P, const AttnMaps& M, const AttnPlan& a, cudaStream_t stream)
{
    if (P.dim == 128)
        return a.row_eights == 1 ? launch_decode<128, 1, 1, 2>(P, M, a.ctas, stream)
             : a.row_warps == 1  ? launch_decode<128, 1, 2, 2>(P, M, a.ctas, stream)
             : a.row_warps == 2  ? launch_decode<128, 2, 2, 3>(P, M, a.ctas, stream) : launch_decode<128, 4, 2, 4>(P, M, a.ctas, stream);
    return a.row_eights == 1 ? launch_decode<64, 1, 1, 3>(P, M, a.ctas, stream)
         : a.row_eights == 2 ? launch_decode<64, 1, 2, 3>(P, M, a.ctas, stream)
         : a.row_warps == 1  ? launch_decode<64, 1, 4, 3>(P, M, a.ctas, stream) : launch_decode<64, 2, 4, 3>(P, M, a.ctas, stream);
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

}  // namespace

// How the keys are shared out: from sizes alone, so that the workspace can be asked for ahead of the call.
namespace {

// wide: heads of 64, 17 to 64 rows: 32 rows a warp (two warps where there are more), else 16 and more CTAs
AttnPlan plan_rows(int64_t n, int64_t seqs, int64_t max_q, int64_t max_len, int64_t window, int q_heads, int kv_heads, int dim, bool wide)
{
    AttnPlan a{};
    const int64_t rows = max_q * (q_heads / kv_heads);
    a.prompt = rows > kPromptRows;
    // a warp holds the output of up to 16 rows of 128 or 32 of 64; more rows are shared out among the CTA's warps
    a.row_eights = rows <= 8 ? 1 : rows <= 16 || dim == 128 || !wide ? 2 : 4;
    a.row_warps = dim == 64 && a.row_eights == 2 ? 1 : (int)(rows <= 8 * a.row_eights ? 1 : rows <= 16 * a.row_eights ? 2 : 4);
    const int64_t tile_rows = a.prompt ? 256 : 8 * a.row_eights * a.row_warps;
    a.row_tiles = ceil_div(rows, tile_rows);
    const int64_t units = seqs * kv_heads * a.row_tiles, tile = a.prompt ? 128 : kTile;
    const int64_t step = a.prompt ? 128 : kTile * (kWarps / a.row_warps);   // keys that a CTA works on at a time
    // Chunks: as many as the CTAs that are resident at a time leave room for; four rounds of them where sequences may differ in
    // length (64 sequences of 2048 ... 8192 keys: one round 152 us, four 135 us).  A chunk is at least eight steps long, so that a
    // CTA's start and the join are worth it (64 sequences of up to 2000 keys: 37 us, five steps 40), or five where half of the places
    // would stay empty (16 sequences: eight 20 us, five 16, 14 with the join as it is now), less only where most SMs would be idle.
    const int64_t resident = (int64_t)kSMs * (a.prompt ? 1 : decode_ctas(dim, a.row_eights));
    int64_t splits = seqs > 1 && !a.prompt ? ceil_div(4 * resident, units) : resident / units;
    // keys that the rows of a tile can see between them
    const int64_t tokens = ceil_div(tile_rows, q_heads / kv_heads) + 1;
    const int64_t span = window > 0 && window + tokens + tile < max_len ? window + tokens + tile : max_len;
    const int64_t least = !a.prompt && 2 * units < resident ? 5 : 8;
    auto most = [&](int64_t keys) {
        const int64_t by_least = ceil_div(keys, least * step), idle = ceil_div(kSMs / 2, units), by_one = ceil_div(keys, step);
        return by_least >= idle ? by_least : by_one < idle ? by_one : idle;
    };
    const int64_t bound = splits < most(max_len) ? splits : most(max_len);   // for the workspace: whatever the window
    a.workspace = bound > 1 ? (size_t)n * q_heads * bound * (dim + 1) * 4 : 0;
    if (splits > most(span)) splits = most(span);
    if (splits < 1) splits = 1;
    a.chunk = ceil_div(ceil_div(span, splits), step) * step;
    if (a.chunk < step) a.chunk = step;
    a.splits = ceil_div(span, a.chunk);
    if (a.splits < 1) a.splits = 1;
    a.ctas = units * a.splits;
    // Up to eight chunks, all of them resident at a time, are joined by the CTAs themselves as a cluster, without a second launch (one
    // sequence of 1000 keys: 6.6 -> 5.8 us; 32 of four drafted tokens and a window of 1024: 25.9 -> 19.1).  Where CTAs queue for
    // places a cluster would hold its places until its longest chunk is done.
    a.cluster = !a.prompt && a.splits > 1 && a.splits <= 8 && a.ctas <= resident;
    // The units of a prompt's last round, if they would keep half of the SMs or fewer busy, are halved to a row tile each (a half takes
    // about two thirds of a unit's time; 512 units of 8192 keys: 450 -> 437 us).
    a.whole_units = a.ctas;
    if (a.prompt && a.splits == 1 && seqs == 1 && units > kSMs && units % kSMs <= kSMs / 2) {
        a.whole_units = units / kSMs * kSMs;
        a.ctas = 2 * units - a.whole_units;
    }
    return a;
}

}  // namespace

AttnPlan plan_attention(int64_t n, int64_t seqs, int64_t max_q, int64_t max_len, int64_t window, int q_heads, int kv_heads, int dim)
{
    if (max_q > n) max_q = n;
    AttnPlan a = plan_rows(n, seqs, max_q, max_len, window, q_heads, kv_heads, dim, true);
    if (a.prompt || a.row_eights != 4) return a;
    // 32 rows a warp save conversions, 16 hide latency better: taken unless a few chunks of all sequences fit side by side
    // (32 sequences of four drafted tokens, window 1024: 32 rows 19 us, 16 rows 29; 64 sequences of 4100 keys: 83 and 79; 16 of
    // 8000, eight tokens: 75 and 66).  The workspace is that of either, whatever the window.
    AttnPlan b = plan_rows(n, seqs, max_q, max_len, window, q_heads, kv_heads, dim, false);
    a.workspace = b.workspace = a.workspace > b.workspace ? a.workspace : b.workspace;
    return a.cluster ? a : b;
}

cudaError_t launch_attention(AttnParams P, const AttnPlan& a, void* workspace, cudaStream_t stream)
{
    P.splits = (int)a.splits;
    P.chunk = a.chunk;
    P.row_tiles = (int)a.row_tiles;
    P.whole_units = (uint32_t)a.whole_units;
    P.cluster = a.cluster;
    P.part_out = static_cast<float*>(workspace);
    P.part_lse = a.splits > 1 ? P.part_out + P.n * P.q_heads * a.splits * P.dim : nullptr;
    AttnMaps M;
    const int tile = a.prompt ? 128 : kTile, box = P.page < tile ? P.page : tile;
    if (!make_map(&M.k, P.k_codes, P, box) || !make_map(&M.v, P.v_codes, P, box)) return cudaErrorInvalidValue;
    cudaError_t e;
    if (a.prompt)
        e = launch_prompt(P, M, a.ctas, stream);
    else
        e = launch_rows(P, M, a, stream);
    if (e != cudaSuccess || a.splits == 1 || a.cluster) return e;
    const int64_t rows = P.n * P.q_heads;
    if (a.splits <= 8)
        return P.dim == 128 ? launch(attn_join_few_kernel<128>, ceil_div(rows, kJoinWarps), 1, kJoinWarps * 32, 0, stream, P)
                            : launch(attn_join_few_kernel<64>, ceil_div(rows, kJoinWarps), 1, kJoinWarps * 32, 0, stream, P);
    return P.dim == 128 ? launch(attn_join_kernel<128>, rows, 1, kJoinWarps * 32, 0, stream, P)
                        : launch(attn_join_kernel<64>, rows, 1, kJoinWarps * 32, 0, stream, P);
}

cudaError_t read_attn_counters(unsigned int* timeouts, unsigned int* bad)
{
    unsigned int more_timeouts = 0, more_bad = 0;
    cudaError_t e = cudaMemcpyFromSymbol(timeouts, g_attn_timeouts, sizeof(unsigned int));
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(bad, g_attn_bad, sizeof(unsigned int));
    if (e == cudaSuccess) e = read_prompt_counters(&more_timeouts, &more_bad);
    *timeouts += more_timeouts;
    *bad += more_bad;
    return e;
}
cudaError_t reset_attn_timeouts()
{
    const unsigned int zero = 0;
    const cudaError_t e = cudaMemcpyToSymbol(g_attn_timeouts, &zero, sizeof(unsigned int));
    return e != cudaSuccess ? e : reset_prompt_counters(true);
}
cudaError_t reset_attn_bad()
{
    const unsigned int zero = 0;
    const cudaError_t e = cudaMemcpyToSymbol(g_attn_bad, &zero, sizeof(unsigned int));
    return e != cudaSuccess ? e : reset_prompt_counters(false);
}

}  // namespace mxn
