// Summed attention weights of the keys for many query rows (prompts): the scores on the 5th-generation tensor cores.
//
//   w_t = earlier_t + sum over rows i of exp(scale q_i . k_t - lse_i),   k_t = 2^(sk - 127) * code
//
// A CTA takes 256 keys of a sequence and head, in two tiles of 128, and walks over the query rows that see them in tiles of up to 128
// (whole tokens of the query heads that share the key head).  Keys are the rows of the products and queries their columns: a thread looks
// after one key, adds its row of scores up in registers, and no sum crosses threads until the end.  The codes become bf16 (exact) once and stay in tensor
// memory as the first operand; the queries come as they are (bf16), by the tensor copy engine, so that every product is exact; the sums of a score are binary32.
// A key enters with most of its scale (a power of two): a product's sum then lies within binary32's range wherever the score does, also where very large
// queries stand over very small keys or the other way round.
// Roles, by warp:
//   0-15   keys to tensor memory; then exponentials and sums, two warpgroups for a product
//   16     copies of query tiles
//   17     issues the products of (query tile, key tile) after (query tile, key tile), into three buffers of tensor memory in turn
//   18     -lse in powers of two for the columns of a query tile
// A cluster of CTAs shares out the query tiles of the same keys where there are too few key tiles for the SMs; their sums are added in a fixed order through
// each other's shared memory.
//
// Bound: at head size 128 a product of 128 keys and 128 rows takes 512 cycles of the tensor cores, its 16384 exponentials 1024 of the special
// function units; three pairs of exponentials in 16 are computed on the multipliers instead.  4096 queries over 8192 keys, 32 query and 8 key heads
// of 128: 255 us, 0.49 of a large library product's measured rate, the special function units busy for two thirds of the time, issue slots for 53 %.
// Eight prompts of up to 1000 queries over up to 1500 keys, 32 and 4 heads of 64: 56 us, of which some 10 are starts and ends of CTAs.
// What mattered (4096 queries): products announced by number and two warpgroups for a product, 64 columns each, instead of whole products in turn
// (280 us); the products that a mask touches in a loop of their own with loads of their own (280 -> 263);
// 32 columns in registers at a time (-> 259).  What did not: six buffers of 64 columns (305: the products are issued one
// every 50 cycles), the next product's columns loaded ahead (276-303), more exponentials on the multipliers (five in 16: 262, seven: 287, in part
// because its constants find no room in registers), three warpgroups for a product of 96 columns (286-302), eight or one CTA for a key tile (340, 328).
// The copies of queries cost nothing (the same time without them).
// Every wait is bounded; see mxn_device_timeouts.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include "mxn_attn.cuh"
#include "mxn_tc.cuh"

namespace mxn {

namespace {

constexpr int kTile = 128, kHalf = 64, kKeys = 256, kThreads = 608, kBuffers = 3, kGroups = 4, kFull = 4, kSlots = 8;
constexpr int kCopies = 16, kProducts = 17, kRowSums = 18;   // warps
constexpr float kLog2e = 1.4426950408889634f;
static_assert(kFull > kBuffers && kFull % 2 == 0);
constexpr int kByMultipliers = 3;   // of 16 pairs of exponentials
// A weight is at most about 1 and a sum of them at most about the number of rows, so a sum that is not below this holds a NaN that went through the
// polynomial.  (A NaN looked for among the exponents themselves took a register and 6 % of the prompts' time.)
constexpr float kMost = 1.70141183e38f;   // 2^127

__device__ unsigned int g_many_timeouts = 0;
__device__ unsigned int g_many_bad = 0;

template <int DIM>
struct ManyShape {
    static constexpr int kStages = DIM == 128 ? 5 : 8;
    static constexpr int kStage = kTile * DIM * 2;
    static constexpr int kSmem = kStages * kStage + 1024;
};

enum { kNan = 1, kUnseeing = 2 };
struct alignas(16) Columns {
    float lse[kTile];     // -lse in powers of two; -infinity for columns without a row
    int special;          // kNan: a NaN is among them; kUnseeing: a row that saw nothing
};

__device__ __forceinline__ void tma_load_queries(uint32_t dst, const CUtensorMap* map, int x, int head, int token, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(map), "r"(x), "r"(head), "r"(token), "r"(bar) : "memory");
}
// two E4M3 codes times a power of two -> two bf16
__device__ __forceinline__ uint32_t bf16_of_codes(uint32_t two, float power)
{
    const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xFFFFu), __NV_E4M3);
    const float2 f = __half22float2(__half2(h));
    const __nv_bfloat162 v = __floats2bfloat162_rn(f.x * power, f.y * power);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// 2^u of two numbers below 2^21 on the multipliers: the polynomial of the prompt attention (mxn_prompt.cu), whose relative error is 1.7e-7 with the
// roundings.  From u = -127 down it is exactly 0 (n = -127 takes the whole exponent of p = 1), so that what gives nothing adds nothing; between
// -127 and -126 it is off by up to 2^-127.  A NaN becomes a NaN or, by the exponent that is added to its bits, a number of 2^127 or more (see kMost).
__device__ __forceinline__ float2 ex2_fma(float2 u)
{
    const float2 v = make_float2(max_nan(u.x, -127.0f), max_nan(u.y, -127.0f)), t = __fadd2_rn(v, f2(12582912.0f));   // 1.5 * 2^23
    const float2 n = __fadd2_rn(t, f2(-12582912.0f)), f = __fadd2_rn(v, make_float2(-n.x, -n.y));
    float2 p = f2(0.00132647273f);
    p = __ffma2_rn(p, f, f2(0.00967151299f));
    p = __ffma2_rn(p, f, f2(0.0555073358f));
    p = __ffma2_rn(p, f, f2(0.240222424f));
    p = __ffma2_rn(p, f, f2(0.693147004f));
    p = __ffma2_rn(p, f, f2(1.0f));
    return make_float2(__uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)),
                       __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

template <int DIM>
__global__ void __launch_bounds__(kThreads, 1) key_weights_many_kernel(const WeightsParams W, const __grid_constant__ CUtensorMap map)
{
    using Sh = ManyShape<DIM>;
    constexpr int ST = Sh::kStages;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * ST + 2 * kSlots + kFull + kBuffers + 1];
    __shared__ Columns columns[kSlots];
    __shared__ float parts[kGroups][kTile], total[kKeys];
    __shared__ uint32_t tmem_at;
    __shared__ int dead_flag;

    pdl_prologue();
    const AttnParams& P = W.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t b = blockIdx.x;
    const int rank = (int)(b % (uint32_t)W.ranks);
    b /= (uint32_t)W.ranks;
    const int h = (int)(b % (uint32_t)P.kv_heads);
    b /= (uint32_t)P.kv_heads;
    const int seq = (int)(b % (uint32_t)P.seqs), k0 = (int)(b / (uint32_t)P.seqs) * kKeys;   // the keys that most rows see first
    const AttnSequence S = attn_sequence(P, seq);
    if (k0 >= S.len) return;   // (all CTAs of the cluster)
    const int k1 = min(S.len, k0 + kKeys), ms = k1 - k0 > kTile ? 2 : 1;
    const int GB = W.tile_heads, T = W.tile_tokens, parts_of_heads = W.head_parts;
    // tokens that see any of these keys, in blocks of T: [block0, block1)
    const int first_token = P.causal ? (int)min((int64_t)S.nq, max((int64_t)0, (int64_t)k0 - S.shift)) : 0;
    const int end_token = P.window > 0 && k0 >= P.sinks ? (int)max((int64_t)0, min((int64_t)S.nq, (int64_t)k1 - 1 + P.window - S.shift)) : S.nq;
    const int block0 = first_token / T, block1 = max(block0, (end_token + T - 1) / T);
    const int all_tiles = end_token > first_token ? (block1 - block0) * parts_of_heads : 0;
    const int tiles = all_tiles > rank ? (all_tiles - rank + W.ranks - 1) / W.ranks : 0;   // rank, rank + ranks, ...
    struct At {
        int token, part;   // first token of a tile among the sequence's, part of the heads
    };
    auto tile_at = [&](int i) {
        const int j = rank + i * W.ranks, blk = parts_of_heads == 1 ? j : j / parts_of_heads;
        return At{(block0 + blk) * T, j - blk * parts_of_heads};
    };

    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u, bar0 = smem_u32(bars);
    const uint32_t q_full = bar0, q_empty = q_full + 8 * ST, n_full = q_empty + 8 * ST, n_empty = n_full + 8 * kSlots, d_full = n_empty + 8 * kSlots,
                   d_empty = d_full + 8 * kFull, a_full = d_empty + 8 * kBuffers;
    volatile int* const dead = &dead_flag;
    if (threadIdx.x == 0) {
        dead_flag = 0;
        for (int i = 0; i < ST; ++i) {
            mbar_init(q_full + 8 * i, 1);
            mbar_init(q_empty + 8 * i, 1);
        }
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(n_full + 8 * i, 1);
            mbar_init(n_empty + 8 * i, 8 * ms);
        }
        // A product is announced by its number, not by its buffer: a warpgroup skips uses of a buffer, and would take the one before for
        // its own.  Four numbers are more than the buffers, so that none comes round before it has been seen.
        for (int i = 0; i < kFull; ++i) mbar_init(d_full + 8 * i, 1);
        for (int i = 0; i < kBuffers; ++i) mbar_init(d_empty + 8 * i, 8);
        mbar_init(a_full, 8 * ms);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == kProducts) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // rows of the stages behind a tile's last, which no copy writes
    const int rows_of_tile = GB * T;
    if (rows_of_tile < kTile) {
        const int words = (kTile - rows_of_tile) * 8;   // 16-byte pieces of a panel
        for (int i = threadIdx.x; i < ST * (DIM / 64) * words; i += kThreads) {
            const uint32_t at = base + (uint32_t)(i / words) * (kTile * 128) + (uint32_t)rows_of_tile * 128 + (uint32_t)(i % words) * 16;
            asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" :: "r"(at), "r"(0u) : "memory");
        }
        fence_async();
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = tmem_at;
    const uint32_t a_col = tmem, d_col = tmem + DIM;   // [key tile][DIM / 2 columns], [buffer][128]

    if (warp == kCopies) {
        bool ok = true;
        const uint32_t bytes = (uint32_t)rows_of_tile * DIM * 2;
        for (int i = 0; i < tiles; ++i) {
            const int st = i % ST;
            if (i >= ST) ok = wait(q_empty + 8 * st, (uint32_t)(i / ST - 1) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            if (lane == 0) {
                const At t = tile_at(i);
                mbar_expect_tx(q_full + 8 * st, bytes);
#pragma unroll
                for (int p = 0; p < DIM / 64; ++p)
                    tma_load_queries(base + st * Sh::kStage + p * kTile * 128, &map, 64 * p, h * P.group + t.part * GB, S.q0 + t.token, q_full + 8 * st);
            }
            __syncwarp();
        }
    } else if (warp == kProducts) {
        const bool one = elect_one();
        bool ok = tiles == 0 || wait(a_full, 0, dead);
        tc_after();
        const uint64_t q_base = operand(base, 1024, 16, 2);
        uint32_t st = 0, st_par = 0, buf = 0, buf_par = 1, number = 0;   // (the buffers' first use waits for nothing)
        for (int i = 0; ok && i < tiles; ++i) {
            ok = wait(q_full + 8 * st, st_par, dead);
            const uint64_t q_desc = q_base + (uint64_t)((st * Sh::kStage) >> 4);
            for (int m = 0; ok && m < ms; ++m) {
                ok = wait(d_empty + 8 * buf, buf_par, dead);
                if (!ok) break;
                tc_after();
                if (one) {
#pragma unroll
                    for (int s = 0; s < DIM / 16; ++s)   // 16 dimensions a step: 8 columns of keys, 32 bytes of the queries' rows
                        mma_values(d_col + buf * kTile, a_col + m * (DIM / 2) + 8 * s, q_desc + (uint64_t)(((s / 4) * kTile * 128 + (s % 4) * 32) >> 4),
                                   idesc_bf16(kTile), s != 0);
                    mma_commit(d_full + 8 * number);
                }
                number = (number + 1) % kFull;
                if (++buf == kBuffers) {
                    buf = 0;
                    buf_par ^= 1u;
                }
            }
            if (ok && one) mma_commit(q_empty + 8 * st);
            if (++st == ST) {
                st = 0;
                st_par ^= 1u;
            }
        }
        if (!ok) {   // what has been issued ends before the tensor memory is given up
            if (one) mma_commit(q_empty);
            (void)mbar_wait_bounded(q_empty, 0, 1u << 14);
            (void)mbar_wait_bounded(q_empty, 1, 1u << 14);
        }
    } else if (warp == kRowSums) {
        // this lane's columns lane, lane + 32, ...: token and head within a tile
        int tok[4], head[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int col = lane + 32 * e;
            tok[e] = col < rows_of_tile ? col / GB : 1 << 30;
            head[e] = col % GB;
        }
        auto load = [&](int i, float (&v)[4]) {
            const At t = tile_at(i);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const bool live = i < tiles && tok[e] < S.nq - t.token && t.part * GB + head[e] < P.group;
                v[e] = live ? __ldg(W.lse + (int64_t)(S.q0 + t.token + tok[e]) * P.q_heads + h * P.group + t.part * GB + head[e]) : INFINITY;
            }
        };
        float v[4], next[4];
        load(0, v);
        for (int i = 0; i < tiles; ++i) {
            load(i + 1, next);
            const int slot = i % kSlots;
            const bool ok = i < kSlots || wait(n_empty + 8 * slot, (uint32_t)(i / kSlots - 1) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            bool nan = false, unseeing = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                nan = nan || v[e] != v[e];
                unseeing = unseeing || v[e] == -INFINITY;
                columns[slot].lse[lane + 32 * e] = v[e] == -INFINITY ? -INFINITY : -v[e] * kLog2e;   // (a row that saw nothing gives nothing)
                v[e] = next[e];
            }
            const int special = (__any_sync(0xFFFFFFFFu, nan) ? kNan : 0) | (__any_sync(0xFFFFFFFFu, unseeing) ? kUnseeing : 0);
            __syncwarp();
            if (lane == 0) {
                columns[slot].special = special;
                mbar_arrive(n_full + 8 * slot);
            }
            __syncwarp();
        }
    } else {
        const int wg = warp >> 2, m = ms == 2 ? wg & 1 : 0, r = threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int key = k0 + m * kTile + r;
        const int32_t page = key < k1 ? __ldg(P.page_table + (int64_t)seq * P.max_pages + (key >> P.page_shift)) : -1;
        const bool real = (uint32_t)page < (uint32_t)P.num_pages;
        const int64_t tile = (int64_t)page * P.kv_heads + h;
        const int in_page = key & (P.page - 1);
        // The key's scale is 2^(byte - 127).  2^in of it enters the operand: 2^16 below the scale, so that a sum has room above the largest score, but no
        // lower than 2^-110, so that the smallest code (2^-9) stays a normal bf16; the largest (448) is one up to byte 254.  2^(byte - 127 - in) is left.
        const int byte = real ? (int)__ldg(P.k_scales + (tile << (P.page_shift - P.block_shift)) + (in_page >> P.block_shift)) : 0;
        const int in = max(byte - 127 - 16, -110);
        auto pow2 = [](int e) { return __uint_as_float((uint32_t)(e + 127) << 23); };
        // ---- keys to tensor memory: half of a row's dimensions a thread (with one key tile the other warpgroups rest) ----
        if (ms == 2 || !(wg & 1)) {
            const int half = wg >> 1;
            uint32_t w[DIM / 4];
#pragma unroll
            for (int i = 0; i < DIM / 32; ++i) {
                uint4 u = make_uint4(0, 0, 0, 0);
                if (real) u = __ldg(reinterpret_cast<const uint4*>(P.k_codes + ((tile << P.page_shift) + in_page) * DIM + half * (DIM / 2)) + i);
                const uint32_t c[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    w[8 * i + 2 * e] = bf16_of_codes(c[e], pow2(in));
                    w[8 * i + 2 * e + 1] = bf16_of_codes(c[e] >> 16, pow2(in));
                }
            }
            const uint32_t at = a_col + m * (DIM / 2) + half * (DIM / 4) + lanes;
            if constexpr (DIM == 128) tm_store32(at, w);
            else tm_store16(at, w);
            tm_store_wait();
            tc_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(a_full);
        }
        if (rank == 0 && wg < ms && __any_sync(0xFFFFFFFFu, key < k1 && !real) && lane == 0) atomicAdd(&g_many_bad, 1u);
        const float scale = real ? P.scale * kLog2e * pow2(byte - 127 - in) : 0.0f;
        const float2 f = f2(scale);
        float2 sum[2] = {f2(0.0f), f2(0.0f)};
        // A product is shared by two warpgroups, half of its columns each: with two key tiles each pair has its own, with one they take turns
        const int items = tiles * ms, col0 = (ms == 2 ? wg >> 1 : wg & 1) * kHalf;
        // First tokens of the query tiles all of whose columns see all of this warp's keys: [see0, see1].  (What a key without a page gets is not used.)
        const int64_t place = (int64_t)key - S.shift;   // of the key, among the call's tokens
        int see0 = P.causal && real ? (int)max(place, (int64_t)0) : 0, see1 = S.nq - T;
        if (P.window > 0 && key >= P.sinks && real) see1 = (int)max((int64_t)-1, min((int64_t)see1, place + P.window - T));
        see0 = __reduce_max_sync(0xFFFFFFFFu, see0);
        see1 = P.group % GB == 0 ? __reduce_min_sync(0xFFFFFFFFu, see1) : -1;
        bool ok = true;
        int buf = ms == 2 ? wg & 1 : wg >> 1;
        for (int item = buf; item < items; item += 2) {
            const int i = ms == 2 ? item >> 1 : item, slot = i % kSlots;
            ok = wait(n_full + 8 * slot, (uint32_t)(i / kSlots) & 1u, dead) && wait(d_full + 8 * (item % kFull), (uint32_t)(item / kFull) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            tc_after();
            const uint32_t at = d_col + buf * kTile + col0 + lanes, free_bar = d_empty + 8 * buf;
            buf = buf > 0 ? buf - 1 : 2;   // two on, of three
            const Columns& C = columns[slot];
            const At t = tile_at(i);
            const float* const cl = C.lse + col0;
            float2 part[2] = {f2(0.0f), f2(0.0f)};
            if (t.token >= see0 && t.token <= see1 && C.special == 0) {
                // 32 columns at a time: with 64 in registers the polynomial's constants found no room (263 us, so 259)
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t y[32];
                    tm_load(y, at + 32 * c);
                    if (c == 1) {   // the buffer is free again before the rest of the arithmetic
                        tc_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(free_bar);
                    }
#pragma unroll
                    for (int e = 0; e < 16; e += 2) {
                        const float4 n = *reinterpret_cast<const float4*>(cl + 32 * c + 2 * e);
                        const float2 u = __ffma2_rn(make_float2(__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])), f, make_float2(n.x, n.y));
                        const float2 v = __ffma2_rn(make_float2(__uint_as_float(y[2 * e + 2]), __uint_as_float(y[2 * e + 3])), f, make_float2(n.z, n.w));
                        // spread over the 16 pairs, so that both kinds run side by side
                        const bool mu = (e * kByMultipliers) / 16 != ((e + 1) * kByMultipliers) / 16;
                        const bool mv = ((e + 1) * kByMultipliers) / 16 != ((e + 2) * kByMultipliers) / 16;
                        part[0] = __fadd2_rn(part[0], mu ? ex2_fma(u) : make_float2(ex2(u.x), ex2(u.y)));
                        part[1] = __fadd2_rn(part[1], mv ? ex2_fma(v) : make_float2(ex2(v.x), ex2(v.y)));
                    }
                }
            } else {
                // Columns [lo, hi) of these see this key.  In a short loop with loads of its own: as a branch over the common path's registers it cost
                // that path 17 of 280 us.
                const int valid = min(T, S.nq - t.token) * min(GB, P.group - t.part * GB);
                const int64_t ahead = place - t.token;
                const int from = P.causal ? (int)max((int64_t)0, min((int64_t)T, ahead)) : 0;
                const int to = P.window == 0 || key < P.sinks ? T : (int)max((int64_t)0, min((int64_t)T, ahead + P.window));
                const int lo = max(from * GB - col0, 0), hi = min((real ? min(to * GB, valid) : 0) - col0, kHalf);
                if (__any_sync(0xFFFFFFFFu, lo < hi)) {
                    const bool unseeing = C.special & kUnseeing;
#pragma unroll 1
                    for (int c = 0; c < kHalf; c += 16) {
                        uint32_t z[16];
                        tm_load16(z, at + c);
                        uint32_t in = ((1u << min(max(hi - c, 0), 16)) - 1u) & (0xFFFFFFFFu << min(max(lo - c, 0), 16));   // bit: the column counts
                        if (unseeing) {   // a row that saw nothing gives nothing, also where its score is a NaN
#pragma unroll 1
                            for (int e = 0; e < 16; ++e) in &= ~((cl[c + e] == -INFINITY ? 1u : 0u) << e);
                        }
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float p = ex2(fmaf(__uint_as_float(z[e]), scale, cl[c + e]));
                            part[e & 1].x += (in >> e) & 1u ? p : 0.0f;
                        }
                    }
                }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(free_bar);
            }
            sum[0] = __fadd2_rn(sum[0], part[0]);
            sum[1] = __fadd2_rn(sum[1], part[1]);
            __syncwarp();
            if (lane == 0) mbar_arrive(n_empty + 8 * slot);
        }
        const float2 both = __fadd2_rn(sum[0], sum[1]);
        const float all = both.x + both.y;
        parts[wg][r] = all < kMost ? all : __uint_as_float(0x7FC00000u);
        tc_before();
    }
    __syncthreads();
    if (threadIdx.x == 0 && dead_flag) {
        // a wait ran out: the copies in flight get a second, shorter wait before the shared memory is given up
        atomicAdd(&g_many_timeouts, 1u);
        for (int i = 0; i < ST; ++i) {
            (void)mbar_wait_bounded(q_full + 8 * i, 0, 1u << 14);
            (void)mbar_wait_bounded(q_full + 8 * i, 1, 1u << 14);
        }
    }
    if (threadIdx.x < kKeys) {
        const int m = threadIdx.x >> 7, r = threadIdx.x & 127;
        total[threadIdx.x] = ms == 2 ? parts[m][r] + parts[m + 2][r] : m == 0 ? (parts[0][r] + parts[1][r]) + (parts[2][r] + parts[3][r]) : 0.0f;
    }
    if (W.ranks > 1) cluster_sync();
    else __syncthreads();
    // the cluster's CTAs share out the keys
    const int share = kKeys / W.ranks, at = rank * share + (int)threadIdx.x, key = k0 + at;
    if ((int)threadIdx.x < share && key < k1) {
        float w = 0.0f;
        if (W.ranks > 1)
            for (int i = 0; i < W.ranks; ++i) w += __uint_as_float(remote_u32(smem_u32(total + at), i));
        else
            w = total[at];
        const int page = __ldg(P.page_table + (int64_t)seq * P.max_pages + (key >> P.page_shift));
        if ((uint32_t)page < (uint32_t)P.num_pages) {
            const int64_t to = (((int64_t)page * P.kv_heads + h) << P.page_shift) + (key & (P.page - 1));
            const bool old = W.earlier != nullptr && (S.nq == 0 || key < S.shift);
            W.sums[to] = (old ? W.earlier[to] : 0.0f) + w;
        }
    }
    if (W.ranks > 1) cluster_sync();   // nobody leaves while its shared memory is read
    if (warp == kProducts) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

template <int DIM>
cudaError_t launch_dim(const WeightsParams& W, const CUtensorMap& map, int64_t ctas, cudaStream_t stream)
{
    const int smem = ManyShape<DIM>::kSmem;
    const cudaError_t e = cudaFuncSetAttribute(key_weights_many_kernel<DIM>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {(unsigned)W.ranks, 1, 1};
    cfg.attrs = attr;
    cfg.numAttrs = W.ranks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, key_weights_many_kernel<DIM>, W, map);
}

}  // namespace

cudaError_t launch_weights_many(const WeightsParams& W, int64_t ctas, cudaStream_t stream)
{
    CUtensorMap map;
    if (!make_query_map(&map, W.a, W.tile_heads, W.tile_tokens)) return cudaErrorInvalidValue;
    return W.a.dim == 128 ? launch_dim<128>(W, map, ctas, stream) : launch_dim<64>(W, map, ctas, stream);
}

cudaError_t read_weights_many_counters(unsigned int* timeouts, unsigned int* bad)
{
    const cudaError_t e = cudaMemcpyFromSymbol(timeouts, g_many_timeouts, sizeof(unsigned int));
    return e != cudaSuccess ? e : cudaMemcpyFromSymbol(bad, g_many_bad, sizeof(unsigned int));
}
cudaError_t reset_weights_many_counters(bool timeouts)
{
    const unsigned int zero = 0;
    return timeouts ? cudaMemcpyToSymbol(g_many_timeouts, &zero, sizeof(unsigned int)) : cudaMemcpyToSymbol(g_many_bad, &zero, sizeof(unsigned int));
}

}  // namespace mxn
