// Which tokens stay in the paged 8-bit cache, and moving them together.
//
// Select: of a sequence's tokens the first `sinks`, the last `recent`, and of those between the largest by weight, equal ones by place, until
// `keep` are chosen; for each key head apart.  A weight's bits, turned so that they order as unsigned numbers, are looked at in three digits
// (11, 11, 10 bits) from the top: a histogram of the digit among what agrees with the digits before gives the next digit of the smallest chosen
// weight.  Then every warp writes the places that it chose, in order, behind those of the warps before it.  A sequence and head is shared out
// over a cluster of CTAs, each with a run of tokens whose weights stay in registers; histograms are read across the cluster.
//
// Compact: token kept[i] goes to place first + i.  A warp takes 32 places (64 with blocks of as many) of a head, for keys and values: it reads
// the listed rows and their blocks' scales, finds for each block of places the scale that its largest value asks for (the append's rule: S =
// 2^(ceil(log2 absmax) - 8)), rounds the codes on it (exact unless they become subnormal; as they are where the scale stays) and writes them.
// In place a row must be read before its place is written. Lists rise and places never lie behind their tokens, so only warps of lower places
// read what a warp is to overwrite; a warp says so once it has read, and waits for those (two at most) whose tokens lie in its places.  Work is
// handed out by a ticket in the order of the places, so that whoever is waited for has started, and nobody waits before it has read: every wait
// ends.  (All waits are bounded; see mxn_device_timeouts.)
//
// Measured, 8 heads of 128 in blocks of 16, choice and move to other pages together: 32 sequences of up to 8192 tokens brought to 2048, 66 us
// (the move 50: 0.27 GB, 5.4 TB/s, HBM busy for 55 %: what its warps wait for is loads that follow one another, list, page, then rows and scales;
// with four CTAs an SM in place of five it took 55); one of 131072 brought to 32768, 55 us, of which the choice takes some 25: 64 CTAs, instructions and three trips across the cluster; 16
// CTAs a cluster took twice that.  In place either move takes 1.4 times what it takes to other pages (74 and 53 us by replays).
#include <cuda_fp16.h>

#include "mxn_async.cuh"
#include "mxn_device.cuh"
#include "mxn_internal.h"

namespace mxn {

namespace {

__device__ unsigned int g_keep_timeouts = 0;
__device__ unsigned int g_keep_bad = 0;   // entries, pages or lengths out of range

constexpr int kBins = 2048;
constexpr int kHeld = 4;   // runs of four tokens of a thread that are held in registers; with more all are read again

// Orders as unsigned numbers: -infinity ... -0 = 0 ... infinity; NaN below all.  0 and kSure are no weight's.
constexpr uint32_t kSure = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t ordered(float w)
{
    if (w != w) return 1u;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint32_t warp_sum_u32(uint32_t v) { return __reduce_add_sync(0xFFFFFFFFu, v); }

template <int WARPS>
__global__ void __launch_bounds__(WARPS * 32, WARPS == 16 ? 2 : 1) select_kernel(const SelectParams P, const int cluster)
{
    constexpr int BINS = kBins / (WARPS * 32);   // of a thread: 4 or 2
    __shared__ alignas(16) uint32_t hist[3][kBins];
    __shared__ uint32_t warp_sums[WARPS];
    __shared__ uint32_t found[2];              // the digit, and how many are chosen at it
    __shared__ uint32_t counts[2];             // of this CTA: above the smallest chosen weight, equal to it
    __shared__ uint32_t warp_counts[WARPS][2];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)(blockIdx.x % (uint32_t)cluster);
    const uint32_t unit = blockIdx.x / (uint32_t)cluster;
    const int h = (int)(unit % (uint32_t)P.heads), seq = (int)(unit / (uint32_t)P.heads);
    const int len = max(0, min(__ldg(P.lens + seq), P.max_len));
    int32_t* const out = P.kept + (int64_t)unit * P.keep;
    if (h == 0 && rank == 0 && threadIdx.x == 0) P.new_lens[seq] = min(len, P.keep);
    if (len <= P.keep) {   // everything stays
        for (int64_t i = rank * WARPS * 32 + threadIdx.x; i < P.keep; i += cluster * WARPS * 32) out[i] = i < len ? (int)i : -1;
        return;
    }
    // this warp's tokens: whole groups of 128, four a lane, kHeld groups of them at a time in registers
    const int groups = (len + 127) >> 7, per_warp = (groups + cluster * WARPS - 1) / (cluster * WARPS);
    const int g0 = (int)min((int64_t)groups, (int64_t)(rank * WARPS + warp) * per_warp), g1 = min(groups, g0 + per_warp);
    const bool once = per_warp <= kHeld;   // else the weights are read again for each step
    const int tail = len - P.recent;
    const int32_t* const table = P.page_table + (int64_t)seq * P.max_pages;
    const float* const weights = P.weights + ((int64_t)h << P.page_shift);
    const int page_mask = (1 << P.page_shift) - 1;
    const bool wide = (reinterpret_cast<uintptr_t>(P.weights) & 15u) == 0u;   // (weights are promised to be 4-byte aligned)
    bool bad = false;
    uint32_t k[kHeld][4];   // of tokens 128 (g + x) + 4 lane + j; 0 where there is none, kSure for the first and the last ones
    auto fetch = [&](int g) {   // all pages, then all weights on their way at once.  Four tokens lie in one page.
        int32_t pg[kHeld];
        float4 w[kHeld];
#pragma unroll
        for (int x = 0; x < kHeld; ++x) {
            const int t = (g + x) * 128 + lane * 4;
            pg[x] = g + x < g1 && t < len ? __ldg(table + (t >> P.page_shift)) : -1;
        }
#pragma unroll
        for (int x = 0; x < kHeld; ++x) {
            const int t = (g + x) * 128 + lane * 4;
            w[x] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if ((uint32_t)pg[x] < (uint32_t)P.num_pages) {
                const float* const at = weights + (((int64_t)pg[x] * P.heads) << P.page_shift) + (t & page_mask);
                w[x] = wide ? __ldg(reinterpret_cast<const float4*>(at)) : make_float4(__ldg(at), __ldg(at + 1), __ldg(at + 2), __ldg(at + 3));
            }
        }
#pragma unroll
        for (int x = 0; x < kHeld; ++x) {
            const int t = (g + x) * 128 + lane * 4;
            const bool real = g + x < g1 && t < len, fits = (uint32_t)pg[x] < (uint32_t)P.num_pages;
            bad |= real && !fits;
            const float v[4] = {w[x].x, w[x].y, w[x].z, w[x].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) k[x][j] = fits ? ordered(v[j]) : 1u;
            if (!real || t < P.sinks || t + 4 > tail) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!real || t + j >= len) k[x][j] = 0u;
                    else if (t + j < P.sinks || t + j >= tail) k[x][j] = kSure;
            }
        }
    };
    for (int i = threadIdx.x; i < 3 * kBins; i += WARPS * 32) (&hist[0][0])[i] = 0u;
    if (once) fetch(g0);
    __syncthreads();

    uint32_t prefix = 0u, need = (uint32_t)(P.keep - P.sinks - P.recent);   // of those that agree with the prefix, how many are chosen
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        constexpr int kShift[3] = {21, 10, 0}, kUp[3] = {32, 21, 10};
        for (int g = g0; g < g1; g += kHeld) {
            if (!once) fetch(g);
#pragma unroll
            for (int x = 0; x < kHeld; ++x)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (k[x][j] - 1u < kSure - 1u && (pass == 0 || k[x][j] >> (kUp[pass] & 31) == prefix))
                        atomicAdd(&hist[pass][(k[x][j] >> kShift[pass]) & (pass == 2 ? 1023u : 2047u)], 1u);
        }
        if (cluster > 1) cluster_sync();
        else __syncthreads();
        // thread i: bins BINS i ... from the top, of all CTAs; an inclusive sum from the top over the block
        const int b0 = kBins - BINS * (1 + (int)threadIdx.x);
        uint32_t n[4] = {0u, 0u, 0u, 0u};   // bins b0 ...
        const uint32_t quad = smem_u32(&hist[pass][b0 & ~3]);
#pragma unroll
        for (int r = 0; r < 8; ++r)
            if (r < cluster) {
                const uint4 v = cluster > 1 ? remote_v4(quad, r) : *reinterpret_cast<const uint4*>(&hist[pass][b0 & ~3]);
                if (BINS == 4 || !(b0 & 2)) {
                    n[0] += v.x;
                    n[1] += v.y;
                }
                if (BINS == 4 || (b0 & 2)) {
                    n[BINS - 2] += v.z;
                    n[BINS - 1] += v.w;
                }
            }
        uint32_t mine = 0u;
#pragma unroll
        for (int x = 0; x < BINS; ++x) mine += n[x];
        uint32_t sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) warp_sums[warp] = sum;
        __syncthreads();
        uint32_t before = warp_sum_u32(lane < warp ? warp_sums[lane & (WARPS - 1)] : 0u) + sum - mine;   // (lane < warp < WARPS)
        // the digit at which the count from the top reaches `need` (with need == 0 there is none)
#pragma unroll
        for (int x = BINS - 1; x >= 0; --x) {
            if (before < need && before + n[x] >= need) {
                found[0] = (uint32_t)(b0 + x);
                found[1] = need - before;
            }
            before += n[x];
        }
        __syncthreads();
        if (need > 0u) {
            prefix = (prefix << (pass == 2 ? 10 : 11)) | found[0];
            need = found[1];
        }
    }
    // a token is chosen if its key is above the smallest chosen one, or equal to it and among the first `need` of those
    const uint32_t least = P.keep == P.sinks + P.recent ? kSure - 1u : prefix;
    uint32_t n_above = 0u, n_equal = 0u;
    for (int g = g0; g < g1; g += kHeld) {
        if (!once) fetch(g);
#pragma unroll
        for (int x = 0; x < kHeld; ++x)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                n_above += k[x][j] > least;
                n_equal += k[x][j] == least;
            }
    }
    n_above = warp_sum_u32(n_above);
    n_equal = warp_sum_u32(n_equal);
    if (lane == 0) {
        warp_counts[warp][0] = n_above;
        warp_counts[warp][1] = n_equal;
    }
    __syncthreads();
    // of the warps before this one in the CTA; the CTA's total
    const uint32_t a = lane < WARPS ? warp_counts[lane][0] : 0u, e = lane < WARPS ? warp_counts[lane][1] : 0u;
    uint32_t a_before = warp_sum_u32(lane < warp ? a : 0u), e_before = warp_sum_u32(lane < warp ? e : 0u);
    if (cluster > 1) {
        const uint32_t all_a = warp_sum_u32(a), all_e = warp_sum_u32(e);
        if (threadIdx.x == 0) {
            counts[0] = all_a;
            counts[1] = all_e;
        }
        cluster_sync();
        const uint32_t other_a = lane < rank ? remote_u32(smem_u32(&counts[0]), lane) : 0u, other_e = lane < rank ? remote_u32(smem_u32(&counts[1]), lane) : 0u;
        a_before += warp_sum_u32(other_a);
        e_before += warp_sum_u32(other_e);
    }
    for (int g = g0; g < g1; g += kHeld) {
        if (!once) fetch(g);
#pragma unroll
        for (int x = 0; x < kHeld; ++x) {
            // above in the low half, equal in the high half, of this lane's four and of the lanes before it
            uint32_t mine = 0u;
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += (k[x][j] > least ? 1u : 0u) + (k[x][j] == least ? 0x10000u : 0u);
            uint32_t upto = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, upto, o);
                if (lane >= o) upto += v;
            }
            const uint32_t all = __shfl_sync(0xFFFFFFFFu, upto, 31), front = upto - mine;
            uint32_t a_front = a_before + (front & 0xFFFFu), e_front = e_before + (front >> 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bool is_above = k[x][j] > least, is_equal = k[x][j] == least;
                const uint32_t at = a_front + min(e_front, need);
                if ((is_above || (is_equal && e_front < need)) && at < (uint32_t)P.keep) out[at] = (g + x) * 128 + lane * 4 + j;
                a_front += is_above;
                e_front += is_equal;
            }
            a_before += all & 0xFFFFu;
            e_before += all >> 16;
        }
    }
    if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicAdd(&g_keep_bad, 1u);
    if (cluster > 1) cluster_sync();   // nobody leaves while its shared memory is read
}

// ---- moving ----------------------------------------------------------------------------------------------------------

constexpr int kMoveWarps = 4;

// largest of the low seven bits of 16 code bytes, in each half of the result
__device__ __forceinline__ uint32_t absmax_codes(uint4 w)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t m = 0u;
#pragma unroll
    for (int i = 0; i < 4; ++i) m = __vmaxu2(m, __vmaxu2(u[i] & 0x007F007Fu, (u[i] >> 8) & 0x007F007Fu));
    return max(m & 0xFFFFu, m >> 16);
}
// the same over numbers only
__device__ __noinline__ uint32_t absmax_numbers(uint4 w)
{
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t m = 0u;
    for (int i = 0; i < 16; ++i) {
        const uint32_t b = (u[i >> 2] >> (8 * (i & 3))) & 0x7Fu;
        if (b != 0x7Fu) m = max(m, b);
    }
    return m;
}
// ceil(log2 of an E4M3 magnitude) - 8
__device__ __forceinline__ int asks(uint32_t m)
{
    const int e = (int)(m >> 3), f = (int)(m & 7u);
    return e > 0 ? e - 15 + (f > 0) : f == 1 ? -17 : f == 2 ? -16 : f <= 4 ? -15 : -14;
}
__device__ __forceinline__ uint32_t half2_of(float v)
{
    const __half2 x = __float2half2_rn(v);
    return *reinterpret_cast<const uint32_t*>(&x);
}
// four codes times a power of two (f16 pairs: exact, or so small that the code rounds to zero either way), rounded to E4M3
__device__ __forceinline__ uint32_t rescale(uint32_t w, uint32_t by)
{
    uint32_t y;
    asm("{ .reg .b16 l, h; .reg .b32 p, q;\n\t"
        "mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 p, l; cvt.rn.f16x2.e4m3x2 q, h;\n\t"
        "mul.rn.f16x2 p, p, %2; mul.rn.f16x2 q, q, %2;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 l, p; cvt.rn.satfinite.e4m3x2.f16x2 h, q; mov.b32 %0, {l, h}; }"
        : "=r"(y) : "r"(w), "r"(by));
    return y;
}
__device__ __forceinline__ void scale_by(uint4& x, int d)   // -24 <= d <= 15
{
    const uint32_t by = half2_of(__uint_as_float((uint32_t)(127 + d) << 23));
    x = make_uint4(rescale(x.x, by), rescale(x.y, by), rescale(x.z, by), rescale(x.w, by));
}

// K: places of a lane; a warp takes 32 K of them, at least a block
template <int DIM, bool IN_PLACE, int K>
__global__ void __launch_bounds__(kMoveWarps * 32, K == 1 ? 5 : 3) compact_kernel(const CompactParams P)
{
    constexpr int kPlaces = 32 * K;
    constexpr int L = DIM / 16;          // lanes of a row
    constexpr int R = 32 / L;            // rows of an access
    constexpr int N = kPlaces / R;       // accesses
    constexpr int PER16 = 16 / R;        // accesses of 16 places
    __shared__ uint32_t ticket;
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, sub = lane % L, grp = lane / L;
    uint32_t cta = blockIdx.x;
    if (IN_PLACE) {
        if (threadIdx.x == 0) ticket = atomicAdd(P.work, 1u);
        __syncthreads();
        cta = ticket;
    }
    const int64_t unit = (int64_t)cta * kMoveWarps + warp, lists = (int64_t)P.seqs * P.heads;
    if (unit >= P.units * lists) return;
    const int u = (int)(unit / lists);
    const uint32_t rest = (uint32_t)(unit % lists);
    const int h = (int)(rest % (uint32_t)P.heads), seq = (int)(rest / (uint32_t)P.heads);
    uint32_t* const flags = P.work + 1;   // of the same list: unit u' at u' * lists + (unit % lists)
    const int64_t flag_at = unit - (int64_t)u * lists;

    const int first = P.first != nullptr ? __ldg(P.first + seq) : 0;
    const int len = __ldg(P.lens + seq);
    const int64_t asked = (int64_t)__ldg(P.new_lens + seq) - first;
    bool bad = first < 0 || first > len || asked > P.max_kept;
    if (bad && lane == 0 && u == 0 && h == 0) atomicAdd(&g_keep_bad, 1u);
    if (first < 0 || first > len) return;   // the sequence is left as it is
    const int end = (int)min(first + min(asked, P.max_kept), (int64_t)0x7FFFFFFF - kPlaces);
    const int from = first / kPlaces * kPlaces, base = (int)min((int64_t)from + (int64_t)u * kPlaces, (int64_t)0x7FFFFFFF - kPlaces);
    if (end <= first || base >= end) return;   // (no unit with places waits for one without)
    bad = false;
    const int32_t* const list = P.kept + ((int64_t)seq * P.kept_heads + (P.kept_heads > 1 ? h : 0)) * P.max_kept;
    const int32_t* const table = P.table + (int64_t)seq * P.width;
    const int32_t* const out_table = P.out_table + (int64_t)seq * P.out_width;
    const int page_mask = (1 << P.page_shift) - 1, per_page = P.page_shift - P.block_shift;

    // ---- this lane's K places: where their tokens are (row numbers in the pool, below 2^31; -1: none), where they go ----
    int src[K], dst[K];
    int scale[2][K];   // of keys and values
    float moved_weight[K];
    bool stays[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        moved_weight[k] = 0.0f;
        const int place = base + 32 * k + lane;
        src[k] = dst[k] = -1;
        scale[0][k] = scale[1][k] = 0;
        stays[k] = true;
        if (place >= end) continue;
        bool wrong = false;
        const int64_t out_page_at = place >> P.page_shift;
        const int out_page = out_page_at < P.out_width ? __ldg(out_table + out_page_at) : -1;
        if ((uint32_t)out_page < (uint32_t)P.num_pages)
            dst[k] = ((out_page * P.heads + h) << P.page_shift) + (place & page_mask);
        else
            wrong = true;
        if (place < first) {   // in front of the list, in the same block: stays where it is
            src[k] = dst[k];
        } else {
            const int token = __ldg(list + (place - first));
            const int prev = place > first ? __ldg(list + (place - first - 1)) : -1;
            const int64_t page_at = token >> P.page_shift;
            const bool fits = token >= 0 && token < len && page_at < P.width && !(IN_PLACE && (token < place || token <= prev));
            const int page = fits ? __ldg(table + page_at) : -1;
            if (fits && (uint32_t)page < (uint32_t)P.num_pages) {
                src[k] = ((page * P.heads + h) << P.page_shift) + (token & page_mask);
                stays[k] = src[k] == dst[k];
            } else {
                wrong = true;
            }
        }
        bad |= wrong;
    }
    // a block with an entry out of range is left as it is, and so is one whose tokens all stay where they are
    const int block = 1 << P.block_shift;
    uint32_t touched[K];   // bit: the place is to be written
    {
        uint64_t moves = 0, off = 0, real = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool there = base + 32 * k + lane < end;
            moves |= (uint64_t)__ballot_sync(0xFFFFFFFFu, !stays[k]) << (32 * k);
            off |= (uint64_t)__ballot_sync(0xFFFFFFFFu, there && (src[k] < 0 || dst[k] < 0)) << (32 * k);
            real |= (uint64_t)__ballot_sync(0xFFFFFFFFu, there) << (32 * k);
        }
        auto spread = [&](uint64_t v) -> uint64_t {   // to all places of the blocks that have a bit
            uint64_t y = 0;
#pragma unroll
            for (int o = 0; o < kPlaces; o += 16) {
                const int first = o & ~(block - 1);
                const uint64_t m = (block == 64 ? ~0ull : (1ull << block) - 1) << first;
                if (v & m) y |= m;
            }
            return y;
        };
        const uint64_t w = spread(moves) & ~spread(off) & real;
#pragma unroll
        for (int k = 0; k < K; ++k) touched[k] = (uint32_t)(w >> (32 * k));
    }
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (!(touched[k] >> lane & 1u)) {
            src[k] = -1;
        } else {
            // row / page * (page / block) + block within the page
            const int64_t at = ((int64_t)(src[k] >> P.page_shift) << per_page) + ((src[k] & page_mask) >> P.block_shift);
            scale[0][k] = P.scales[0][at];
            scale[1][k] = P.scales[1][at];
            if (P.weights != nullptr) moved_weight[k] = P.weights[src[k]];
        }
    }
    uint4 x[2][N];
#pragma unroll
    for (int which = 0; which < 2; ++which)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int row = __shfl_sync(0xFFFFFFFFu, src[i * R / 32], (i * R + grp) & 31);
            x[which][i] = make_uint4(0u, 0u, 0u, 0u);
            if (row >= 0) x[which][i] = *reinterpret_cast<const uint4*>(P.codes[which] + (int64_t)row * DIM + 16 * sub);
        }
    bool ok = true;
    if (IN_PLACE) {
        // While the rows are on their way: list entries whose tokens lie in this warp's places [base, base + kPlaces).  They stand in front of its own;
        // the first of them, 32 probes at a time
        int u0 = 0, u1 = -1;   // the warps that read them
        const int mine = max(0, base - first);   // list entries in front of this unit's
        if (mine > 0 && __ldg(list + (mine - 1)) >= base) {
            int at = 0, n = mine;   // the first entry >= base is in [at, at + n)
            while (n > 1) {
                const int step = (n + 31) / 32, probe = at + min(lane * step, n - 1);
                const unsigned less = __ballot_sync(0xFFFFFFFFu, lane * step < n && __ldg(list + probe) < base);
                if (less == 0u) break;   // the first one already is
                const int skip = (31 - __clz(less)) * step + 1;   // behind the last probe below
                at += skip;
                n = min(step, n - skip);
            }
            // rising entries: at most kPlaces lie in the places
            const int stop = min(mine, at + kPlaces) - 1;
            u0 = (first + at - from) / kPlaces;
            u1 = min((first + stop - from) / kPlaces, u - 1);
        }
        // every lane's reads are done before the flag is up
        __threadfence();
        __syncwarp();
        if (lane == 0) asm volatile("st.release.gpu.global.u32 [%0], %1;" :: "l"(flags + unit), "r"(1u) : "memory");
        for (int w = u0 + lane; w <= u1; w += 32) {
            uint32_t there = 0u;
            for (uint32_t spin = 0; spin < (1u << 20) && there == 0u; ++spin)
                asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(there) : "l"(flags + (int64_t)w * lists + flag_at) : "memory");
            ok = ok && there != 0u;
        }
        ok = __all_sync(0xFFFFFFFFu, ok);
        __syncwarp();
        if (!ok) {
            if (lane == 0) atomicAdd(&g_keep_timeouts, 1u);
            return;
        }
    }
    if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicAdd(&g_keep_bad, 1u);
    if (touched[0] == 0u && touched[K - 1] == 0u) return;

#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (!(touched[k] >> lane & 1u)) dst[k] = -1;
        else if (P.weights != nullptr) P.weights[dst[k]] = moved_weight[k];
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        // ---- scales of the blocks: the largest that a token asks for ----
        // A normal code m asks for ceil(m / 8) - 15 above its token's scale.  Fewer is asked only where all of a token's codes are below 8 (8 itself asks
        // for as much as the formula gives these), and a NaN (0x7F) has no say: where a piece of 16 codes has its largest among these, all are looked at one by one.
        int ask[2 * K];   // of 16 places each
        bool odd = false;
#pragma unroll
        for (int q = 0; q < 2 * K; ++q) {
            int most = -1024;
#pragma unroll
            for (int i = q * PER16; i < (q + 1) * PER16; ++i) {
                const uint32_t m = absmax_codes(x[which][i]);
                const int s = __shfl_sync(0xFFFFFFFFu, scale[which][i * R / 32], (i * R + grp) & 31);
                odd = odd || m - 8u >= 0x7Fu - 8u;
                most = max(most, s + (int)((m + 7u) >> 3) - 15);
            }
            ask[q] = __reduce_max_sync(0xFFFFFFFFu, most);
        }
        if (__any_sync(0xFFFFFFFFu, odd)) {
#pragma unroll 1
            for (int q = 0; q < 2 * K; ++q) {
                int most = -1024;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const uint32_t m = absmax_numbers(x[which][i]);
                    const int s = __shfl_sync(0xFFFFFFFFu, scale[which][i * R / 32], (i * R + grp) & 31);
                    if (i / PER16 == q && m != 0u) most = max(most, s + asks(m));
                }
                most = __reduce_max_sync(0xFFFFFFFFu, most);
#pragma unroll
                for (int y = 0; y < 2 * K; ++y)
                    if (y == q) ask[y] = most;
            }
        }
        if (block >= 32) {
#pragma unroll
            for (int k = 0; k < K; ++k) ask[2 * k] = ask[2 * k + 1] = max(ask[2 * k], ask[2 * k + 1]);
            if (K == 2 && block == 64) ask[0] = ask[1] = ask[2 * K - 2] = ask[2 * K - 1] = max(ask[0], ask[2 * K - 1]);
        }
#pragma unroll
        for (int q = 0; q < 2 * K; ++q) ask[q] = min(max(ask[q], 0), 254);
#pragma unroll
        for (int k = 0; k < K; ++k)   // the block's scale: by the block's first place
            if (dst[k] >= 0 && ((base + 32 * k + lane) & (block - 1)) == 0)
                P.scales[which][((int64_t)(dst[k] >> P.page_shift) << per_page) + ((dst[k] & page_mask) >> P.block_shift)] =
                    (uint8_t)(lane < 16 ? ask[2 * k] : ask[2 * k + 1]);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int from_lane = (i * R + grp) & 31;
            const int s = __shfl_sync(0xFFFFFFFFu, scale[which][i * R / 32], from_lane);
            const int row = __shfl_sync(0xFFFFFFFFu, dst[i * R / 32], from_lane);
            const int d = max(s - ask[i / PER16], -24);   // at most 17; below -24 nothing is left of any code
            if (__any_sync(0xFFFFFFFFu, row >= 0 && d != 0)) {
                const int d1 = min(d, 15);
                scale_by(x[which][i], d1);
                if (__any_sync(0xFFFFFFFFu, d > 15)) scale_by(x[which][i], min(d, 30) - d1);   // (a power that f16 does not hold; exact in two steps: 1 where it is none)
            }
            if (row >= 0) *reinterpret_cast<uint4*>(P.codes[which] + (int64_t)row * DIM + 16 * sub) = x[which][i];
        }
    }
}

template <class K, class... Args>
cudaError_t launch(K kernel, int64_t ctas, int cluster, int threads, cudaStream_t stream, const Args&... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(threads);
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

}  // namespace

cudaError_t launch_select(const SelectParams& P, cudaStream_t stream)
{
    // CTAs of a sequence and head: more while one an SM is not reached and each still has 1024 tokens; of 32 warps where 16 would not hold their tokens
    const int64_t lists = (int64_t)P.seqs * P.heads;
    int cluster = 1;
    while (cluster < 8 && lists * cluster * 2 <= kSMs && P.max_len > 1024 * cluster) cluster *= 2;
    if (P.max_len > (int64_t)cluster * 16 * 128 * kHeld) return launch(select_kernel<32>, lists * cluster, cluster, 1024, stream, P, cluster);
    return launch(select_kernel<16>, lists * cluster, cluster, 512, stream, P, cluster);
}

// units of places that max_kept entries reach into, wherever the first stands
int64_t compact_units(int64_t max_kept, int places) { return max_kept > 0 ? ceil_div(max_kept + places - 1, places) : 0; }

cudaError_t launch_compact(CompactParams P, cudaStream_t stream)
{
    // 32 places a warp, 64 where a block has as many: half the registers let more warps hide the chain of loads in front of the rows
    const bool wide = P.block_shift == 6;
    P.units = compact_units(P.max_kept, wide ? 64 : 32);
    const int64_t units = P.units * P.seqs * P.heads, ctas = ceil_div(units, kMoveWarps);
    const bool in_place = P.out_table == P.table;
    if (in_place) {
        const cudaError_t e = cudaMemsetAsync(P.work, 0, (size_t)(units + 1) * 4, stream);
        if (e != cudaSuccess) return e;
    }
    auto go = [&](auto kernel) { return launch(kernel, ctas, 1, kMoveWarps * 32, stream, P); };
    if (P.dim == 128) return wide ? (in_place ? go(compact_kernel<128, true, 2>) : go(compact_kernel<128, false, 2>))
                                  : (in_place ? go(compact_kernel<128, true, 1>) : go(compact_kernel<128, false, 1>));
    return wide ? (in_place ? go(compact_kernel<64, true, 2>) : go(compact_kernel<64, false, 2>))
                : (in_place ? go(compact_kernel<64, true, 1>) : go(compact_kernel<64, false, 1>));
}

cudaError_t read_keep_counters(unsigned int* timeouts, unsigned int* bad)
{
    const cudaError_t e = cudaMemcpyFromSymbol(timeouts, g_keep_timeouts, sizeof(unsigned int));
    return e != cudaSuccess ? e : cudaMemcpyFromSymbol(bad, g_keep_bad, sizeof(unsigned int));
}
cudaError_t reset_keep_counters(bool timeouts)
{
    const unsigned int zero = 0;
    return timeouts ? cudaMemcpyToSymbol(g_keep_timeouts, &zero, sizeof(unsigned int)) : cudaMemcpyToSymbol(g_keep_bad, &zero, sizeof(unsigned int));
}

}  // namespace mxn
