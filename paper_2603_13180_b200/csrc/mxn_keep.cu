// Which tokens stay in the paged 8-bit cache, and moving them together.
//
// Select: of a sequence's tokens the first `sinks`, the last `recent`, and of those between the largest by weight, equal ones by place, until
// `keep` are chosen; for each key head apart.  A weight's bits, turned so that they order as unsigned numbers, are looked at in three digits
// (11, 11, 10 bits) from the top: a histogram of the digit among what agrees with the digits before gives the next digit of the smallest
// chosen weight.  Then every warp writes the places that it chose, in order, behind those of the warps before it.  A sequence and head is
// shared out over a cluster of CTAs, each with a run of tokens that it holds in shared memory; histograms are read across the cluster.
//
// Compact: token kept[i] goes to place first + i.  A warp takes 64 places of the keys or the values of a head: it reads the listed rows and their blocks' scales,
// finds for each block of places the scale that its largest value asks for (the append's rule: S = 2^(ceil(log2 absmax) - 8)), rounds the codes
// on it (exact unless they become subnormal; as they are where the scale stays) and writes them.  In place a row must be read before its place is written.
// Lists rise and places never lie behind their tokens, so only warps of lower places read what a warp is to overwrite; a warp says so once it
// has read, and waits for those (two at most) whose tokens lie in its 64 places.  Work is handed out by a ticket in the order of the places, so that whoever is
// waited for has started, and nobody waits before it has read: every wait ends.  (All waits are bounded; see mxn_device_timeouts.)
#include <cuda_fp16.h>

#include "mxn_device.cuh"
#include "mxn_internal.h"

namespace mxn {

namespace {

__device__ unsigned int g_keep_timeouts = 0;
__device__ unsigned int g_keep_bad = 0;   // entries, pages or lengths out of range

constexpr int kSelectThreads = 1024, kSelectWarps = 32, kBins = 2048;
constexpr int kHeld = 32768;   // tokens of a CTA's run that are held in shared memory; more are read again

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\n\tbarrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote_u32(uint32_t addr, int rank)
{
    uint32_t at, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.b32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
    return v;
}

// orders as unsigned numbers: -infinity ... -0 = 0 ... infinity; NaN below all
__device__ __forceinline__ uint32_t ordered(float w)
{
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__global__ void __launch_bounds__(kSelectThreads) select_kernel(const SelectParams P, const int cluster, const int held)
{
    extern __shared__ uint32_t keys[];
    __shared__ uint32_t hist[3][kBins];
    __shared__ uint32_t warp_sums[kSelectWarps];
    __shared__ uint32_t found[2];              // the digit, and how many are chosen at it
    __shared__ uint32_t counts[2];             // of this CTA: above the smallest chosen weight, equal to it
    __shared__ uint32_t warp_counts[kSelectWarps][2];
    pdl_prologue();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int rank = (int)(blockIdx.x % (uint32_t)cluster);
    const uint32_t unit = blockIdx.x / (uint32_t)cluster;
    const int h = (int)(unit % (uint32_t)P.heads), seq = (int)(unit / (uint32_t)P.heads);
    const int len = max(0, min(__ldg(P.lens + seq), P.max_len));
    int32_t* const out = P.kept + (int64_t)unit * P.keep;
    if (h == 0 && rank == 0 && threadIdx.x == 0) P.new_lens[seq] = min(len, P.keep);
    if (len <= P.keep) {   // everything stays
        for (int i = rank * kSelectThreads + threadIdx.x; i < P.keep; i += cluster * kSelectThreads) out[i] = i < len ? i : -1;
        return;
    }
    // this CTA's tokens, and this warp's: whole groups of 32
    const int groups = (len + 31) >> 5, per_warp = (groups + cluster * kSelectWarps - 1) / (cluster * kSelectWarps);
    const int g0 = min((int64_t)groups, (int64_t)(rank * kSelectWarps + warp) * per_warp), g1 = min(groups, g0 + per_warp);
    const int slot0 = warp * per_warp * 32;   // of the warp's first token among the CTA's
    const int tail = len - P.recent;
    const int32_t* const table = P.page_table + (int64_t)seq * P.max_pages;
    const int page_mask = (1 << P.page_shift) - 1;
    bool bad = false;
    auto fetch = [&](int t) -> uint32_t {
        if (t >= len) return 0u;
        const int pg = __ldg(table + (t >> P.page_shift));
        if ((uint32_t)pg >= (uint32_t)P.num_pages) {
            bad = true;
            return 0u;
        }
        return ordered(__ldg(P.weights + (((int64_t)pg * P.heads + h) << P.page_shift) + (t & page_mask)));
    };
    auto key = [&](int g) -> uint32_t {   // of this lane's token of group g of this warp
        const int slot = slot0 + (g - g0) * 32 + lane;
        return slot < held ? keys[slot] : fetch(g * 32 + lane);
    };
    auto between = [&](int t) { return t >= P.sinks && t < tail; };
    for (int i = threadIdx.x; i < 3 * kBins; i += kSelectThreads) (&hist[0][0])[i] = 0u;
    __syncthreads();

    uint32_t prefix = 0u, need = (uint32_t)(P.keep - P.sinks - P.recent);   // of those that agree with the prefix, how many are chosen
    const int first_group = g0;
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t mask = pass == 2 ? 1023u : 2047u;
        if (pass == 0) {
            for (int g = first_group; g < g1; g += 4) {
                uint32_t k[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) k[x] = g + x < g1 ? fetch((g + x) * 32 + lane) : 0u;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (g + x >= g1) continue;
                    const int slot = slot0 + (g + x - g0) * 32 + lane;
                    if (slot < held) keys[slot] = k[x];
                    if (between((g + x) * 32 + lane)) atomicAdd(&hist[0][k[x] >> 21], 1u);
                }
            }
        } else {
            const int up = pass == 1 ? 21 : 10;
            for (int g = first_group; g < g1; ++g) {
                const uint32_t k = key(g);
                if (between(g * 32 + lane) && (k >> up) == prefix) atomicAdd(&hist[pass][(k >> shift) & mask], 1u);
            }
        }
        cluster > 1 ? cluster_sync() : __syncthreads();
        // thread i: bins 2 i and 2 i + 1 from the top; an inclusive sum from the top over the block
        const int b0 = kBins - 1 - 2 * (int)threadIdx.x;
        uint32_t n0 = 0u, n1 = 0u;
        for (int r = 0; r < cluster; ++r) {
            n0 += cluster > 1 ? remote_u32(smem_at(&hist[pass][b0]), r) : hist[pass][b0];
            n1 += cluster > 1 ? remote_u32(smem_at(&hist[pass][b0 - 1]), r) : hist[pass][b0 - 1];
        }
        uint32_t sum = n0 + n1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xFFFFFFFFu, sum, o);
            if (lane >= o) sum += v;
        }
        if (lane == 31) warp_sums[warp] = sum;
        __syncthreads();
        uint32_t above = 0u;   // of the warps before
        {
            uint32_t v = warp_sums[lane];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(0xFFFFFFFFu, v, o);
                if (lane >= o) v += u;
            }
            above = warp > 0 ? __shfl_sync(0xFFFFFFFFu, v, warp - 1) : 0u;
        }
        const uint32_t before0 = above + sum - n0 - n1, before1 = before0 + n0;
        // the digit at which the count from the top reaches `need` (with need == 0: none, and every digit is above)
        if (before0 < need && before0 + n0 >= need) {
            found[0] = (uint32_t)b0;
            found[1] = need - before0;
        }
        if (before1 < need && before1 + n1 >= need) {
            found[0] = (uint32_t)(b0 - 1);
            found[1] = need - before1;
        }
        __syncthreads();
        if (need == 0u) break;
        prefix = (prefix << (pass == 2 ? 10 : 11)) | found[0];
        need = found[1];
    }
    // a token is chosen if its key is above the prefix, or equal to it and among the first `need` of those
    const bool none = P.keep == P.sinks + P.recent;
    auto above_it = [&](int t, uint32_t k) { return t < len && (!between(t) || (!none && k > prefix)); };
    auto equal_to = [&](int t, uint32_t k) { return !none && t < len && between(t) && k == prefix; };
    uint32_t n_above = 0u, n_equal = 0u;
    for (int g = g0; g < g1; ++g) {
        const uint32_t k = key(g);
        const int t = g * 32 + lane;
        n_above += __popc(__ballot_sync(0xFFFFFFFFu, above_it(t, k)));
        n_equal += __popc(__ballot_sync(0xFFFFFFFFu, equal_to(t, k)));
    }
    if (lane == 0) {
        warp_counts[warp][0] = n_above;
        warp_counts[warp][1] = n_equal;
    }
    __syncthreads();
    // of the warps before this one in the CTA; the CTA's total
    uint32_t a = warp_counts[lane][0], e = warp_counts[lane][1], a_before = lane < warp ? a : 0u, e_before = lane < warp ? e : 0u;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        a += __shfl_xor_sync(0xFFFFFFFFu, a, o);
        e += __shfl_xor_sync(0xFFFFFFFFu, e, o);
        a_before += __shfl_xor_sync(0xFFFFFFFFu, a_before, o);
        e_before += __shfl_xor_sync(0xFFFFFFFFu, e_before, o);
    }
    if (cluster > 1) {
        if (threadIdx.x == 0) {
            counts[0] = a;
            counts[1] = e;
        }
        cluster_sync();
        for (int r = 0; r < rank; ++r) {
            a_before += remote_u32(smem_at(&counts[0]), r);
            e_before += remote_u32(smem_at(&counts[1]), r);
        }
    }
    const uint32_t below = (1u << lane) - 1u;
    for (int g = g0; g < g1; ++g) {
        const uint32_t k = key(g);
        const int t = g * 32 + lane;
        const uint32_t ua = __ballot_sync(0xFFFFFFFFu, above_it(t, k)), ue = __ballot_sync(0xFFFFFFFFu, equal_to(t, k));
        const uint32_t e_mine = e_before + __popc(ue & below);   // equal ones in front of this token
        const bool chosen = (ua >> lane & 1u) || ((ue >> lane & 1u) && e_mine < need);
        const uint32_t at = a_before + __popc(ua & below) + min(e_mine, need);
        if (chosen && at < (uint32_t)P.keep) out[at] = t;
        a_before += __popc(ua);
        e_before += __popc(ue);
    }
    if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicAdd(&g_keep_bad, 1u);
    if (cluster > 1) cluster_sync();   // nobody leaves while its shared memory is read
}

// ---- moving ----------------------------------------------------------------------------------------------------------

constexpr int kPlaces = 64, kMoveWarps = 4;

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
// ceil(log2 of an E4M3 magnitude) - 8; far below every other for 0
__device__ __forceinline__ int asks(uint32_t m)
{
    if (m == 0u) return -1024;
    const int e = (int)(m >> 3), f = (int)(m & 7u);
    return e > 0 ? e - 15 + (f > 0) : f == 1 ? -17 : f == 2 ? -16 : f <= 4 ? -15 : -14;
}
__device__ __forceinline__ uint32_t half2_of(float v)
{
    const __half2 x = __float2half2_rn(v);
    return *reinterpret_cast<const uint32_t*>(&x);
}
// four codes times 2^a times 2^b (f16 pairs: exact, or so small that the code rounds to zero either way), rounded to E4M3
__device__ __forceinline__ uint32_t rescale(uint32_t w, uint32_t by_a, uint32_t by_b)
{
    uint32_t y;
    asm("{ .reg .b16 l, h; .reg .b32 p, q;\n\t"
        "mov.b32 {l, h}, %1; cvt.rn.f16x2.e4m3x2 p, l; cvt.rn.f16x2.e4m3x2 q, h;\n\t"
        "mul.rn.f16x2 p, p, %2; mul.rn.f16x2 q, q, %2; mul.rn.f16x2 p, p, %3; mul.rn.f16x2 q, q, %3;\n\t"
        "cvt.rn.satfinite.e4m3x2.f16x2 l, p; cvt.rn.satfinite.e4m3x2.f16x2 h, q; mov.b32 %0, {l, h}; }"
        : "=r"(y) : "r"(w), "r"(by_a), "r"(by_b));
    return y;
}
__device__ __forceinline__ int64_t shfl64(int64_t v, int from) { return __shfl_sync(0xFFFFFFFFu, v, from); }

template <int DIM, bool IN_PLACE>
__global__ void __launch_bounds__(kMoveWarps * 32, 4) compact_kernel(const CompactParams P)
{
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
    const int64_t unit = (int64_t)cta * kMoveWarps + warp, lists = (int64_t)P.seqs * P.heads * 2;
    if (unit >= P.units * lists) return;
    const int u = (int)(unit / lists);
    uint32_t rest = (uint32_t)(unit % lists);
    const int which = (int)(rest & 1u);
    rest >>= 1;
    const int h = (int)(rest % (uint32_t)P.heads), seq = (int)(rest / (uint32_t)P.heads);
    uint32_t* const flags = P.work + 1;   // of the same list: unit u' at u' * lists + (unit % lists)
    const int64_t flag_at = unit - (int64_t)u * lists;

    const int first = P.first != nullptr ? __ldg(P.first + seq) : 0;
    const int len = __ldg(P.lens + seq);
    const int64_t asked = (int64_t)__ldg(P.new_lens + seq) - first;
    bool bad = first < 0 || first > len || asked > P.max_kept;
    if (bad && lane == 0 && u == 0 && h == 0 && which == 0) atomicAdd(&g_keep_bad, 1u);
    if (first < 0 || first > len) return;   // the sequence is left as it is
    const int end = (int)min(first + min(asked, P.max_kept), (int64_t)0x7FFFFFFF - kPlaces);
    const int from = first / kPlaces * kPlaces, base = (int)min((int64_t)from + (int64_t)u * kPlaces, (int64_t)0x7FFFFFFF - kPlaces);
    if (end <= first || base >= end) return;   // (no unit with places waits for one without)
    bad = false;
    const int32_t* const list = P.kept + ((int64_t)seq * P.kept_heads + (P.kept_heads > 1 ? h : 0)) * P.max_kept;
    const int32_t* const table = P.table + (int64_t)seq * P.width;
    const int32_t* const out_table = P.out_table + (int64_t)seq * P.out_width;
    const int page_mask = (1 << P.page_shift) - 1, per_page = P.page_shift - P.block_shift;

    // ---- this lane's two places: where their tokens are (row numbers in the pool; -1: none), where they go ----
    int64_t src[2], dst[2];
    int scale[2];
    float moved_weight[2] = {0.0f, 0.0f};
    bool stays[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int place = base + 32 * k + lane;
        src[k] = dst[k] = -1;
        scale[k] = 0;
        stays[k] = true;
        if (place >= end) continue;
        bool wrong = false;
        const int64_t out_page_at = place >> P.page_shift;
        const int out_page = out_page_at < P.out_width ? __ldg(out_table + out_page_at) : -1;
        if ((uint32_t)out_page < (uint32_t)P.num_pages)
            dst[k] = (((int64_t)out_page * P.heads + h) << P.page_shift) + (place & page_mask);
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
                src[k] = (((int64_t)page * P.heads + h) << P.page_shift) + (token & page_mask);
                stays[k] = src[k] == dst[k];
            } else {
                wrong = true;
            }
        }
        bad |= wrong;
    }
    // a block with an entry out of range is left as it is, and so is one whose tokens all stay where they are
    const int block = 1 << P.block_shift;
    uint32_t touched[2];   // bit: the place is to be written
    {
        const uint32_t moves0 = __ballot_sync(0xFFFFFFFFu, !stays[0]), moves1 = __ballot_sync(0xFFFFFFFFu, !stays[1]);
        const uint32_t off0 = __ballot_sync(0xFFFFFFFFu, base + lane < end && (src[0] < 0 || dst[0] < 0)),
                       off1 = __ballot_sync(0xFFFFFFFFu, base + 32 + lane < end && (src[1] < 0 || dst[1] < 0));
        const uint32_t real0 = __ballot_sync(0xFFFFFFFFu, base + lane < end), real1 = __ballot_sync(0xFFFFFFFFu, base + 32 + lane < end);
        auto spread = [&](uint64_t v) -> uint64_t {   // to all places of the blocks that have a bit
            uint64_t y = 0;
            for (int o = 0; o < kPlaces; o += block) {
                const uint64_t m = (block == 64 ? ~0ull : (1ull << block) - 1) << o;
                if (v & m) y |= m;
            }
            return y;
        };
        const uint64_t w = spread((uint64_t)moves1 << 32 | moves0) & ~spread((uint64_t)off1 << 32 | off0) & ((uint64_t)real1 << 32 | real0);
        touched[0] = (uint32_t)w;
        touched[1] = (uint32_t)(w >> 32);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!(touched[k] >> lane & 1u)) {
            src[k] = -1;
        } else {
            // row / page * (page / block) + block within the page
            scale[k] = P.scales[which][((src[k] >> P.page_shift) << per_page) + ((src[k] & page_mask) >> P.block_shift)];
            if (which == 0 && P.weights != nullptr) moved_weight[k] = P.weights[src[k]];
        }
    }
    uint4 x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int place = i * R + grp;
        const int64_t row = shfl64(i * R < 32 ? src[0] : src[1], place & 31);
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row >= 0) x[i] = *reinterpret_cast<const uint4*>(P.codes[which] + row * DIM + 16 * sub);
    }
    bool ok = true;
    if (IN_PLACE) {
        // every lane's reads are done before the flag is up
        __threadfence();
        __syncwarp();
        if (lane == 0) {
            asm volatile("st.release.gpu.global.u32 [%0], %1;" :: "l"(flags + unit), "r"(1u) : "memory");
        }
        // list entries whose tokens lie in this warp's places [base, base + 64): they stand in front of its own.  The first of them, 32 probes at a time
        const int mine = max(0, base - first);   // list entries in front of this unit's
        if (mine > 0 && __ldg(list + (mine - 1)) >= base) {
            int at = 0, n = mine;   // the first entry >= base is in [at, at + n)
            while (n > 1) {
                const int step = (n + 31) / 32, probe = at + min(lane * step, n - 1);
                const unsigned less = __ballot_sync(0xFFFFFFFFu, lane * step < n && __ldg(list + probe) < base);
                if (less == 0u) break;   // the first one already is
                const int last = 31 - __clz(less);   // the last probe below
                const int skip = last * step + 1;
                at += skip;
                n = min(step, n - skip);
            }
            // rising entries: at most 64 lie in the places
            const int stop = min(mine, at + kPlaces) - 1;
            const int u0 = (first + at - from) / kPlaces, u1 = min((first + stop - from) / kPlaces, u - 1);
            for (int w = u0 + lane; w <= u1; w += 32) {
                uint32_t there = 0u;
                for (uint32_t spin = 0; spin < (1u << 20) && there == 0u; ++spin)
                    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(there) : "l"(flags + (int64_t)w * lists + flag_at) : "memory");
                ok = ok && there != 0u;
            }
            ok = __all_sync(0xFFFFFFFFu, ok);
            __syncwarp();
        }
        if (!ok) {
            if (lane == 0) atomicAdd(&g_keep_timeouts, 1u);
            return;
        }
    }
    if (__any_sync(0xFFFFFFFFu, bad) && lane == 0) atomicAdd(&g_keep_bad, 1u);
    if (touched[0] == 0u && touched[1] == 0u) return;

    // ---- scales of the blocks: the largest that a token asks for ----
    int ask[4];   // of 16 places each
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        int most = -1024;
#pragma unroll
        for (int i = q * PER16; i < (q + 1) * PER16; ++i) {
            uint32_t m = absmax_codes(x[i]);
            if (__any_sync(0xFFFFFFFFu, m == 0x7Fu)) m = absmax_numbers(x[i]);   // a NaN has no say in the scale
            const int s = __shfl_sync(0xFFFFFFFFu, i * R < 32 ? scale[0] : scale[1], (i * R + grp) & 31);
            most = max(most, m == 0u ? -1024 : s + asks(m));
        }
        ask[q] = __reduce_max_sync(0xFFFFFFFFu, most);
    }
    if (block >= 32) {
        ask[0] = ask[1] = max(ask[0], ask[1]);
        ask[2] = ask[3] = max(ask[2], ask[3]);
        if (block == 64) ask[0] = ask[1] = ask[2] = ask[3] = max(ask[0], ask[2]);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) ask[q] = min(max(ask[q], 0), 254);
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (!(touched[k] >> lane & 1u)) {
            dst[k] = -1;
            continue;
        }
        if (which == 0 && P.weights != nullptr) P.weights[dst[k]] = moved_weight[k];
        const int place = base + 32 * k + lane;
        // the block's scale: by the block's first place
        if ((place & (block - 1)) == 0)
            P.scales[which][((dst[k] >> P.page_shift) << per_page) + ((dst[k] & page_mask) >> P.block_shift)] =
                (uint8_t)(lane < 16 ? ask[2 * k] : ask[2 * k + 1]);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int from_lane = (i * R + grp) & 31;
        const int s = __shfl_sync(0xFFFFFFFFu, i * R < 32 ? scale[0] : scale[1], from_lane);
        const int64_t row = shfl64(i * R < 32 ? dst[0] : dst[1], from_lane);
        const int d = max(s - ask[i / PER16], -24);   // at most 17; below -24 nothing is left of any code
        if (__any_sync(0xFFFFFFFFu, row >= 0 && d != 0)) {
            const int d1 = min(d, 15);
            const uint32_t a = half2_of(__uint_as_float((uint32_t)(127 + d1) << 23)), b = half2_of(__uint_as_float((uint32_t)(127 + min(d, 30) - d1) << 23));
            x[i].x = rescale(x[i].x, a, b);
            x[i].y = rescale(x[i].y, a, b);
            x[i].z = rescale(x[i].z, a, b);
            x[i].w = rescale(x[i].w, a, b);
        }
        if (row >= 0) *reinterpret_cast<uint4*>(P.codes[which] + row * DIM + 16 * sub) = x[i];
    }
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

template <class K, class... Args>
cudaError_t launch(K kernel, int64_t ctas, int cluster, int threads, int smem, cudaStream_t stream, const Args&... args)
{
    if (smem > 16 * 1024) {
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

}  // namespace

cudaError_t launch_select(const SelectParams& P, cudaStream_t stream)
{
    // CTAs of a sequence and head: more while two an SM are not reached and each still has 2048 tokens
    const int64_t lists = (int64_t)P.seqs * P.heads;
    int cluster = 1;
    while (cluster < 8 && lists * cluster * 2 <= 2 * 148 && P.max_len > 2048 * cluster) cluster *= 2;
    const int64_t run = ceil_div(ceil_div(P.max_len, 32), cluster * kSelectWarps) * 32 * kSelectWarps;   // a CTA's tokens at most
    const int held = (int)(run < kHeld ? run : kHeld);
    return launch(select_kernel, lists * cluster, cluster, kSelectThreads, held * 4, stream, P, cluster, held);
}

// units of 64 places that max_kept entries reach into, wherever the first stands
int64_t compact_units(int64_t max_kept) { return max_kept > 0 ? ceil_div(max_kept + kPlaces - 1, kPlaces) : 0; }

cudaError_t launch_compact(const CompactParams& P, cudaStream_t stream)
{
    const int64_t units = P.units * P.seqs * P.heads * 2, ctas = ceil_div(units, kMoveWarps);
    const bool in_place = P.out_table == P.table;
    if (in_place) {
        const cudaError_t e = cudaMemsetAsync(P.work, 0, (size_t)(units + 1) * 4, stream);
        if (e != cudaSuccess) return e;
    }
    if (P.dim == 128) return in_place ? launch(compact_kernel<128, true>, ctas, 1, kMoveWarps * 32, 0, stream, P)
                                      : launch(compact_kernel<128, false>, ctas, 1, kMoveWarps * 32, 0, stream, P);
    return in_place ? launch(compact_kernel<64, true>, ctas, 1, kMoveWarps * 32, 0, stream, P)
                    : launch(compact_kernel<64, false>, ctas, 1, kMoveWarps * 32, 0, stream, P);
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
