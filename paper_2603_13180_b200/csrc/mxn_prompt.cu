// Attention over the paged 8-bit cache for many query rows (prompts): both products on the 5th-generation tensor cores.
//
//   o = sum_t softmax(scale q . k_t) v_t,   k_t = 2^(sk - 127) * code, v_t likewise
//
// Work of a CTA: 256 query rows of one sequence and key head (query heads that share a key head are rows like any other: row =
// token * group + head), in two tiles of 128, over a chunk of the keys in tiles of 128 tokens.  Tensor memory holds the scores
// and the output of both tiles (2 * (128 + dim) columns of binary32).  Roles, by warp:
//   0      copies: codes of keys and values by the tensor copy engine, a box for each page; scales by plain loads; starts while q is read
//   1, 2   issue the products, one warp for each row tile
//   4-7    values: E4M3 codes -> f16 (exact), zeros for what no row may see; before that, with 8-15, q
//   8-15   softmax, one warpgroup for each row tile, a thread for each row
// The two row tiles alternate: while one's scores are in the softmax, the other's products run.
//
// Scores: E4M3 x E4M3 products on the key codes as they are; q is scaled by a power of two to [128, 256) at its row's largest
//   and written as a sum of two E4M3 numbers, hi + lo, which is exact but for elements below 2^-10 of the row's largest (to 2^-18
//   of it).  Two products of twice f16's rate cost what one in f16 would, and the keys need no conversion.
// Weights: w_t = 2^(s_t + sv_t - R + 1) in f16 (11 significant bits): the value block's scale is folded into the weight, so that the
//   codes enter the second product without a scale.  R (an integer: corrections are exact) is the first tile's largest s + sv and
//   is moved only when a step's largest is 14 above or 16 below it, so that the output in tensor memory rarely has to be corrected.
//   f16 drops what is below 2^-25, i.e. 2^-26 of the weight at R and 2^-10 of the largest of a step at the window's lower end.
// The softmax's sum is l = sum of w_t 2^(c0 - sv_t) with unrounded w, a factor for each run of 16 tokens, c0 near the scales;
// a tile with scales far from c0 is summed apart (see kApart), and c0 follows a tile whose scales are all elsewhere.
// The weights replace their scores in tensor memory and are the second product's first operand from there; the values are its
// second operand as they lie ([token][dim] is the "MN-major" form), so nothing is transposed.
//
// Bound: at head size 128 the two products of a 256 x 128 tile take 2048 cycles at the tensor cores' rate, its 32768 exponentials
// 2048 cycles of the special function units.  4096 queries over 8192 keys, 32 query and 8 key heads of 128: 450 us, 916 TFLOP/s, 55 %
// of a large library product's measured rate (482 us in turn with other work, at lower clocks); a tile takes some 3900 cycles.  Without
// the softmax's arithmetic the same kernel takes 310 us: what is left is the softmax's chain of loads, maxima, exponentials and stores,
// two warps for each scheduler, with the special function units busy for half of the time.  Four warps for each scheduler (two for a
// row) took 595 us: twice the fixed costs of a step.  What shortened the chain: barriers and scales looked at a step ahead, while
// shared memory is busy with the products' operands (499 -> 478); a rounding of the maximum taken out of it (501 -> 493); q read by
// rows, 12 warps at it, and the output written by rows through shared memory (464 -> 450), the last units in halves (-> 437).  NaN
// scores kept as such: 446, sums apart: 450.  The products alone do not reach their rate either: scores in products of 64 tokens read
// 6 KB of shared memory in 48 cycles for 32 of the tensor cores.
//
// Every wait is bounded; see mxn_device_timeouts.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <type_traits>

#include "mxn_attn.cuh"

namespace mxn {

namespace {

constexpr int kTile = 128;        // tokens of a key tile, rows of a row tile
constexpr int kStep = 64;         // tokens of a step of the softmax: half a tile
constexpr int kThreads = 512;
constexpr int kKeyStages = 3, kValStages = 2, kHalfStages = 2, kScaleSlots = 8;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kRun = 16;          // tokens that share a scale at the finest
// Weights: 2^kTop at the reference; the reference is moved when a tile's largest is more than kUp above or kDown below it, but to
// no more than kDepth below the largest so far (the output's sums must not overflow)
constexpr float kTop = 1.0f, kUp = 14.0f, kDown = 16.0f, kDepth = 40.0f;

__device__ unsigned int g_prompt_timeouts = 0;
__device__ unsigned int g_prompt_bad = 0;

template <int DIM>
struct PromptShape {
    static constexpr int kCodes = kTile * DIM;                 // bytes of a tile of codes (keys, values, q hi, q lo)
    static constexpr int kHalf = kTile * DIM * 2;              // bytes of a tile of f16 values
    static constexpr int kQ = 0;                               // [row tile][hi, lo]
    static constexpr int kK = kQ + 4 * kCodes;
    static constexpr int kV = kK + kKeyStages * kCodes;
    static constexpr int kH = kV + kValStages * kCodes;
    static constexpr int kEnd = kH + kHalfStages * kHalf;
    static constexpr int kSmem = kEnd + 1024;
};

constexpr uint32_t kWide = 1, kMoved = 2;
// one slot of the scales' ring: what the softmax needs to know about a key tile.  The ring is deeper than the keys': a slot is
// written again once the keys kKeyStages tiles before are free, i.e. when the softmax of both row tiles is past the tile before those.
struct alignas(16) TileScales {
    float k[kTile / kRun];        // 2^(sk - 127)
    float v[kTile / kRun];        // sv - 127
    float l[kTile / kRun];        // 2^(c0 - v): from weights to the softmax's sum
    uint32_t readable;            // bit i: the page of run i could be read
    uint32_t apart;               // kWide: a value scale lies so far from c0 that the tile is summed apart; kMoved: c0 is another than before
    float c0;
};

// ---- tensor core plumbing ------------------------------------------------------------------------------------
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// shared-memory operand descriptor: address, stride between groups of 8 rows (`group`), between repeats along the other
// axis (`repeat`), and the swizzle (2: 128 bytes, 4: 64 bytes)
__device__ __forceinline__ uint64_t operand(uint32_t addr, uint32_t group, uint32_t repeat, uint32_t swizzle)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(repeat >> 4) << 16) | ((uint64_t)(group >> 4) << 32) | (1ull << 46) |
           ((uint64_t)swizzle << 61);
}
// instruction descriptors: binary32 sums, M = 128
__host__ __device__ constexpr uint32_t idesc_e4m3(int n) { return (1u << 4) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }
__host__ __device__ constexpr uint32_t idesc_f16_bt(int n) { return (1u << 4) | (1u << 16) | ((uint32_t)(n >> 3) << 17) | (8u << 24); }

__device__ __forceinline__ void mma_scores(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p; }"
                 :: "r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_values(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add)
{
    asm volatile("{ .reg .pred p; setp.ne.u32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
                 :: "r"(d), "r"(a), "l"(b), "r"(idesc), "r"(add) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" :: "r"(bar) : "memory");
}
#define MXN_R8(r, i) "=r"(r[i]), "=r"(r[i + 1]), "=r"(r[i + 2]), "=r"(r[i + 3]), "=r"(r[i + 4]), "=r"(r[i + 5]), "=r"(r[i + 6]), "=r"(r[i + 7])
#define MXN_U8(r, i) "+r"(r[i]), "+r"(r[i + 1]), "+r"(r[i + 2]), "+r"(r[i + 3]), "+r"(r[i + 4]), "+r"(r[i + 5]), "+r"(r[i + 6]), "+r"(r[i + 7])
#define MXN_I8(r, i) "r"(r[i]), "r"(r[i + 1]), "r"(r[i + 2]), "r"(r[i + 3]), "r"(r[i + 4]), "r"(r[i + 5]), "r"(r[i + 6]), "r"(r[i + 7])
// 32 columns of this warp's 32 lanes, a lane's row in its thread
__device__ __forceinline__ void tm_load(uint32_t (&r)[32], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\ttcgen05.wait::ld.sync.aligned;"
                 : MXN_R8(r, 0), MXN_R8(r, 8), MXN_R8(r, 16), MXN_R8(r, 24) : "r"(addr) : "memory");
}
// the same in two steps: the values are there after tm_arrived of the same registers
__device__ __forceinline__ void tm_request(uint32_t (&r)[32], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : MXN_R8(r, 0), MXN_R8(r, 8), MXN_R8(r, 16), MXN_R8(r, 24) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_arrived(uint32_t (&r)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;" : MXN_U8(r, 0), MXN_U8(r, 8), MXN_U8(r, 16), MXN_U8(r, 24) :: "memory");
}
__device__ __forceinline__ void tm_store32(uint32_t addr, const uint32_t (&r)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 :: "r"(addr), MXN_I8(r, 0), MXN_I8(r, 8), MXN_I8(r, 16), MXN_I8(r, 24) : "memory");
}
__device__ __forceinline__ void tm_store16(uint32_t addr, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 :: "r"(addr), MXN_I8(r, 0), MXN_I8(r, 8) : "memory");
}
__device__ __forceinline__ void tm_load16(uint32_t (&r)[16], uint32_t addr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
                 "tcgen05.wait::ld.sync.aligned;"
                 : MXN_R8(r, 0), MXN_R8(r, 8) : "r"(addr) : "memory");
}
__device__ __forceinline__ void tm_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ bool elect_one()
{
    uint32_t is;
    asm volatile("{ .reg .pred p; elect.sync _|p, 0xFFFFFFFF; selp.u32 %0, 1, 0, p; }" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{ .reg .pred p; mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// waits with a limit; a wait that runs out, or one that sees another's, ends the CTA's work
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* dead)
{
    if (mbar_test(bar, parity)) return true;
    for (uint32_t spin = 0; spin < (1u << 20); ++spin) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((spin & 255u) == 255u && *dead) return false;
    }
    *dead = 1;
    return false;
}

__device__ __forceinline__ float max3(uint32_t a, uint32_t b, uint32_t c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(__uint_as_float(a)), "f"(__uint_as_float(b)), "f"(__uint_as_float(c)));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ float2 f2(float a) { return make_float2(a, a); }

// 2^u of two numbers below 2^21 on the multipliers: u = n + f with n the nearest integer (what is below -126 counts as that: 2^-126 is
// nothing to a sum whose terms reach 2^-15, and rounds to 0 in f16), and 2^f by a polynomial fitted to the least relative error over
// [-1/2, 1/2] with 1 as its constant: 1.09e-7, with the roundings 1.7e-7 (2^-22.4)
__device__ __forceinline__ float2 ex2_fma(float2 u)
{
    const float2 v = make_float2(fmaxf(u.x, -126.0f), fmaxf(u.y, -126.0f)), t = __fadd2_rn(v, f2(12582912.0f));   // 1.5 * 2^23
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
__global__ void __launch_bounds__(kThreads, 1) attn_prompt_kernel(const AttnParams P, const __grid_constant__ AttnMaps M)
{
    using Sh = PromptShape<DIM>;
    constexpr uint32_t SW = DIM == 128 ? 2 : 4;         // swizzle of a tile of codes: its rows are DIM bytes
    constexpr uint32_t GROUP = 8 * DIM;                 // bytes of 8 rows of codes
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * kKeyStages + 2 * kValStages + 2 * kHalfStages + 8 + kScaleSlots];
    __shared__ TileScales scales[kScaleSlots];
    __shared__ float row_factors[2 * kTile];
    __shared__ uint32_t tmem_at;
    __shared__ int dead_flag;

    pdl_prologue();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    uint32_t b = blockIdx.x;
    int half = -1;   // the last units may be in two halves of a row tile each
    if (b >= P.whole_units) {
        half = (int)((b - P.whole_units) & 1u);
        b = P.whole_units + (b - P.whole_units) / 2;
    }
    const int split = (int)(b % (uint32_t)P.splits);
    b /= (uint32_t)P.splits;
    const int seq = (int)(b % (uint32_t)P.seqs);
    b /= (uint32_t)P.seqs;
    const int h = (int)(b % (uint32_t)P.kv_heads);
    const int block = P.row_tiles - 1 - (int)(b / (uint32_t)P.kv_heads);   // the rows that see most keys first

    const AttnSequence S = attn_sequence(P, seq);
    const int q0 = S.q0, len = S.len, shift = S.shift, nq = S.nq;
    const int G = P.group, row0 = (2 * block + (half == 1)) * kTile, rows = min(nq * G, row0 + (half < 0 ? 2 : 1) * kTile);
    if (row0 >= rows) return;
    const bool two = rows - row0 > kTile;   // else nothing is done for the second row tile
    const int hi = max(0, min(len, P.causal ? shift + P.by_group(rows - 1) + 1 : len));
    const int seen = first_seen(shift + P.by_group(row0), P.window);   // nothing before it, not even its page, has any influence
    const int lo = seen / kTile * kTile;
    const int k0 = (int)min((int64_t)hi, lo + (int64_t)split * P.chunk), k1 = (int)min((int64_t)hi, (int64_t)k0 + P.chunk);
    const int tiles = (k1 - k0 + kTile - 1) / kTile;

    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t bar0 = smem_u32(bars);
    const uint32_t k_full = bar0, k_empty = k_full + 8 * kKeyStages, v_full = k_empty + 8 * kKeyStages, v_empty = v_full + 8 * kValStages,
                   h_full = v_empty + 8 * kValStages, h_empty = h_full + 8 * kHalfStages, s_full = h_empty + 8 * kHalfStages,
                   p_full = s_full + 32, sc_full = p_full + 32;   // [row tile][buffer]
    volatile int* const dead = &dead_flag;
    if (threadIdx.x == 0) {
        dead_flag = 0;
        for (int i = 0; i < kKeyStages; ++i) {
            mbar_init(k_full + 8 * i, 1);
            mbar_init(k_empty + 8 * i, two ? 2 : 1);
        }
        for (int i = 0; i < kValStages; ++i) {
            mbar_init(v_full + 8 * i, 1);
            mbar_init(v_empty + 8 * i, 4);
        }
        for (int i = 0; i < kHalfStages; ++i) {
            mbar_init(h_full + 8 * i, 4);
            mbar_init(h_empty + 8 * i, two ? 2 : 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(s_full + 8 * i, 1);
            mbar_init(p_full + 8 * i, 4);
        }
        for (int i = 0; i < kScaleSlots; ++i) mbar_init(sc_full + 8 * i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" :: "r"(smem_u32(&tmem_at)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }

    const int rt = (warp >> 2) & 1;                       // row tile of warps 8-15
    const int r_in = threadIdx.x & 127;                   // row within its tile
    // q, by warps 4-15: DIM / 8 threads for a row, so that a row is read in one piece.  It is split into hi and lo for the tensor cores.
    if (warp >= 4) {
        constexpr int kLanes = DIM / 8, kAtOnce = 32 / kLanes, kPass = 12 * kAtOnce, kPasses = (2 * kTile + kPass - 1) / kPass;
        const int c = lane % kLanes, first = (warp - 4) * kAtOnce + lane / kLanes;
        uint4 w[kPasses];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int r = first + i * kPass, rr = row0 + r;
            w[i] = make_uint4(0, 0, 0, 0);
            if (r < 2 * kTile && rr < rows) {
                const int t = P.by_group(rr);
                w[i] = __ldg(reinterpret_cast<const uint4*>(P.q + (q0 + t) * P.q_stride + (int64_t)(h * G + rr - t * G) * DIM) + c);
            }
        }
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int r = first + i * kPass;
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
            float m = hmax_abs_to_f32(absmax_bf16x2(absmax_bf16x2(absmax_bf16x2(absmax_bf16x2(0u, u[0]), u[1]), u[2]), u[3]));
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
            const uint32_t E = __float_as_uint(m) >> 23, Ec = min(max(E, 8u), 254u);
            float up = __uint_as_float((261u - Ec > 254u ? 254u : 261u - Ec) << 23);             // 2^(7 - (E - 127))
            if (P.scale < 0.0f) up = -up;
            if (E == 255u) up = __uint_as_float(0x7FC00000u);   // an infinity or NaN: the row's result is NaN (E4M3 has no infinity)
            uint32_t hh[4], ll[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const __half2 v = __floats2half2_rn(bf16_lo(u[y]) * up, bf16_hi(u[y]) * up);
                hh[y] = __nv_cvt_halfraw2_to_fp8x2(static_cast<__half2_raw>(v), __NV_SATFINITE, __NV_E4M3);
                const __half2 left = __hsub2(v, __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)hh[y], __NV_E4M3)));
                ll[y] = __nv_cvt_halfraw2_to_fp8x2(static_cast<__half2_raw>(left), __NV_SATFINITE, __NV_E4M3);
            }
            if (r < 2 * kTile) {
                const int rl = r & (kTile - 1);
                const uint32_t at = base + Sh::kQ + (uint32_t)(r / kTile) * 2 * Sh::kCodes + (uint32_t)rl * DIM
                                  + (uint32_t)(((c >> 1) ^ (DIM == 128 ? rl & 7 : (rl >> 1) & 3)) << 4) + (uint32_t)(c & 1) * 8;
                asm volatile("st.shared.v2.b32 [%0], {%1,%2};" :: "r"(at), "r"(hh[0] | (hh[1] << 16)), "r"(hh[2] | (hh[3] << 16)) : "memory");
                asm volatile("st.shared.v2.b32 [%0], {%1,%2};" :: "r"(at + Sh::kCodes), "r"(ll[0] | (ll[1] << 16)), "r"(ll[2] | (ll[3] << 16)) : "memory");
                if (c == 0) row_factors[r] = fabsf(P.scale) * kLog2e * __uint_as_float((Ec - 7u) << 23);
            }
        }
        fence_async();
    }
    // warp 0 made the barriers and waits for nobody: its copies start while q is read
    if (warp == 0) {
        __syncwarp();
        asm volatile("barrier.arrive 1, %0;" :: "n"(kThreads) : "memory");
    } else {
        tc_before();
        asm volatile("barrier.sync 1, %0;" :: "n"(kThreads) : "memory");
        tc_after();
    }
    const uint32_t tmem = warp == 0 ? 0u : tmem_at;
    const uint32_t s_col[2] = {tmem, tmem + 128}, o_col[2] = {tmem + 256, tmem + 256 + DIM};

    // 512 threads at 128 registers: the softmax warps take what the others give up (256 * 56 + 256 * 200 = 512 * 128)
#define MXN_FEW_REGISTERS() asm volatile("setmaxnreg.dec.sync.aligned.u32 56;")
    if (warp == 0) {
        // ---- copies ----
        MXN_FEW_REGISTERS();
        const int32_t* const table = P.page_table + (int64_t)seq * P.max_pages;
        const int box = min(P.page, kTile), boxes = kTile / box;     // tokens of a box, boxes of a tile
        const int per_page_shift = P.page_shift - P.block_shift;
        bool any_bad = false;
        float c0 = 0.0f;
        int page_next = -1;                                          // lane i: page of run i (lanes 0-7) of the next tile
        auto look_up = [&](int j) {
            const int t = k0 + j * kTile + kRun * (lane & 7);
            int pg = -1;
            if (j < tiles && lane < 8 && t < k1 && (t | (box - 1)) >= seen) {
                pg = __ldg(table + (t >> P.page_shift));
                if (pg < 0 || pg >= P.num_pages) {
                    pg = -1;
                    any_bad = true;
                }
            }
            return pg;
        };
        page_next = look_up(0);
        bool ok = true;
        for (int j = 0; j < tiles; ++j) {
            const int pg = page_next;
            page_next = look_up(j + 1);
            const int t0 = k0 + j * kTile, ks = j % kKeyStages, vs = j % kValStages;
            // scales
            uint32_t sk = 0, sv = 0;
            if (pg >= 0) {
                const int64_t at = (((int64_t)pg * P.kv_heads + h) << per_page_shift) + (((t0 + kRun * lane) & (P.page - 1)) >> P.block_shift);
                sk = __ldg(P.k_scales + at);
                sv = __ldg(P.v_scales + at);
            }
            const uint32_t readable = __ballot_sync(0xFFFFFFFFu, pg >= 0);
            // this lane's box starts at run lane * (box / 16)
            const int src = lane * (box / kRun);
            const int box_page = __shfl_sync(0xFFFFFFFFu, pg, src & 7);
            const bool mine = lane < boxes && box_page >= 0;
            const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, mine)) * (uint32_t)(box * DIM);
            const int y = (t0 + src * kRun) & (P.page - 1), z = box_page * P.kv_heads + h;

            if (j >= kKeyStages) ok = ok && wait(k_empty + 8 * ks, (uint32_t)(j / kKeyStages - 1) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            TileScales& slot = scales[j % kScaleSlots];
            const float v = (float)(int)sv - 127.0f;
            // c0, near the value scales: the largest of the first tile, or of the first one whose scales are all elsewhere
            bool wide = __any_sync(0xFFFFFFFFu, pg >= 0 && fabsf(v - c0) > kApart);
            const float c0_before = c0;
            if (j == 0 || wide) {
                float top = v;   // (a run without tokens has the least)
#pragma unroll
                for (int o = 4; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                top = fminf(fmaxf(__shfl_sync(0xFFFFFFFFu, top, 0), -60.0f), 60.0f);
                const bool still = __any_sync(0xFFFFFFFFu, pg >= 0 && fabsf(v - top) > kApart);
                if (j == 0 || !still) {
                    c0 = top;
                    wide = still;
                }
            }
            if (lane < 8) {
                slot.k[lane] = e8m0_to_f32(sk);
                slot.v[lane] = v;
                slot.l[lane] = ex2(fminf(fmaxf(c0 - v, -40.0f), 40.0f));
            }
            if (lane == 0) {
                slot.readable = readable;
                slot.apart = (wide ? kWide : 0u) | (c0 != c0_before ? kMoved : 0u);
                slot.c0 = c0;
            }
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(sc_full + 8 * (j % kScaleSlots));
                if (bytes) mbar_expect_tx(k_full + 8 * ks, bytes);
                else mbar_arrive(k_full + 8 * ks);
            }
            __syncwarp();
            if (mine) tma_load_codes(base + Sh::kK + ks * Sh::kCodes + lane * box * DIM, &M.k, y, z, k_full + 8 * ks);
            if (j >= kValStages) ok = ok && wait(v_empty + 8 * vs, (uint32_t)(j / kValStages - 1) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            if (lane == 0) {
                if (bytes) mbar_expect_tx(v_full + 8 * vs, bytes);
                else mbar_arrive(v_full + 8 * vs);
            }
            __syncwarp();
            if (mine) tma_load_codes(base + Sh::kV + vs * Sh::kCodes + lane * box * DIM, &M.v, y, z, v_full + 8 * vs);
        }
        if (__any_sync(0xFFFFFFFFu, any_bad) && lane == 0) atomicAdd(&g_prompt_bad, 1u);
    } else if (warp == 1 || warp == 2) {
        // ---- products: a warp for each row tile, so that neither waits for the other's softmax ----
        MXN_FEW_REGISTERS();
        if (tiles > 0 && (warp == 1 || two)) {
            // Step i is half a key tile.  Scores are two steps ahead of the weights: while the softmax works on one buffer, the
            // other's scores are made.  The weights of step i lie in their scores' columns, so the scores of step i + 2 are
            // issued behind the product that reads those weights; products run in the order of issue.
            // One thread issues a row tile's products, one every 50 cycles: the whole warp goes through the loop, so that descriptors (bases
            // plus constants) are uniform values.
            const bool one = elect_one();
            const int r = warp - 1;
            const uint32_t s_mine = s_col[0] + r * 128, o_mine = o_col[0] + r * DIM, s_bar = s_full + 16 * r, p_bar = p_full + 16 * r;
            bool ok = true;
            const uint64_t q_desc = operand(base + Sh::kQ + r * 2 * Sh::kCodes, GROUP, 16, SW), k_base = operand(base + Sh::kK, GROUP, 16, SW),
                           h_base = operand(base + Sh::kH, 1024, kTile * 128, 2);
            uint32_t ks = 0, k_par = 0, hs = 0, h_par = 0, p_par = 0;
            uint64_t k_desc = k_base;
            auto scores = [&](int half) {   // S = (hi + lo) K^T
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int s = 0; s < DIM / 32; ++s)
                        mma_scores(s_mine + half * kStep, q_desc + (uint64_t)((part * Sh::kCodes + 32 * s) >> 4),
                                   k_desc + (uint64_t)((half * kStep * DIM + 32 * s) >> 4), idesc_e4m3(kStep), (part | s) != 0);
            };
            auto next_keys = [&]() {   // the next key tile
                if (++ks == kKeyStages) {
                    ks = 0;
                    k_par ^= 1u;
                }
                k_desc = k_base + (uint64_t)((ks * Sh::kCodes) >> 4);
            };
            ok = wait(k_full, 0, dead);
            if (ok) {
                tc_after();
#pragma unroll
                for (int half = 0; half < 2; ++half)
                    if (one) {
                        scores(half);
                        mma_commit(s_bar + 8 * half);
                    }
                if (one) mma_commit(k_empty);
                next_keys();
            }
            for (int j = 0; ok && j < tiles; ++j) {
                const bool more = j + 1 < tiles;
                ok = wait(h_full + 8 * hs, h_par, dead) && (!more || wait(k_full + 8 * ks, k_par, dead));
                if (!ok) break;
                const uint64_t h_desc = h_base + (uint64_t)((hs * Sh::kHalf) >> 4);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    ok = ok && wait(p_bar + 8 * half, p_par, dead);
                    if (!ok) continue;
                    tc_after();
                    if (one) {
#pragma unroll
                        for (int s = 0; s < kStep / 16; ++s)   // 16 tokens a step: 8 columns of weights, two groups of 8 token rows
                            mma_values(o_mine, s_mine + half * kStep + 8 * s, h_desc + (uint64_t)((half * kStep * 128 + s * 2048) >> 4),
                                       idesc_f16_bt(DIM), (half | s) != 0 || j > 0);
                        if (more) scores(half);
                        mma_commit(s_bar + 8 * half);   // the scores two steps on, and the output up to this step
                    }
                }
                if (one) {
                    mma_commit(h_empty + 8 * hs);
                    if (more) mma_commit(k_empty + 8 * ks);
                }
                if (more) next_keys();
                if (++hs == kHalfStages) {
                    hs = 0;
                    h_par ^= 1u;
                }
                p_par ^= 1u;
            }
            if (!ok) {   // what has been issued ends before the tensor memory is given up
                if (one) mma_commit(k_empty);
                (void)mbar_wait_bounded(k_empty, 0, 1u << 14);
                (void)mbar_wait_bounded(k_empty, 1, 1u << 14);
            }
        }
    } else if (warp >= 4 && warp < 8) {
        // ---- values to f16 ----
        MXN_FEW_REGISTERS();
        const int t = threadIdx.x - 128;   // token row of the tile
        bool ok = true;
        for (int j = 0; j < tiles; ++j) {
            const int vs = j % kValStages, hs = j % kHalfStages;
            ok = wait(v_full + 8 * vs, (uint32_t)(j / kValStages) & 1u, dead) && wait(sc_full + 8 * (j % kScaleSlots), (uint32_t)(j / kScaleSlots) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            const int place = k0 + j * kTile + t;
            const bool real = place >= seen && place < k1 && ((scales[j % kScaleSlots].readable >> (t / kRun)) & 1u);
            if (j >= kHalfStages) ok = wait(h_empty + 8 * hs, (uint32_t)(j / kHalfStages - 1) & 1u, dead);
            if (!__all_sync(0xFFFFFFFFu, ok)) break;
            const uint32_t src = base + Sh::kV + vs * Sh::kCodes + (uint32_t)t * DIM;
            // panels of 64 dimensions: [token][128 bytes], 128-byte swizzle
            const uint32_t dst = base + Sh::kH + hs * Sh::kHalf + (uint32_t)t * 128;
#pragma unroll
            for (int i = 0; i < DIM / 16; ++i) {
                uint4 w = lds_v4(src + (uint32_t)((DIM == 128 ? i ^ (t & 7) : i ^ ((t >> 1) & 3)) << 4));
                if (!real) w = make_uint4(0, 0, 0, 0);
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
                uint32_t o[8];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u[x] & 0xFFFFu), __NV_E4M3);
                    const __half2_raw c = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(u[x] >> 16), __NV_E4M3);
                    o[2 * x] = (uint32_t)a.x | ((uint32_t)a.y << 16);
                    o[2 * x + 1] = (uint32_t)c.x | ((uint32_t)c.y << 16);
                }
                const uint32_t panel = dst + (uint32_t)(i / 4) * (kTile * 128);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const uint32_t at = panel + (uint32_t)(((2 * (i % 4) + x) ^ (t & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(o[4 * x]), "r"(o[4 * x + 1]), "r"(o[4 * x + 2]), "r"(o[4 * x + 3]) : "memory");
                }
            }
            fence_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(v_empty + 8 * vs);
                mbar_arrive(h_full + 8 * hs);
            }
        }
    } else if (warp >= 8 && (rt == 0 || two)) {
        // ---- softmax ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 200;");
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t o_at = o_col[rt] + lanes;
        const int row = row0 + rt * kTile + r_in;
        const bool row_live = row < rows;
        const int q_tok = row_live ? P.by_group(row) : 0;
        const int64_t tok = q0 + q_tok;
        const int head = h * G + (row_live ? row - q_tok * G : 0);
        const float row_factor = row_factors[rt * kTile + r_in];
        const int pos = shift + (row_live ? q_tok : nq - 1);
        const int see_hi = P.causal ? min(pos + 1, len) : len;
        const int see_lo = first_seen(pos, P.window);
        const float kNone = -INFINITY;
        float ref = kNone, top_all = kNone, l = 0.0f, c0 = 0.0f;
        // l's unit is 2^(ref - kTop - c0) until a tile is wide or c0 changes; from then on (`by_own`) 2^sum_ref, and `unit` the former in the
        // latter.  Where ref lies so far above the scores (a wide tile's larger scales) that weights vanish which the sum has to count, the
        // warp sums by exponentials of their own (`slow`).
        float sum_ref = kNone, unit = 1.0f;
        bool ok = true, by_own = false, slow = false;
        const int steps = 2 * tiles;
        // a row that nothing hides in a step needs no mask: the range that holds for the warp's rows
        const int all_lo = __reduce_max_sync(0xFFFFFFFFu, see_lo), all_hi = __reduce_min_sync(0xFFFFFFFFu, min(see_hi, k1));
        bool here = false, scales_here = false;
        for (int i = 0; i < steps; ++i) {
            const int j = i >> 1, buf = i & 1;
            const TileScales& slot = scales[j % kScaleSlots];
            if (!here && !__all_sync(0xFFFFFFFFu, wait(s_full + 16 * rt + 8 * buf, (uint32_t)j & 1u, dead))) ok = false;
            if (!buf && !scales_here && !__all_sync(0xFFFFFFFFu, wait(sc_full + 8 * (j % kScaleSlots), (uint32_t)(j / kScaleSlots) & 1u, dead))) ok = false;
            if (!ok) break;
            tc_after();
            const uint32_t s_at = s_col[rt] + lanes + buf * kStep;
            const int t0 = k0 + i * kStep;
            uint32_t x[2][32];
            tm_request(x[0], s_at);
            tm_request(x[1], s_at + 32);
            const float4 k4 = *reinterpret_cast<const float4*>(slot.k + 4 * buf), v4 = *reinterpret_cast<const float4*>(slot.v + 4 * buf),
                         l4 = *reinterpret_cast<const float4*>(slot.l + 4 * buf);
            const float slot_k[4] = {k4.x, k4.y, k4.z, k4.w}, slot_v[4] = {v4.x, v4.y, v4.z, v4.w}, slot_l[4] = {l4.x, l4.y, l4.z, l4.w};
            const uint32_t readable = (slot.readable >> (4 * buf)) & 0xFu;
            const uint32_t special = slot.apart & (kWide | (buf ? 0u : kMoved));
            // bit e: the row sees token 32 c + e of the step
            auto visible = [&](int c) -> uint32_t {
                const int tc = t0 + 32 * c, up = min(max(min(see_hi, k1) - tc, 0), 32), down = min(max(see_lo - tc, 0), 32);
                const uint32_t below = up == 32 ? 0xFFFFFFFFu : (1u << up) - 1u, above = down == 32 ? 0u : 0xFFFFFFFFu << down;
                return below & above & (((readable >> (2 * c)) & 1u ? 0xFFFFu : 0u) | ((readable >> (2 * c + 1)) & 1u ? 0xFFFF0000u : 0u));
            };
            const bool all = t0 >= all_lo && t0 + kStep <= all_hi && readable == 0xFu;
            float fac[4], utop = kNone;
#pragma unroll
            for (int g = 0; g < 4; ++g) fac[g] = fmaxf(row_factor * slot_k[g], 1.17549435e-38f);
            tm_arrived(x[0]);
            tm_arrived(x[1]);
            if (!all) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const uint32_t see = visible(c);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!((see >> e) & 1u)) x[c][e] = 0xFF800000u;   // -infinity; a factor is never 0, so it stays that
                }
            }
            // the step's largest s + sv, and the reference
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t* const y = &x[g >> 1][16 * (g & 1)];
                float m = max3(y[0], y[1], y[2]);
#pragma unroll
                for (int e = 3; e < 15; e += 2) m = max3(__float_as_uint(m), y[e], y[e + 1]);
                m = max_nan(m, __uint_as_float(y[15]));
                utop = max_nan(utop, fmaf(m, fac[g], slot_v[g]));
            }
            top_all = fmaxf(top_all, utop);
            const bool move = utop > ref + kUp || (utop < ref - kDown && utop > kNone);   // (ref + kUp is -infinity without a reference)
            float counts = unit;   // what the step's weights count in the sum
            if (__any_sync(0xFFFFFFFFu, move || special || slow)) {   // one branch for all that is rare
                const bool summed = slow || (special && (i > 0 || (special & kWide)));
                if (summed && !by_own) {
                    by_own = true;
                    if (ref > kNone) sum_ref = ref - kTop - c0;
                }
                c0 = slot.c0;
                // from the scores as they still stand, by the whole warp
                float ztop = kNone;
#pragma unroll 1
                for (int pass = 0; summed && pass < 2; ++pass) {
#pragma unroll 1
                    for (int g = 0; g < 4; ++g) {
                        uint32_t z[16];
                        tm_load16(z, s_at + 16 * g);
                        const uint32_t see = visible(g >> 1) >> (16 * (g & 1));
                        const float f = fmaxf(row_factor * slot.k[4 * buf + g], 1.17549435e-38f);
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float s = (see >> e) & 1u ? __uint_as_float(z[e]) * f : kNone;
                            if (pass == 0) ztop = fmaxf(ztop, s);
                            else if (sum_ref > kNone) l += ex2(s - sum_ref);
                        }
                    }
                    if (pass == 0 && ztop > sum_ref + kLift) {
                        const float next = ceilf(ztop);
                        if (sum_ref > kNone) l = times_pow2(l, sum_ref - next);
                        sum_ref = next;
                    }
                }
                float next = ref;
                if (utop > ref + kUp) next = ceilf(utop);
                else if (utop < ref - kDown && utop > kNone) next = ceilf(fmaxf(utop, top_all - kDepth));
                const bool up = next > ref;
                const float alpha = ref == kNone ? 0.0f : ex2(ref - next);
                l *= by_own ? 1.0f : alpha;
                ref = next;
                if (by_own) {
                    float d = ref == kNone ? 0.0f : ref - kTop - c0 - sum_ref;
                    if (d > kApart && up && !(special & kWide)) {   // ref comes from a score of this step within kApart of it
                        if (sum_ref > kNone) l = times_pow2(l, -d);
                        sum_ref = ref - kTop - c0;
                        d = 0.0f;
                    }
                    unit = ex2(fminf(d, kApart));
                    slow = __any_sync(0xFFFFFFFFu, d > kApart);
                }
                counts = summed ? 0.0f : unit;
                if (i > 0 && __any_sync(0xFFFFFFFFu, move)) {   // the output up to the last step: its end is signalled with the next step's scores
                    ok = wait(s_full + 16 * rt + 8 * (buf ^ 1), (uint32_t)((i + 1) >> 1) & 1u, dead);
                    if (!__all_sync(0xFFFFFFFFu, ok)) break;
                    tc_after();
#pragma unroll 1
                    for (int c = 0; c < DIM / 16; ++c) {
                        uint32_t z[16];
                        tm_load16(z, o_at + 16 * c);
#pragma unroll
                        for (int e = 0; e < 16; ++e) z[e] = __float_as_uint(__uint_as_float(z[e]) * alpha);
                        tm_store16(o_at + 16 * c, z);
                    }
                }
            }
            // weights, over their scores
            // a NaN among the scores reaches all of the step's weights: the polynomial below would take it for a small number
            const float shift_by = utop != utop ? utop : ref == kNone ? 0.0f : kTop - ref;
            uint32_t w[32];
            float more = 0.0f;
            bool probe[3];
            probe[2] = mbar_test(sc_full + 8 * ((i + 1) / 2 % kScaleSlots), (uint32_t)((i + 1) / 2 / kScaleSlots) & 1u);
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const uint32_t* const y = &x[g >> 1][16 * (g & 1)];
                const float2 f = f2(fac[g]), add = f2(slot_v[g] + shift_by);
                float2 sum[2] = {f2(0.0f), f2(0.0f)};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 u = __ffma2_rn(make_float2(__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])), f, add);
                    // one pair in eight by the multipliers: the special function units are the busier ones (none 450 us, one 437, two 454)
                    const float2 p = e == 7 ? ex2_fma(u) : make_float2(ex2(u.x), ex2(u.y));
                    sum[e & 1] = __fadd2_rn(sum[e & 1], p);
                    const __half2 q = __floats2half2_rn(p.x, p.y);
                    w[8 * g + e] = *reinterpret_cast<const uint32_t*>(&q);
                }
                const float2 both = __fadd2_rn(sum[0], sum[1]);
                more = fmaf(both.x + both.y, slot_l[g], more);
                if (g & 1) probe[g >> 1] = mbar_test(s_full + 16 * rt + 8 * (buf ^ 1), (uint32_t)((i + 1) >> 1) & 1u);
            }
            l = fmaf(more, counts, l);   // (a NaN among the weights reaches the sum all the same)
            tm_store32(s_at, w);
            here = __all_sync(0xFFFFFFFFu, i + 1 < steps && (probe[0] || probe[1]));
            scales_here = __all_sync(0xFFFFFFFFu, probe[2]);
            tm_store_wait();
            tc_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full + 16 * rt + 8 * buf);
        }
        // ---- output ----
        if (ok && tiles > 0) ok = wait(s_full + 16 * rt + 8, (uint32_t)tiles & 1u, dead);   // behind the last step's product
        ok = __all_sync(0xFFFFFFFFu, ok);
        tc_after();
        // out = acc 2^c0 / l;  log2 of the softmax's sum = log2 l + R - 1 - c0.  Summed apart, with a reference r of l: out = acc 2^(R - 1 - r) / l,
        // the power in two factors, since it may lie outside binary32's range where the product does not
        const bool some = ref > kNone || l != l;   // (NaN scores set no reference)
        float inv = some ? __fdiv_rn(ex2(c0), l) : 0.0f, inv2 = 1.0f, lse2 = some ? log2f(l) + (ref - kTop - c0) : kNone;
        if (by_own && ref > kNone) {
            const int e = min(max((int)(__float_as_uint(l) >> 23) - 127, -126), 127);
            const float d = ref - kTop - sum_ref - (float)e, half = floorf(0.5f * d);
            inv = __fdiv_rn(ex2(half), times_pow2(l, (float)-e));   // l in [1, 2)
            inv2 = ex2(d - half);
            lse2 = log2f(l) + sum_ref;
        }
        const int64_t out_row = tok * P.q_heads + head;
        const uint32_t out_at = base + Sh::kQ + (uint32_t)(warp - 8) * 32 * 2 * DIM;
#pragma unroll
        for (int c = 0; c < DIM / 32; ++c) {
            uint32_t x[32];
            if (tiles > 0) {
                tm_load(x, o_at + 32 * c);
            }
            __syncwarp();
            float* const o = reinterpret_cast<float*>(x);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] = some ? o[e] * inv * inv2 : 0.0f;
            if (P.splits == 1) {   // to shared memory (q's, which no product reads any more): 16-byte pieces, as swizzled as its rows are long
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t r[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const __nv_bfloat162 v = __floats2bfloat162_rn(o[8 * e + 2 * i], o[8 * e + 2 * i + 1]);
                        r[i] = *reinterpret_cast<const uint32_t*>(&v);
                    }
                    const uint32_t at = out_at + (uint32_t)lane * 2 * DIM + (uint32_t)(((4 * c + e) ^ (lane & 7)) << 4);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" :: "r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]) : "memory");
                }
            } else if (row_live && some) {
                float* const y = P.part_out + (out_row * P.splits + split) * DIM + 32 * c;
#pragma unroll
                for (int e = 0; e < 8; ++e) *reinterpret_cast<float4*>(y + 4 * e) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
            }
            __syncwarp();
        }
        if (P.splits == 1) {   // and from there a row in one piece
            constexpr int kLanes = DIM / 8, kAtOnce = 32 / kLanes;
            const int c = lane % kLanes;
#pragma unroll 4
            for (int i = 0; i < 32; i += kAtOnce) {
                const int r = i + lane / kLanes, rr = row0 + (warp - 8) * 32 + r;
                const uint4 v = lds_v4(out_at + (uint32_t)r * 2 * DIM + (uint32_t)((c ^ (r & 7)) << 4));
                if (rr < rows) {
                    const int t = P.by_group(rr);
                    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
                    st_v4(P.out + (q0 + t) * P.out_stride + (int64_t)(h * G + rr - t * G) * DIM + 8 * c, u);
                }
            }
        }
        if (row_live) {
            if (P.splits > 1) P.part_lse[out_row * P.splits + split] = lse2;
            else if (P.lse != nullptr) P.lse[out_row] = lse2 * kLn2;
        }
        tc_before();
    } else {
        MXN_FEW_REGISTERS();
    }
    __syncthreads();
    if (threadIdx.x == 0 && dead_flag) {
        // a wait ran out: the copies in flight get a second, shorter wait before the shared memory is given up
        atomicAdd(&g_prompt_timeouts, 1u);
        for (int i = 0; i < kKeyStages + kValStages; ++i) {
            const uint32_t bar = i < kKeyStages ? k_full + 8 * i : v_full + 8 * (i - kKeyStages);
            (void)mbar_wait_bounded(bar, 0, 1u << 14);
            (void)mbar_wait_bounded(bar, 1, 1u << 14);
        }
    }
    __syncwarp();
    if (warp == 1) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" :: "r"(tmem) : "memory");
    }
}

template <int DIM>
cudaError_t launch_dim(const AttnParams& P, const AttnMaps& M, int64_t ctas, cudaStream_t stream)
{
    const int smem = PromptShape<DIM>::kSmem;
    const cudaError_t e = cudaFuncSetAttribute(attn_prompt_kernel<DIM>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, attn_prompt_kernel<DIM>, P, M);
}

}  // namespace

cudaError_t launch_prompt(const AttnParams& P, const AttnMaps& M, int64_t ctas, cudaStream_t stream)
{
    return P.dim == 128 ? launch_dim<128>(P, M, ctas, stream) : launch_dim<64>(P, M, ctas, stream);
}

cudaError_t read_prompt_counters(unsigned int* timeouts, unsigned int* bad)
{
    const cudaError_t e = cudaMemcpyFromSymbol(timeouts, g_prompt_timeouts, sizeof(unsigned int));
    return e != cudaSuccess ? e : cudaMemcpyFromSymbol(bad, g_prompt_bad, sizeof(unsigned int));
}
cudaError_t reset_prompt_counters(bool timeouts)
{
    const unsigned int zero = 0;
    return timeouts ? cudaMemcpyToSymbol(g_prompt_timeouts, &zero, sizeof(unsigned int)) : cudaMemcpyToSymbol(g_prompt_bad, &zero, sizeof(unsigned int));
}

}  // namespace mxn
