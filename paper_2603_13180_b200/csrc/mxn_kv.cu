// Append of keys and values to a paged cache of E4M3 codes with one E8M0 scale for each block of tokens and head.
//
//   k' = R(position) k (when a rotation is given);  S = 2^(ceil(log2 absmax) - 8) over a block's tokens of one head;
//   codes = E4M3(k' / S).
// A block that already holds earlier tokens keeps at least its scale; where the new tokens raise it, the earlier codes are
// rounded again on the new scale (exact but for codes that become subnormal).  Power-of-two scales are what makes appending
// one token at a time cheap and repeatable: appending the same tokens to the same places again changes nothing.
//
// One warp owns one (block of tokens, head) of the keys or of the values, so that no two warps ever meet in a block and no
// atomic is needed.  A warp is given a run of token rows and works on the blocks whose first new token lies in its run; the
// first 16 tokens (8 of heads beyond 128) of a block are copied to shared memory all at once and read there for the maximum and
// for the codes, the others are read again from L1.  The run's rows are asked into L2 while the warp looks up its sequence.
//
// Bound: HBM, 3 bytes an element (2 read, 1 written); a decode step of a few tokens is bound by the latency of one warp's chain of
// loads.  Measured, 8 heads of 128 in blocks of 16: six prompts of up to 4096 tokens 31 us, 3.5 TB/s, which is no bound: a warp does one
// block of one head and ends, so that its chain of loads (sequence, length, page, rows, angles) hides behind no other block of its own;
// half of the issue slots are busy.  One token for each of 64 sequences 4.0 us.
#include "mxn_async.cuh"
#include "mxn_internal.h"
#include "mxn_rope.cuh"

namespace mxn {

namespace {

constexpr int kWarps = 4;

__device__ unsigned int g_kv_bad = 0;   // blocks whose page, position or length is out of range

// index of the sequence that row j belongs to: the last s with cu[s] <= j, found 32 probes at a time
__device__ __forceinline__ int find_sequence(const int32_t* cu, int seqs, int j, int lane)
{
    int lo = 0, n = seqs;   // the answer is in [lo, lo + n)
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const bool below = lane * step < n && __ldg(cu + at) <= j;
        const unsigned b = __ballot_sync(0xFFFFFFFFu, below);
        const int k = b ? 31 - __clz(b) : 0;
        lo += k * step;
        n = min(step, n - k * step);
    }
    return lo;
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}

__device__ __forceinline__ float largest(float top, const Lane16& x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
        top = fmaxf(fmaxf(fmaxf(top, fabsf(x.a[i].x)), fmaxf(fabsf(x.a[i].y), fabsf(x.b[i].x))), fabsf(x.b[i].y));
    return top;
}

// 16 bytes to shared memory, or zeros (bytes = 0)
__device__ __forceinline__ void copy16(uint32_t dst, const uint16_t* src, int bytes)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(dst), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void sts_v4(uint32_t at, float2 a, float2 b)
{
    asm volatile("st.shared.v4.f32 [%0], {%1,%2,%3,%4};" :: "r"(at), "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y) : "memory");
}

// four E4M3 bytes -> binary32
__device__ __forceinline__ void e4m3x4_to_f32(uint32_t w, float* f)
{
    uint32_t a, b;
    asm("{ .reg .b16 lo, hi; mov.b32 {lo, hi}, %2; cvt.rn.f16x2.e4m3x2 %0, lo; cvt.rn.f16x2.e4m3x2 %1, hi; }" : "=r"(a), "=r"(b) : "r"(w));
    asm("{ .reg .f16 lo, hi; mov.b32 {lo, hi}, %2; cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi; }" : "=f"(f[0]), "=f"(f[1]) : "r"(a));
    asm("{ .reg .f16 lo, hi; mov.b32 {lo, hi}, %2; cvt.f32.f16 %0, lo; cvt.f32.f16 %1, hi; }" : "=f"(f[2]), "=f"(f[3]) : "r"(b));
}

template <int LP, bool PAIRS>
__global__ void __launch_bounds__(kWarps * 32, 6) kv_append_kernel(const KvAppendParams P)
{
    constexpr int G = 32 / LP;   // tokens a warp holds at a time
    constexpr int kStaged = LP == 16 ? 8 : 16;        // tokens of a block that go through shared memory
    constexpr int kTurns = G < kStaged ? kStaged / G : 1, kTurnBytes = 2048;
    __shared__ __align__(16) uint8_t staged[kWarps][kTurns * kTurnBytes];
    pdl_prologue();
    const int lane = threadIdx.x & 31, sub = lane % LP, grp = lane / LP;
    const uint32_t stage = smem_u32(staged[threadIdx.x >> 5]) + lane * 16;
    const int hv = (int)blockIdx.y * kWarps + (threadIdx.x >> 5);   // keys' heads, then values' heads
    if (hv >= 2 * P.heads) return;
    const int which = hv >= P.heads, h = hv - which * P.heads;
    const bool rotate = which == 0 && P.cos_sin != nullptr;
    const bool live = 16 * sub < P.dim;
    const int rot = rotate ? P.rot : 0;
    const LanePairs lp = lane_pairs(live ? sub : 0, P.dim, rot, PAIRS);
    const int n = (int)P.n, rows = min(__ldg(P.cu + P.seqs), n), first_row = __ldg(P.cu);
    int j = (int)blockIdx.x * P.run;
    const int j_end = min(j + P.run, rows);
    {
        const int per_row = (2 * P.dim + 127) / 128;   // lines of a head
        for (int i = lane; i < P.run * per_row; i += 32) {
            const int row = j + i / per_row;
            if (row < n) {
                const char* at = reinterpret_cast<const char*>(P.x[which] + row * P.x_stride[which] + h * P.dim) + 128 * (i % per_row);
                asm volatile("prefetch.global.L2 [%0];" :: "l"(at));
            }
        }
    }
    if (j < first_row) j = first_row;
    int s = -1, c0 = 0, c1 = 0, start = 0;
    while (j < j_end) {
        if (s < 0 || j >= c1) {
            s = find_sequence(P.cu, P.seqs, j, lane);
            c0 = __ldg(P.cu + s);
            const int c_end = __ldg(P.cu + s + 1);
            c1 = min(c_end, rows);
            start = (int)max((int64_t)-1, (int64_t)__ldg(P.lens + s) - ((int64_t)c_end - c0));   // place of the sequence's first new token
            if (c0 < 0 || j < c0 || j >= c1) {   // no sequence holds this row (cu is not a rising list): leave it
                ++j;
                s = -1;
                continue;
            }
        }
        if (start < 0) {   // more new tokens than the sequence is long
            if (lane == 0 && j == c0) atomicAdd(&g_kv_bad, 1u);
            j = c1;
            continue;
        }
        const int pos = start + (j - c0), in_block = pos & (P.block - 1), count = min(P.block - in_block, c1 - j);
        if (in_block != 0 && j != c0) {   // the block belongs to the warp of its first new token
            j += count;
            continue;
        }
        const int page_at = pos >> P.page_shift;
        const int page = page_at < P.max_pages ? __ldg(P.page_table + s * P.max_pages + page_at) : -1;
        if (page < 0 || page >= P.num_pages || (rotate && (int64_t)pos + count > P.table_rows)) {
            if (lane == 0) atomicAdd(&g_kv_bad, 1u);
            j += count;
            continue;
        }
        const int off = pos & (P.page - 1);   // of the first new token within its page
        const int64_t tile = (int64_t)page * P.heads + h;
        uint8_t* const codes = P.codes[which] + (tile * P.page + (off - in_block)) * P.dim;   // the block's first token
        uint8_t* const scale = P.scales[which] + (tile << (P.page_shift - P.block_shift)) + (off >> P.block_shift);
        const uint16_t* const x0 = P.x[which] + j * P.x_stride[which] + h * P.dim;

        // The block's first kStaged tokens on their way to shared memory all at once; a thread reads back only its own pieces.
        // Rotated elements are left there in binary32 for the second reading.
#pragma unroll
        for (int k = 0; k < kTurns; ++k) {
            const int i = k * G + grp, bytes = live && i < count ? 16 : 0;
            const uint16_t* p = x0 + (bytes ? i : 0) * P.x_stride[which];
            copy16(stage + k * kTurnBytes, p + lp.o0, bytes);
            copy16(stage + k * kTurnBytes + 512, p + lp.o1, bytes);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        const bool turns = rot != 0 && lp.turns;
        const float* const angles = P.cos_sin + (int64_t)pos * rot;
        auto load = [&](int i, uint32_t at, Lane16& x) {   // token i of the new ones, rotated
            uint4 w[2];
            if (i < kStaged) {
                w[0] = lds_v4(at);
                w[1] = lds_v4(at + 512);
            } else {
                w[0] = w[1] = make_uint4(0u, 0u, 0u, 0u);
                if (live && i < count) {
                    const uint16_t* p = x0 + i * P.x_stride[which];
                    w[0] = __ldg(reinterpret_cast<const uint4*>(p + lp.o0));
                    w[1] = __ldg(reinterpret_cast<const uint4*>(p + lp.o1));
                }
            }
            unpack<PAIRS>(x, w);
            if (turns && i < count) {
                Turn turn;
                load_turn<PAIRS>(turn, angles + i * rot, lp, rot);
                apply_turn<false, false, PAIRS>(x, turn, lp);
            }
        };
        float top = 0.0f;
        uint32_t at = stage;
#pragma unroll 2
        for (int i = grp; i - grp < count; i += G, at += kTurnBytes) {
            Lane16 x;
            load(i, at, x);
            top = largest(top, x);
            if (turns && i < kStaged) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    sts_v4(at + 512 * e, x.a[2 * e], x.a[2 * e + 1]);
                    sts_v4(at + 1024 + 512 * e, x.b[2 * e], x.b[2 * e + 1]);
                }
            }
        }
        uint32_t sb = e8m0_scale_rceil_pow2<8>(warp_max(top));
        if (in_block != 0) {
            const uint32_t old = *scale;
            if (old >= sb) {
                sb = old;
            } else if (old != sb) {
                // earlier tokens on the new scale; 2^(old - sb) below 2^-126 leaves nothing of any code
                const int d = (int)sb - (int)old;
                const float by = d > 126 ? 0.0f : __uint_as_float((uint32_t)(127 - d) << 23);
                for (int i = grp; i < in_block; i += G) {
                    if (!live) continue;
                    uint4* p = reinterpret_cast<uint4*>(codes + i * P.dim + 16 * sub);
                    uint4 w = *p;
                    uint32_t* v = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float f[4];
                        e4m3x4_to_f32(v[e], f);
                        v[e] = cvt_e4m3x4(__fmul_rn(f[0], by), __fmul_rn(f[1], by), __fmul_rn(f[2], by), __fmul_rn(f[3], by));
                    }
                    *p = w;
                }
            }
        }
        __syncwarp();
        if (lane == 0) *scale = (uint8_t)sb;
        const float inv = inv_scale(sb);
        auto store = [&](int i, Lane16& x) {
            if (!live || i >= count) return;
            const float2 f = make_float2(inv, inv);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                x.a[e] = __fmul2_rn(x.a[e], f);
                x.b[e] = __fmul2_rn(x.b[e], f);
            }
            uint32_t w[4];
            if (PAIRS) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = cvt_e4m3x4(x.a[e].x, x.b[e].x, x.a[e].y, x.b[e].y);
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    w[e] = cvt_e4m3x4(x.a[2 * e].x, x.a[2 * e].y, x.a[2 * e + 1].x, x.a[2 * e + 1].y);
                    w[2 + e] = cvt_e4m3x4(x.b[2 * e].x, x.b[2 * e].y, x.b[2 * e + 1].x, x.b[2 * e + 1].y);
                }
            }
            uint8_t* y = codes + (in_block + i) * P.dim;
            if (lp.o1 == lp.o0 + 8) {
                st_v4(y + lp.o0, w);
            } else {
                st_v2(y + lp.o0, w);
                st_v2(y + lp.o1, w + 2);
            }
        };
        at = stage;
#pragma unroll 2
        for (int i = grp; i - grp < count; i += G, at += kTurnBytes) {
            Lane16 x;
            if (turns && i < kStaged) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    *reinterpret_cast<uint4*>(&x.a[2 * e]) = lds_v4(at + 512 * e);
                    *reinterpret_cast<uint4*>(&x.b[2 * e]) = lds_v4(at + 1024 + 512 * e);
                }
            } else {
                load(i, at, x);
            }
            store(i, x);
        }
        j += count;
    }
}

template <int LP>
cudaError_t launch_lp(const KvAppendParams& P, cudaStream_t stream)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((P.n + P.run - 1) / P.run), (unsigned)((2 * P.heads + kWarps - 1) / kWarps));
    cfg.blockDim = dim3(kWarps * 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return P.pairs ? cudaLaunchKernelEx(&cfg, kv_append_kernel<LP, true>, P) : cudaLaunchKernelEx(&cfg, kv_append_kernel<LP, false>, P);
}

}  // namespace

cudaError_t launch_kv_append(KvAppendParams P, cudaStream_t stream)
{
    // rows a warp looks after: a block's worth for prompts; one where sequences bring about one token each, so that each
    // block has a warp of its own
    P.run = P.n >= (int64_t)P.seqs * P.block ? P.block : 1;
    switch (lanes_per_head(P.dim)) {
        case 1: return launch_lp<1>(P, stream);
        case 2: return launch_lp<2>(P, stream);
        case 4: return launch_lp<4>(P, stream);
        case 8: return launch_lp<8>(P, stream);
        default: return launch_lp<16>(P, stream);
    }
}

cudaError_t read_kv_bad(unsigned int* out) { return cudaMemcpyFromSymbol(out, g_kv_bad, sizeof(unsigned int)); }
cudaError_t reset_kv_bad()
{
    const unsigned int zero = 0;
    return cudaMemcpyToSymbol(g_kv_bad, &zero, sizeof(unsigned int));
}

}  // namespace mxn
