// extern "C" entry points of libmxnorm: argument checks and dispatch only.
#include <mutex>

#include "../../include/mxnorm.h"
#include "mxn_internal.h"

namespace {

inline bool misaligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) != 0; }

// the paper's printed correction constants RMS / G_p for Gaussian blocks (implementation appendix)
float paper_coef(int B, int p)
{
    switch (B * 4 + p) {
        case 16 * 4 + 1: return 0.4814f;
        case 16 * 4 + 2: return 0.4688f;
        case 32 * 4 + 1: return 0.4261f;
        case 32 * 4 + 2: return 0.4185f;
        case 64 * 4 + 1: return 0.3852f;
        case 64 * 4 + 2: return 0.3803f;
        default: return 0.0f;
    }
}

mxn_status check_common(const void* x, int64_t T, int64_t D, int B, const void* codes, const void* scales,
                        int round, int layout)
{
    if (T < 0 || D <= 0 || !mxn::fwd_shape_supported(D, B)) return MXN_ERR_SHAPE;
    if (round < 0 || round > MXN_ROUND_RCEIL_MAX) return MXN_ERR_ENUM;
    if (layout != MXN_SCALES_ROWMAJOR && layout != MXN_SCALES_SWIZZLE_128x4) return MXN_ERR_ENUM;
    if (T == 0) return MXN_OK;
    if (x == nullptr || codes == nullptr || scales == nullptr) return MXN_ERR_NULL;
    if (misaligned(x, 32) || misaligned(codes, 32)) return MXN_ERR_ALIGN;
    return MXN_OK;
}

// padding bytes of a tiled scale buffer are defined to be zero: clear the buffer when it has any
cudaError_t clear_scale_padding(void* scales, int64_t T, int64_t K, int layout, cudaStream_t s)
{
    if (layout == MXN_SCALES_SWIZZLE_128x4 && (T % 128 != 0 || K % 4 != 0))
        return cudaMemsetAsync(scales, 0, mxn_scale_bytes(T, K, MXN_SCALES_SWIZZLE_128x4), s);
    return cudaSuccess;
}

mxn_status run_fwd(int stat, bool nvfp4, const void* x, const void* gain, int64_t T, int64_t D, int B, int p,
                   float coef, float eps, float global_scale, void* codes, void* scales, float* rms,
                   int round, int layout, void* stream, int elem = mxn::ELEM_E4M3)
{
    mxn_status st = check_common(x, T, D, B, codes, scales, round, layout);
    if (st != MXN_OK || T == 0) return st;
    if (gain != nullptr && misaligned(gain, 16)) return MXN_ERR_ALIGN;
    if (rms != nullptr && misaligned(rms, 4)) return MXN_ERR_ALIGN;
    if (stat == mxn::STAT_MX) {
        if (p != 1 && p != 2) return MXN_ERR_SHAPE;
        if (coef == 0.0f) coef = paper_coef(B, p);
    }
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    mxn::FwdParams P{};
    P.x = static_cast<const uint16_t*>(x);
    P.gain = static_cast<const uint16_t*>(gain);
    P.codes = static_cast<uint8_t*>(codes);
    P.scales = static_cast<uint8_t*>(scales);
    P.rms_out = rms;
    P.T = T;
    P.D = (int)D;
    P.K = (int)(D / B);
    P.p = p;
    P.coef = coef;
    P.eps = eps;
    P.global_scale = global_scale;
    P.round = round;
    P.layout = layout;
    P.elem = nvfp4 ? mxn::ELEM_E2M1 : elem;
    if (clear_scale_padding(scales, T, P.K, layout, s) != cudaSuccess) return MXN_ERR_CUDA;
    return mxn::launch_fwd(P, B, stat, nvfp4, s) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t mxn_scale_bytes(int64_t T, int64_t K, mxn_scale_layout layout)
{
    if (T < 0 || K < 0) return 0;
    if (layout == MXN_SCALES_ROWMAJOR) return (size_t)T * (size_t)K;
    if (layout == MXN_SCALES_SWIZZLE_128x4) return (size_t)((T + 127) / 128) * (size_t)((K + 3) / 4) * 512;
    return 0;
}

const char* mxn_status_string(mxn_status s)
{
    switch (s) {
        case MXN_OK: return "ok";
        case MXN_ERR_NULL: return "a required pointer is NULL";
        case MXN_ERR_SHAPE: return "unsupported shape, block size or p";
        case MXN_ERR_ALIGN: return "a pointer is not aligned as required";
        case MXN_ERR_ENUM: return "unknown rounding mode or scale layout";
        case MXN_ERR_WORKSPACE: return "workspace missing or too small";
        case MXN_ERR_CUDA: return "CUDA runtime error at launch";
        case MXN_ERR_TIMEOUT: return "a bounded device-side wait ran out";
        case MXN_ERR_TOO_LARGE: return "the problem needs more built-in scratch than the library holds";
        case MXN_ERR_INDEX: return "an index held in device memory was out of range";
        default: return "unknown status";
    }
}

mxn_status mxn_device_timeouts(unsigned int* count_out)
{
    unsigned int n = 0, attn = 0, bad = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || mxn::read_timeouts(&n) != cudaSuccess ||
        mxn::read_attn_counters(&attn, &bad) != cudaSuccess)
        return MXN_ERR_CUDA;
    n += attn;
    if (count_out != nullptr) *count_out = n;
    return n == 0 ? MXN_OK : MXN_ERR_TIMEOUT;
}

mxn_status mxn_device_timeouts_reset(void)
{
    return cudaDeviceSynchronize() == cudaSuccess && mxn::reset_timeouts() == cudaSuccess &&
                   mxn::reset_attn_timeouts() == cudaSuccess
               ? MXN_OK : MXN_ERR_CUDA;
}

mxn_status mxn_device_bad_indices(unsigned int* count_out)
{
    unsigned int heads = 0, kv = 0, attn = 0, timeouts = 0;
    if (cudaDeviceSynchronize() != cudaSuccess || mxn::read_heads_bad(&heads) != cudaSuccess ||
        mxn::read_kv_bad(&kv) != cudaSuccess || mxn::read_attn_counters(&timeouts, &attn) != cudaSuccess)
        return MXN_ERR_CUDA;
    const unsigned int n = heads + kv + attn;
    if (count_out != nullptr) *count_out = n;
    return n == 0 ? MXN_OK : MXN_ERR_INDEX;
}

mxn_status mxn_device_bad_indices_reset(void)
{
    return cudaDeviceSynchronize() == cudaSuccess && mxn::reset_heads_bad() == cudaSuccess &&
                   mxn::reset_kv_bad() == cudaSuccess && mxn::reset_attn_bad() == cudaSuccess
               ? MXN_OK : MXN_ERR_CUDA;
}

mxn_status mxn_selftest_bounded_wait(unsigned int polls, void* cuda_stream)
{
    if (polls == 0 || polls > (1u << 16)) return MXN_ERR_SHAPE;
    return mxn::selftest_bounded_wait(polls, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

mxn_status mxn_selftest_division(unsigned long long* mismatches_out)
{
    unsigned long long n = 0;
    if (mxn::selftest_division(&n) != cudaSuccess) return MXN_ERR_CUDA;
    if (mismatches_out != nullptr) *mismatches_out = n;
    return MXN_OK;
}

mxn_status mxn_selftest_dispatch(int64_t max_D, long long* missing_out, int64_t* first_D_out, int* first_case_out)
{
    if (missing_out == nullptr) return MXN_ERR_NULL;
    if (max_D < 16) return MXN_ERR_SHAPE;
    int64_t first_D = 0;
    int first_case = 0;
    int64_t missing = mxn::selftest_dispatch(max_D, &first_D, &first_case);
    {
        int64_t d = 0;
        int c = 0;
        const int64_t bad = mxn::selftest_bwd_plans(max_D, &d, &c);
        if (missing == 0 && bad != 0) {
            first_D = d;
            first_case = c;
        }
        missing += bad;
    }
    *missing_out = (long long)missing;
    if (first_D_out != nullptr) *first_D_out = first_D;
    if (first_case_out != nullptr) *first_case_out = first_case;
    return MXN_OK;
}

mxn_status mx_cast(const void* x_bf16, int64_t T, int64_t D, int block, void* codes_u8, void* scales_u8,
                   mxn_round round, mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_NONE, false, x_bf16, nullptr, T, D, block, 2, 1.0f, 0.0f, 1.0f, codes_u8, scales_u8,
                   nullptr, round, layout, cuda_stream);
}

mxn_status rmsnorm_mxfp8_fwd(const void* x_bf16, const void* gain_bf16_or_null, int64_t T, int64_t D, int block,
                             float eps, void* codes_u8, void* scales_u8, float* rms_out_or_null,
                             mxn_round round, mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_RMS, false, x_bf16, gain_bf16_or_null, T, D, block, 2, 1.0f, eps, 1.0f, codes_u8,
                   scales_u8, rms_out_or_null, round, layout, cuda_stream);
}

mxn_status mxnorm_fwd(const void* x_bf16, const void* gain_bf16_or_null, int64_t T, int64_t D, int block, int p,
                      float coef_or_0, float eps, void* codes_u8, void* scales_u8, float* rms_est_out_or_null,
                      mxn_round round, mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_MX, false, x_bf16, gain_bf16_or_null, T, D, block, p, coef_or_0, eps, 1.0f, codes_u8,
                   scales_u8, rms_est_out_or_null, round, layout, cuda_stream);
}

mxn_status mxnorm_nvfp4_fwd(const void* x_bf16, int64_t T, int64_t D, int p, float coef_or_0, float eps,
                            float global_scale, void* codes_u8_packed, void* scales_e4m3,
                            float* rms_est_out_or_null, mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_MX, true, x_bf16, nullptr, T, D, 16, p, coef_or_0, eps, global_scale, codes_u8_packed,
                   scales_e4m3, rms_est_out_or_null, MXN_ROUND_RCEIL_POW2, layout, cuda_stream);
}

mxn_status mx_cast_nvfp4(const void* x_bf16, int64_t T, int64_t D, float global_scale, void* codes_u8_packed,
                      void* scales_e4m3, mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_NONE, true, x_bf16, nullptr, T, D, 16, 2, 1.0f, 0.0f, global_scale, codes_u8_packed,
                   scales_e4m3, nullptr, MXN_ROUND_RCEIL_POW2, layout, cuda_stream);
}

mxn_status rmsnorm_nvfp4_fwd(const void* x_bf16, int64_t T, int64_t D, float eps, float global_scale,
                             void* codes_u8_packed, void* scales_e4m3, float* rms_out_or_null,
                             mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_RMS, true, x_bf16, nullptr, T, D, 16, 2, 1.0f, eps, global_scale, codes_u8_packed,
                   scales_e4m3, rms_out_or_null, MXN_ROUND_RCEIL_POW2, layout, cuda_stream);
}

mxn_status mxnorm_add_fwd(const void* x_bf16, const void* residual_bf16, int64_t T, int64_t D, int block, int p,
                          float coef_or_0, float eps, void* h_out_bf16, void* codes_u8, void* scales_u8,
                          float* rms_est_out_or_null, mxn_scale_layout layout, void* cuda_stream)
{
    mxn_status st = check_common(x_bf16, T, D, block, codes_u8, scales_u8, MXN_ROUND_RCEIL_POW2, layout);
    if (st != MXN_OK || T == 0) return st;
    if (residual_bf16 == nullptr || h_out_bf16 == nullptr) return MXN_ERR_NULL;
    if (misaligned(residual_bf16, 32) || misaligned(h_out_bf16, 32)) return MXN_ERR_ALIGN;
    if (p != 1 && p != 2) return MXN_ERR_SHAPE;
    if (rms_est_out_or_null != nullptr && misaligned(rms_est_out_or_null, 4)) return MXN_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    mxn::FwdParams P{};
    P.x = static_cast<const uint16_t*>(x_bf16);
    P.residual = static_cast<const uint16_t*>(residual_bf16);
    P.h_out = static_cast<uint16_t*>(h_out_bf16);
    P.codes = static_cast<uint8_t*>(codes_u8);
    P.scales = static_cast<uint8_t*>(scales_u8);
    P.rms_out = rms_est_out_or_null;
    P.T = T;
    P.D = (int)D;
    P.K = (int)(D / block);
    P.p = p;
    P.coef = coef_or_0 == 0.0f ? paper_coef(block, p) : coef_or_0;
    P.eps = eps;
    P.global_scale = 1.0f;
    P.round = MXN_ROUND_RCEIL_POW2;
    P.layout = layout;
    P.elem = mxn::ELEM_E4M3;
    if (clear_scale_padding(scales_u8, T, P.K, layout, s) != cudaSuccess) return MXN_ERR_CUDA;
    return mxn::launch_fwd(P, block, mxn::STAT_MX, false, s) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

mxn_status mxnorm_postround_fwd(const void* x_bf16, int64_t T, int64_t D, int block, float eps, void* codes_u8,
                                void* scales_u8, float* rms_est_out_or_null, mxn_scale_layout layout, void* cuda_stream)
{
    mxn_status st = check_common(x_bf16, T, D, block, codes_u8, scales_u8, MXN_ROUND_RCEIL_POW2, layout);
    if (st != MXN_OK || T == 0) return st;
    if (mxn::postround_prepare(block) != cudaSuccess) return MXN_ERR_CUDA;
    return run_fwd(mxn::STAT_POSTROUND, false, x_bf16, nullptr, T, D, block, 2, 1.0f, eps, 1.0f, codes_u8, scales_u8,
                   rms_est_out_or_null, MXN_ROUND_RCEIL_POW2, layout, cuda_stream);
}

mxn_status mx_cast_fp4(const void* x_bf16, int64_t T, int64_t D, int block, void* codes_u8_packed, void* scales_u8,
                       mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_NONE, false, x_bf16, nullptr, T, D, block, 2, 1.0f, 0.0f, 1.0f, codes_u8_packed, scales_u8,
                   nullptr, MXN_ROUND_RCEIL_POW2, layout, cuda_stream, mxn::ELEM_E2M1);
}

mxn_status rmsnorm_mxfp4_fwd(const void* x_bf16, int64_t T, int64_t D, int block, float eps, void* codes_u8_packed,
                             void* scales_u8, float* rms_out_or_null, mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_RMS, false, x_bf16, nullptr, T, D, block, 2, 1.0f, eps, 1.0f, codes_u8_packed, scales_u8,
                   rms_out_or_null, MXN_ROUND_RCEIL_POW2, layout, cuda_stream, mxn::ELEM_E2M1);
}

mxn_status mxnorm_mxfp4_fwd(const void* x_bf16, int64_t T, int64_t D, int block, int p, float coef_or_0, float eps,
                            void* codes_u8_packed, void* scales_u8, float* rms_est_out_or_null,
                            mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_MX, false, x_bf16, nullptr, T, D, block, p, coef_or_0, eps, 1.0f, codes_u8_packed, scales_u8,
                   rms_est_out_or_null, MXN_ROUND_RCEIL_POW2, layout, cuda_stream, mxn::ELEM_E2M1);
}

namespace {
mxn_status run_transposed(const void* x_bf16, const float* rms_or_null, int64_t T, int64_t D, float eps, void* codes_t_u8,
                          void* scales_t_u8, int round, int layout, int elem, void* cuda_stream);
}

mxn_status mx_cast_e5m2(const void* x_bf16, int64_t T, int64_t D, int block, void* codes_u8, void* scales_u8,
                        mxn_scale_layout layout, void* cuda_stream)
{
    return run_fwd(mxn::STAT_NONE, false, x_bf16, nullptr, T, D, block, 2, 1.0f, 0.0f, 1.0f, codes_u8, scales_u8, nullptr,
                   MXN_ROUND_RCEIL_POW2, layout, cuda_stream, mxn::ELEM_E5M2);
}

mxn_status mx_cast_transposed_e5m2(const void* x_bf16, int64_t T, int64_t D, void* codes_t_u8, void* scales_t_u8,
                                   mxn_scale_layout layout, void* cuda_stream)
{
    return run_transposed(x_bf16, nullptr, T, D, 0.0f, codes_t_u8, scales_t_u8, MXN_ROUND_RCEIL_POW2, layout, mxn::ELEM_E5M2,
                          cuda_stream);
}

mxn_status mx_cast_transposed(const void* x_bf16, const float* rms_or_null, int64_t T, int64_t D, float eps,
                              void* codes_t_u8, void* scales_t_u8, mxn_round round, mxn_scale_layout layout,
                              void* cuda_stream)
{
    return run_transposed(x_bf16, rms_or_null, T, D, eps, codes_t_u8, scales_t_u8, round, layout, mxn::ELEM_E4M3, cuda_stream);
}

namespace {
mxn_status run_transposed(const void* x_bf16, const float* rms_or_null, int64_t T, int64_t D, float eps, void* codes_t_u8,
                          void* scales_t_u8, int round, int layout, int elem, void* cuda_stream)
{
    if (T < 0 || D <= 0 || T % 32 != 0 || D % 4 != 0 || D > 0x7FFFFFFF || T / 128 > 65535) return MXN_ERR_SHAPE;
    if (round < 0 || round > MXN_ROUND_RCEIL_MAX) return MXN_ERR_ENUM;
    if (layout != MXN_SCALES_ROWMAJOR && layout != MXN_SCALES_SWIZZLE_128x4) return MXN_ERR_ENUM;
    if (T == 0) return MXN_OK;
    if (x_bf16 == nullptr || codes_t_u8 == nullptr || scales_t_u8 == nullptr) return MXN_ERR_NULL;
    if (misaligned(x_bf16, 8) || misaligned(codes_t_u8, 32) || (rms_or_null != nullptr && misaligned(rms_or_null, 4)))
        return MXN_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (clear_scale_padding(scales_t_u8, D, T / 32, layout, s) != cudaSuccess) return MXN_ERR_CUDA;
    mxn::TransposedParams P{};
    P.x = static_cast<const uint16_t*>(x_bf16);
    P.rms = rms_or_null;
    P.codes = static_cast<uint8_t*>(codes_t_u8);
    P.scales = static_cast<uint8_t*>(scales_t_u8);
    P.T = T;
    P.D = (int)D;
    P.eps = eps;
    P.round = round;
    P.layout = layout;
    P.elem = elem;
    return mxn::launch_cast_transposed(P, s) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}
}  // namespace

mxn_status mxnorm_bwd(const void* x_bf16, const void* grad_out_bf16, const void* gain_bf16_or_null,
                      const float* rms, int64_t T, int64_t D, void* dx, int dx_is_fp32, float* dgain_f32_or_null,
                      void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (T < 0 || D <= 0 || !mxn::bwd_shape_supported(D)) return MXN_ERR_SHAPE;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (T == 0) {
        if (dgain_f32_or_null != nullptr &&
            cudaMemsetAsync(dgain_f32_or_null, 0, sizeof(float) * (size_t)D, s) != cudaSuccess)
            return MXN_ERR_CUDA;
        return MXN_OK;
    }
    if (x_bf16 == nullptr || grad_out_bf16 == nullptr || rms == nullptr || dx == nullptr) return MXN_ERR_NULL;
    if (misaligned(x_bf16, 16) || misaligned(grad_out_bf16, 16) || misaligned(dx, 16) || misaligned(rms, 4) ||
        (gain_bf16_or_null != nullptr && misaligned(gain_bf16_or_null, 16)) ||
        (dgain_f32_or_null != nullptr && misaligned(dgain_f32_or_null, 16)))
        return MXN_ERR_ALIGN;
    if (dgain_f32_or_null != nullptr) {
        if (workspace == nullptr || workspace_bytes < mxnorm_bwd_workspace_bytes(T, D)) return MXN_ERR_WORKSPACE;
        if (misaligned(workspace, 16)) return MXN_ERR_ALIGN;
    }
    mxn::BwdParams P{};
    P.x = static_cast<const uint16_t*>(x_bf16);
    P.g = static_cast<const uint16_t*>(grad_out_bf16);
    P.gain = static_cast<const uint16_t*>(gain_bf16_or_null);
    P.rms = rms;
    P.dx = dx;
    P.dgain = dgain_f32_or_null;
    P.partial = static_cast<float*>(workspace);
    P.T = T;
    P.D = (int)D;
    P.dx_is_fp32 = dx_is_fp32 != 0;
    P.parts = mxn::bwd_parts(T, D);
    return mxn::launch_bwd(P, s) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

size_t mxnorm_bwd_workspace_bytes(int64_t T, int64_t D)
{
    if (T <= 0 || D <= 0 || !mxn::bwd_shape_supported(D)) return 0;
    return (size_t)mxn::bwd_parts(T, D) * (size_t)D * sizeof(float);
}

// ---- host-memory front end ----------------------------------------------------------------------
namespace {

struct HostPipe {
    bool ready = false;
    cudaStream_t in = nullptr, out = nullptr;
    cudaEvent_t fork = nullptr, copied = nullptr, join = nullptr;
};
constexpr int kMaxDevices = 64;
HostPipe g_pipes[kMaxDevices];
std::mutex g_pipes_mutex;

// call with g_pipes_mutex held
HostPipe* host_pipe()
{
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return nullptr;
    HostPipe& hp = g_pipes[dev];
    if (!hp.ready) {
        if (cudaStreamCreateWithFlags(&hp.in, cudaStreamNonBlocking) != cudaSuccess ||
            cudaStreamCreateWithFlags(&hp.out, cudaStreamNonBlocking) != cudaSuccess ||
            cudaEventCreateWithFlags(&hp.fork, cudaEventDisableTiming) != cudaSuccess ||
            cudaEventCreateWithFlags(&hp.copied, cudaEventDisableTiming) != cudaSuccess ||
            cudaEventCreateWithFlags(&hp.join, cudaEventDisableTiming) != cudaSuccess)
            return nullptr;
        hp.ready = true;
    }
    return &hp;
}

inline size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
constexpr int64_t kHostChunkRows = 2048;   // multiple of the 128-row scale tile

}  // namespace

size_t mxnorm_fwd_host_workspace_bytes(int64_t T, int64_t D, int block, mxn_scale_layout layout)
{
    if (T <= 0 || D <= 0 || !mxn::fwd_shape_supported(D, block)) return 0;
    const size_t sb = mxn_scale_bytes(T, D / block, layout);
    if (sb == 0) return 0;
    return align_up((size_t)T * D * 2, 256) + align_up((size_t)T * D, 256) + align_up(sb, 256) +
           align_up((size_t)T * 4, 256);
}

mxn_status mxnorm_fwd_host(const void* x_host_bf16, int64_t T, int64_t D, int block, int p, float coef_or_0,
                           float eps, void* codes_host, void* scales_host, float* rms_est_host_or_null,
                           mxn_round round, mxn_scale_layout layout, void* workspace, size_t workspace_bytes,
                           void* cuda_stream)
{
    if (T < 0 || D <= 0 || !mxn::fwd_shape_supported(D, block) || (p != 1 && p != 2)) return MXN_ERR_SHAPE;
    if (round < 0 || round > MXN_ROUND_RCEIL_MAX) return MXN_ERR_ENUM;
    if (layout != MXN_SCALES_ROWMAJOR && layout != MXN_SCALES_SWIZZLE_128x4) return MXN_ERR_ENUM;
    if (T == 0) return MXN_OK;
    if (x_host_bf16 == nullptr || codes_host == nullptr || scales_host == nullptr) return MXN_ERR_NULL;
    if (workspace == nullptr || workspace_bytes < mxnorm_fwd_host_workspace_bytes(T, D, block, layout))
        return MXN_ERR_WORKSPACE;
    if (misaligned(workspace, 256)) return MXN_ERR_ALIGN;
    // the internal streams and events of a device are shared by every call on it: one call enqueues at a time
    std::lock_guard<std::mutex> pipe_lock(g_pipes_mutex);
    HostPipe* hp = host_pipe();
    if (hp == nullptr) return MXN_ERR_CUDA;
    cudaStream_t user = static_cast<cudaStream_t>(cuda_stream);

    const int64_t K = D / block;
    const size_t sbytes = mxn_scale_bytes(T, K, layout);
    uint8_t* base = static_cast<uint8_t*>(workspace);
    uint16_t* dx = reinterpret_cast<uint16_t*>(base);
    uint8_t* dcodes = base + align_up((size_t)T * D * 2, 256);
    uint8_t* dscales = dcodes + align_up((size_t)T * D, 256);
    float* drms = reinterpret_cast<float*>(dscales + align_up(sbytes, 256));
    const uint16_t* hx = static_cast<const uint16_t*>(x_host_bf16);
    uint8_t* hcodes = static_cast<uint8_t*>(codes_host);
    uint8_t* hscales = static_cast<uint8_t*>(scales_host);

    if (cudaEventRecord(hp->fork, user) != cudaSuccess) return MXN_ERR_CUDA;   // nothing forked yet
    bool ok = cudaStreamWaitEvent(hp->in, hp->fork, 0) == cudaSuccess &&
              cudaStreamWaitEvent(hp->out, hp->fork, 0) == cudaSuccess;
    mxn_status failed = MXN_OK;
    const bool tiled = layout == MXN_SCALES_SWIZZLE_128x4;
    const int64_t tiles_per_row = (K + 3) / 4;
    for (int64_t r0 = 0; ok && r0 < T; r0 += kHostChunkRows) {
        const int64_t rows = (T - r0 < kHostChunkRows) ? T - r0 : kHostChunkRows;
        ok = cudaMemcpyAsync(dx + r0 * D, hx + r0 * D, (size_t)rows * D * 2, cudaMemcpyHostToDevice, hp->in) == cudaSuccess &&
             cudaEventRecord(hp->copied, hp->in) == cudaSuccess &&
             cudaStreamWaitEvent(hp->out, hp->copied, 0) == cudaSuccess;
        if (!ok) break;
        // a chunk starts on a 128-row boundary, so its scales are a contiguous slice in either layout
        const size_t soff = tiled ? (size_t)(r0 / 128) * tiles_per_row * 512 : (size_t)r0 * K;
        const size_t slen = tiled ? (size_t)((rows + 127) / 128) * tiles_per_row * 512 : (size_t)rows * K;
        mxn_status st = run_fwd(mxn::STAT_MX, false, dx + r0 * D, nullptr, rows, D, block, p, coef_or_0, eps, 1.0f,
                                dcodes + r0 * D, dscales + soff, drms + r0, round, layout, hp->out);
        if (st != MXN_OK) {   // leave through the join below: the chunks already enqueued must stay ordered
            failed = st;
            break;
        }
        ok = cudaMemcpyAsync(hcodes + r0 * D, dcodes + r0 * D, (size_t)rows * D, cudaMemcpyDeviceToHost, hp->out) == cudaSuccess &&
             cudaMemcpyAsync(hscales + soff, dscales + soff, slen, cudaMemcpyDeviceToHost, hp->out) == cudaSuccess;
        if (ok && rms_est_host_or_null != nullptr)
            ok = cudaMemcpyAsync(rms_est_host_or_null + r0, drms + r0, (size_t)rows * 4, cudaMemcpyDeviceToHost, hp->out) == cudaSuccess;
    }
    // Join on every path that forked: the caller's stream waits for both internal streams, so whatever was enqueued
    // (copies into the caller's buffers included) is ordered before anything the caller enqueues next.
    const bool joined = cudaEventRecord(hp->copied, hp->in) == cudaSuccess &&
                        cudaStreamWaitEvent(hp->out, hp->copied, 0) == cudaSuccess &&
                        cudaEventRecord(hp->join, hp->out) == cudaSuccess &&
                        cudaStreamWaitEvent(user, hp->join, 0) == cudaSuccess;
    if (failed != MXN_OK) return failed;
    return ok && joined ? MXN_OK : MXN_ERR_CUDA;
}

// ---- queries, keys and values around attention ------------------------------------------------------

namespace {

constexpr int64_t kMaxTokens = 0x7FFFFFFF;   // positions and row counts are 32-bit in device memory
constexpr int kMaxHeads = 4096;

bool head_dim_supported(int dim) { return dim >= 16 && dim <= 256 && dim % 16 == 0; }

// one operand of `heads` heads of `dim` elements a token: pointer, token stride, alignment of 16 bytes
mxn_status check_heads(const void* p, int64_t stride, int heads, int dim)
{
    if (heads == 0) return MXN_OK;
    if (p == nullptr) return MXN_ERR_NULL;
    if (stride < (int64_t)heads * dim) return MXN_ERR_SHAPE;
    if (misaligned(p, 16) || stride % 8 != 0) return MXN_ERR_ALIGN;
    return MXN_OK;
}

mxn_status check_rotation(const float* cos_sin, int64_t table_rows, int rot, int dim, int pairing)
{
    if (pairing != MXN_ROPE_HALVES && pairing != MXN_ROPE_PAIRS) return MXN_ERR_ENUM;
    if (cos_sin == nullptr) return MXN_OK;
    if (rot < 16 || rot > dim || rot % 16 != 0 || table_rows < 1) return MXN_ERR_SHAPE;
    return misaligned(cos_sin, 16) ? MXN_ERR_ALIGN : MXN_OK;
}

mxn_status check_rope(int64_t T, int q_heads, int k_heads, int dim, int normalise, const void* q_gain, const void* k_gain, float eps,
                      const float* cos_sin, int64_t table_rows, int rot, int pairing, const int32_t* positions)
{
    if (T < 0 || T > kMaxTokens || q_heads < 0 || k_heads < 0 || q_heads + k_heads < 1 || q_heads > kMaxHeads || k_heads > kMaxHeads ||
        !head_dim_supported(dim))
        return MXN_ERR_SHAPE;
    if (normalise != 0 && normalise != 1) return MXN_ERR_ENUM;
    if (!(eps >= 0.0f) || (normalise == 0 && (q_gain != nullptr || k_gain != nullptr))) return MXN_ERR_SHAPE;
    const mxn_status st = check_rotation(cos_sin, table_rows, rot, dim, pairing);
    if (st != MXN_OK) return st;
    if ((q_gain != nullptr && misaligned(q_gain, 16)) || (k_gain != nullptr && misaligned(k_gain, 16)) ||
        (positions != nullptr && misaligned(positions, 4)))
        return MXN_ERR_ALIGN;
    return MXN_OK;
}

mxn::HeadsParams rope_params(int64_t T, int q_heads, int k_heads, int dim, int normalise, const void* q_gain, const void* k_gain, float eps,
                             const float* cos_sin, int64_t table_rows, int rot, int pairing, const int32_t* positions)
{
    mxn::HeadsParams P{};
    P.T = T;
    P.heads[0] = q_heads;
    P.heads[1] = k_heads;
    P.dim = dim;
    P.norm = normalise;
    P.gain[0] = static_cast<const uint16_t*>(q_gain);
    P.gain[1] = static_cast<const uint16_t*>(k_gain);
    P.eps = eps;
    P.inv_dim = 1.0f / (float)dim;
    P.cos_sin = cos_sin;
    P.table_rows = table_rows;
    P.rot = cos_sin != nullptr ? rot : 0;
    P.pairs = pairing == MXN_ROPE_PAIRS;
    P.positions = positions;
    return P;
}

mxn_status check_cache(int kv_heads, int dim, int64_t n_seqs, int64_t max_pages, int64_t num_pages, int page_size, int block,
                       const void* cu, const void* lens, const void* table, const void* kc, const void* ks, const void* vc, const void* vs)
{
    if (kv_heads < 1 || kv_heads > kMaxHeads || !head_dim_supported(dim) || n_seqs < 0 || n_seqs > kMaxTokens || max_pages < 1 || num_pages < 1)
        return MXN_ERR_SHAPE;
    if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1)) != 0) return MXN_ERR_SHAPE;
    if ((block != 16 && block != 32 && block != 64) || block > page_size) return MXN_ERR_SHAPE;
    if (max_pages > kMaxTokens / page_size || num_pages > kMaxTokens / kv_heads) return MXN_ERR_SHAPE;
    if (n_seqs == 0) return MXN_OK;
    if (cu == nullptr || lens == nullptr || table == nullptr || kc == nullptr || ks == nullptr || vc == nullptr || vs == nullptr) return MXN_ERR_NULL;
    if (misaligned(cu, 4) || misaligned(lens, 4) || misaligned(table, 4) || misaligned(kc, 16) || misaligned(vc, 16)) return MXN_ERR_ALIGN;
    return MXN_OK;
}

int log2_of(int v)
{
    int n = 0;
    while ((1 << n) < v) ++n;
    return n;
}

bool attention_shape_ok(int64_t n_tokens, int64_t n_seqs, int64_t max_q_len, int64_t max_kv_len, int q_heads, int kv_heads, int dim)
{
    return n_tokens >= 0 && n_tokens <= kMaxTokens && n_seqs >= 0 && n_seqs <= kMaxTokens && max_q_len >= 1 && max_q_len <= kMaxTokens &&
           max_kv_len >= 0 && max_kv_len <= kMaxTokens - 511 && kv_heads >= 1 && q_heads >= kv_heads && q_heads <= kMaxHeads &&
           q_heads % kv_heads == 0 && (dim == 64 || dim == 128);
}

}  // namespace

mxn_status rmsnorm_rope_fwd(const void* q_bf16, int64_t q_stride, int q_heads, const void* k_bf16, int64_t k_stride, int k_heads, int64_t T,
                            int head_dim, int normalise, const void* q_gain_bf16_or_null, const void* k_gain_bf16_or_null, float eps,
                            const float* cos_sin_or_null, int64_t table_rows, int rot_dim, mxn_rope pairing, const int32_t* positions_or_null,
                            void* q_out_bf16, int64_t q_out_stride, void* k_out_bf16, int64_t k_out_stride, void* cuda_stream)
{
    mxn_status st = check_rope(T, q_heads, k_heads, head_dim, normalise, q_gain_bf16_or_null, k_gain_bf16_or_null, eps, cos_sin_or_null,
                               table_rows, rot_dim, pairing, positions_or_null);
    if (st != MXN_OK || T == 0) return st;
    if ((st = check_heads(q_bf16, q_stride, q_heads, head_dim)) != MXN_OK || (st = check_heads(k_bf16, k_stride, k_heads, head_dim)) != MXN_OK ||
        (st = check_heads(q_out_bf16, q_out_stride, q_heads, head_dim)) != MXN_OK ||
        (st = check_heads(k_out_bf16, k_out_stride, k_heads, head_dim)) != MXN_OK)
        return st;
    mxn::HeadsParams P = rope_params(T, q_heads, k_heads, head_dim, normalise, q_gain_bf16_or_null, k_gain_bf16_or_null, eps, cos_sin_or_null,
                                     table_rows, rot_dim, pairing, positions_or_null);
    P.x[0] = static_cast<const uint16_t*>(q_bf16);
    P.x[1] = static_cast<const uint16_t*>(k_bf16);
    P.x_stride[0] = q_stride;
    P.x_stride[1] = k_stride;
    P.y[0] = static_cast<uint16_t*>(q_out_bf16);
    P.y[1] = static_cast<uint16_t*>(k_out_bf16);
    P.y_stride[0] = q_out_stride;
    P.y_stride[1] = k_out_stride;
    return mxn::launch_rope_fwd(P, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

size_t rmsnorm_rope_bwd_workspace_bytes(int64_t T, int q_heads, int k_heads, int head_dim)
{
    if (check_rope(T, q_heads, k_heads, head_dim, 1, nullptr, nullptr, 0.0f, nullptr, 0, 0, MXN_ROPE_HALVES, nullptr) != MXN_OK) return 0;
    return (size_t)mxn::rope_bwd_ctas(T, q_heads, k_heads, head_dim) * head_dim * 4;
}

mxn_status rmsnorm_rope_bwd(const void* q_bf16_or_null, int64_t q_stride, int q_heads, const void* k_bf16_or_null, int64_t k_stride, int k_heads,
                            const void* grad_q_bf16, int64_t grad_q_stride, const void* grad_k_bf16, int64_t grad_k_stride, int64_t T,
                            int head_dim, int normalise, const void* q_gain_bf16_or_null, const void* k_gain_bf16_or_null, float eps,
                            const float* cos_sin_or_null, int64_t table_rows, int rot_dim, mxn_rope pairing, const int32_t* positions_or_null,
                            void* dq_bf16, int64_t dq_stride, void* dk_bf16, int64_t dk_stride, float* q_dgain_f32_or_null,
                            float* k_dgain_f32_or_null, void* workspace, size_t workspace_bytes, void* cuda_stream)
{
    mxn_status st = check_rope(T, q_heads, k_heads, head_dim, normalise, q_gain_bf16_or_null, k_gain_bf16_or_null, eps, cos_sin_or_null,
                               table_rows, rot_dim, pairing, positions_or_null);
    if (st != MXN_OK) return st;
    const bool dgain = q_dgain_f32_or_null != nullptr || k_dgain_f32_or_null != nullptr;
    if (normalise == 0 && dgain) return MXN_ERR_SHAPE;
    if ((q_dgain_f32_or_null != nullptr && misaligned(q_dgain_f32_or_null, 4)) ||
        (k_dgain_f32_or_null != nullptr && misaligned(k_dgain_f32_or_null, 4)))
        return MXN_ERR_ALIGN;
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (T == 0) {
        const size_t bytes = (size_t)head_dim * 4;
        if ((q_dgain_f32_or_null != nullptr && cudaMemsetAsync(q_dgain_f32_or_null, 0, bytes, s) != cudaSuccess) ||
            (k_dgain_f32_or_null != nullptr && cudaMemsetAsync(k_dgain_f32_or_null, 0, bytes, s) != cudaSuccess))
            return MXN_ERR_CUDA;
        return MXN_OK;
    }
    if (normalise != 0 && ((st = check_heads(q_bf16_or_null, q_stride, q_heads, head_dim)) != MXN_OK ||
                           (st = check_heads(k_bf16_or_null, k_stride, k_heads, head_dim)) != MXN_OK))
        return st;
    if ((st = check_heads(grad_q_bf16, grad_q_stride, q_heads, head_dim)) != MXN_OK ||
        (st = check_heads(grad_k_bf16, grad_k_stride, k_heads, head_dim)) != MXN_OK ||
        (st = check_heads(dq_bf16, dq_stride, q_heads, head_dim)) != MXN_OK || (st = check_heads(dk_bf16, dk_stride, k_heads, head_dim)) != MXN_OK)
        return st;
    if (dgain) {
        if (workspace == nullptr || workspace_bytes < rmsnorm_rope_bwd_workspace_bytes(T, q_heads, k_heads, head_dim)) return MXN_ERR_WORKSPACE;
        if (misaligned(workspace, 16)) return MXN_ERR_ALIGN;
    }
    mxn::HeadsParams P = rope_params(T, q_heads, k_heads, head_dim, normalise, q_gain_bf16_or_null, k_gain_bf16_or_null, eps, cos_sin_or_null,
                                     table_rows, rot_dim, pairing, positions_or_null);
    P.x[0] = static_cast<const uint16_t*>(q_bf16_or_null);
    P.x[1] = static_cast<const uint16_t*>(k_bf16_or_null);
    P.x_stride[0] = q_stride;
    P.x_stride[1] = k_stride;
    P.grad[0] = static_cast<const uint16_t*>(grad_q_bf16);
    P.grad[1] = static_cast<const uint16_t*>(grad_k_bf16);
    P.grad_stride[0] = grad_q_stride;
    P.grad_stride[1] = grad_k_stride;
    P.y[0] = static_cast<uint16_t*>(dq_bf16);
    P.y[1] = static_cast<uint16_t*>(dk_bf16);
    P.y_stride[0] = dq_stride;
    P.y_stride[1] = dk_stride;
    P.dgain[0] = q_dgain_f32_or_null;
    P.dgain[1] = k_dgain_f32_or_null;
    P.partial = dgain ? static_cast<float*>(workspace) : nullptr;
    return mxn::launch_rope_bwd(P, s) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

mxn_status mxkv_append(const void* k_bf16, int64_t k_stride, const void* v_bf16, int64_t v_stride, int64_t n_tokens, int kv_heads, int head_dim,
                       const int32_t* cu_tokens, int64_t n_seqs, const int32_t* kv_lens, const int32_t* page_table, int64_t max_pages,
                       int64_t num_pages, int page_size, int block, const float* cos_sin_or_null, int64_t table_rows, int rot_dim,
                       mxn_rope pairing, void* k_codes_u8, void* k_scales_u8, void* v_codes_u8, void* v_scales_u8, void* cuda_stream)
{
    mxn_status st = check_cache(kv_heads, head_dim, n_seqs, max_pages, num_pages, page_size, block, cu_tokens, kv_lens, page_table, k_codes_u8,
                                k_scales_u8, v_codes_u8, v_scales_u8);
    if (st != MXN_OK) return st;
    if (n_tokens < 0 || n_tokens > kMaxTokens) return MXN_ERR_SHAPE;
    if ((st = check_rotation(cos_sin_or_null, table_rows, rot_dim, head_dim, pairing)) != MXN_OK) return st;
    if (n_tokens == 0 || n_seqs == 0) return MXN_OK;
    if ((st = check_heads(k_bf16, k_stride, kv_heads, head_dim)) != MXN_OK || (st = check_heads(v_bf16, v_stride, kv_heads, head_dim)) != MXN_OK)
        return st;
    mxn::KvAppendParams P{};
    P.x[0] = static_cast<const uint16_t*>(k_bf16);
    P.x[1] = static_cast<const uint16_t*>(v_bf16);
    P.x_stride[0] = k_stride;
    P.x_stride[1] = v_stride;
    P.codes[0] = static_cast<uint8_t*>(k_codes_u8);
    P.codes[1] = static_cast<uint8_t*>(v_codes_u8);
    P.scales[0] = static_cast<uint8_t*>(k_scales_u8);
    P.scales[1] = static_cast<uint8_t*>(v_scales_u8);
    P.cu = cu_tokens;
    P.lens = kv_lens;
    P.page_table = page_table;
    P.cos_sin = cos_sin_or_null;
    P.n = n_tokens;
    P.num_pages = num_pages;
    P.max_pages = max_pages;
    P.table_rows = table_rows;
    P.seqs = (int)n_seqs;
    P.heads = kv_heads;
    P.dim = head_dim;
    P.page = page_size;
    P.block = block;
    P.page_shift = log2_of(page_size);
    P.block_shift = log2_of(block);
    P.rot = rot_dim;
    P.pairs = pairing == MXN_ROPE_PAIRS;
    return mxn::launch_kv_append(P, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

size_t mxkv_attention_workspace_bytes(int64_t n_tokens, int64_t n_seqs, int64_t max_q_len, int64_t max_kv_len, int q_heads, int kv_heads,
                                      int head_dim)
{
    if (!attention_shape_ok(n_tokens, n_seqs, max_q_len, max_kv_len, q_heads, kv_heads, head_dim) || n_tokens == 0 || n_seqs == 0) return 0;
    return mxn::plan_attention(n_tokens, n_seqs, max_q_len, max_kv_len, 0, q_heads, kv_heads, head_dim).workspace;
}

mxn_status mxkv_attention(const void* q_bf16, int64_t q_stride, int64_t n_tokens, int q_heads, int kv_heads, int head_dim,
                          const int32_t* cu_q, int64_t n_seqs, int64_t max_q_len, const int32_t* kv_lens, int64_t max_kv_len,
                          const int32_t* page_table, int64_t max_pages, int64_t num_pages, int page_size, int block, const void* k_codes_u8,
                          const void* k_scales_u8, const void* v_codes_u8, const void* v_scales_u8, float scale, int causal, int64_t window,
                          void* out_bf16, int64_t out_stride, float* lse_out_or_null, void* workspace, size_t workspace_bytes,
                          void* cuda_stream)
{
    if (!attention_shape_ok(n_tokens, n_seqs, max_q_len, max_kv_len, q_heads, kv_heads, head_dim)) return MXN_ERR_SHAPE;
    mxn_status st = check_cache(kv_heads, head_dim, n_seqs, max_pages, num_pages, page_size, block, cu_q, kv_lens, page_table, k_codes_u8,
                                k_scales_u8, v_codes_u8, v_scales_u8);
    if (st != MXN_OK) return st;
    if (max_kv_len > max_pages * page_size || window < 0 || window > kMaxTokens || !(scale == scale)) return MXN_ERR_SHAPE;
    if (causal != 0 && causal != 1) return MXN_ERR_ENUM;
    if (n_tokens == 0 || n_seqs == 0) return MXN_OK;
    if ((st = check_heads(q_bf16, q_stride, q_heads, head_dim)) != MXN_OK || (st = check_heads(out_bf16, out_stride, q_heads, head_dim)) != MXN_OK)
        return st;
    if (lse_out_or_null != nullptr && misaligned(lse_out_or_null, 4)) return MXN_ERR_ALIGN;
    const mxn::AttnPlan plan = mxn::plan_attention(n_tokens, n_seqs, max_q_len, max_kv_len, causal ? window : 0, q_heads, kv_heads,
                                                    head_dim);
    if (plan.ctas > 0x7FFFFFFF || n_tokens * q_heads > 0x7FFFFFFF) return MXN_ERR_SHAPE;
    if (plan.splits > 1) {
        if (workspace == nullptr || workspace_bytes < plan.workspace) return MXN_ERR_WORKSPACE;
        if (misaligned(workspace, 16)) return MXN_ERR_ALIGN;
    }
    mxn::AttnParams P{};
    P.q = static_cast<const uint16_t*>(q_bf16);
    P.out = static_cast<uint16_t*>(out_bf16);
    P.lse = lse_out_or_null;
    P.k_codes = static_cast<const uint8_t*>(k_codes_u8);
    P.k_scales = static_cast<const uint8_t*>(k_scales_u8);
    P.v_codes = static_cast<const uint8_t*>(v_codes_u8);
    P.v_scales = static_cast<const uint8_t*>(v_scales_u8);
    P.cu_q = cu_q;
    P.lens = kv_lens;
    P.page_table = page_table;
    P.n = n_tokens;
    P.q_stride = q_stride;
    P.out_stride = out_stride;
    P.max_pages = max_pages;
    P.num_pages = (int)num_pages;
    P.seqs = (int)n_seqs;
    P.q_heads = q_heads;
    P.kv_heads = kv_heads;
    P.group = q_heads / kv_heads;
    // with s = ceil(log2 group) and mul = ceil(2^(31 + s) / group) the product's error stays below 2^(31 + s) / group for rows < 2^31
    P.group_shift = P.group > 1 ? (uint32_t)log2_of(P.group) - 1 : 0;
    P.group_mul = P.group > 1 ? (uint32_t)(((1ull << (32 + P.group_shift)) + P.group - 1) / P.group) : 0;
    P.dim = head_dim;
    P.page = page_size;
    P.page_shift = log2_of(page_size);
    P.block_shift = log2_of(block);
    P.max_q = (int)(max_q_len < n_tokens ? max_q_len : n_tokens);
    P.max_len = (int)max_kv_len;
    P.causal = causal;
    P.window = (int)window;
    P.scale = scale;
    return mxn::launch_attention(P, plan, workspace, static_cast<cudaStream_t>(cuda_stream)) == cudaSuccess ? MXN_OK : MXN_ERR_CUDA;
}

}  // extern "C"
