// extern "C" surface of the token-major products: plan life cycle, argument checks, choice of the kernel.
#include <cuda_runtime.h>

#include <cstring>

#include "ubp_internal.h"
#include "ubp_linear.h"
#include "ubp_types.cuh"

namespace ubp {

// Kernel and tile of a launch. Estimates in us, fitted to back-to-back launches on B200 (26 random layers of 256 .. 10000
// rows and channels, bf16 and e4m3, 1, 2, 4, 8 rows an entry, 50 .. 90 % pruned, 1 .. 24 tokens; the kept blocks and the
// dense form both timed; the choice costs 2 % on average over always taking the faster one, "eight tokens or fewer" 3.5 %):
//   kept blocks   2.8 + (entries (24 + 6.6 t) + kept weights x 27 t) ns / 1000 over the SMs + 85 ns a thousand channels and
//                 token, t = tokens a block takes: instruction-bound, in the entries and in the products
//   dense, few    3.3 + 0.9 for a split reduction + 6.4 ns a KB of weights a block streams + 0.12 us a MB in all
// From 17 tokens on (three blocks to a row range) the kept blocks lost everywhere. A call of the few-token kernel covers 256
// tokens; with more (4096 x 4096, 384 tokens, 22.5 us) the pair kernel is as fast (22.2) and from 512 on faster. Its tile is
// 128 rows wide while those tiles fit one round (8192 x 2048, 256 tokens: 14.1 us against 16.8), else 256 (384 tokens: 17.3
// against 22.2).
LinearChoice linear_choose(const ubp_linear_plan *p, int64_t T, int sms)
{
    const int b = p->dtype == UBP_E4M3 ? 1 : 2;
    const int rows = p->gated ? (p->F + 15) / 16 * 32 : p->M, rt = (rows + 127) / 128, nk = p->img.Kp * b / 128;
    int S = 1;                       // split as far as the blocks find SMs and keep four chunks of the reduction each
    while (S < 8 && rt * S * 2 <= sms && nk / (S * 2) >= 4) S *= 2;
    if (T <= 16) {
        int t;
        int64_t nchunk;
        linear_sparse_tokens(p, T, &t, &nchunk);
        const double kept = (double)p->img.entries * p->img.nbk, share = (double)nchunk / sms;
        const double sparse = 2.8 + ((double)p->img.entries * (24 + 6.6 * t) + kept * 27 * t) * share * 1e-6 + 85e-6 * p->C * t;
        const double waves = (rt * S + sms - 1) / sms;
        const double dense = 3.3 + (S > 1 ? 0.9 : 0.0) + 128.0 * p->img.Kp * b / S * waves * 6.4e-6 + 128e-6 * rt * p->img.Kp * b * 0.12;
        if (sparse <= dense) return {LIN_SPARSE, t, 0};
    }
    if (T <= 256) return {LIN_FEW, (int)((T + 15) / 16 * 16), S};
    const int64_t t128 = ((T + 255) / 256) * ((rows + 127) / 128);
    return {LIN_MANY, t128 <= sms / 2 ? 128 : 256, 0};
}

// SMs of the current device (asked once per device)
int device_sms()
{
    static int known[64] = {};
    int dev = 0, sms = 148;
    if (cudaGetDevice(&dev) != cudaSuccess) return sms;
    if (dev < 64 && known[dev]) return known[dev];
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
    if (dev < 64) known[dev] = sms;
    return sms;
}

}  // namespace ubp

static bool live(const ubp_linear_plan *p) { return p && p->magic == ubp::kLinearMagic; }

extern "C" {

int ubp_linear_plan_size(const void *blob, size_t len, int dtype, int gated, size_t *dev_bytes)
{
    if (!dev_bytes) return UBP_E_ARG;
    ubp_view_t v;
    if (int rc = ubp::blob_view(blob, len, &v)) return rc;
    try {
        ubp::LinearImage img;
        if (int rc = ubp::build_linear_image(v, dtype, gated != 0, true, img)) return rc;
        *dev_bytes = img.total;
    } catch (...) { return UBP_E_SPACE; }
    return UBP_OK;
}

int ubp_linear_plan_image(const void *blob, size_t len, int dtype, int gated, void *host_buf, size_t cap, int32_t geom[6],
                          int64_t offs[5])
{
    if (!host_buf || !geom || !offs) return UBP_E_ARG;
    ubp_view_t v;
    if (int rc = ubp::blob_view(blob, len, &v)) return rc;
    try {
        ubp::LinearImage img;
        if (int rc = ubp::build_linear_image(v, dtype, gated != 0, false, img)) return rc;
        if (cap < img.total) return UBP_E_SPACE;
        std::memcpy(host_buf, img.bytes.data(), img.total);
        geom[0] = img.nbk; geom[1] = img.epc; geom[2] = img.Mp; geom[3] = img.Kp; geom[4] = ubp::dtype_size(dtype);
        geom[5] = img.lanes;
        offs[0] = (int64_t)img.scale_off; offs[1] = (int64_t)img.off_off; offs[2] = (int64_t)img.idx_off;
        offs[3] = (int64_t)img.val_off; offs[4] = (int64_t)img.dense_off;
    } catch (...) { return UBP_E_SPACE; }
    return UBP_OK;
}

int ubp_linear_plan_build(const void *blob, size_t len, int dtype, int gated, void *dev_buf, size_t dev_bytes, void *stream,
                          ubp_linear_plan_t **plan)
{
    if (!plan || !dev_buf || (reinterpret_cast<uintptr_t>(dev_buf) & 255)) return UBP_E_ARG;
    *plan = nullptr;
    ubp_view_t v;
    if (int rc = ubp::blob_view(blob, len, &v)) return rc;
    ubp_linear_plan *p = nullptr;
    try {
        p = new ubp_linear_plan();
        int rc = ubp::build_linear_image(v, dtype, gated != 0, true, p->img);
        if (!rc && dev_bytes < p->img.total) rc = UBP_E_SPACE;
        if (!rc) rc = ubp::build_linear_image(v, dtype, gated != 0, false, p->img);
        if (rc) { delete p; return rc; }
    } catch (...) { delete p; return UBP_E_SPACE; }
    p->magic = ubp::kLinearMagic;
    p->M = v.M; p->C = v.C; p->Nb = v.Nb; p->m = v.m;
    p->dtype = dtype; p->gated = gated != 0;
    p->F = p->gated ? v.M / 2 : v.M;
    p->dev = static_cast<uint8_t *>(dev_buf);
    const cudaError_t e = cudaMemcpyAsync(dev_buf, p->img.bytes.data(), p->img.total, cudaMemcpyHostToDevice,
                                          static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { ubp::set_last_cuda_error((int)e); delete p; return UBP_E_CUDA; }
    *plan = p;
    return UBP_OK;
}

void ubp_linear_plan_free(ubp_linear_plan_t *plan)
{
    if (live(plan)) { plan->magic = 0; delete plan; }
}

int ubp_linear_plan_check(const ubp_linear_plan_t *plan, void *stream)
{
    if (!live(plan)) return UBP_E_ARG;
    int word = 0;
    cudaError_t e = cudaMemcpyAsync(&word, plan->dev, sizeof word, cudaMemcpyDeviceToHost, static_cast<cudaStream_t>(stream));
    if (e == cudaSuccess) e = cudaStreamSynchronize(static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { ubp::set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return word == 0 ? UBP_OK : UBP_E_DEVICE;
}

int ubp_linear_plan_clear_status(const ubp_linear_plan_t *plan, void *stream)
{
    if (!live(plan)) return UBP_E_ARG;
    const cudaError_t e = cudaMemsetAsync(plan->dev, 0, sizeof(int), static_cast<cudaStream_t>(stream));
    if (e != cudaSuccess) { ubp::set_last_cuda_error((int)e); return UBP_E_CUDA; }
    return UBP_OK;
}

size_t ubp_linear_workspace_size(const ubp_linear_plan_t *plan, const void *x, int64_t ldx, int64_t T)
{
    if (!live(plan) || T <= 0) return 0;
    if (ubp::linear_choose(plan, T, ubp::device_sms()).kernel == ubp::LIN_SPARSE || ubp::linear_x_direct(plan, x, ldx, T)) return 0;
    return (size_t)T * (size_t)plan->img.Kp * (size_t)ubp::dtype_size(plan->dtype);
}

int ubp_linear_choice(const ubp_linear_plan_t *plan, int64_t T, int *kernel, int *tile, int *split)
{
    if (!live(plan) || T < 0 || !kernel || !tile || !split) return UBP_E_ARG;
    const ubp::LinearChoice ch = ubp::linear_choose(plan, T, ubp::device_sms());
    *kernel = ch.kernel; *tile = ch.cols; *split = ch.split;
    return UBP_OK;
}

int ubp_linear(const ubp_linear_plan_t *plan, const void *x, int64_t ldx, const float *x_scales, int64_t T, const float *bias,
               int act, const void *residual, int64_t ldr, void *y, int64_t ldy, int y_dtype, void *workspace,
               size_t workspace_bytes, void *stream)
{
    if (!live(plan) || T < 0 || act < UBP_ACT_NONE || act > UBP_ACT_SILU) return UBP_E_ARG;
    const bool q = plan->dtype == UBP_E4M3;
    if (y_dtype != UBP_F32 && y_dtype != plan->dtype && !(q && (y_dtype == UBP_BF16 || y_dtype == UBP_F16))) return UBP_E_ARG;
    if (y_dtype == UBP_E4M3) return UBP_E_ARG;
    if (q ? (!x_scales && T > 0) : x_scales != nullptr) return UBP_E_ARG;
    if (T == 0) return UBP_OK;
    const uintptr_t b = (uintptr_t)ubp::dtype_size(plan->dtype), o = (uintptr_t)ubp::dtype_size(y_dtype);
    if (!x || !y || (T > 1 && (ldx < plan->C || ldy < plan->F || (residual && ldr < plan->F)))) return UBP_E_ARG;
    auto off = [](const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) != 0; };
    if (off(x, b) || off(y, o) || off(residual, o) || off(bias, 4) || off(x_scales, 4) || off(workspace, 16)) return UBP_E_ARG;
    if (workspace_bytes < ubp_linear_workspace_size(plan, x, ldx, T)) return UBP_E_SPACE;
    ubp::LinearArgs a;
    a.x = x; a.ldx = ldx; a.xs = x_scales; a.T = T; a.bias = bias; a.act = act;
    a.res = residual; a.ldr = ldr; a.y = y; a.ldy = ldy;
    a.status = reinterpret_cast<int *>(plan->dev);
    a.M = plan->M; a.C = plan->C; a.F = plan->F; a.gated = plan->gated;
    const int sms = ubp::device_sms();
    const ubp::LinearChoice ch = ubp::linear_choose(plan, T, sms);
    if (ch.kernel == ubp::LIN_SPARSE) return ubp::launch_linear_sparse(plan, a, y_dtype, sms, stream);
    return ubp::launch_linear_tc(plan, a, y_dtype, ch, workspace, sms, stream);
}

}  // extern "C"
