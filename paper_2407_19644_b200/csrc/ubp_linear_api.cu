// extern "C" surface of the token-major products: plan life cycle, argument checks, choice of the kernel.
#include <cuda_runtime.h>

#include <atomic>
#include <cstring>

#include "ubp_internal.h"
#include "ubp_linear.h"
#include "ubp_types.cuh"

namespace ubp {

// Kernel and tile of a launch, by estimates in us that were fitted to back-to-back launches on B200.
//   kept blocks   2.4 + (entries x 10 t + kept weights x 70 + rows (1000 + 700 b t)) / 10^6 over the SMs + 100 a million
//                 channels and token; t = tokens a block takes, b = rows of an entry: instructions for the entries, the
//                 products and the joining of a row's sums (40 random layers of 256 .. 16000 rows, 256 .. 8192 channels, all
//                 types, blocks of 2 .. 16 rows, 50 .. 90 % pruned, 1 .. 16 tokens: error 11 %; choosing by it costs 1.3 % on
//                 average over the faster of the two forms, the dense form always 20 %, the kept blocks always 13 %). From 17
//                 tokens on, three blocks to a row range, the kept blocks lost everywhere.
//   few           2.9 + 0.55 for a split reduction + rounds x (chunks a block takes (0.15 + 0.0008 n) + 0.023 n) + 0.052 a MB
//                 of weights, n = tokens of a tile: bound by what the copies bring a block, 16 KB + 128 n bytes a chunk
//   many          4.2 / 5.2 + rounds x (chunks x 0.233 / 0.26 + 2.1 / 4.6) for tiles of 128 / 256 rows, + 0.02 a MB of weights;
//                 a round after the first starts under the one before it: 0.022 / 0.043 a chunk less
// (The dense forms: 60 layers of 256 .. 18000 rows, 256 .. 8192 channels, bf16 and e4m3, 8 .. 5600 tokens, 1200 launches,
// error 7 and 11 %. Choosing by them costs 1 % on average over the best of all tiles and splits. A few-token tile of all
// tokens up to 256 and the pair kernel beyond cost 10 %: 512 x 5000, 1024 tokens, 24.4 us where 128 tokens x 4 parts take 12.3;
// 2048 x 8192, 24 tokens, 15.7 in 8 parts, two rounds, where 4 parts take 10.9.)
// A round is what the SMs hold at once: clusters of 2, 4, 8 blocks leave 0, 16, 28 of the 148 SMs without one
// (cudaOccupancyMaxActiveClusters).
LinearChoice linear_choose(const ubp_linear_plan *p, int64_t T, int sms)
{
    const int b = p->dtype == UBP_E4M3 ? 1 : 2;
    const int rows = p->gated ? (p->F + 15) / 16 * 32 : p->M, rt = (rows + 127) / 128, nk = p->img.Kp * b / 128;
    const double mb = 128e-6 * rt * p->img.Kp * b;
    if (T < 1) T = 1;                // (asked for no tokens: as for one)
    LinearChoice best{LIN_MANY, 256, 0};
    double least = 1e30;
    auto offer = [&](double us, LinearChoice c) { if (us < least) { least = us; best = c; } };
    for (int S = 1; S <= 8 && (S == 1 || nk >= 2 * S); S *= 2) {
        const int64_t fit = (int64_t)sms * (S == 4 ? 132 : S == 8 ? 120 : 148) / 148, ranges = fit / ((int64_t)rt * S);
        if (ranges == 0 && S > 1) break;
        // as many token tiles as one round holds, of 64 tokens at least, all alike
        int64_t n = (T + (ranges > 1 ? ranges : 1) - 1) / (ranges > 1 ? ranges : 1);
        if (n < 64) n = T < 64 ? T : 64;
        const int64_t ntt = (T + n - 1) / n;
        n = ((T + ntt - 1) / ntt + 15) / 16 * 16;
        if (n > 256) continue;
        const double rounds = (double)((rt * ntt * S + fit - 1) / fit), chunks = (nk + S - 1) / S;
        offer(2.9 + (S > 1 ? 0.55 : 0.0) + rounds * (chunks * (0.15 + 0.0008 * n) + 0.023 * n) + 0.052 * mb, {LIN_FEW, (int)n, S});
    }
    if (T <= 16) {
        int t;
        int64_t nchunk;
        linear_sparse_tokens(p, T, &t, &nchunk);
        const double e = (double)p->img.entries, nbk = p->img.nbk;
        const double ns = e * 10 * t + e * nbk * 70 + (double)p->M * (1000 + 700 * nbk * t);
        offer(2.4 + ns * (double)nchunk / sms * 1e-6 + 100e-6 * p->C * t, {LIN_SPARSE, t, 0});
    } else if (T > 64) {
        for (int wide = 0; wide < 2; ++wide) {
            const int nt = wide ? 256 : 128;
            const double tiles = (double)((T + 255) / 256) * ((rows + nt - 1) / nt), pairs = sms / 2;
            const double rounds = (double)(int64_t)((tiles + pairs - 1) / pairs), more = tiles > pairs ? tiles / pairs - 1 : 0;
            offer((wide ? 5.2 : 4.2) + rounds * (nk * (wide ? 0.26 : 0.233) + (wide ? 4.6 : 2.1)) + 0.02 * mb - more * nk * (wide ? 0.043 : 0.022),
                  {LIN_MANY, nt, 0});
        }
    }
    return best;
}

// SMs of the current device (asked once per device)
int device_sms()
{
    static std::atomic<int> known[64] = {};          // (calls come from any thread)
    int dev = 0, sms = 148;
    if (cudaGetDevice(&dev) != cudaSuccess) return sms;
    if (dev < 64)
        if (const int n = known[dev].load(std::memory_order_relaxed)) return n;
    if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 148;
    if (dev < 64) known[dev].store(sms, std::memory_order_relaxed);
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
    // The copy is waited for, so the host image (as large as the device's, 168 MB for 16384 x 4096 in 16 bits) need not stay:
    // launches read the geometry only. A stream under capture cannot be waited for and may replay the copy: there it stays.
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(st, &capture);
    if (e == cudaSuccess) e = cudaMemcpyAsync(dev_buf, p->img.bytes.data(), p->img.total, cudaMemcpyHostToDevice, st);
    if (e == cudaSuccess && capture == cudaStreamCaptureStatusNone) {
        e = cudaStreamSynchronize(st);
        std::vector<uint8_t>().swap(p->img.bytes);
    }
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
    if (y == x || (residual == y && T > 1 && ldr != ldy)) return UBP_E_ARG;      // (read whole rows; element by element)
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
