// Plan builder of the token-major products: the canonical blocks as (a) per start row streams of (input channel, nbk
// weights) entries for few tokens and (b) a densified K-major matrix for many. Host code only.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <thread>

#include "ubp_linear.h"
#include "ubp_internal.h"

namespace ubp {

namespace {

constexpr size_t round_up(size_t x, size_t n) { return (x + n - 1) / n * n; }

// rounding of one weight to the plan's type (to nearest, ties to even; 8 bits: after division by the row's scale)
inline void put_weight(uint8_t *dst, float w, float scale, int dtype)
{
    if (dtype == UBP_BF16) {
        const __nv_bfloat16 v = __float2bfloat16_rn(w);
        std::memcpy(dst, &v, 2);
    } else if (dtype == UBP_F16) {
        const __half v = __float2half_rn(w);
        std::memcpy(dst, &v, 2);
    } else {
        *dst = __nv_cvt_float_to_fp8(w / scale, __NV_SATFINITE, __NV_E4M3);
    }
}

// fn(first, last) over [0, n) in contiguous shares, a thread each where the work is worth it (a plan of a large layer is tens
// of millions of weights: 0.8 s on one core). An exception in a share is passed on; threads that cannot be had are done
// without.
template <typename Fn> void in_shares(int n, size_t work, Fn &&fn)
{
    unsigned most = std::thread::hardware_concurrency();
    most = most > 16 ? 16 : most;
    const int shares = work < (1u << 20) || most < 2 ? 1 : std::min((int)most, n);
    std::vector<std::exception_ptr> failed((size_t)shares);
    auto run = [&](int k) {
        try { fn((int)((int64_t)n * k / shares), (int)((int64_t)n * (k + 1) / shares)); }
        catch (...) { failed[(size_t)k] = std::current_exception(); }
    };
    std::vector<std::thread> threads;
    threads.reserve((size_t)shares);
    int started = 1;
    try { for (; started < shares; ++started) threads.emplace_back(run, started); }
    catch (...) {}
    run(0);
    for (int k = started; k < shares; ++k) run(k);
    for (auto &t : threads) t.join();
    for (auto &e : failed)
        if (e) std::rethrow_exception(e);
}

}  // namespace

int build_linear_image(const ubp_view_t &v, int dtype, bool gated, bool count_only, LinearImage &img)
{
    const int M = v.M, C = v.C, Nb = v.Nb;
    const int b = dtype == UBP_E4M3 ? 1 : (dtype == UBP_BF16 || dtype == UBP_F16) ? 2 : 0;
    if (!b) return UBP_E_ARG;
    if (v.R != 1 || C > 65536) return UBP_E_UNSUPPORTED;           // channel indices are 16 bits
    if (gated && M % 2 != 0) return UBP_E_ARG;
    img = LinearImage();
    int nbk = 1;                                                   // rows per entry: the largest of 1, 2, 4, 8 that divides Nb
    while (nbk < 8 && Nb % (nbk * 2) == 0) nbk *= 2;
    const int sub = Nb / nbk;
    img.nbk = nbk;
    img.entries = (int64_t)v.m * sub;
    if (img.entries >= (1ll << 31)) return UBP_E_UNSUPPORTED;
    const int epc = 16 / (nbk * b);
    img.epc = epc;
    std::vector<uint32_t> count((size_t)M, 0);                     // entries of each start row
    for (int i = 0; i < M; ++i)
        for (int s = 0; s < sub; ++s) count[(size_t)std::min(i + s * nbk, M - 1)] += (uint32_t)(v.indptr[i + 1] - v.indptr[i]);
    // Lanes a row: long rows to whole warps (few rows make few tasks for a block's sixteen warps), short ones to eight lanes
    // (a row's last step is half empty on average).
    const double mean = (double)img.entries / epc / M;
    const int lanes = mean >= 192 ? 32 : mean >= 80 ? 16 : 8, rb = 32 / lanes;
    img.lanes = lanes;
    img.bundles = (M + rb - 1) / rb;
    std::vector<uint32_t> off((size_t)img.bundles + 1, 0);
    for (int q = 0; q < img.bundles; ++q) {
        uint32_t most = 0;
        for (int i = q * rb; i < std::min(M, (q + 1) * rb); ++i) most = std::max(most, count[(size_t)i]);
        const uint32_t chunks = (most + (uint32_t)epc - 1) / (uint32_t)epc;
        off[(size_t)q + 1] = off[(size_t)q] + (chunks + (uint32_t)lanes - 1) / (uint32_t)lanes;
    }
    img.steps = off[(size_t)img.bundles];
    if (img.steps >= (1ll << 26)) return UBP_E_UNSUPPORTED;        // (chunk numbers stay below 2^31)
    const int F = gated ? M / 2 : M;
    img.Kp = (int)round_up((size_t)C, 128 / b);
    img.Mp = (int)round_up(gated ? round_up((size_t)F, 16) * 2 : (size_t)M, 128);
    size_t at = 256;
    img.scale_off = at;
    if (dtype == UBP_E4M3) at += round_up((size_t)M * 4, 256);
    img.off_off = at; at += round_up(((size_t)img.bundles + 1) * 4, 256);
    img.idx_off = at; at += round_up((size_t)img.steps * 32 * epc * 2, 256);
    img.val_off = at; at += round_up((size_t)img.steps * 512, 256);
    img.dense_off = at; at += round_up((size_t)img.Mp * img.Kp * b, 256);
    img.cnt_off = at; at += round_up((size_t)M * 4, 256);
    img.total = at;
    if (count_only) return UBP_OK;

    img.bytes.assign(at, 0);
    uint8_t *base = img.bytes.data();
    std::vector<float> scale((size_t)M, 1.f);
    // weight of output row `row` in block blk: the rotation keeps it in slot row mod Nb
    auto weight = [&](int32_t blk, int row) { return v.values[(size_t)blk * Nb + (size_t)(row % Nb)]; };
    if (dtype == UBP_E4M3) {
        in_shares(M, (size_t)v.m * Nb, [&](int r0, int r1) {
            for (int r = r0; r < r1; ++r) scale[(size_t)r] = 0.f;
            for (int i = std::max(0, r0 - Nb + 1); i < r1; ++i)
                for (int32_t k = v.indptr[i]; k < v.indptr[i + 1]; ++k)
                    for (int r = std::max(i, r0); r < std::min(i + Nb, r1); ++r) scale[(size_t)r] = std::max(scale[(size_t)r], std::fabs(weight(k, r)));
            for (int r = r0; r < r1; ++r) scale[(size_t)r] = std::max(scale[(size_t)r] / 448.f, 1.17549435e-38f);
        });
        std::memcpy(base + img.scale_off, scale.data(), (size_t)M * 4);
    }
    std::memcpy(base + img.off_off, off.data(), off.size() * 4);
    std::memcpy(base + img.cnt_off, count.data(), count.size() * 4);
    // place of entry n of start row i
    auto place = [&](int i, uint32_t n) {
        const uint32_t c = n / (uint32_t)epc, step = off[(size_t)(i / rb)] + c / (uint32_t)lanes;
        return ((size_t)step * 32 + (size_t)((i % rb) * lanes) + c % (uint32_t)lanes) * (size_t)epc + n % (uint32_t)epc;
    };
    uint16_t *idx = reinterpret_cast<uint16_t *>(base + img.idx_off);
    uint8_t *val = base + img.val_off, *dense = base + img.dense_off;
    // Start row i of entries: the blocks that start s * nbk rows above it, s-th part of each. Every row's entries and every
    // weight's place in the dense matrix belong to one start row, so shares of rows do not meet.
    in_shares(M, (size_t)img.entries * nbk, [&](int r0, int r1) {
        for (int i = r0; i < r1; ++i) {
            uint32_t n = 0;
            uint16_t last = 0;
            for (int s = 0; s < sub; ++s) {
                const int start = i - s * nbk;
                if (start < 0) break;
                for (int32_t k = v.indptr[start]; k < v.indptr[start + 1]; ++k) {
                    const int j = v.indices[k];
                    const size_t e = place(i, n++);
                    idx[e] = last = (uint16_t)j;
                    for (int t = 0; t < nbk; ++t) {
                        const int row = i + t;
                        uint8_t *w = val + (e * (size_t)nbk + (size_t)t) * b;
                        put_weight(w, weight(k, row), scale[(size_t)row], dtype);
                        const int f = row < F ? row : row - F;
                        const size_t d = !gated ? (size_t)row : (size_t)(f / 16) * 32 + (row < F ? 0 : 16) + (size_t)(f % 16);
                        std::memcpy(dense + (d * (size_t)img.Kp + (size_t)j) * b, w, (size_t)b);
                    }
                }
            }
            const uint32_t all = (off[(size_t)(i / rb) + 1] - off[(size_t)(i / rb)]) * (uint32_t)(lanes * epc);
            for (; n < all; ++n) idx[place(i, n)] = last;
        }
    });
    return UBP_OK;
}

}  // namespace ubp
