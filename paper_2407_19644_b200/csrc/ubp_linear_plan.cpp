// Plan builder of the token-major products: the canonical blocks as (a) per start row streams of (input channel, nbk
// weights) entries for few tokens and (b) a densified K-major matrix for many. Host code only.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp8.h>

#include <algorithm>
#include <cmath>
#include <cstring>

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
    img.total = at;
    if (count_only) return UBP_OK;

    img.bytes.assign(at, 0);
    uint8_t *base = img.bytes.data();
    std::vector<float> scale((size_t)M, 1.f);
    // weight of output row `row` in block blk: the rotation keeps it in slot row mod Nb
    auto weight = [&](int32_t blk, int row) { return v.values[(size_t)blk * Nb + (size_t)(row % Nb)]; };
    if (dtype == UBP_E4M3) {
        std::fill(scale.begin(), scale.end(), 0.f);
        for (int i = 0; i < M; ++i)
            for (int32_t k = v.indptr[i]; k < v.indptr[i + 1]; ++k)
                for (int t = 0; t < Nb; ++t) scale[(size_t)(i + t)] = std::max(scale[(size_t)(i + t)], std::fabs(weight(k, i + t)));
        for (auto &s : scale) s = std::max(s / 448.f, 1.17549435e-38f);
        std::memcpy(base + img.scale_off, scale.data(), (size_t)M * 4);
    }
    std::memcpy(base + img.off_off, off.data(), off.size() * 4);
    std::vector<uint32_t> next((size_t)M, 0);                        // entries of each start row placed so far
    // place of entry n of start row i
    auto place = [&](int i, uint32_t n) {
        const uint32_t c = n / (uint32_t)epc, step = off[(size_t)(i / rb)] + c / (uint32_t)lanes;
        return ((size_t)step * 32 + (size_t)((i % rb) * lanes) + c % (uint32_t)lanes) * (size_t)epc + n % (uint32_t)epc;
    };
    uint16_t *idx = reinterpret_cast<uint16_t *>(base + img.idx_off);
    uint8_t *val = base + img.val_off, *dense = base + img.dense_off;
    for (int i = 0; i < M; ++i)
        for (int32_t k = v.indptr[i]; k < v.indptr[i + 1]; ++k) {
            const int j = v.indices[k];
            for (int s = 0; s < sub; ++s) {
                const size_t e = place(i + s * nbk, next[(size_t)(i + s * nbk)]++);
                idx[e] = (uint16_t)j;
                for (int t = 0; t < nbk; ++t) {
                    const int row = i + s * nbk + t;
                    uint8_t *w = val + (e * (size_t)nbk + (size_t)t) * b;
                    put_weight(w, weight(k, row), scale[(size_t)row], dtype);
                    const int f = row < F ? row : row - F;
                    const size_t d = !gated ? (size_t)row : (size_t)(f / 16) * 32 + (row < F ? 0 : 16) + (size_t)(f % 16);
                    std::memcpy(dense + (d * (size_t)img.Kp + (size_t)j) * b, w, (size_t)b);
                }
            }
        }
    for (int i = 0; i < M; ++i) {
        const uint32_t all = (off[(size_t)(i / rb) + 1] - off[(size_t)(i / rb)]) * (uint32_t)(lanes * epc);
        const uint16_t last = next[(size_t)i] ? idx[place(i, next[(size_t)i] - 1)] : 0;
        for (uint32_t n = next[(size_t)i]; n < all; ++n) idx[place(i, n)] = last;
    }
    return UBP_OK;
}

}  // namespace ubp
