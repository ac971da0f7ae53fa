// Token-major products with a block-pruned weight: plan of one layer and what its two kernels share.
#ifndef UBP_LINEAR_H_
#define UBP_LINEAR_H_

#include <cuda.h>

#include <cstddef>
#include <cstdint>
#include <vector>

#include "ubp.h"

namespace ubp {

// Device image (all offsets from its base, which is 256-byte aligned):
//   [0, 256)      header; int32 status word at byte 0
//   scale_off     float[M]: scale of each weight row (8-bit plans only)
//   off_off       uint32[bundles + 1]: first step of a bundle. A bundle is 32 / lanes consecutive start rows, a row is dealt
//                 to `lanes` lanes of a warp in chunks of 16 bytes of weights = epc entries of nbk weights each, and a step is
//                 one chunk for each of the warp's 32 lanes (lane = row in the bundle * lanes + place): chunk i of a row lies in
//                 step i / lanes, place i mod lanes. Rows are filled up to their bundle's steps with entries of weight zero.
//   idx_off       uint16[steps][32][epc]: input channel of an entry (of a filler: the row's last channel, 0 in an empty row)
//   val_off       weights [steps][32][epc][nbk]: consecutive output rows from the entry's start row (plan's type)
//   dense_off     the densified weight [Mp][Kp] (plan's type), K contiguous. Gated plans interleave the two halves in
//                 groups of 16 rows: dense row 32 g + i is gate row 16 g + i, dense row 32 g + 16 + i is up row 16 g + i.
//                 Kp = C rounded up to 128 bytes, Mp = rows rounded up to 128; the padding is zero.
//   cnt_off       uint32[M]: entries of a start row without the fillers
struct LinearImage {
    std::vector<uint8_t> bytes;
    size_t scale_off = 0, off_off = 0, idx_off = 0, val_off = 0, dense_off = 0, cnt_off = 0, total = 0;
    int nbk = 1, epc = 1, lanes = 8, bundles = 0, Mp = 0, Kp = 0;
    int64_t entries = 0, steps = 0;
};
int build_linear_image(const ubp_view_t &v, int dtype, bool gated, bool count_only, LinearImage &img);

constexpr uint32_t kLinearMagic = 0x4c504255u;   // "UBPL": first word of a live handle

}  // namespace ubp

struct ubp_linear_plan {
    uint32_t magic;
    int M, C, Nb, m;
    int dtype, gated;
    int F;                          // output features: M, or M / 2 of a gated plan
    ubp::LinearImage img;           // geometry and offsets (its bytes are released after the upload)
    uint8_t *dev;                   // caller's device buffer
};

namespace ubp {

// One product, as the kernels get it (device pointers; strides in elements).
struct LinearArgs {
    const void *x;
    int64_t ldx;
    const float *xs;                // scale of each token, 8-bit plans only
    int64_t T;
    const float *bias;              // [M] or null
    int act;
    const void *res;                // null or [T][F] in y's type
    int64_t ldr;
    void *y;
    int64_t ldy;
    int *status;
    int M, C, F, gated;
};

// Which kernel a launch takes and its tile.
enum { LIN_SPARSE = 0, LIN_FEW = 1, LIN_MANY = 2 };
struct LinearChoice {
    int kernel;                     // LIN_*
    int cols;                       // LIN_SPARSE, LIN_FEW: tokens per block; LIN_MANY: dense weight rows per tile
    int split;                      // LIN_FEW: blocks of a cluster that share a reduction
};
LinearChoice linear_choose(const ubp_linear_plan *p, int64_t T, int sms);

// tokens a block of the kept-block kernel takes (1, 2, 4 or 8) and the number of such groups
void linear_sparse_tokens(const ubp_linear_plan *p, int64_t T, int *tokens, int64_t *groups);
int launch_linear_sparse(const ubp_linear_plan *p, const LinearArgs &a, int y_dtype, int sms, void *stream);
int device_sms();
// whether the tensor-core kernels can copy x's rows as they are (else they go through the workspace, [T][Kp])
bool linear_x_direct(const ubp_linear_plan *p, const void *x, int64_t ldx, int64_t T);
int launch_linear_tc(const ubp_linear_plan *p, const LinearArgs &a, int y_dtype, const LinearChoice &ch, void *workspace, int sms,
                     void *stream);

}  // namespace ubp
#endif
