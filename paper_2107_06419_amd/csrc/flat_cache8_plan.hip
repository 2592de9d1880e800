// Host-side planning of attention over the 8-bit cache, and the frequencies of rotary positions (no device code).
#include <math.h>

#include "flat_cache8.hpp"

namespace flat {

// How many units a launch aims at: what the chip holds at once (256 compute units, two workgroups each, one at d = 256), over the heads of the
// cache.  Which entry gets how many is settled on the device from the lengths.  With more entries than kMaxEntries nothing is divided: they fill
// the chip by themselves, and finding one's unit would cost more than it gives.
void cache8_plan(int B, int H, int heads, int Nq, int max_tokens, int d, Cache8Plan* out) {
    constexpr int kMaxEntries = 1024, kLeastTiles = 8;
    const long long rows = (long long)Nq * (H / heads);
    out->rows_per_block = 32;
    out->row_blocks = (int)((rows + out->rows_per_block - 1) / out->rows_per_block);
    const long long entries = (long long)B * out->row_blocks;
    out->entries = (int)entries;
    out->least_tiles = kLeastTiles;
    const long long tiles = ((long long)max_tokens + 2 * kCacheBlock - 1) / (2 * kCacheBlock);
    const int slots = (d == 256 ? 256 : 512) / heads;
    out->target = 0;
    if (entries <= kMaxEntries && tiles > kLeastTiles) out->target = slots > entries ? slots : (int)entries;
    out->max_units = (int)entries + out->target;
    out->workspace_bytes = out->target ? (size_t)out->max_units * heads * out->rows_per_block * (d + 2) * sizeof(float) : 0;
}

}  // namespace flat

extern "C" int flat_attn_rope_freqs(double* out, int rot_d, double base, int scaling, double factor, double original_len, double low, double high) {
    if (!out) return FLAT_ERR_NULL;
    if (rot_d < 2 || rot_d > 256 || rot_d % 2) return FLAT_ERR_UNSUPPORTED;
    if (scaling < FLAT_ROPE_SCALE_NONE || scaling > FLAT_ROPE_SCALE_BANDS) return FLAT_ERR_UNSUPPORTED;
    if (!(base > 1.0) || isinf(base)) return FLAT_ERR_UNSUPPORTED;
    if (scaling != FLAT_ROPE_SCALE_NONE && (!(factor >= 1.0) || isinf(factor))) return FLAT_ERR_UNSUPPORTED;
    if (scaling == FLAT_ROPE_SCALE_BANDS && (!(original_len > 0.0) || isinf(original_len) || !(low >= 0.0) || !(high > low) || isinf(high))) return FLAT_ERR_UNSUPPORTED;
    if (scaling == FLAT_ROPE_SCALE_BASE && rot_d > 2) base *= pow(factor, (double)rot_d / (rot_d - 2));
    for (int i = 0; i < rot_d / 2; ++i) {
        double f = pow(base, -2.0 * i / rot_d);
        if (scaling == FLAT_ROPE_SCALE_LINEAR) f /= factor;
        if (scaling == FLAT_ROPE_SCALE_BANDS) {
            const double turns = original_len * f / (2.0 * 3.14159265358979323846);
            const double share = (turns - low) / (high - low), keep = share < 0.0 ? 0.0 : share > 1.0 ? 1.0 : share;
            f = f * keep + f / factor * (1.0 - keep);
        }
        out[i] = f;
    }
    return FLAT_OK;
}
