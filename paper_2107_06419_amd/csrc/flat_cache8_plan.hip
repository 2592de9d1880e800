// Host-side planning of attention over the 8-bit cache, and the frequencies of rotary positions (no device code).
#include <math.h>

#include "flat_cache8.hpp"

namespace flat {

void cache8_plan(int B, int H, int heads, int Nq, int max_tokens, int d, Cache8Plan* out) {
    constexpr int kMaxEntries = 1024, kLeastKeys = 256;
    const long long rows = (long long)Nq * (H / heads);
    out->rows_per_block = rows <= 32 ? 32 : rows <= 64 && d != 256 ? 64 : 128;
    out->tile_keys = out->rows_per_block > 32 ? 64 : d == 32 ? 128 : d == 64 ? 64 : 32;
    out->row_blocks = (int)((rows + out->rows_per_block - 1) / out->rows_per_block);
    const long long entries = (long long)B * out->row_blocks;
    out->entries = (int)entries;
    out->least_tiles = kLeastKeys / out->tile_keys;
    const long long tiles = ((long long)max_tokens + out->tile_keys - 1) / out->tile_keys;
    // units that the chip holds at once: 256 compute units of two workgroups (d = 256: one; 64 rows of up to 64 channels: four)
    const int slots = 256 * (d == 256 ? 1 : out->rows_per_block == 64 && d <= 64 ? 4 : 2) / heads;
    out->aim = out->limit = 0;
    out->parts_at = out->workspace_bytes = 0;
    // With more entries than kMaxEntries nothing is divided: they fill the chip by themselves, and finding a unit would cost more than it gives.  Neither
    // are blocks of many rows that fill it: their lengths differ little, and putting their many rows together costs more.
    if (entries <= kMaxEntries && tiles > out->least_tiles && (out->rows_per_block == 32 || entries < slots)) {
        out->aim = slots > entries ? slots : (int)entries;
        out->limit = 2 * entries <= out->aim ? out->aim : out->aim + (int)entries;
        out->parts_at = ((size_t)entries * 8 + 15) / 16 * 16;
        out->workspace_bytes = out->parts_at + (size_t)out->limit * heads * out->rows_per_block * (d + 2) * sizeof(float);
    }
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
