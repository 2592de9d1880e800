// Host-side planning of attention over the 8-bit cache, and the frequencies of rotary positions (no device code).
#include <math.h>

#include "flat_cache8.hpp"

namespace flat {

// Which kernel an attention call takes, and whether the keys of its entries are divided over workgroups.  Figures: e4m3, 4 query heads to a head of the cache,
// us, a hipGraph of ten calls; BH = batch entries * heads of the cache.
//
// Blocks of 16 or 32 rows, whose keys the four wavefronts of a workgroup share, or of 256 (d = 256: 128), whose tiles are widened once for eight (four) wavefronts of 32 rows.
// The latter are ahead where there is one for each of the 256 compute units and 7 of 8 of their wavefronts have rows.  256 blocks of 4096 keys, blocks of 32 / 256 rows: d = 128
// 199 / 155, d = 64 109 / 104; d = 32, 2048 keys 54 / 51; d = 96 78 / 76; d = 256 121 / 107; half as many blocks, d = 128 98 / 131, d = 64 59 / 94, d = 256 66 / 101; a quarter of the
// wavefronts without rows, d = 128 157 / 155, d = 64 86 / 105, d = 32 42 / 48, d = 96 61 / 73, d = 256 98 / 104.
//
// Dividing costs a launch and the parts' way through memory, 5 us and more, and gives shorter walks over the keys and even shares of a ragged batch.  A workgroup takes
// about 5.5 us and `round` per step of its four wavefronts, but no less than the memory takes for the codes of all of them at 5.2 TB/s, counted at 0.45: a batch is as often
// ragged as not, and its longest walk counts.  What dividing saves is the difference, step by step.  Up to 16 rows, ragged batches of 0.1 to 1 times the keys, undivided / divided: d = 64,
// BH = 64, 2048 keys 10.7 / 10.8, 4096 17.3 / 13.8; BH = 128, 2048 11.3 / 13.5, 16384 59 / 36; BH = 256, 16384 70 / 67; d = 128, BH = 64, 2048 14.1 / 14.6, 4096 21.7 / 17.6; BH = 128, 4096 22.1 /
// 22.0, 16384 90 / 65; BH = 256, 4096 33.6 / 35.6; d = 256, BH = 64, 1024 16.9 / 15.7; BH = 128, 1024 17.7 / 18.7, 4096 51 / 40.
void cache8_plan(int B, int H, int heads, int Nq, int max_tokens, int d, Cache8Plan* out) {
    constexpr int kLeastKeys = 256;
    const int held = d == 256 ? 256 : 512;  // workgroups that 256 compute units hold at once
    const long long rows = (long long)Nq * (H / heads);
    const int many = d == 256 ? 128 : 256;
    const long long blocks = (rows + many - 1) / many;
    const bool filled = blocks * B * heads >= 256 && 8 * ((rows + 31) / 32) >= 7 * blocks * (many / 32);
    out->rows_per_block = filled ? many : rows <= 16 && d % 64 == 0 ? 16 : 32;
    out->row_blocks = (int)((rows + out->rows_per_block - 1) / out->rows_per_block);
    const long long entries = (long long)B * out->row_blocks, grid = entries * heads;
    out->entries = (int)entries;
    out->tile_keys = out->rows_per_block > 32 ? 64 : cache8_step_keys(out->rows_per_block, d);
    out->least_tiles = kLeastKeys / out->tile_keys;
    out->aim = out->limit = 0;
    out->parts_at = out->workspace_bytes = 0;
    if (out->rows_per_block > 32 || grid >= held) return;
    const double round = out->rows_per_block == 16 ? (d == 64 ? 0.62 : d == 128 ? 0.95 : 2.4) : d == 32 ? 1.5 : d == 64 ? 0.87 : d == 96 ? 0.64 : d == 128 ? 0.67 : 1.2;  // us
    const long long round_keys = 4 * out->tile_keys, rounds = (max_tokens + round_keys - 1) / round_keys;
    const double memory = 0.45 * (double)grid * (double)(round_keys * 2 * d) / 5.2e6;
    if ((double)rounds * (round - memory) <= 5.5 + (double)(rows < 32 ? rows : 32) / 16.0) return;
    out->aim = held / heads > entries ? held / heads : (int)entries;
    out->limit = 2 * entries <= out->aim ? out->aim : out->aim + (int)entries;
    out->parts_at = ((size_t)entries * 8 + 15) / 16 * 16;
    out->workspace_bytes = out->parts_at + (size_t)out->limit * heads * out->rows_per_block * (d + 2) * sizeof(float);
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
