// How a product with an epilogue runs: tiles, parts of the reduction, way of the operands.  (Host code alone.)
#pragma once

#include <algorithm>
#include <cstdint>

namespace capgnn {

struct LinearPlan {
    int tile;                   // rows and columns of a tile, where the operands' rows start on 4 bytes; 0: a few rows
    int parts;                  // of the reduction
    int64_t part_k;
};
constexpr int FEW_ROWS = 16;            // (32 by two such groups: 32 x 4096 x 4096 bf16 15.3 us, 33 rows by tiles of 64 in parts 13.5)

inline bool cut_pays(int64_t M, int64_t N, int64_t K) { return M * N >= ((int64_t(1) << 28) + K - 1) / std::max<int64_t>(K, 1); }

inline LinearPlan linear_plan(int64_t M, int64_t N, int64_t K, int es) {
    LinearPlan p{0, 1, K};
    auto tiles = [&](int64_t b) { return ((M + b - 1) / b) * ((N + b - 1) / b); };
    const int64_t lines = (K * es + 127) / 128;         // steps
    int64_t groups, most;
    if (M <= FEW_ROWS) {
        groups = (N + 15) / 16;
        most = lines / 32;
    } else {
        // Large tiles read their operands less often, where there are enough of them for the compute units, little of them lies beyond the matrix
        // and the reduction is long enough for what a workgroup alone on its compute unit cannot overlap: its first loads and its results.
        // us, tiles of 256 / 128 / 64: 8192 x 8192 x 2048 bf16 298 / 329 / 463, x 1024 206 / 208 / 272, x 256 133 / 111 / 147; x 1024 fp32
        // 647 / 717 / 1047, x 256 222 / 215 / 305; x 1024 e4m3 166 / 145 / 187, x 2048 216 / 204 / 266; 612000 x 47 x 256 bf16 274 / 157 / 107,
        // fp32 660 / 296 / 233; 3000^3 bf16 (144 tiles of 256) 123 with them, 105 / 117 with the others.
        auto wide = [&](int64_t b) { return tiles(b) * b * b * 4 <= tiles(b / 2) * (b / 2) * (b / 2) * 5; };
        // Tiles of 128 in parts of 32 steps and more, where that gives every compute unit one: 6095 x 376 x 5188 fp32 177, tiles of 64 281;
        // 1500 x 1500 x 6000 bf16 60 / 84; 100 x 8192 x 8192 bf16 45.5 / 44.3, 300 x 4096 x 8192 37.6 / 47.6 (with parts of 16, 2048 x 1024 x 2048
        // bf16 23.8 / 17.7).
        const int64_t split = tiles(128) < 256 ? std::min<int64_t>(std::min<int64_t>(lines / 32, 512 / tiles(128)), 32) : 1;
        p.tile = tiles(256) >= 200 && wide(256) && lines >= (es == 1 ? 32 : 16) ? 256 : tiles(128) * split >= 256 && wide(128) ? 128 : 64;
        groups = tiles(p.tile);
        most = p.tile == 64 ? lines / 8 : p.tile == 128 ? split : 1;
    }
    // (enough workgroups for the chip, parts of 8 steps or more; of a few rows 32)
    const int64_t parts = std::min<int64_t>(std::min<int64_t>(most, (p.tile ? 512 : 256) / groups), 32);
    if (parts > 1) {
        const int64_t each = (lines + parts - 1) / parts;
        p.part_k = each * (128 / es);
        p.parts = static_cast<int>((lines + each - 1) / each);
        if (p.parts == 1) p.part_k = K;
    }
    return p;
}

// The kernel that a plan's product takes.  es: bytes of an operand's element (4: fp32); rows_of_4: both operands' rows start on 4 bytes and
// are shorter than 2^23 bytes apart.
struct LinearWay {
    int tile;                   // as it runs
    bool cut;                   // fp32 operands in three bf16 pieces
    bool direct;                // operands straight to LDS
    int waves;                  // of a workgroup, a few rows only
};
constexpr int FEW_WAVES = 16;           // of a workgroup, at most

inline LinearWay linear_way(const LinearPlan &p, int64_t M, int64_t N, int64_t K, int es, bool rows_of_4) {
    LinearWay w{0, false, false, 1};
    if (p.tile == 0) {
        const int64_t lines = (p.part_k * es + 127) / 128;          // a line of a row per wave and turn
        while (w.waves < FEW_WAVES && w.waves < lines / 4 + 1) w.waves *= 2;
        while ((N + 15) / 16 * w.waves * 64 >= int64_t(1) << 32 && w.waves > 1) w.waves /= 2;      // (of a launch: fewer than 2^32 threads)
        return w;
    }
    w.cut = es == 4 && rows_of_4 && cut_pays(M, N, K);
    // One or two steps pay for no loads ahead: through registers more workgroups share a compute unit (us, to LDS / through registers:
    // 612000 x 47 x 100 bf16 104 / 80, x 128 82 / 65, 100000 x 256 x 100 44 / 37, 16311 x 2503 x 2 fp32 74 / 63; two whole steps of larger
    // tiles, 8192 x 4096 x 128 28.2 / 30.6; three steps and more the same or less).  Below 256 bytes larger tiles straight to LDS and those of 64
    // through registers are near one another: 8192 x 4096 x 64 bf16 25.0 / 26.4, 8192 x 8192 x 64 45 / 48, 180000 x 256 x 64 30.6 / 30.8,
    // 612000 x 256 x 100 213 / 225, 100000 x 256 x 100 42 / 36, 8192 x 4096 x 16 34.6 / 30.5.
    w.direct = w.cut || (rows_of_4 && K * es >= (p.tile == 64 ? 257 : 256));
    w.tile = !w.direct || (es == 4 && !w.cut) ? 64 : p.tile;
    return w;
}

}  // namespace capgnn
