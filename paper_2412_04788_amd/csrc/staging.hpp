// Where the 16-byte pieces are that loads take from memory straight to LDS.  Plain arithmetic, which a host compiler takes as well.
//
// Such a load names a buffer (a base and a number of bytes), an offset of the lane's and one of the wave's, and gives zeros
// for what is beyond the buffer.  Only the lane's offset is sure to be held against the end.  So rows are reached by it alone: a
// lane whose row or piece is not there has an offset at or beyond the end, whatever is added to it, and the wave's offset
// stays within a row that is there.
#pragma once

#include <stdint.h>

namespace guide {

constexpr uint32_t kBeyond = 0x80000000u;                            // past the end of any buffer here

// Staged operands of a product have rows of 128 bytes, so that a load takes whole cache lines (rows of 64 bytes cost 7 % of a large
// product).
constexpr int kRow = 128;

// Place of 16-byte piece c of row r in it: sixteen rows' pieces of one c fall into sixteen different slots of the 256 bytes that
// LDS serves at once.
constexpr int swizzled(int r, int c) { return c ^ ((r >> 1) & 7); }

// ROWS rows of codes.  An instruction of a wave moves 1024 bytes, which it lays down in the lanes' order, so that the swizzle is on
// the memory's side (it repeats with every other instruction).
template <int ROWS, int WAVES>
struct TilePlaces {
    static constexpr int kLoads = ROWS * kRow / 1024 / WAVES, kRowsPer = 1024 / kRow, kForms = 2;       // instructions of a wave, rows of one
    uint32_t off[kForms] = {}, piece[kForms] = {}, stride = 0;

    constexpr void init(int64_t row_stride, int wave, int lane) {
        stride = (uint32_t)row_stride;
        for (int i = 0; i < kForms; ++i) {
            const int r = (wave * kLoads + i) * kRowsPer + lane / (kRow / 16);
            piece[i] = (uint32_t)swizzled(r, lane % (kRow / 16)) * 16;
            off[i] = (uint32_t)r * stride + piece[i];
        }
    }
    // Instruction i of the wave's kLoads; of the rows' bytes from the wave's offset on, `left` are there.
    constexpr uint32_t of_lane(int i, int left) const {
        return (int)piece[i % kForms] >= left ? kBeyond : off[i % kForms] + (uint32_t)(i / kForms * kForms * kRowsPer) * stride;
    }
    static constexpr uint32_t of_wave(int at, int left) { return left > 0 ? (uint32_t)at : 0u; }
    // Bytes of the buffer: up to the end of the tile's last row that is there (row_stride < 2^22).
    static constexpr uint32_t bytes(uint32_t rows, int64_t row_stride, int64_t row_bytes) {
        return (uint32_t)((int64_t)((rows < (uint32_t)ROWS ? rows : (uint32_t)ROWS) - 1) * row_stride + row_bytes);
    }
};

// Staged keys or values: tiles of 64 rows of D elements.  KEYS: rows are read 16 or 32 at a time, one piece of each; else (values)
// four at a time, 32 bytes of each.
constexpr int kTileK = 64;

template <int D, bool KEYS>
constexpr int piece_of(int r, int c) {
    if (KEYS) return D == 128 ? c ^ (r % 16) : c ^ (r / 2 % 8);
    return c ^ (r % 4 * (D / 32));
}

template <int D, bool KEYS, int WAVES>
struct KeyPlaces {
    static constexpr int kRow = D * 2, kRowsPer = 1024 / kRow, kLoads = kTileK / kRowsPer / WAVES, kRows = kLoads * kRowsPer;      // rows of a wave
    // From one instruction to the next, the pieces of keys change by an exclusive or with a constant (D = 128: row bits 2 and
    // 3, D = 64: row bit 3), those of values not at all.
    static constexpr uint32_t kFlip = KEYS ? 64 : 0;
    uint32_t row_off = 0, piece = 0;                                 // the lane's place in the wave's first instruction

    constexpr void init(int64_t stride, int wave, int lane) {        // stride in bytes, at most 2^25
        const int r = lane / (kRow / 16);
        row_off = (uint32_t)r * (uint32_t)stride;
        piece = (uint32_t)piece_of<D, KEYS>(wave * kRows + r, lane % (kRow / 16)) * 16;
    }
    // Instruction i of the wave's kLoads, from the first of the wave's rows on.
    constexpr uint32_t of_lane(int i, int64_t stride) const {
        return row_off + (uint32_t)(i * kRowsPer) * (uint32_t)stride + (piece ^ (uint32_t)i * kFlip);
    }
    // Bytes of the buffer, of which `left` rows are there.
    static constexpr uint32_t bytes(int left, int64_t stride) {
        return left <= 0 ? 0u : (uint32_t)((left < kRows ? left : kRows) - 1) * (uint32_t)stride + kRow;
    }
};

}  // namespace guide
