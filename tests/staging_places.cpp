// Every offset that loads from memory straight to LDS are given, at every number of rows that is there: pieces that exist are reached
// where they are; a lane's offset of any other piece is at or beyond the buffer's end by itself, and the wave's is below it.
#include <cstdio>
#include <cstdlib>
#include <set>

#include "staging.hpp"

using namespace guide;

static long checked = 0;
static void expect(bool ok, const char *what, long a, long b, long c) {
    ++checked;
    if (ok) return;
    std::printf("%s: %ld %ld %ld\n", what, a, b, c);
    std::exit(1);
}

template <int ROWS>
static void tiles(uint32_t rows, int64_t stride, int64_t row_bytes) {
    using P = TilePlaces<ROWS, 4>;
    const uint64_t end = P::bytes(rows, stride, row_bytes);
    const uint32_t there = rows < ROWS ? rows : ROWS;
    expect(end == (there - 1) * (uint64_t)stride + row_bytes && end < kBeyond, "bytes of a tile", ROWS, rows, stride);
    for (int64_t at = 0; at < row_bytes + 3 * kRow; at += kRow) {
        const int left = (int)(row_bytes - at);
        expect(P::of_wave((int)at, left) < end, "the wave's offset", ROWS, rows, at);
        std::set<uint32_t> seen;
        for (int wave = 0; wave < 4; ++wave)
            for (int lane = 0; lane < 64; ++lane) {
                P p;
                p.init(stride, wave, lane);
                for (int i = 0; i < P::kLoads; ++i) {
                    const int r = (wave * P::kLoads + i) * P::kRowsPer + lane / 8, c = swizzled(r, lane % 8);      // what the lane's place in LDS stands for
                    const uint64_t lane_off = p.of_lane(i, left), wave_off = P::of_wave((int)at, left);
                    if ((uint32_t)r < there && c * 16 < left) {
                        expect(lane_off + wave_off == r * (uint64_t)stride + at + c * 16 && lane_off + wave_off + 16 <= end, "a piece that is there", ROWS, r, c);
                    } else {
                        expect(lane_off >= end, "a piece that is not there", ROWS, r, c);
                    }
                    seen.insert((uint32_t)(r * 8 + c));
                }
            }
        expect(seen.size() == ROWS * 8u, "every piece has a place", ROWS, rows, at);
    }
}

template <int D, bool KEYS, int WAVES>
static void keys(int left_of_tile, int64_t stride) {
    using P = KeyPlaces<D, KEYS, WAVES>;
    std::set<uint32_t> seen;
    for (int wave = 0; wave < WAVES; ++wave) {
        const int left = left_of_tile - wave * P::kRows;
        const uint64_t end = P::bytes(left, stride);
        expect(end < kBeyond && (left > 0) == (end > 0), "bytes of keys", D, left, stride);
        for (int lane = 0; lane < 64; ++lane) {
            P p;
            p.init(stride, wave, lane);
            for (int i = 0; i < P::kLoads; ++i) {
                const int r = i * P::kRowsPer + lane / (D / 8), c = piece_of<D, KEYS>(wave * P::kRows + r, lane % (D / 8));
                const uint64_t off = p.of_lane(i, stride);
                if (r < left) expect(off == r * (uint64_t)stride + c * 16 && off + 16 <= end, "a piece of a key", D, r, c);
                else expect(off >= end, "a piece beyond the last key", D, r, c);
                seen.insert((uint32_t)((wave * P::kRows + r) * (D / 8) + c));
            }
        }
    }
    expect(seen.size() == kTileK * (D / 8u), "every piece has a place", D, left_of_tile, stride);
}

template <int D, int WAVES>
static void both(int left, int64_t stride) {
    keys<D, true, WAVES>(left, stride);
    keys<D, false, WAVES>(left, stride);
}

int main() {
    for (uint32_t rows = 1; rows < 300; rows += rows < 140 ? 1 : 7) {
        const int64_t sizes[][2] = {{16, 16}, {32, 16}, {4096, 4096}, {1040, 1024 + 16}, {(1 << 22) - 16, 160}};       // row stride, bytes of a row
        for (const auto &s : sizes) {
            tiles<64>(rows, s[0], s[1]);
            tiles<128>(rows, s[0], s[1]);
            tiles<256>(rows, s[0], s[1]);
        }
    }
    for (int left = -70; left < 140; ++left)
        for (int64_t stride : {256ll, 258ll, 1280ll, 1ll << 25}) {
            both<64, 4>(left, stride);
            both<128, 4>(left, stride);
            both<128, 8>(left, stride);
        }
    std::printf("%ld\n", checked);
    return 0;
}
