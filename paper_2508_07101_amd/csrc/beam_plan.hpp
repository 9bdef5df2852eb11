// How attention over a group's pages is cut into workgroups.  Plain host code, no HIP: the rules can be looked at without a GPU.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace cusa {

constexpr int BEAM_ROWS = 32;           // rows (row of the group, query head) of one KV head in a workgroup
constexpr int BEAM_CUS = 256;
constexpr int BEAM_LIST = 8192;         // pages of a piece: a bit each in LDS
constexpr int BEAM_MAX_SPLITS = 64;     // pieces of a group's pages: one lane each in the merge
constexpr int BEAM_MIN_PIECE = 128;     // tokens: a tile for each wave (4 beams of 4096 tokens 8.7 us, by 256 9.5; 8 of 2000 10.4 and 11.8; longer ones alike)
constexpr int BEAM_PIECE_COST = 16;     // tiles of 32 tokens that a piece costs besides its own
inline bool beam_pages_served(int64_t pages) { return pages <= (int64_t)BEAM_LIST * BEAM_MAX_SPLITS; }

// The host knows no more than a bound, width * max_seq_len tokens or the pool's, of which rows that share have a fraction.  Few groups stay whole up to a bound that costs little whether it is near the truth or far above it,
// a lower one where a workgroup has more than 16 rows; many up to a higher one.  Us a call, whole and cut, 8 KV heads: one group of 4 beams, 500 tokens 10.4 and 14.5, 900 12.6 and 14.2, 1200 15.6 and 14.1, 1700 19.8 and 14.0;
// of 8 beams (32 rows) 400 12.5 and 13.8, 600 14.1 and 13.9, 1000 18.1 and 13.6; 4 groups of 4, bound 1800, 500 tokens 10.0 and 13.9; 16 of 4, 1200 19.0 and 20.9, 2700 34 and 34; 24 of 4 28 and 31 at 1700.
// Where all CUs have two workgroups, pieces only make up for lengths.
constexpr int BEAM_WHOLE = 1280, BEAM_WHOLE_WIDE = 768, BEAM_WHOLE_MANY = 4096;   // tokens

struct BeamPlan {
    int blocks;      // workgroups that share a KV head's pages
    int n_splits;    // pieces of a group's pages at most; the kernel makes fewer of a short list
};
inline BeamPlan plan_beams(int64_t max_pages, int groups, int G, int rows) {
    const int64_t max_len = max_pages * 16;
    BeamPlan p;
    p.blocks = (rows + BEAM_ROWS - 1) / BEAM_ROWS;
    const int64_t wgs = (int64_t)groups * G * p.blocks;
    const int64_t want = groups == 1 ? 2 * BEAM_CUS / wgs : wgs >= 16 * BEAM_CUS ? 1 : std::max<int64_t>(4, 4 * BEAM_CUS / wgs);
    const int64_t by_list = (max_pages + BEAM_LIST - 1) / BEAM_LIST, least = wgs >= 2 * BEAM_CUS ? 4096 : BEAM_MIN_PIECE;
    const int64_t pieces = max_len <= (wgs >= BEAM_CUS / 2 ? BEAM_WHOLE_MANY : rows <= 16 ? BEAM_WHOLE : BEAM_WHOLE_WIDE) ? 1 : (max_len + least - 1) / least;
    p.n_splits = (int)std::max<int64_t>({1, by_list, std::min<int64_t>({want, pieces, BEAM_MAX_SPLITS})});
    return p;
}

// Workgroups of the launch: blocks of rows for each piece and KV head, rounded up to 8 XCDs.  A launch has fewer than 2^32 threads.
inline int64_t beam_units(const BeamPlan& p, int groups, int G) { return ((int64_t)p.n_splits * G * groups + 7) / 8 * 8 * p.blocks; }
inline bool beam_units_served(int64_t units) { return units < 1 << 24; }

// Bytes of partial results: 128 sums, a maximum and a denominator per row and piece.
struct BeamAttnWs {
    size_t acc, ml, pieces, total;
};
inline BeamAttnWs beam_attn_workspace(const BeamPlan& p, int batch, int H, int groups) {
    const size_t rows = p.n_splits > 1 ? (size_t)batch * H * p.n_splits : 0;
    BeamAttnWs w;
    w.acc = 0;
    w.ml = (rows * 128 * 4 + 255) / 256 * 256;
    w.pieces = w.ml + (rows * 2 * 4 + 255) / 256 * 256;
    w.total = w.pieces + ((size_t)groups * 4 + 255) / 256 * 256;
    return w;
}

}  // namespace cusa
