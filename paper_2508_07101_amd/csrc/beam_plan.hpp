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
constexpr int BEAM_MIN_PIECE = 256;     // tokens
constexpr int BEAM_PIECE_COST = 16;     // tiles of 32 tokens that a piece costs besides its own
inline bool beam_pages_served(int64_t pages) { return pages <= (int64_t)BEAM_LIST * BEAM_MAX_SPLITS; }

// The host knows no more than width * max_seq_len tokens, of which rows that share have a fraction: a group stays whole up to a bound that costs little if they share nothing (4 beams of one group,
// 8 KV heads: 1000 tokens whole 14.2 us, cut and merged 14.4; 700: 10.8 and 12.4; 1550: 17.7 and 14.8), a higher one where half of the CUs have a workgroup anyway (16 groups of 4 beams: 600 tokens, bound 2600,
// whole 13.2, cut 16.5; 1000, bound 4100, 17.1 and 19.9).  Where all have two already, pieces only make up for lengths.
constexpr int BEAM_WHOLE = 2048, BEAM_WHOLE_MANY = 4096;   // tokens

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
    const int64_t pieces = max_len <= (wgs >= BEAM_CUS / 2 ? BEAM_WHOLE_MANY : BEAM_WHOLE) ? 1 : (max_len + least - 1) / least;
    p.n_splits = (int)std::max<int64_t>({1, by_list, std::min<int64_t>({want, pieces, BEAM_MAX_SPLITS})});
    return p;
}

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
