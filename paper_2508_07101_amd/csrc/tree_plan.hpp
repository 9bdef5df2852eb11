// How attention over trees of drafted tokens is cut into workgroups.  Plain host code, no HIP: the rules can be looked at without a GPU.
#pragma once

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace cusa {

constexpr int TREE_MAX_NODES = 256;
constexpr int TREE_MAX_SPLITS = 64;     // pieces of a sequence's tokens: one lane each in the merge
constexpr int TREE_MIN_PIECE = 256;     // tokens
constexpr int TREE_CUS = 256;           // with a workgroup each at a time
constexpr int TREE_PIECE_COST = 16;     // tiles of 32 tokens that a piece costs besides its own

constexpr int TREE_ROWS = 256;          // rows (node, query head) of one KV head that a workgroup has registers for

// Entries of a workgroup's list of cache rows: tokens of a chosen prefix, pages of 16 of a whole one.
constexpr int TREE_LIST = 5120;
enum TreeKind { TREE_FULL, TREE_CHOSEN };
inline int tree_piece_most(TreeKind kind) { return kind == TREE_CHOSEN ? TREE_LIST : TREE_LIST * 16; }
inline bool tree_len_served(TreeKind kind, int64_t len) { return len <= (int64_t)tree_piece_most(kind) * TREE_MAX_SPLITS; }

// Tokens up to which sequences stay whole: what a workgroup of up to 64 rows takes in three steps (its teams take 256 or 128 tokens a step), which is less than the
// merge's launch costs (1 sequence, 4 rows, 300 tokens: whole 9.8 us, in pieces 12.5; 520: 11.7 and 12.8; 1020, four steps: 14.9 and 13.7; 8 sequences, 64 rows,
// 300 tokens: 14.8 and 16.8; 1020: 28.0 and 22.5), and for more rows one piece.  Where half of the CUs have a workgroup anyway, up to 1536 tokens (256 rows, 16 sequences
// of 1064 tokens: whole 38 us, cut 59; 25: 55 and 61).  Of 2000 equal tokens 18 still gain, 81 and 100, but of 100 to 2000 they lose, 72 and 64.
inline int tree_whole(int rows, int64_t wgs) { return std::max(rows <= 32 ? 768 : rows <= 64 ? 384 : TREE_MIN_PIECE, wgs >= TREE_CUS / 2 ? 1536 : 0); }

// Where every CU has a workgroup already, pieces only make up for lengths, and room for them costs what starting workgroups without work does: 40 sequences of
// 2000 tokens, 256 rows, 183 us with room for pieces of 256, 167 without; of 250 to 4000 tokens 206 and 163.  From 4096 on there is room: 40 of 10000 tokens 567,
// without 647, 33 of 8192 under 3 nodes 226 and 263.  (Ragged batches of many would do without, 40 of 600 to 10000 tokens 357 and 336, but then a single long sequence
// among short ones holds up the rest.)
inline int tree_pieces(int rows, int64_t wgs, int max_len) {
    const int least = wgs >= TREE_CUS ? 4096 : TREE_MIN_PIECE;
    return max_len <= tree_whole(rows, wgs) ? 1 : (int)(((int64_t)max_len + least - 1) / least);
}

// Rows of a workgroup.  Half as many of twice as many workgroups where these and all their pieces run at once and sequences are not long: half as many steps
// for the same tokens (a workgroup's two teams share them) and half the partial sums, but the tiles come twice from L2.  (60 nodes, 4 heads each: 1 sequence of 520
// tokens 22.3 us, so 18.6; 8000: 31.0 and 27.1; 16 of 2000: 72 and 55; 256 nodes, 4 of 520: 53 and 36.)  In more than a round the ones without work, of trees and
// sequences that differ, leave the last ones waiting: 8 of 520 under 256 nodes 58 and 70, 8 of 500 to 8000 under 20 to 60 nodes 79 and 88, though 3 of up to 2000
// 28 and 24.  Beyond 8192 tokens a single sequence would gain up to 30000 (10000: 35.4 and 30.4; 30000: 53.8 and 53.2; 131072: 166 and 176), several lose (8 of 30000: 302
// and 319).  Where the last workgroup's rows are few, waves that idle in the large form are the cheaper ones from 2048 tokens on (36 nodes: 1 of 2000 23.5 and 19.5, of
// 30000 46 and 52).
inline int tree_tile_rows(int rows, int64_t pairs, int batch, int max_len) {
    const int tiles = (rows + 127) / 128;
    const int64_t wgs = pairs * tiles, at_once = batch == 1 ? wgs : wgs * tree_pieces(rows, wgs, max_len);   // (one sequence is cut for the CUs that there are)
    return rows > 128 && at_once <= TREE_CUS && max_len <= (rows > 96 * tiles ? 8192 : 2048) ? 128 : TREE_ROWS;
}

struct TreePlan {
    int rows;        // that a workgroup holds at most
    int m_tiles;     // workgroups that share a KV head's tokens
    int n_splits;    // pieces of a sequence's tokens at most; the kernel makes fewer of a short one
};

inline TreePlan plan_tree(TreeKind kind, int max_len, int batch, int G, int g, int max_nodes) {
    const int64_t pairs = (int64_t)batch * G;
    TreePlan p;
    p.rows = tree_tile_rows(max_nodes * g, pairs, batch, max_len);
    p.m_tiles = (max_nodes * g + p.rows - 1) / p.rows;
    // One sequence: a piece for each CU.  Several: room for as many as make up for their lengths' differences (64 of 8192 to 32768 tokens, 8 KV heads:
    // pieces of the longest alone 1437 us, see tree_work).
    const int64_t wgs = pairs * p.m_tiles, want = batch == 1 ? TREE_CUS / wgs : wgs >= 8 * TREE_CUS ? 1 : std::max<int64_t>(4, 2 * TREE_CUS / wgs);
    const int64_t by_list = ((int64_t)max_len + tree_piece_most(kind) - 1) / tree_piece_most(kind);
    p.n_splits = (int)std::max<int64_t>({1, by_list, std::min<int64_t>({want, tree_pieces(max_nodes * g, wgs, max_len), TREE_MAX_SPLITS})});
    return p;
}

// Bytes of partial results: 128 sums, a maximum and a denominator per row and piece.  Trees of fewer nodes may be cut into more
// pieces, but have fewer rows: the bound is over all of them, so that a workspace serves every smaller batch of tokens as well.
struct TreeWs {
    size_t acc, ml, pieces, total;
};
inline TreeWs tree_workspace(TreeKind kind, int max_len, int batch, int H, int G, int max_tokens, int max_nodes) {
    const int g = H / G;
    size_t worst = 0;
    for (int rows = 32;; rows += 32) {               // (all that a plan asks of the rows changes behind multiples of 32)
        const int nodes = std::min(max_nodes, rows / g);
        const TreePlan p = plan_tree(kind, max_len, batch, G, g, nodes);
        const size_t tokens = (size_t)std::min<int64_t>(max_tokens, (int64_t)batch * nodes);
        if (p.n_splits > 1) worst = std::max(worst, tokens * H * p.n_splits);
        if (nodes == max_nodes) break;
    }
    TreeWs w;
    w.acc = 0;
    w.ml = (worst * 128 * 4 + 255) / 256 * 256;
    w.pieces = w.ml + (worst * 2 * 4 + 255) / 256 * 256;
    w.total = w.pieces + ((size_t)batch * 4 + 255) / 256 * 256;
    return w;
}

}  // namespace cusa
