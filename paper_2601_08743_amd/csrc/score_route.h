// Which kernel scores a call's tokens where one launch for scores and list does not do (block_attn.hip): plain C++, so that it also builds
// without the HIP headers.
#pragma once
#include <algorithm>
#include <cstdint>

namespace tc {

constexpr int kScoreBlocks = 256;                        // candidates of a work-group

// Tokens that share a work-group in the grouped kernel: four tiles of 16 query rows.
inline int score_group_tokens(int G) { return G <= 16 ? 4 * (16 / G) : 1; }

inline int64_t score_parts(int64_t max_blocks) { return (max_blocks + kScoreBlocks - 1) / kScoreBlocks; }

// Whether tokens share work-groups.  One token to a work-group costs some 4 ns for each (token, KV head, range), of which there are
// `by_token`.  A group reads the digests once for all of its tokens of one request, but takes its requests one after the other, each
// a chain of round trips, 4 to 5 us: `passes` of them, if a table row brings as many tokens as another.  Padded rows count as tokens, so a
// batch of one token each has some more than one to a row: below three nothing is shared that pays (700 rows of two, 32 / 8 heads, 1700
// entries: 275 us for 319, the best of many; 8 / 8 heads 396 for 313).  Both kernels, us a call with its lists, 32 / 8, 28 / 4 and 8 / 8 heads:
//   rows x tokens, table entries    64 x 1 + 3, 1700   64 x 2, 1700    16 x 4, 1700    64 x 4, 700     16 x 8, 1700    4 x 16, 1700
//   a token each                    24.1 16.8  24.0    37.2 24.3  37.6 23.6 16.4 23.7  35.9 21.8 35.5  35.9 23.2 37.5  23.5 16.2 23.8
//   grouped                         71.9 40.2 330.3    47.2 29.4 173.2 27.3 18.5 92.6  30.5 19.4 95.4  22.6 16.8 55.0  15.3 14.7 33.1
inline bool scores_by_group(int64_t n_tokens, int64_t rows, int G, int Hkv, int64_t max_blocks)
{
    const int64_t group = score_group_tokens(G);
    if (group == 1 || n_tokens < 3 * rows) return false;
    const int64_t passes = std::min(group, std::max<int64_t>(1, (group * rows + n_tokens - 1) / std::max<int64_t>(n_tokens, 1)));
    const int64_t by_token = n_tokens * Hkv * score_parts(max_blocks);
    return by_token > 1200 * passes;
}

}  // namespace tc
