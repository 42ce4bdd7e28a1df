// Attention of a few queries of each of B sequences over key/value rows that live in pages (decode time).
//
//   s_j = scale <q, k_j>,  lse = log sum_j exp s_j,  o = sum_j exp(s_j - lse) v_j   over the rows j that the query sees.
//
// Bound: HBM.  A visible row is fetched once for all queries of its kv head (they share the matrix instructions' columns),
// 4 * d * (queries of the head) operations per 4 * d bytes, far below the matrix pipe's rate.
//
// Split.  The visible rows of an entry are counted in blocks of 32.  The blocks of all entries, one behind the other, are cut into
// as many equal runs as there are workers, so sequences of any mix of lengths fill the chip alike and the host needs no lengths.  A
// worker is one workgroup for each kv head (and row block); its four waves take every fourth block of an entry and are joined
// through LDS.  An entry that one worker has to itself is finished there; of the others each worker leaves the unnormalised sum,
// the maximum and the weight of its part in the workspace, and a second launch joins them in the order of the rows.  Where workers suffice
// for it, each entry is cut for itself instead, so that no worker has two, and few short entries go to a workgroup each, in one launch.
//
// Measured (MI355X; rows of 8 kv heads, 32 query heads unless said; a graph's replays): 48 sequences of up to 4096 rows 95 us
// (462 MB, 4.9 TB/s), 4 of up to 32768 with 40 heads 357 (1974 MB, 5.5; a kernel that only reads reaches 6.0), 12 of up to 4096
// with 10 queries each under a tree 47.4, one of 777 rows of 32 kv heads 10.3.  The counters have every visible row fetched once from HBM, and
// vector and matrix instructions issue in a tenth of the waves' time (under the tree a fifth): they wait for rows, or for room to ask for more.
//
// Layout.  A wave keeps everything in registers and shares nothing until its end: S^T = K Q^T puts a query in a
// column (lane % 16) and four keys in a lane, which is at once the layout that O^T = V^T P^T wants of P^T.  V rows are
// read in 16-byte pieces of eight (float: four) channels; the channel that a lane's row of V^T stands for is free to
// choose, so the transposition is a matter of picking halves of registers.
#include "paged_attend.h"

namespace beagle {

// The parts, and for each entry who has them.
size_t paged_attn_ws_bytes(int32_t B, int32_t M, int32_t H, int32_t G) {
  return (size_t)part_rows(M * (H / G), G) * (128 + 2) * sizeof(float) + (size_t)B * sizeof(int2);
}

void launch_paged_attn(bool bf16, PagedAttnArgs a, void* ws, hipStream_t s) { launch_attend<PLAIN>(bf16, a, ws, s); }

}  // namespace beagle
