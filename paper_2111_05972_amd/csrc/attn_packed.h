// Attention of packed sequences with grouped heads: the plan of a batch, and how rows are numbered.  Shared by the plan kernel
// (attn_packed_plan.hip) and the bf16 and float kernels.
//
// Flattened rows.  The G = nq / nkv query heads of a key head read the same keys, so to that key head they are one sequence of
// len * G query rows: row r is head r % G of query r / G.  Its keys are 0 .. r / G under the causal mask, that is, key j is seen
// by the rows r >= j G.  A block of 128 rows is then full where there are short sequences and many heads to a key head, crosses a
// short piece of the diagonal, and dK, dV of a key head need no sum over heads besides the one over rows.
//
// Plan (device memory, 32-bit words): positions [M], keys that a token sees [M] (0: it is in no sequence), a header, offsets of the sequences, block counts, and lists of work items.
// A strip is a block of 128 rows (forward, dQ) or 128 keys (dK, dV) of a sequence with the 64-row tiles that it visits on the other
// side.  Strips much longer than a compute unit's share of all tiles are cut into chunks, each an item of its own that leaves float
// sums in a slot of the workspace, and joined in chunk order by another kernel.  Lists are ordered by length, longest first (what
// starts last should be short), those of up to three tiles about as the rows are; items of equal length come in any order, which no result depends on.
#pragma once
#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace tpl {

constexpr int PACK_BLK = 128, PACK_TILE = 64;
constexpr int PACK_MAX_GROUP = 128;
constexpr int PACK_MIN_CHUNK = 8;         // tiles, half of it where strips are few, see pack_shares

struct PackItem {
    int t0, len;           // the sequence: first row of the batch, length
    int first;             // first flattened row (forward, dQ) or key (dK, dV) of the strip
    int tile0, tile1;      // tiles of the other side: [tile0, tile1)
    int slot;              // of this chunk's sums (of chunk 0's in the join lists), -1: the whole strip
    int chunks;            // of the strip
    int pad;
};
struct PackHeader {
    int sequences, tokens, nq, nkv, causal;
    int items[2];          // [0]: forward and dQ, [1]: dK, dV
    int joins[2];          // strips that were cut
    int first_short[2];    // items of one or two tiles stand from here on (longer ones, and chunks of cut strips, may be among them)
    int pad[5];
};
// Word offsets of the plan's parts; a function of what the host knows, so host and device agree without a copy.
struct PackLayout {
    int64_t seen, header, start, pre[2], items[2], joins[2], words;
    int64_t cap[2], join_cap[2];
};
inline int64_t pack_up(int64_t x) { return (x + 63) / 64 * 64; }
// Shares[side]: all tiles of a launch, per key head, are cut into that many of the average length at most (0: nothing is cut).
struct PackShares { int64_t of[2]; };
inline PackLayout pack_layout(int64_t sequences, int64_t M, int64_t nq, int64_t nkv, const PackShares& shares) {
    PackLayout L;
    const int64_t G = nq / nkv;
    int64_t w = pack_up(M);
    L.seen = w; w += pack_up(M);
    L.header = w; w += pack_up(sizeof(PackHeader) / 4);
    L.start = w; w += pack_up(sequences + 1);
    for (int s = 0; s < 2; ++s) {
        L.cap[s] = M * (s == 0 ? G : 1) / PACK_BLK + sequences + shares.of[s];      // a strip of n tiles has less than n / chunk + 1 chunks
        L.join_cap[s] = shares.of[s];                                               // strips longer than a chunk
        L.pre[s] = w; w += pack_up(sequences + 1);
        L.items[s] = w; w += pack_up(L.cap[s] * 8);
        L.joins[s] = w; w += pack_up(L.join_cap[s] * 8);
    }
    L.words = w;
    return L;
}
// A chunk is no shorter than what a compute unit would have of all tiles if they were spread evenly, one workgroup to a unit: twice and four times
// as many shares took 320, 330 and 351 us instead of 314 backward (12 documents of 8192 tokens, 16 / 2 heads of 128), 88, 92 and 110 instead of 87
// forward, in sums written and read.  At least 8 tiles, or 4 where all chunks then still find a unit (5 tiles of both sides to a share): 1000 tokens,
// 8 heads of 128 forward 24.4 -> 16.3 us, backward 47.5 -> 40.4, 4 heads of 64 17.2 -> 13.0, 35.8 -> 24.9; 4 everywhere took 2 to 6 us more
// of 15 and 30 us where strips fill the chip (4096 tokens in 24 sequences).  Nothing is cut, and no kernel joins, below 768 rows: 500 tokens of a head of 64
// take 10.4 and 22.1 us, cut 11.3 and 20.3, 300 of 4 heads 8.1 and 15.5, with a join that finds nothing 9.7 and 17.8.
inline PackShares pack_shares(int64_t M, int64_t nq, int64_t nkv, int units) {
    if (M * (nq / nkv) < 768) return PackShares{{0, 0}};
    const int64_t each = (units + nkv - 1) / nkv;
    return PackShares{{each, each}};
}

#ifdef __HIPCC__
__device__ __forceinline__ const PackItem* pack_items(const int* plan, int64_t at) { return reinterpret_cast<const PackItem*>(plan + at); }
// Whether the plan at hand was made for this call.
__device__ __forceinline__ bool pack_matches(const PackHeader* h, int sequences, int tokens, int nq, int nkv, int causal) {
    return h->sequences == sequences && h->tokens == tokens && h->nq == nq && h->nkv == nkv && h->causal == causal;
}
#endif

// What an attention call of packed sequences works on.
struct PackAttnArgs {
    int dtype;
    int64_t sequences, M;
    int nq, nkv, dh, causal;
    const int* plan;
    const void* qkv; void* o; float* lse;                         // lse [M, nq]
    const void* d_o; void* dqkv; float* dsum;                     // dsum [M, nq]
    void* ws; size_t ws_bytes;
    hipStream_t stream;
};
hipError_t pack_plan(int64_t sequences, int64_t M, const int* offsets, int nq, int nkv, int causal, int* plan, hipStream_t s);
size_t attn_packed_workspace_bytes(const PackAttnArgs& a, bool bwd);
hipError_t attn_packed_bf16(const PackAttnArgs& a, bool bwd);
hipError_t attn_packed_f32(const PackAttnArgs& a, bool bwd);

}  // namespace tpl
