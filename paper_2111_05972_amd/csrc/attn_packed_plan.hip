// The plan of a packed batch (attn_packed.h), made on the device from the offsets of its sequences: one launch, no host copy, so
// that it can be enqueued ahead of a step or captured with it.  Workgroup 0 makes the lists, the others the positions.  Bound by the dependent
// passes of that workgroup: 9 us for 2 sequences, 17 for 24 of 4096 tokens, 31 for 64 of 65536, 81 for 3000, once for all layers of a step.
//
// Offsets are taken as their running maximum, clamped to [0, M]: whatever the caller's memory holds, sequences neither overlap
// nor leave the rows, and the lists stay within their capacity.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attn_packed_dev.h"
#include "kernels.h"

namespace tpl {
namespace {

constexpr int PLAN_THREADS = 1024;
constexpr int BUCKETS = 1024;
constexpr int NEAR = 2048;

// Inclusive scan over the workgroup, sum or maximum, by wavefronts and then over their totals; total: of all.
template <bool MAX> __device__ __forceinline__ int join(int a, int b) { return MAX ? max(a, b) : a + b; }
template <bool MAX> __device__ int block_scan(int v, int* tmp, int& total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int o = __shfl_up(v, d, 64);
        if (lane >= d) v = join<MAX>(v, o);
    }
    __syncthreads();                                               // the scan before has been read
    if (lane == 63) tmp[wave] = v;
    __syncthreads();
    int before = MAX ? -1 : 0;
    total = before;
#pragma unroll
    for (int w = 0; w < PLAN_THREADS / 64; ++w) {
        const int o = tmp[w];
        if (w < wave) before = join<MAX>(before, o);
        total = join<MAX>(total, o);
    }
    return join<MAX>(v, before);
}

struct PlanParams {
    int n, M, nq, nkv, mask, window, sinks;
    PackShares shares;
    PackCut cut;
    const int* offsets;
    int* plan;
    PackLayout L;
};

// Strip `i` of a sequence: its first row or key and its tiles.
template <bool WIN> __device__ __forceinline__ int mask_of(const PlanParams& p) { return WIN ? PACK_WINDOW : p.mask == PACK_CAUSAL ? PACK_CAUSAL : PACK_ALL; }
template <bool WIN> __device__ __forceinline__ PackTiles strip_of(const PlanParams& p, int side, int len, int i) {
    return pack_tiles(mask_of<WIN>(p), p.window, p.sinks, (unsigned)(p.nq / p.nkv), side, len, i * PACK_BLK);
}
// Longest first, `top` above the longest.  Strips of up to LEVEL tiles, which memory bounds and not their length, stay in the order of the
// rows: sorted, the units would all read the same part of every sequence at a time, and where lengths are equal and even those parts lie on the same channels
// (forward, 8192 tokens, 16 / 2 heads of 128: 64 sequences of 128 42.5 -> 28.7 us, 32 of 256 37.6 -> 35.0, other lengths within 2 %; LEVEL = 4
// takes 3 % more in backward).
constexpr int LEVEL = 3;
__device__ __forceinline__ int bucket_of(int tiles, int top) {
    return BUCKETS - 1 - min(BUCKETS - 1, (int)((float)max(tiles, LEVEL) * ((float)(BUCKETS - 1) / (float)top)));
}

// WIN: with a window, whose questions took the others 0.4 to 0.6 us.
template <bool WIN> __global__ __launch_bounds__(PLAN_THREADS) void pack_plan_kernel(PlanParams p) {
    __shared__ int tmp[PLAN_THREADS / 64];
    __shared__ int hist[2][BUCKETS];
    __shared__ int longest[2], slots[2], joins[2], first_short[2];
    __shared__ unsigned long long tiles[2];
    __shared__ int near[3][NEAR];                                  // what the searches read, where it fits
    const int t = threadIdx.x, G = p.nq / p.nkv;
    const bool fits = p.n < NEAR;
    int* start = fits ? near[2] : p.plan + p.L.start;
    int* const before[2] = {fits ? near[0] : p.plan + p.L.pre[0], fits ? near[1] : p.plan + p.L.pre[1]};   // strips before each sequence
    auto offset = [&](int i) { return min(max(p.offsets[i], 0), p.M); };
    if (blockIdx.x > 0) {
        // This workgroup's tokens, each looking for its sequence among the running maxima of the offsets, 1024 sequences at a time.
        const int64_t step = (int64_t)(gridDim.x - 1) * PLAN_THREADS, m0 = (int64_t)(blockIdx.x - 1) * PLAN_THREADS + t;
        for (int64_t m = m0; m < p.M; m += step) p.plan[m] = p.plan[p.L.seen + m] = 0;
        int* begin = near[0];                                      // of these sequences, and the end of the last
        int carry = 0;
        for (int base = 0; base < p.n; base += PLAN_THREADS) {
            const int i = base + t, count = min(p.n - base, PLAN_THREADS);
            int all;
            begin[t] = max(block_scan<true>(i <= p.n ? offset(i) : 0, tmp, all), carry);
            carry = max(carry, all);
            if (t == 0) begin[PLAN_THREADS] = max(carry, base + PLAN_THREADS <= p.n ? offset(base + PLAN_THREADS) : 0);
            __syncthreads();
            for (int64_t m = m0; m < p.M; m += step) {
                if (m < begin[0] || m >= begin[count]) continue;
                int lo = 0, hi = count - 1;                        // the last with begin <= m
                while (lo < hi) {
                    const int mid = (lo + hi + 1) >> 1;
                    if (begin[mid] <= m) lo = mid; else hi = mid - 1;
                }
                p.plan[m] = (int)m - begin[lo];
                const int at = (int)m - begin[lo];
                int seen = WIN || p.mask != PACK_ALL ? at + 1 : begin[lo + 1] - begin[lo];
                if (WIN) seen = min(seen, p.window) + min(p.sinks, max(0, seen - p.window));
                p.plan[p.L.seen + m] = seen;
            }
            __syncthreads();
        }
        return;
    }
    if (t < 2) { first_short[t] = 0; longest[t] = 0; slots[t] = 0; joins[t] = 0; tiles[t] = 0; }
    hist[0][t] = hist[1][t] = 0;
    __syncthreads();
    // offsets as running maxima, and the strips before each sequence
    int carry_max = 0, carry[2] = {0, 0};
    for (int base = 0; base <= p.n; base += PLAN_THREADS) {
        const int i = base + t;
        int all;
        const int c = max(block_scan<true>(i <= p.n ? offset(i) : 0, tmp, all), carry_max);
        if (i <= p.n) start[i] = c;
        carry_max = max(carry_max, all);
    }
    __threadfence_block();
    __syncthreads();
    for (int base = 0; base <= p.n; base += PLAN_THREADS) {
        const int i = base + t;
        const int len = i < p.n ? start[i + 1] - start[i] : 0;
        for (int side = 0; side < 2; ++side) {
            const int blocks = ((side == 0 ? len * G : len) + PACK_BLK - 1) / PACK_BLK;
            int all;
            const int pre = block_scan<false>(blocks, tmp, all) + carry[side];
            if (i <= p.n) before[side][i] = pre - blocks;
            carry[side] += all;
        }
    }
    __threadfence_block();
    __syncthreads();
    auto find = [&](const int* pre, int item) {                    // the sequence that strip `item` belongs to
        int lo = 0, hi = p.n - 1;                                  // the last i with pre[i] <= item: sequences without strips lie before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (pre[mid] <= item) lo = mid; else hi = mid - 1;
        }
        return lo;
    };
    for (int side = 0; side < 2; ++side) {
        const int* pre = before[side];
        unsigned long long mine = 0;
        int most = 0;
        for (int k = t; k < carry[side]; k += PLAN_THREADS) {
            const int b = find(pre, k);
            const PackTiles s = strip_of<WIN>(p, side, start[b + 1] - start[b], k - pre[b]);
            mine += (unsigned)(s.tile1 - s.tile0);
            most = max(most, s.tile1 - s.tile0);
        }
        if (mine) {
            atomicAdd(&tiles[side], mine);
            atomicMax(&longest[side], most);
        }
    }
    __syncthreads();
    for (int side = 0; side < 2; ++side) {
        const int* pre = before[side];
        int chunk = 1 << 30;
        const bool few = (int64_t)(tiles[0] + tiles[1]) <= 5 * p.shares.of[side];          // a compute unit and a quarter to a chunk at most
        if (p.cut.of[side]) chunk = max(few ? PACK_MIN_CHUNK / 2 : PACK_MIN_CHUNK, (int)((tiles[side] + p.shares.of[side] - 1) / p.shares.of[side]));
        const int top = min(longest[side], chunk) + 1;
        PackItem* items = reinterpret_cast<PackItem*>(p.plan + p.L.items[side]);
        PackItem* join = reinterpret_cast<PackItem*>(p.plan + p.L.joins[side]);
        for (int pass = 0; pass < 2; ++pass) {                     // count, then place
            for (int k = t; k < carry[side]; k += PLAN_THREADS) {
                const int b = find(pre, k);
                PackItem it{};
                it.t0 = start[b];
                it.len = start[b + 1] - start[b];
                it.first = (k - pre[b]) * PACK_BLK;
                const PackTiles s = strip_of<WIN>(p, side, it.len, k - pre[b]);
                const int a = s.tile0, z = s.tile1;
                it.skip = s.skip;
                it.chunks = (z - a + chunk - 1) / chunk;
                const int each = (z - a + it.chunks - 1) / it.chunks;
                const int bucket = bucket_of(each, top);
                if (pass == 0) {
                    atomicAdd(&hist[side][bucket], it.chunks);
                    continue;
                }
                const int at = atomicAdd(&hist[side][bucket], it.chunks);
                int slot = -1;
                if (it.chunks > 1) {
                    slot = atomicAdd(&slots[side], it.chunks);
                    const int j = atomicAdd(&joins[side], 1);
                    it.slot = slot;
                    it.tile0 = a;
                    it.tile1 = z;
                    if (j < p.L.join_cap[side]) join[j] = it;
                }
                for (int c = 0; c < it.chunks; ++c) {
                    it.slot = slot < 0 ? -1 : slot + c;
                    it.tile0 = a + c * each;
                    it.tile1 = min(z, a + (c + 1) * each);
                    if (at + c < p.L.cap[side]) items[at + c] = it;
                }
            }
            __syncthreads();
            if (pass == 0) {                                       // counts -> first places
                int all;
                const int v = hist[side][t], at = block_scan<false>(v, tmp, all) - v;
                hist[side][t] = at;
                if (t == bucket_of(2, top)) first_short[side] = at;
                __syncthreads();
            }
        }
        if (t == 0) {
            PackHeader* h = reinterpret_cast<PackHeader*>(p.plan + p.L.header);
            h->items[side] = min(hist[side][BUCKETS - 1], (int)p.L.cap[side]);   // the end of the last bucket
            h->joins[side] = min(joins[side], (int)p.L.join_cap[side]);
            h->first_short[side] = min(first_short[side], h->items[side]);
            if (side == 0) { h->sequences = p.n; h->tokens = p.M; h->nq = p.nq; h->nkv = p.nkv; h->mask = p.mask; h->window = p.window; h->sinks = p.sinks; }
        }
    }
}

}  // namespace

size_t attn_packed_workspace_bytes(const PackAttnArgs& a, bool bwd) { return ws_of(a, bwd).total; }

hipError_t pack_plan(int64_t sequences, int64_t M, const int* offsets, int nq, int nkv, int mask, int window, int sinks, int* plan, hipStream_t s) {
    PlanParams p{};
    p.n = (int)sequences; p.M = (int)M; p.nq = nq; p.nkv = nkv; p.mask = mask; p.window = window; p.sinks = sinks;
    p.shares = pack_shares(M, nq, nkv, compute_units());
    p.cut = pack_cut(mask, window, sinks, M, nq, nkv, compute_units());
    p.offsets = offsets; p.plan = plan;
    p.L = pack_layout(sequences, M, nq, nkv, p.shares);
    static_assert(BUCKETS == PLAN_THREADS && NEAR > PLAN_THREADS, "a thread to a bucket, 1024 sequences and an end in LDS");
    const int64_t groups = std::min<int64_t>((M + PLAN_THREADS - 1) / PLAN_THREADS, 1024);
    hipLaunchKernelGGL(mask == PACK_WINDOW ? pack_plan_kernel<true> : pack_plan_kernel<false>, dim3((unsigned)(1 + groups)), dim3(PLAN_THREADS), 0, s, p);
    return hipGetLastError();
}

}  // namespace tpl
