// Definitions shared by the tensor-core attention kernels.
#pragma once
#include "sm100_ptx.cuh"

namespace attn_tc {

using namespace sm100;

constexpr int kStatusTimeout = 9;  // ATTN_ERR_DEVICE_TIMEOUT

// Last key (index inside this K/V shard) that query row `row` may see, or a negative number when it
// sees none: all Sk keys without a mask; with the causal mask key j of a shard that starts at global
// key index k_offset is visible iff k_offset + j <= row.
__device__ __forceinline__ int last_visible_key(int row, int Sk, int causal, int k_offset) {
    const int all = Sk - 1;
    if (!causal) return all;
    const int c = row - k_offset;
    return c < all ? c : all;
}

// Bits 0 .. n-1 (n below 0: none, above 32: all).
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u); }

// Sliding window: which of the 32 keys from key0 the query at position p sees (bit e: key0 + e).  One word of bits per 32
// elements, so that masking an element is a bit test and a select.
__device__ __forceinline__ uint32_t window_keys(int key0, int p, int Sk, int window, int sinks) {
    const int last = p < Sk - 1 ? p : Sk - 1;
    int low = p - window + 1;
    low = low > 0 ? low : 0;
    return low_bits(last - key0 + 1) & (~low_bits(low - key0) | low_bits(sinks - key0));
}

// The other way round: which of the 32 queries at positions p0, p0 + 1, .. see key `key`.
__device__ __forceinline__ uint32_t window_queries(int p0, int key, int Sk, int window, int sinks) {
    if (key >= Sk) return 0u;
    const int64_t past = static_cast<int64_t>(key) + window - p0;      // first position whose window has left the key
    const uint32_t until = (key < sinks || past >= 32) ? 0xffffffffu : low_bits(past < 0 ? 0 : static_cast<int>(past));
    return ~low_bits(key - p0) & until;
}

// End of a CTA in which a wait ran out, executed by one thread once no role asks for anything more.  Copies and products that the
// CTA did ask for may still be on their way into its shared and tensor memory, which therefore has to stay its own for a while:
// those that arrive at all take microseconds.
constexpr uint64_t kSettleNs = 200000;
__device__ __forceinline__ void report_timeout(int* status) {
    const uint64_t t0 = sm100::globaltimer_ns();
    while (sm100::globaltimer_ns() - t0 < kSettleNs) __nanosleep(1000);
    atomicExch(status, kStatusTimeout);
}

// End of a persistent kernel, executed by one thread per CTA after the CTA's last draw from the work
// counter: reports a timed-out wait, and hands the counter back zeroed.  counter[0] is the next work
// item, counter[1] the number of CTAs that have finished; the CTA that finishes last resets both, so
// the next launch that uses this counter (launches that share one are ordered on one stream) starts
// from zero without a memset.  Every CTA reaches this point, also after a timed-out wait.
__device__ __forceinline__ void finish_cta(int* status, bool timed_out, unsigned int* counter) {
    if (timed_out) report_timeout(status);
    if (counter) {
        __threadfence();
        if (atomicAdd(counter + 1, 1u) == gridDim.x - 1) {
            counter[0] = 0u;
            counter[1] = 0u;
            __threadfence();
        }
    }
}

}  // namespace attn_tc
