// Rows that several workgroups share: the words they hand to one another (see SplitRow in ppv_internal.h), shared by the kernels of
// libppv_hip.so that split rows.
#pragma once
#include "ppv_device.h"
#include "ppv_internal.h"

namespace {

// Words that the workgroups of a split row hand to one another (see SplitRow) are written and read with device-scope
// accesses (each goes to the level of the memory system that all compute units share), so that no fence over the whole
// cache is needed: a device-wide fence per wavefront cost 30 us per launch.
template <typename W> __device__ __forceinline__ void shared_put(W *p, W v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename W> __device__ __forceinline__ W shared_get(const W *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// A row shared by `parts` workgroups (see SplitRow); parts == 1: one workgroup has the row to itself and
// nothing else here is looked at.
struct Split {
    int parts;
    int part;             // this workgroup's number, 0 .. parts-1
    SplitRow *row;        // the row's scratch
    uint32_t *arrivals;   // the row's arrival counter
    uint32_t mark;        // of the call
};
template <bool SPLIT> __device__ __forceinline__ Split split_of(int shift) {
    if (!SPLIT) return {1, 0, nullptr, nullptr, 0u};
    return {1 << shift, (int)(blockIdx.x & ((1u << shift) - 1u)), nullptr, nullptr, 0u};
}
// (Where it is needed, not when the kernel starts: on the way through the index there is no room for it in the scalar registers.)
template <bool SPLIT> __device__ __forceinline__ void find_area(Split &sp, SplitScratch *scratch, int b, uint32_t mark) {
    if (!SPLIT) return;
    sp.row = &scratch->row[b];
    sp.arrivals = &scratch->arrivals[b];
    sp.mark = mark;
}
__device__ __forceinline__ void send(Marked *p, float v, uint32_t mark) { shared_put(p, (uint64_t)mark << 32 | __float_as_uint(v)); }
__device__ __forceinline__ void send(MarkedPair *p, float a, float b, uint32_t mark) {
    send(&p->first, a, mark);
    send(&p->second, b, mark);
}
__device__ __forceinline__ void clear(MarkedPair *p) {
    shared_put(&p->first, (Marked)0);
    shared_put(&p->second, (Marked)0);
}
__device__ __forceinline__ MarkedPair look(const MarkedPair *p) { return {shared_get(&p->first), shared_get(&p->second)}; }
__device__ __forceinline__ bool has(Marked w, uint32_t mark) { return (uint32_t)(w >> 32) == mark; }
__device__ __forceinline__ bool has(const MarkedPair &w, uint32_t mark) { return has(w.first, mark) && has(w.second, mark); }
__device__ __forceinline__ float value(Marked w) { return __uint_as_float((uint32_t)w); }
// Waits for words that have been sent, by a whole wavefront: look_again() at all of them as long as one lane's there() is false.  False if they
// do not come: two launches use one area at a time, which no caller may do.  (The row then has no result, and says so: id -1, masses NaN.)
constexpr uint32_t MOST_LOOKS = 1u << 16;      // a word that has been sent comes within microseconds
template <typename THERE, typename LOOK> __device__ __forceinline__ bool wait_for(const Split &sp, THERE there, LOOK look_again) {
    uint32_t n = 0;
    while (__ballot(!there()) != 0ull) {   // (uniform: what is live here is in scalar registers, of which there are too few)
        if (n++ >= MOST_LOOKS || (sp.mark & PPV_LOOK_ONCE)) return false;
        look_again();
    }
    return true;
}
// Counts this workgroup: true for the one that arrives last.  (The count goes from parts - 1 to 0, and from anything that is more: what launches
// that may not have met here leave in it makes some workgroup of a later one the last, which waits for the words of the others.)
__device__ __forceinline__ bool arrive(const Split &sp) { return atomicInc(sp.arrivals, (uint32_t)sp.parts - 1u) >= (uint32_t)sp.parts - 1u; }

}  // namespace
