// Rows dealt to experts: which rows a workgroup takes (device code).
#pragma once
#include "internal.hpp"

namespace alpa {

// Group g of `experts` + 2: expert g's rows, then the rows behind the last expert's, then those before the first one's.
// Offsets are taken as they come, cut to 0 .. rows, so that no value of theirs leads out of the tensors.
__device__ __forceinline__ void group_rows(const int32_t *offsets, int experts, int rows, int g, int &first, int &end)
{
    first = end = 0;
    if (g > experts + 1) return;
    const int a = min(max(offsets[g > experts ? 0 : g], 0), rows);
    if (g < experts) {
        first = a;
        end = max(a, min(max(offsets[g + 1], 0), rows));
    } else if (g == experts) {
        first = a;
        end = rows;
    } else {
        end = a;
    }
}

struct Slot {
    int expert;          // -1: no such slot; >= experts: rows of no expert
    int first, end;      // its rows
};

// The slot-th run of up to `tile` rows of one group, in the order of the groups.  One wave looks at 64 groups at a time; the whole
// wave has to be here.
__device__ __forceinline__ Slot find_slot(const int32_t *offsets, int experts, int rows, int tile, int slot)
{
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));         // (what follows from it is not kept in registers between two calls)
    int before = 0;
    for (int base = 0; base < experts + 2; base += 64) {
        int first, end;
        group_rows(offsets, experts, rows, base + lane, first, end);
        const int n = (end - first + tile - 1) / tile;
        int sum = n;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const int o = __shfl_up(sum, off, 64);
            if (lane >= off) sum += o;
        }
        const unsigned long long past = __ballot(before + sum > slot);
        if (past) {
            const int l = __ffsll(past) - 1;
            const int f = __builtin_amdgcn_readlane(first, l), e = __builtin_amdgcn_readlane(end, l);
            const int s = before + __builtin_amdgcn_readlane(sum, l) - __builtin_amdgcn_readlane(n, l);
            const int at = f + (slot - s) * tile;
            return Slot{base + l, at, min(at + tile, e)};
        }
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return Slot{-1, 0, 0};
}

// slots of the groups in front of `group`
__device__ __forceinline__ int slots_before(const int32_t *offsets, int experts, int rows, int tile, int group)
{
    const int lane = threadIdx.x & 63;
    int sum = 0;
    for (int base = 0; base < group; base += 64) {
        int first, end;
        group_rows(offsets, experts, rows, base + lane, first, end);
        int n = base + lane < group ? (end - first + tile - 1) / tile : 0;
#pragma unroll
        for (int off = 32; off; off >>= 1) n += __shfl_xor(n, off, 64);
        sum += __builtin_amdgcn_readfirstlane(n);
    }
    return sum;
}

}  // namespace alpa
