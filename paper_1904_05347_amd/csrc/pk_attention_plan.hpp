// pk_attention_plan.hpp -- how the work of one attention call is divided.  Plain
// integer arithmetic, which the kernels and the CPU tests evaluate alike.
//
// The rows of one sequence that read one head of the cache (its tokens times the
// query heads that share it) are cut into groups; a group of rows with its head is
// an item.  An item's positions are cut into units.  All items' units form one
// line: sequence by sequence, head by head, group by group.  A work-group takes an
// equal share of the line, whatever the sequences' lengths, and what lies on both
// sides of a share's border is joined afterwards.
//
// 32-bit integers throughout (a 64-bit division takes a GPU hundreds of
// instructions): a line has fewer than 2^31 units, by the host's bound on it.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define PK_PLAN __host__ __device__ inline
#else
#define PK_PLAN inline
#endif

namespace pk::attention {

constexpr int kMostTokens = 64;  // of a sequence: a mask's bits
constexpr int64_t kMostLine = ((int64_t)1 << 31) - 1;

struct Shape {
    int M;           // tokens of the call, at most 2^30
    int capacity;    // positions that a row of the page table names, at most 2^30
    int heads;       // of the cache
    int group;       // query heads of each
    int most;        // tokens of a sequence
    int rows_shift;  // rows of an item: a power of two
    int unit_shift;  // positions of a unit: a power of two; -1: an item is one unit
    int tail;        // positions that an item's last unit takes beyond a unit's
};

struct Sequence {
    int first;   // its first token
    int tokens;
    int length;  // positions before its tokens, at most capacity
    int keys;    // positions in all, at most capacity
    int groups;  // of rows, for each head
    int units;   // of an item
    PK_PLAN unsigned cost(int heads) const { return (unsigned)heads * (unsigned)groups * (unsigned)units; }
};

// What a sequence's indices say, held to what the tensors have.
PK_PLAN Sequence sequence(const Shape &s, int start, int end, int length)
{
    Sequence q;
    int64_t t = (int64_t)end - start;
    if (t > s.most) t = s.most;
    if (start < 0 || start > s.M) t = 0;
    if (t > s.M - start) t = s.M - start;
    if (t < 0) t = 0;
    q.first = start;
    q.tokens = (int)t;
    q.length = length < 0 ? 0 : length > s.capacity ? s.capacity : length;
    q.keys = q.length + (int)t < s.capacity ? q.length + (int)t : s.capacity;
    q.groups = ((int)t * s.group + (1 << s.rows_shift) - 1) >> s.rows_shift;
    // An item without positions still writes its rows.
    q.units = s.unit_shift < 0 ? 1 : (q.keys - s.tail + (1 << s.unit_shift) - 1) >> s.unit_shift;
    if (q.units < 1) q.units = 1;
    return q;
}

// Units of a work-group's share.
PK_PLAN unsigned share(unsigned total, unsigned groups) { return total > groups ? (total + groups - 1) / groups : 1; }

// A part of an item lies in its work-group's first slot if it begins the share, in
// the second if it does not: at most one part of each kind is not a whole item.
PK_PLAN int slot_of(unsigned part_begin, unsigned share_begin) { return part_begin == share_begin ? 0 : 1; }

}  // namespace pk::attention
