// pk_attention_plan.hpp -- how the work of one attention call is divided.  Plain
// integer arithmetic, which the kernels and the CPU tests evaluate alike.
//
// The rows of one sequence that read one head of the cache (its tokens times the
// query heads that share it) are cut into groups; a group of rows with its head is
// an item.  An item's positions are cut into units.  All items' units form one
// line: sequence by sequence, head by head, group by group.  A work-group takes an
// equal share of the line, whatever the sequences' lengths, and what lies on both
// sides of a share's border is joined afterwards.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define PK_PLAN __host__ __device__ inline
#else
#define PK_PLAN inline
#endif

namespace pk::attention {

constexpr int kMostTokens = 64;  // of a sequence: a mask's bits

struct Shape {
    int64_t M;         // tokens of the call
    int64_t capacity;  // positions that a row of the page table names
    int heads, group;  // of the cache; query heads of each
    int most;          // tokens of a sequence
    int rows;          // of an item
    int unit;          // positions of a unit; 0: an item is one unit
};

struct Sequence {
    int64_t first;   // its first token
    int64_t length;  // positions before its tokens, at most capacity
    int64_t keys;    // positions in all, at most capacity
    int tokens;
    int groups;      // of rows, for each head
    int64_t units;   // of an item
    PK_PLAN int64_t cost(int heads) const { return (int64_t)heads * groups * units; }
};

// What a sequence's indices say, held to what the tensors have.
PK_PLAN Sequence sequence(const Shape &s, int64_t start, int64_t end, int64_t length)
{
    Sequence q;
    q.first = start;
    int64_t t = end - start;
    if (t > s.most) t = s.most;
    if (start < 0 || start > s.M) t = 0;
    if (t > s.M - start) t = s.M - start;
    if (t < 0) t = 0;
    q.tokens = (int)t;
    q.length = length < 0 ? 0 : length > s.capacity ? s.capacity : length;
    q.keys = q.length + t < s.capacity ? q.length + t : s.capacity;
    q.groups = (int)((t * s.group + s.rows - 1) / s.rows);
    // an item without positions still writes its rows
    q.units = !s.unit ? 1 : q.keys ? (q.keys + s.unit - 1) / s.unit : 1;
    return q;
}

// Units of a work-group's share.
PK_PLAN int64_t share(int64_t total, int64_t groups) { return total > groups ? (total + groups - 1) / groups : 1; }

// A part of an item lies in its work-group's first slot if it begins the share, in
// the second if it does not: at most one part of each kind is not a whole item.
PK_PLAN int slot_of(int64_t part_begin, int64_t share_begin) { return part_begin == share_begin ? 0 : 1; }

}  // namespace pk::attention
