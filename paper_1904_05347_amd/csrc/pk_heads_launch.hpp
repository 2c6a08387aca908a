// pk_heads_launch.hpp -- how heads are laid over lanes and work-groups.  Plain
// integer arithmetic, which the CPU tests evaluate too.
#pragma once

#include <stdint.h>

namespace pk {

// A lane holds two vectors of E elements (16 bytes each) of a head: of a pair's
// two channels where pairs are halves apart, of neighbours elsewhere.
struct HeadTiling {
    int pair_chunks;  // lanes that hold rotated channels, E pairs each
    int chunks;       // lanes that hold a head
    int team;         // the next power of two: a head's lanes
};

constexpr HeadTiling head_tiling(int d, int pairs, int E)
{
    HeadTiling t = {(pairs + E - 1) / E, 0, 1};
    t.chunks = t.pair_chunks + (d - 2 * pairs + 2 * E - 1) / (2 * E);
    while (t.team < t.chunks) t.team *= 2;
    return t;
}

constexpr int kMostHeadThreads = 512;

struct HeadGroup {
    int threads;  // of a work-group, a multiple of 64
    int teams;    // heads that it has in work at once
    int tokens;   // tokens of a work-group: several where a token's heads are few
};

// `rows` heads a token.  A work-group has the teams that its heads need, in equal
// rounds; several tokens where they are few.
constexpr HeadGroup head_group(int64_t rows, int team, int pairs)
{
    const int most = kMostHeadThreads / team;
    HeadGroup g = {64, 1, 1};
    if (rows * 2 <= 256 / team) {
        g.tokens = (int)(256 / team / rows);
        // the tokens' angles stay within 16 KB of LDS
        while (g.tokens > 1 && (int64_t)g.tokens * pairs > 2048) g.tokens -= 1;
        const int64_t need = g.tokens * rows * team;
        g.threads = (int)((need + 63) / 64 * 64);
    } else {
        const int64_t rounds = (rows + most - 1) / most;
        const int64_t need = (rows + rounds - 1) / rounds * team;
        g.threads = (int)((need + 63) / 64 * 64);
    }
    g.teams = g.threads / team;
    return g;
}

// Which of its work-group's tokens and of their rows a team begins with.  A team without
// any has the row `rows`, which is none, of a token whose angles are in LDS like the others'.
struct HeadStart {
    int token, row;
};

constexpr HeadStart head_start(int slot, int tokens, int rows)
{
    if (tokens == 1) return {0, slot};
    const int token = slot / rows;
    if (token >= tokens) return {0, rows};
    return {token, slot - token * rows};
}

}  // namespace pk
