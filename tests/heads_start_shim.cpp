// Which rows a work-group's teams begin with (pk_heads_launch.hpp), for the CPU tests.
#include "../paper_1904_05347_amd/csrc/pk_heads_launch.hpp"

#include <stdint.h>

extern "C" {

// out: threads, teams, tokens, a team's lanes, those that hold pairs
void shim_layout(int d, int pairs, int E, int64_t rows, int *out)
{
    const pk::HeadTiling t = pk::head_tiling(d, pairs, E);
    const pk::HeadGroup g = pk::head_group(rows, t.team, pairs);
    out[0] = g.threads;
    out[1] = g.teams;
    out[2] = g.tokens;
    out[3] = t.team;
    out[4] = t.pair_chunks;
}

void shim_start(int slot, int tokens, int rows, int *out)
{
    const pk::HeadStart s = pk::head_start(slot, tokens, rows);
    out[0] = s.token;
    out[1] = s.row;
}
}
