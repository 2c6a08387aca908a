// The plain integer arithmetic of the attention operators for the CPU tests: where
// tensors lie (pk_heads_checks.hpp), how heads are laid over lanes
// (pk_heads_launch.hpp), how an attention's work is divided (pk_attention_plan.hpp).
#include "../paper_1904_05347_amd/csrc/pk_attention_plan.hpp"
#include "../paper_1904_05347_amd/csrc/pk_heads_checks.hpp"
#include "../paper_1904_05347_amd/csrc/pk_heads_launch.hpp"

extern "C" {

// a, b: at, run, then three pairs of count and stride
static pk::heads::Region region(const int64_t *v)
{
    pk::heads::Region r = pk::heads::flat((const void *)v[0], v[1]);
    for (int i = 0; i < 3; ++i) r.add(v[2 + 2 * i], v[3 + 2 * i]);
    return r;
}

int shim_shared(const int64_t *a, const int64_t *b) { return pk::heads::shared(region(a), region(b)); }
int shim_distinct(const int64_t *a) { return region(a).distinct(); }

void shim_tiling(int d, int pairs, int E, int64_t rows, int *out)
{
    const pk::HeadTiling t = pk::head_tiling(d, pairs, E);
    const pk::HeadGroup g = pk::head_group(rows, t.team, pairs);
    out[0] = t.pair_chunks;
    out[1] = t.chunks;
    out[2] = t.team;
    out[3] = g.threads;
    out[4] = g.teams;
    out[5] = g.tokens;
}

void shim_sequence(int64_t M, int64_t capacity, int group, int most, int rows, int unit, int tail, int64_t start, int64_t end,
                   int64_t length, int64_t *out)
{
    int rows_shift = 0, unit_shift = unit ? 0 : -1;
    while (1 << rows_shift < rows) ++rows_shift;
    while (unit && 1 << unit_shift < unit) ++unit_shift;
    const pk::attention::Shape s = {(int)M, (int)capacity, 1, group, most, rows_shift, unit_shift, tail};
    const pk::attention::Sequence q = pk::attention::sequence(s, (int)start, (int)end, (int)length);
    out[0] = q.first;
    out[1] = q.length;
    out[2] = q.keys;
    out[3] = q.tokens;
    out[4] = q.groups;
    out[5] = q.units;
}

int64_t shim_share(int64_t total, int64_t groups) { return pk::attention::share((unsigned)total, (unsigned)groups); }
int shim_slot(int64_t part, int64_t share) { return pk::attention::slot_of((unsigned)part, (unsigned)share); }
}
