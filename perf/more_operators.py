"""The calls of the attention operators whose time is followed from change to change.

Between the products of an attention layer a network runs these:

- ``rope_qk``: queries and keys of new tokens, each head normed to its root mean
  square and rotated by its token's position; ``rope_qk_backward`` the gradients
  of both and of the norms' weights;
- ``cache_append``: the same where tokens are generated: the keys go, normed and
  rotated, to their slots of a paged cache, the values beside them, the queries to
  the attention that follows;
- ``attention_tree``: that attention: the drafted tokens of each sequence (one, a
  chain or a tree of them, told by a bit mask) over the sequence's pages.

``own`` chooses between those calls and the same operators in their plain form,
elementary torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6


# ------------------------------------------------------------------ the cases

def _rope(name, M, Hq, Hk, d, rot, dtype, layout="half", norm=True, far=4096, back=False):
    """M tokens, Hq query and Hk key heads of d channels, the first rot of them rotated; positions up to `far`."""
    return {"name": name, "op": "back" if back else "rope", "M": M, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot, "dtype": dtype,
            "layout": layout, "norm": norm, "far": far}


def _append(name, M, Hq, Hk, d, rot, dtype, page, pages, layout="half", norm=True, far=4096, padded=0):
    """The same into a cache of `pages` pages; the last `padded` tokens are a batch's padding and have no slot."""
    return {"name": name, "op": "append", "M": M, "Hq": Hq, "Hk": Hk, "d": d, "rot": rot, "dtype": dtype, "layout": layout,
            "norm": norm, "far": far, "page": page, "pages": pages, "padded": padded}


def _attention(name, B, T, L, Hk, G, d, dtype, page, tree=True, ragged=True, cap=0.0, lse=False):
    """B sequences of up to L cached positions and up to T drafted tokens, Hk key heads with G query heads each."""
    return {"name": name, "op": "attention", "B": B, "T": T, "L": L, "Hk": Hk, "G": G, "d": d, "dtype": dtype, "page": page,
            "tree": tree, "ragged": ragged, "cap": cap, "lse": lse}


def listed():
    return [
        # a small model's heads, an odd number of prompt tokens, half of each head rotated, neighbours as pairs
        _rope("rope_odd", 777, 12, 3, 80, 40, "f32", layout="interleaved", norm=False),
        # prompts of 8192 tokens, normed heads, far into a long context
        _rope("rope_prompts", 8192, 32, 8, 128, 128, "bf16", far=1 << 20),
        # gradients of a small training batch
        _rope("rope_back_odd", 1003, 12, 4, 96, 48, "f32", back=True),
        # gradients of a training batch of 8192 tokens
        _rope("rope_back_train", 8192, 32, 8, 128, 128, "bf16", far=8192, back=True),
        # one token of one sequence: latency
        _append("append_token", 1, 32, 8, 128, 128, "bf16", 16, 256),
        # a padded batch of prompts into a cache, pairs of neighbours, no norm
        _append("append_prompts", 4100, 32, 8, 128, 64, "f16", 64, 128, layout="interleaved", norm=False, padded=37),
        # one sequence generating one token: latency, and the cache read by the whole card
        _attention("attention_token", 1, 1, 4096, 8, 4, 128, "bf16", 16, tree=False, ragged=False),
        # 32 sequences of uneven lengths that generate together
        _attention("attention_batch", 32, 1, 8192, 8, 4, 128, "bf16", 16, tree=False),
        # trees of up to 16 drafted tokens
        _attention("attention_tree", 16, 16, 16384, 8, 4, 128, "bf16", 64),
        # odd heads, few positions to a page, capped scores
        _attention("attention_odd", 5, 7, 3001, 3, 5, 80, "f16", 24, cap=30.0, lse=True),
        # 32 bits throughout
        _attention("attention_f32", 3, 4, 5000, 4, 2, 64, "f32", 32, lse=True),
        # the widest trees over long contexts
        _attention("attention_wide", 4, 64, 32768, 8, 8, 128, "bf16", 128),
    ]


MOST_BYTES = 4e8          # of a drawn case: below the largest listed ones, as is
MOST_FLOPS = 9e10         # (32 bits have a sixteenth of the rate)
MOST_CACHED = 1 << 27     # elements of K that an attention's plain form lays out
MOST_SCORES = 1 << 28     # and of its scores


def _log(rng, lo, hi):
    return min(max(int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))), lo), hi)


def _heads(rng):
    return rng.choice([1, 2, 3, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 8, 8, 16])


def _draw_one(rng):
    op = rng.choice(["rope", "back", "append", "attention", "attention", "attention"])
    Hk, G = _heads(rng)
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op == "attention":
        T = rng.choice([1, 1, _log(rng, 1, 64)])
        return {"op": op, "B": _log(rng, 1, 64), "T": T, "L": _log(rng, 16, 32768), "Hk": Hk, "G": G,
                "d": rng.choice([64, 80, 96, 128, 128, 128, 256, rng.randrange(16, 257)]), "dtype": dtype,
                "page": rng.choice([1, 8, 16, 16, 24, 32, 64, 128, 256]), "tree": T > 1 and rng.random() < 0.7,
                "ragged": rng.random() < 0.7, "cap": rng.choice([0.0, 0.0, 30.0]), "lse": rng.random() < 0.3}
    d = rng.choice([64, 80, 96, 128, 128, 256, 2 * rng.randrange(8, 129)])
    rot = rng.choice([d, d, max(2, d // 4 * 2), max(2, d // 8 * 2)])
    M = _log(rng, 1, 64) if rng.random() < 0.4 else _log(rng, 64, 8192)
    case = {"op": op, "M": M, "Hq": Hk * G, "Hk": Hk, "d": d, "rot": rot, "dtype": dtype,
            "layout": rng.choice(["half", "half", "interleaved"]), "norm": rng.random() < 0.6,
            "far": rng.choice([4096, 1 << 17, 1 << 20])}
    if op == "append":
        page = rng.choice([8, 16, 24, 64, 256])
        case.update(page=page, pages=-(-M // page) + rng.randrange(1, 64), padded=rng.choice([0, 0, M // 3]))
    return case


def draw(rng):
    while True:
        c = _draw_one(rng)
        w = work(c)
        if w["bytes"] > MOST_BYTES or w["flops"] * (16 if c["dtype"] == "f32" else 1) > MOST_FLOPS:
            continue
        heads = c["B"] * c["Hk"] * (c["L"] + c["T"]) if c["op"] == "attention" else 0
        if heads * c["d"] <= MOST_CACHED and heads * c.get("T", 0) * c.get("G", 0) <= MOST_SCORES:
            return c


def _lengths(case):
    """(cached positions, drafted tokens) of each sequence: spread evenly from a quarter of L (of T) to the whole where ragged."""
    B, T, L = case["B"], case["T"], case["L"]
    if not case["ragged"] or B == 1:
        return [L] * B, [T] * B
    order = [(7 * b + 3) % B if B % 7 else b for b in range(B)]  # long and short ones mixed
    return ([max(1, L * (B + 3 * o) // (4 * B - 3)) for o in order],
            [max(1, T * (B + 3 * o) // (4 * B - 3)) for o in reversed(order)])


def work(case):
    size, d = SIZE[case["dtype"]], case["d"]
    if case["op"] == "attention":
        lengths, drafted = _lengths(case)
        seen = [n + t for n, t in zip(lengths, drafted)]
        Hq = case["Hk"] * case["G"]
        rows = sum(drafted) * Hq
        return {"bytes": 2 * sum(seen) * case["Hk"] * d * size + 2 * rows * d * size + (4 * rows if case["lse"] else 0)
                + 4 * sum(-(-n // case["page"]) for n in seen) + 8 * sum(drafted),
                "flops": 4 * sum(n * t for n, t in zip(seen, drafted)) * Hq * d}
    M, heads = case["M"], case["Hq"] + case["Hk"]
    wide = 1 if not case["norm"] else 2  # a gradient reads what the norm read
    read = {"rope": heads, "append": heads + case["Hk"], "back": heads * wide}[case["op"]]
    written = {"rope": heads, "append": heads + case["Hk"], "back": heads}[case["op"]]
    return {"bytes": M * d * size * (read + written) + 8 * M + 4 * case["rot"] + (4 * d * size if case["norm"] else 0),
            "flops": M * heads * (3 * case["rot"] + (4 * d if case["norm"] else 0)) * (2 if case["op"] == "back" else 1)}


# ------------------------------------------------------------------ inputs

def _frequencies(rot):
    return 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)


def _prepare_heads(case, g):
    M, Hq, Hk, d, dtype = case["M"], case["Hq"], case["Hk"], case["d"], TYPES[case["dtype"]]

    def projected():
        # one product's output for queries, keys and values
        p = torch.randn((M, (Hq + 2 * Hk) * d), generator=g, device="cuda").to(dtype)
        return (p[:, :Hq * d].view(M, Hq, d), p[:, Hq * d:(Hq + Hk) * d].view(M, Hk, d), p[:, (Hq + Hk) * d:].view(M, Hk, d))

    def weight():
        return (1 + 0.1 * torch.randn(d, generator=g, device="cuda")).to(dtype) if case["norm"] else None

    q, k, v = projected()
    s = {"case": case, "q": q, "k": k, "v": v, "qw": weight(), "kw": weight(), "f": _frequencies(case["rot"]),
         "positions": torch.randint(0, case["far"], (M,), generator=g, device="cuda")}
    if case["op"] == "back":
        s["dq"] = torch.randn((M, Hq, d), generator=g, device="cuda").to(dtype)
        s["dk"] = torch.randn((M, Hk, d), generator=g, device="cuda").to(dtype)
    if case["op"] == "append":
        shape = (case["pages"], case["page"], Hk, d)
        s["kc"] = torch.randn(shape, generator=g, device="cuda").to(dtype)
        s["vc"] = torch.randn(shape, generator=g, device="cuda").to(dtype)
        slots = torch.randperm(case["pages"] * case["page"], generator=g, device="cuda")[:M].contiguous()
        if case["padded"]:
            slots[M - case["padded"]:] = -1
        s["slots"] = slots
    return s


def _prepare_attention(case, g):
    lengths, drafted = _lengths(case)
    Hk, G, d, page, dtype = case["Hk"], case["G"], case["d"], case["page"], TYPES[case["dtype"]]
    need = [-(-(n + t) // page) for n, t in zip(lengths, drafted)]
    pages = sum(need) + 3
    shape = (pages, page, Hk, d)
    kc = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)
    vc = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(dtype)
    # pages in the order in which a pool hands them out after a while: any
    order = torch.randperm(pages, generator=g, device="cuda").int()
    table = torch.zeros((case["B"], max(need)), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    starts, mask = [0], []
    cpu = torch.Generator().manual_seed(int(torch.randint(1 << 30, (1,), generator=g, device="cuda")))
    for t in drafted:
        starts.append(starts[-1] + t)
        parents = (torch.rand(t, generator=cpu) * torch.arange(t)).long().tolist()
        for i in range(t):
            # a drafted token sees itself and its ancestors
            mask.append((mask[starts[-2] + parents[i]] if i else 0) | 1 << i)
    mask = torch.tensor([m - (1 << 64) if m >> 63 else m for m in mask], dtype=torch.int64, device="cuda") if case["tree"] else None
    q = (1.5 * torch.randn((starts[-1], Hk * G, d), generator=g, device="cuda")).to(dtype)
    return {"case": case, "q": q, "kc": kc, "vc": vc, "table": table, "mask": mask,
            "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            "starts": torch.tensor(starts, dtype=torch.int32, device="cuda")}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return _prepare_attention(case, g) if case["op"] == "attention" else _prepare_heads(case, g)


# ------------------------------------------------------------------ the framework's operators

def _run_own(s):
    import paper_1904_05347_amd as pk
    case = s["case"]
    if case["op"] == "attention":
        return pk.attention_tree(s["q"], s["kc"], s["vc"], s["table"], s["lengths"], s["starts"], case["T"], mask=s["mask"],
                                 cap=case["cap"], lse=case["lse"])
    if case["op"] == "rope":
        return pk.rope_qk(s["q"], s["k"], s["positions"], s["f"], s["qw"], s["kw"], eps=EPS, layout=case["layout"])
    if case["op"] == "append":
        q = pk.cache_append(s["k"], s["v"], s["kc"], s["vc"], s["slots"], s["positions"], s["f"], s["kw"], q=s["q"],
                            q_weight=s["qw"], eps=EPS, layout=case["layout"])
        return q, s["kc"], s["vc"]
    grads = pk.rope_qk_backward(s["dq"], s["dk"], s["q"], s["k"], s["positions"], s["f"], s["qw"], s["kw"], eps=EPS,
                                layout=case["layout"])
    return grads if case["norm"] else grads[:2]


# ------------------------------------------------------------------ the plain forms

def _turned(x, s, inverse=False):
    """x (fp32, tokens x heads x d) with its pairs rotated by their angles."""
    case = s["case"]
    angles = s["positions"].double()[:, None] * s["f"]
    cos, sin = angles.cos().float()[:, None], angles.sin().float()[:, None]
    if inverse:
        sin = -sin
    rot = case["rot"]
    if case["layout"] == "half":
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, x[..., rot:]), dim=-1)
    a, b = x[..., 0:rot:2], x[..., 1:rot:2]
    return torch.cat((torch.stack((a * cos - b * sin, b * cos + a * sin), dim=-1).flatten(-2), x[..., rot:]), dim=-1)


def _normed(x, w):
    return x if w is None else x * torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS) * w.float()


def _plain_backward(dy, x, w, s):
    g = _turned(dy.float(), s, inverse=True)
    if w is None:
        return g.to(dy.dtype), None
    x = x.float()
    n = torch.rsqrt((x * x).mean(dim=-1, keepdim=True) + EPS)
    gw = g * w.float()
    dx = n * (gw - x * (n * n * (gw * x).mean(dim=-1, keepdim=True)))
    return dx.to(dy.dtype), (g * x * n).sum(dim=(0, 1)).to(w.dtype)


def _plain_append(s):
    case = s["case"]
    q = _turned(_normed(s["q"].float(), s["qw"]), s).to(s["q"].dtype)
    k = _turned(_normed(s["k"].float(), s["kw"]), s).to(s["k"].dtype)
    # a padded token writes what the first token writes, where that writes it
    kept = s["slots"] >= 0
    at = torch.where(kept, s["slots"], s["slots"][:1])
    kept = kept[:, None, None]
    shape = (case["pages"] * case["page"],) + tuple(k.shape[1:])
    s["kc"].view(shape)[at] = torch.where(kept, k, k[:1])
    s["vc"].view(shape)[at] = torch.where(kept, s["v"], s["v"][:1])
    return q, s["kc"], s["vc"]


def _plain_attention(s):
    case = s["case"]
    Hk, G, d, T, page = case["Hk"], case["G"], case["d"], case["T"], case["page"]
    B, P = s["table"].shape
    N = P * page
    lengths, starts, device = s["lengths"].long()[:, None], s["starts"].long(), s["q"].device
    t = torch.arange(T, device=device)
    row = starts[:-1, None] + t                                  # B x T: the tokens' rows, some of them the next sequence's
    row = row.clamp(max=s["q"].shape[0] - 1)
    j = torch.arange(N, device=device) - lengths                 # B x N: a position's number among the drafted ones
    if s["mask"] is None:
        seen = j[:, None, :] <= t[:, None]
    else:
        drafted = j.clamp(0, 63)
        seen = (j[:, None, :] < 0) | ((s["mask"][row][:, :, None] >> drafted[:, None, :] & 1 == 1) & (j[:, None, :] < 64))
    seen = seen[:, None, :, None, :]                             # B x 1 x T x 1 x N
    q = s["q"].float()[row].view(B, T, Hk, G, d).permute(0, 2, 1, 3, 4).reshape(B * Hk, T * G, d)
    k = s["kc"][s["table"].long()].float().view(B, N, Hk, d).permute(0, 2, 3, 1).reshape(B * Hk, d, N)
    score = torch.matmul(q, k).mul_(d ** -0.5).view(B, Hk, T, G, N)
    del k
    if case["cap"]:
        score = torch.tanh(score / case["cap"]).mul_(case["cap"])
    score.masked_fill_(~seen, -math.inf)
    most = score.amax(dim=-1, keepdim=True)
    p = score.sub_(most).exp_()
    total = p.sum(dim=-1, keepdim=True)
    v = s["vc"][s["table"].long()].float().view(B, N, Hk, d).permute(0, 2, 1, 3).reshape(B * Hk, N, d)
    o = torch.matmul(p.view(B * Hk, T * G, N), v).view(B, Hk, T, G, d) / total
    # back to the tokens' rows: token m is number m - starts[b] of its sequence b
    m = torch.arange(s["q"].shape[0], device=device)
    b = torch.searchsorted(starts, m, right=True) - 1
    i = m - starts[b]
    out = o.permute(0, 2, 1, 3, 4).reshape(B, T, Hk * G, d)[b, i].to(s["q"].dtype)
    if not case["lse"]:
        return out
    lse = (most + total.log()).permute(0, 2, 1, 3, 4).reshape(B, T, Hk * G)[b, i]
    return out, lse


def run(state):
    if own:
        return _run_own(state)
    s, op = state, state["case"]["op"]
    if op == "attention":
        return _plain_attention(s)
    if op == "append":
        return _plain_append(s)
    if op == "rope":
        return (_turned(_normed(s["q"].float(), s["qw"]), s).to(s["q"].dtype),
                _turned(_normed(s["k"].float(), s["kw"]), s).to(s["k"].dtype))
    dq, dqw = _plain_backward(s["dq"], s["q"], s["qw"], s)
    dk, dkw = _plain_backward(s["dk"], s["k"], s["kw"], s)
    return (dq, dk) if dqw is None else (dq, dk, dqw, dkw)


# ------------------------------------------------------------------ from the definitions, in 64 bits

def _rotation(s):
    """For each token the d x d matrix that a head's row is multiplied by, as (partner of each channel, its factor, the own one's)."""
    case = s["case"]
    d, rot, device = case["d"], case["rot"], s["q"].device
    c = torch.arange(d, device=device)
    if case["layout"] == "half":
        partner = torch.where(c < rot // 2, c + rot // 2, torch.where(c < rot, c - rot // 2, c))
        pair, second = torch.where(c < rot // 2, c, c - rot // 2), c >= rot // 2
    else:
        partner = torch.where(c < rot, c ^ 1, c)
        pair, second = c // 2, c % 2 == 1
    turned = c < rot
    angle = s["positions"].double()[:, None] * s["f"][torch.where(turned, pair, 0)] * turned
    return partner, torch.where(second, 1.0, -1.0) * turned * torch.sin(angle), torch.cos(angle)


def _exact_heads(x, w, s):
    x = x.double()
    if w is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS) * w.double()
    partner, sin, cos = _rotation(s)
    return x * cos[:, None] + x[..., partner] * sin[:, None]


def _exact_backward(dy, x, w, s):
    dy = dy.double()
    partner, sin, cos = _rotation(s)
    # y_c = cos x_c + sin_c x_partner(c): x_c takes cos from y_c and its partner's sine from y_partner
    g = dy * cos[:, None] + dy[..., partner] * sin[:, partner][:, None]
    if w is None:
        return g, None
    x = x.double()
    n = (x.square().mean(-1, keepdim=True) + EPS) ** -0.5
    h = g * w.double()
    return n * h - n ** 3 * x * (h * x).sum(-1, keepdim=True) / x.shape[-1], (g * x * n).sum((0, 1))


def _exact_attention(s):
    """Sequence by sequence, key head by key head, over the positions that it has."""
    case = s["case"]
    lengths, drafted = _lengths(case)
    Hk, G, d, page = case["Hk"], case["G"], case["d"], case["page"]
    out = torch.empty((sum(drafted), Hk * G, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((sum(drafted), Hk * G), dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, t) in enumerate(zip(lengths, drafted)):
        pages = s["table"][b, :-(-(n + t) // page)].long()
        hidden = torch.zeros((t, n + t), dtype=torch.bool, device="cuda")
        for i in range(t):
            word = (1 << i + 1) - 1 if s["mask"] is None else int(s["mask"][at + i])
            hidden[i, n:] = torch.tensor([not word >> j & 1 for j in range(t)], device="cuda")
        for h in range(Hk):
            k = s["kc"][pages, :, h].reshape(-1, d)[:n + t].double()
            v = s["vc"][pages, :, h].reshape(-1, d)[:n + t].double()
            for e in range(h * G, (h + 1) * G):
                score = s["q"][at:at + t, e].double() @ k.t() / math.sqrt(d)
                if case["cap"]:
                    score = case["cap"] * torch.tanh(score / case["cap"])
                score[hidden] = -math.inf
                lse[at:at + t, e] = torch.logsumexp(score, dim=1)
                out[at:at + t, e] = torch.exp(score - lse[at:at + t, e, None]) @ v
        at += t
    return (out, lse) if case["lse"] else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "attention":
        return _exact_attention(s)
    if case["op"] == "back":
        dq, dqw = _exact_backward(s["dq"], s["q"], s["qw"], s)
        dk, dkw = _exact_backward(s["dk"], s["k"], s["kw"], s)
        return (dq, dk, dqw, dkw) if case["norm"] else (dq, dk)
    q, k = _exact_heads(s["q"], s["qw"], s), _exact_heads(s["k"], s["kw"], s)
    if case["op"] == "rope":
        return q, k
    kc, vc = s["kc"].double(), s["vc"].double()
    kept = s["slots"] >= 0
    page, place = s["slots"][kept] // case["page"], s["slots"][kept] % case["page"]
    kc[page, place] = k[kept]
    vc[page, place] = s["v"][kept].double()
    return q, kc, vc
