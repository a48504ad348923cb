"""The operators of a step that verifies drafted tokens, and the norms of q and k, and how their speed is measured.

A case is one pass through one of

  norm_fwd, norm_bwd   each head of q and k normalised, scaled by a gain and rotated; and the gradients
  norm_append          the same on the way of q, and of k with v into a paged cache
  tree_map             which drafted tokens each drafted token descends from, and their positions
  tree_attn            attention of requests' drafted trees over that cache
  logits               penalties for repeated tokens, biases and grammar masks on the rows of a step

``run`` computes them in elementary torch operations; with ``own`` set it makes the calls of
``paper_2502_10940_amd.cola`` instead.  Head layouts are those of the LLaMA shapes in
``paper_2502_10940_amd/inputs.py`` (8 and 32 heads of 64, 32 heads of 128), or such with fewer key heads.  Rows of
q, k, v and gradients follow N(0, 1), gains lie around 1; lengths are spread evenly up to the case's largest, in an
order that the seed gives; pages lie in the cache in a seeded random order.  A request's tree has its root in its
first drafted row, and each further row descends from an earlier one drawn evenly, so that depths grow with the
logarithm of the tree's size, as those of trees drawn by a drafting model's best guesses do.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


def _norm(kind, T, hq, hk, hd, rot=None, dtype="bf16", layout="half", scaling="none", base=10000.0, factor=1.0, orig=0,
          low=0.0, high=0.0, seq_len=0, far=0, pad=0):
    """far: positions are drawn below it (0: a row's index in its sequence of seq_len); pad: elements after each row."""
    return dict(kind=kind, T=T, hq=hq, hk=hk, hd=hd, rot=hd if rot is None else rot, dtype=dtype, layout=layout,
                scaling=scaling, base=base, factor=factor, orig=orig, low=low, high=high, seq_len=seq_len, far=far, pad=pad)


def _append(T, hq, hk, hd, page, far, idle=0, **norm):
    """idle: rows at the end of the batch that hold no token."""
    return dict(_norm("norm_append", T, hq, hk, hd, far=far, **norm), page=page, idle=idle)


def _map(n_req, max_old, max_nodes, idle=0, pos0=0):
    """Requests that hold 0 .. max_old tokens and have trees of 1 .. max_nodes drafted ones."""
    return dict(kind="tree_map", n_req=n_req, max_old=max_old, max_nodes=max_nodes, idle=idle, pos0=pos0)


def _attn(n_req, prefix, max_old, max_nodes, hq, hk, hd, page, idle=0):
    """Requests of 0 .. max_old cached tokens after a shared prefix, then trees of 1 .. max_nodes drafted ones."""
    return dict(kind="tree_attn", n_req=n_req, prefix=prefix, max_old=max_old, max_nodes=max_nodes, hq=hq, hk=hk, hd=hd,
                page=page, idle=idle)


def _logits(n_req, max_nodes, V, dtype, max_hist, n_bias=0, grammar=False, pad=0):
    """max_nodes 0: one row each, no drafted tokens; n_bias biased tokens a request; grammar: masks of the rows."""
    return dict(kind="logits", n_req=n_req, max_nodes=max_nodes, V=V, dtype=dtype, max_hist=max_hist, n_bias=n_bias,
                grammar=grammar, pad=pad)


def listed():
    cases = [
        # one short fp32 sequence of the 60M shape, as gradient checks and small experiments normalise it
        ("norm_fwd_60m_fp32", _norm("norm_fwd", 256, 8, 8, 64, dtype="f32", seq_len=256)),
        # the gradients in a pre-training step of the 1B shape: 128 sequences of 256 tokens
        ("norm_bwd_1b_train", _norm("norm_bwd", 32768, 32, 32, 64, seq_len=256)),
        # the gradients in long-context fine-tuning: an odd number of rows of packed q, k, v, half of each head
        # rotated in neighbouring pairs, positions up to 128 Ki stretched by wavelengths
        ("norm_bwd_long_odd", _norm("norm_bwd", 8191, 32, 8, 128, rot=64, layout="interleaved", scaling="wavelength",
                                    base=500000.0, factor=8.0, orig=8192, low=1.0, high=4.0, far=131072, pad=1024)),
        # the drafted tokens of 48 requests on their way into the cache, a padded batch with fewer key heads
        ("norm_append_verify_gqa", _append(1536, 32, 8, 128, page=64, far=32768, idle=37)),
        # the masks of a step of four requests with small trees: latency
        ("tree_map_few", _map(4, 700, 16)),
        # a large batch whose trees need up to four words of mask a row
        ("tree_map_many", _map(1000, 4000, 201, idle=50, pos0=1024)),
        # one request of the 60M shape, a small tree: latency
        ("tree_attn_60m_one", _attn(1, 0, 200, 12, 8, 8, 64, page=16)),
        # a batch that verifies trees of up to 32 nodes, four query heads to a key head
        ("tree_attn_verify_gqa", _attn(32, 0, 4000, 32, 32, 8, 128, page=64)),
        # the 1B shape behind a prompt that all requests share, a padded batch
        ("tree_attn_prefix_1b", _attn(24, 2048, 1500, 48, 32, 32, 64, page=128, idle=9)),
        # few requests with long documents and large trees
        ("tree_attn_long_gqa", _attn(8, 0, 32000, 64, 32, 8, 128, page=32)),
        # one greedy answer, fp32 logits of a 32000-token vocabulary: latency
        ("logits_one", _logits(1, 0, 32000, "f32", 2000, n_bias=10)),
        # a verifying step of 40 requests over an odd vocabulary: every rule at once
        ("logits_verify", _logits(40, 48, 128003, "bf16", 8000, n_bias=200, grammar=True)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = ((8, 8, 64), (16, 16, 64), (32, 32, 64), (32, 32, 128), (32, 8, 128), (16, 2, 64), (20, 4, 128), (12, 12, 128))


def _draw_norm(rng, kind):
    hq, hk, hd = rng.choice(_HEADS + ((20, 5, 80), (9, 3, 96)))
    far = rng.choice([0, _log(rng, 16, 1000000)]) if kind != "norm_append" else _log(rng, 16, 1000000)
    scaling = rng.choice(["none", "none", "linear", "wavelength"])
    norm = dict(rot=hd // rng.choice([1, 1, 2]), layout=rng.choice(["half", "interleaved"]), scaling=scaling,
                dtype=rng.choice(["bf16", "bf16", "f32"]), base=rng.choice([10000.0, 500000.0]),
                factor=1.0 if scaling == "none" else rng.choice([2.0, 4.0, 8.5]))
    if scaling == "wavelength":
        norm.update(orig=rng.choice([2048, 4096, 8192]), low=1.0, high=4.0)
    # no more than the bytes of the largest listed pass
    T = _log(rng, 1, 32768 * 4096 * (1 if norm["dtype"] == "bf16" else 0.5) / ((hq + hk) * hd))
    if kind == "norm_append":
        return _append(T, hq, hk, hd, rng.choice([16, 32, 64, 128]), far, rng.randrange(0, T // 3 + 1), **norm)
    return _norm(kind, T, hq, hk, hd, seq_len=_log(rng, 1, T), far=far, pad=rng.choice([0, 0, 64, 37]), **norm)


def draw(rng):
    kind = rng.choice(["norm_fwd", "norm_bwd", "norm_append", "tree_map", "tree_attn", "tree_attn", "tree_attn", "logits",
                       "logits"])
    if kind.startswith("norm"):
        return _draw_norm(rng, kind)
    if kind == "tree_map":
        return _map(_log(rng, 1, 1000), _log(rng, 1, 4000), _log(rng, 1, 201), rng.randrange(64), rng.randrange(5000))
    if kind == "logits":
        while True:
            c = _logits(_log(rng, 1, 256), rng.choice([0, _log(rng, 1, 64)]), _log(rng, 1000, 150000),
                        rng.choice(["bf16", "f32"]), _log(rng, 1, 8000), rng.choice([0, _log(rng, 1, 300)]),
                        rng.random() < 0.5, rng.choice([0, 0, 5, 64]))
            if work(c)["bytes"] <= 5e8:
                return c
    while True:
        hq, hk, hd = rng.choice(_HEADS)
        c = _attn(_log(rng, 1, 128), rng.choice([0, 0, 1]) * _log(rng, 1, 8192), _log(rng, 1, 32000), _log(rng, 1, 200), hq,
                  hk, hd, rng.choice([16, 32, 64, 128, 256]), rng.randrange(9))
        w = work(c)
        # the plain form's scores stay within 4 GB as well
        if w["bytes"] <= 5.9e8 and w["flops"] <= 7.5e10 and c["n_req"] * hq * c["max_nodes"] * c["max_old"] <= 1e9:
            return c


# ---------------------------------------------------------------------------
# lengths of a case: the same multiset for every seed, in the seed's order
# ---------------------------------------------------------------------------

def _spread(n, lo, hi):
    """n whole numbers spread evenly over lo .. hi, hi among them."""
    return [hi - (hi - lo) * i // n for i in range(n)]


def _lengths(case):
    """(tokens that each request held before, its drafted ones)."""
    n = case["n_req"]
    nodes = _spread(n, 1, case["max_nodes"])
    return _spread(n, 0, case["max_old"]), nodes[n // 2:] + nodes[:n // 2]


def _tokens(case):
    """Rows of the batch: its drafted tokens, and the idle rows behind them."""
    return sum(_lengths(case)[1]) + case["idle"]


def _logit_lengths(case):
    """(tokens of each request's history, rows)."""
    n = case["n_req"]
    rows = _spread(n, 1, case["max_nodes"]) if case["max_nodes"] else [1] * n
    return _spread(n, 1, case["max_hist"]), rows[n // 2:] + rows[:n // 2]


def _words(case):
    return -(-case["max_nodes"] // 64)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _dtype(case):
    return torch.float32 if case.get("dtype") == "f32" else torch.bfloat16


def _normal(g, shape, dtype):
    return torch.empty(shape, dtype=torch.float32, device=DEV).normal_(0.0, 1.0, generator=g).to(dtype)


def _uniform(g, n):
    return torch.rand(n, generator=g, device=DEV, dtype=torch.float64)


def _rows(T, width, pad, dtype):
    return torch.zeros((T, width + pad), dtype=dtype, device=DEV)[:, :width]


def _i32(x):
    return torch.as_tensor(x, dtype=torch.int32, device=DEV)


def _order(g, *lists):
    """The same seeded permutation of each list, as int32 tensors."""
    p = torch.randperm(len(lists[0]), generator=g, device=DEV)
    return [_i32(x)[p] for x in lists]


def _cumulated(n):
    return torch.cat([n.new_zeros(1), n.cumsum(0).int()])


def _owner(start, T):
    """The request of each row (rows behind the last: the last request)."""
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(start[1:].long(), t, right=True).clamp(max=start.numel() - 2)
    return r, t - start.long()[r]


def _trees(g, start, T):
    """parent[t]: the row that row t descends from, counted in its request; -1: the root."""
    r, i = _owner(start, T)
    parent = (_uniform(g, T) * i).long().clamp(max=i - 1)
    return torch.where(torch.arange(T, device=DEV) < start[-1], parent, -1).int()


def _masks(parent, start, n_req, width, words):
    """Bit j of row i: i is j or descends from it; int64 words of 64 bits."""
    r, i = _owner(start, parent.numel())
    live = torch.arange(parent.numel(), device=DEV) < start[-1]
    up = torch.zeros((n_req, width, 64 * words), device=DEV)
    p = parent.long()
    has = live & (p >= 0) & (p < i)
    # rows of no request write into the diagonal, which is set anyway
    own_row = torch.where(live, i, 0)
    up[r, own_row, torch.where(has, p, own_row)] = 1.0
    up[:, torch.arange(width, device=DEV), torch.arange(width, device=DEV)] = 1.0
    steps = max(1, math.ceil(math.log2(max(width, 2))))
    sq = up[:, :, :width]
    for _ in range(steps):                                      # descent in up to 2, 4, 8 .. steps
        sq = ((sq @ sq) > 0).float()
    up[:, :, :width] = sq
    mine = (up[r, own_row] > 0) & live[:, None]
    bits = mine.view(-1, words, 64).long() << torch.arange(64, device=DEV)
    return bits.sum(-1), mine


def _prepare_norm(case, seed):
    g, dt = _gen(seed), _dtype(case)
    T, hq, hk, hd, pad = (case[k] for k in ("T", "hq", "hk", "hd", "pad"))
    s = dict(case=case, positions=None)
    for name, h in (("q", hq), ("k", hk)):
        s[name] = _rows(T, h * hd, pad, dt)
        s[name].copy_(_normal(g, (T, h * hd), dt))
        s["g" + name] = (1.0 + 0.25 * _normal(g, (hd,), torch.float32)).to(dt)
        s[name + "_out"] = _rows(T, h * hd, pad, dt)
        if case["kind"] == "norm_bwd":
            s["d" + name + "_out"] = _rows(T, h * hd, pad, dt)
            s["d" + name + "_out"].copy_(_normal(g, (T, h * hd), dt))
            s["dg" + name] = torch.zeros(hd, dtype=torch.float32, device=DEV)
    if case["far"]:
        s["positions"] = torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32)
    return s


def _prepare_append(case, seed):
    s = _prepare_norm(case, seed)
    g, dt = _gen(seed + 1), _dtype(case)
    T, hk, hd, page = case["T"], case["hk"], case["hd"], case["page"]
    used = T - case["idle"]
    pages = -(-T // page) + 3
    s["v"] = _normal(g, (T, hk * hd), dt)
    s["used"] = used
    s["slots"] = torch.randperm(pages * page, generator=g, device=DEV)[:T].int()
    s["slots"][used:] = -1
    s["K"] = _normal(g, (pages, hk, page, hd), dt)
    s["V"] = _normal(g, (pages, hk, page, hd), dt)
    s["n_pages"] = pages
    return s


def _prepare_map(case, seed):
    g = _gen(seed)
    T = _tokens(case)
    old, nodes = _order(g, *_lengths(case))
    start = _cumulated(nodes)
    return dict(case=case, T=T, kv_len=old + nodes, start=start, parent=_trees(g, start, T),
                mask=torch.zeros((T, _words(case)), dtype=torch.int64, device=DEV),
                positions=torch.zeros(T, dtype=torch.int32, device=DEV))


def _prepare_attn(case, seed):
    g = _gen(seed)
    page, n, L, hq, hk, hd = (case[k] for k in ("page", "n_req", "prefix", "hq", "hk", "hd"))
    T = _tokens(case)
    old, nodes = _order(g, *_lengths(case))
    total, start = old + nodes, _cumulated(nodes)
    pages = -(-total // page)
    width = -(-(case["max_old"] + case["max_nodes"]) // page)
    shared = -(-L // page)
    n_pages = int(pages.sum()) + shared + 2
    ids = torch.randperm(n_pages, generator=g, device=DEV).int()
    table = torch.full((n, width), -1, dtype=torch.int32, device=DEV)
    table[torch.arange(width, device=DEV) < pages[:, None]] = ids[shared:-2]
    bf = torch.bfloat16
    mask = _masks(_trees(g, start, T), start, n, case["max_nodes"], _words(case))[0]
    return dict(case=case, T=T, used=T - case["idle"], q=_normal(g, (T, hq * hd), bf),
                K=_normal(g, (n_pages, hk, page, hd), bf), V=_normal(g, (n_pages, hk, page, hd), bf), mask=mask,
                prefix_table=ids[:shared].clone(), table=table, kv_len=total, start=start, max_kv=int(total.max()),
                out=torch.zeros((T, hq * hd), dtype=bf, device=DEV),
                lse=torch.zeros((hq, T), dtype=torch.float32, device=DEV), n_pages=n_pages)


def _prepare_logits(case, seed):
    g, dt = _gen(seed), _dtype(case)
    n, V, H = case["n_req"], case["V"], case["max_hist"]
    hist, rows = _order(g, *_logit_lengths(case))
    start = _cumulated(rows)
    T = int(start[-1])
    tokens = lambda *shape: (V * torch.rand(shape, generator=g, device=DEV) ** 3).int().clamp(max=V - 1)  # few are frequent
    s = dict(case=case, T=T, logits=_rows(T, V, case["pad"], dt), out=_rows(T, V, case["pad"], dt), start=start,
             history=tokens(n, H), hist_len=hist, prompt_len=(hist * _uniform(g, n)).int(), draft=None, mask=None,
             bias_start=None, bias_token=None, bias=None, allowed=None, allowed_row=None)
    s["logits"].copy_(_normal(g, (T, V), torch.float32) * 3.0)
    # a request in four asks for no penalty of a kind
    off = lambda: (_uniform(g, n) < 0.75).float()
    s["repetition"] = 1.0 + 0.3 * off() * _uniform(g, n).float()
    s["presence"] = off() * _uniform(g, n).float()
    s["frequency"] = off() * _uniform(g, n).float()
    if case["max_nodes"]:
        s["draft"] = tokens(T)
        s["mask"] = _masks(_trees(g, start, T), start, n, case["max_nodes"], _words(case))[0]
    b = min(case["n_bias"], V)
    if b:
        at = torch.randint(0, V, (n, 1), generator=g, device=DEV) + torch.arange(b, device=DEV) * (V // b)
        s["bias_token"] = (at % V).int().flatten()
        s["bias"] = _normal(g, (n * b,), torch.float32) * 5.0
        s["bias_start"] = (torch.arange(n + 1, device=DEV) * b).int()
    if case["grammar"]:
        states = T // 2 + 1
        s["allowed"] = torch.randint(-2 ** 31, 2 ** 31, (states, -(-V // 32)), generator=g, device=DEV).int()
        s["allowed_row"] = torch.randint(-1, states, (T,), generator=g, device=DEV).int()
    return s


def prepare(case, seed):
    make = {"norm_append": _prepare_append, "tree_map": _prepare_map, "tree_attn": _prepare_attn, "logits": _prepare_logits}
    return make.get(case["kind"], _prepare_norm)(case, seed)


# ---------------------------------------------------------------------------
# one pass: the plain forms
# ---------------------------------------------------------------------------

def _cos_sin(case, positions, T):
    """Cosines and sines of the rotated pairs, their angles in 64 bits."""
    i = torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV)
    f, factor = case["base"] ** (-2.0 * i / case["rot"]), case["factor"]
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "wavelength":
        turns = case["orig"] * f / (2.0 * math.pi)
        w = ((turns - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
        f = (1.0 - w) * f / factor + w * f
    if positions is None:
        positions = torch.arange(T, device=DEV) % (case["seq_len"] or T)
    angle = positions.double()[:, None] * f
    return angle.cos().float()[:, None], angle.sin().float()[:, None]


def _turned(case, y, cos, sin):
    rot = case["rot"]
    if case["layout"] == "half":
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned, y[..., rot:]], -1)


def _normed(case, x, gain, cos, sin):
    y = x.float().reshape(x.shape[0], -1, case["hd"])
    y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * gain.float()
    return _turned(case, y, cos, sin).flatten(1).to(x.dtype)


def _plain_norm_fwd(s):
    case = s["case"]
    cos, sin = _cos_sin(case, s["positions"], case["T"])
    return {"q": _normed(case, s["q"], s["gq"], cos, sin), "k": _normed(case, s["k"], s["gk"], cos, sin)}


def _plain_norm_bwd(s):
    case, out = s["case"], {}
    cos, sin = _cos_sin(case, s["positions"], case["T"])
    for name in ("q", "k"):
        x = s[name].float().reshape(case["T"], -1, case["hd"])
        dz = _turned(case, s["d" + name + "_out"].float().reshape(x.shape), cos, -sin)
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        xh = x * r
        w = dz * s["g" + name].float()
        out["d" + name] = (r * (w - xh * (w * xh).mean(-1, keepdim=True))).flatten(1).to(s[name].dtype)
        out["dg" + name] = (dz * xh).sum((0, 1))
    return out


def _plain_append(s):
    case, n = s["case"], s["used"]
    cos, sin = _cos_sin(case, s["positions"], case["T"])
    q, k = _normed(case, s["q"], s["gq"], cos, sin), _normed(case, s["k"], s["gk"], cos, sin)
    slots = s["slots"][:n].long()
    page, off = slots // case["page"], slots % case["page"]
    s["K"][page, :, off] = k[:n].view(n, case["hk"], case["hd"])
    s["V"][page, :, off] = s["v"][:n].view(n, case["hk"], case["hd"])
    return {"q": q, "K": s["K"], "V": s["V"]}


def _plain_map(s):
    case = s["case"]
    words, mine = _masks(s["parent"], s["start"], case["n_req"], case["max_nodes"], _words(case))
    r, _ = _owner(s["start"], s["T"])
    old = s["kv_len"].long() - (s["start"][1:] - s["start"][:-1]).long()
    depth = mine.sum(-1) - 1
    return {"mask": words, "positions": torch.where(depth >= 0, case["pos0"] + old[r] + depth, 0).int()}


def _bits(words):
    """[..][words] of int64 to [..][64 words] of truth values."""
    return ((words[..., None] >> torch.arange(64, device=DEV)) & 1).bool().flatten(-2)


def _plain_attn(s):
    case = s["case"]
    n, L, N, hq, hk, hd = (case[k] for k in ("n_req", "prefix", "max_nodes", "hq", "hk", "hd"))
    T, g, scale = s["used"], hq // hk, case["hd"] ** -0.5
    q = s["q"][:T].float().view(T, hk, g, hd)
    # every row against the shared keys, a product for each key head
    Kp, Vp = (c[s["prefix_table"].long()].transpose(0, 1).reshape(hk, -1, hd)[:, :L].float() for c in (s["K"], s["V"]))
    sp = q.transpose(0, 1).reshape(hk, T * g, hd) @ Kp.transpose(1, 2).contiguous() * scale
    # every request's rows against its own keys
    start, kv, pages = s["start"].long(), s["kv_len"].long(), s["table"].long().clamp(min=0)
    Ks, Vs = (c[pages].transpose(1, 2).reshape(n, hk, -1, hd).float() for c in (s["K"], s["V"]))
    i = torch.arange(N, device=DEV)
    rows = (start[:-1, None] + i).clamp(max=T - 1)
    qs = q[rows].transpose(1, 2).reshape(n, hk, N * g, hd)
    ss = (qs @ Ks.transpose(2, 3).contiguous() * scale).view(n, hk, N, g, -1)
    old = kv - (start[1:] - start[:-1])
    node = torch.arange(Ks.shape[2], device=DEV) - old[:, None]          # which drafted token a key is
    tree = _bits(s["mask"][rows]).gather(2, node.clamp(0, 64 * _words(case) - 1)[:, None].expand(n, N, -1))
    inside = (node >= 0) & (node < (start[1:] - start[:-1])[:, None])
    seen = (node < 0)[:, None] | (tree & inside[:, None])
    ss = torch.where(seen[:, None, :, None], ss, -math.inf)
    # back to the batch's rows, and one softmax over both parts
    mine = _owner(s["start"], T)
    m = ss.amax(-1).transpose(1, 2)[mine]
    if L:
        m = torch.maximum(m, sp.view(hk, T, g, L).amax(-1).transpose(0, 1))
    mb = torch.zeros((n, N, hk, g), device=DEV).index_put(mine, m).transpose(1, 2)
    es = torch.exp(ss - mb[..., None])
    den = es.sum(-1).transpose(1, 2)[mine]
    out = (es.view(n, hk, N * g, -1) @ Vs).view(n, hk, N, g, hd).transpose(1, 2)[mine]
    if L:
        ep = torch.exp(sp.view(hk, T, g, L) - m.transpose(0, 1)[..., None])
        den = den + ep.sum(-1).transpose(0, 1)
        out = out + (ep.view(hk, T * g, L) @ Vp).view(hk, T, g, hd).transpose(0, 1)
    s["out"][:T] = (out / den[..., None]).view(T, hq * hd).bfloat16()
    s["lse"][:, :T] = (m + den.log()).view(T, hq).T
    return {"out": s["out"], "lse": s["lse"]}


def _plain_logits(s):
    case, T = s["case"], s["T"]
    n, V, H, N = case["n_req"], case["V"], case["max_hist"], case["max_nodes"]
    r, _ = _owner(s["start"], T)
    j, tokens = torch.arange(H, device=DEV), s["history"].long()
    held = j < s["hist_len"][:, None]
    answer = held & (j >= s["prompt_len"][:, None])
    none = torch.zeros((n, V), device=DEV)
    count, seen = none.scatter_add(1, tokens, answer.float())[r], (none.scatter_add(1, tokens, held.float()) > 0)[r]
    if N:
        t = (s["start"].long()[r][:, None] + torch.arange(64 * _words(case), device=DEV)).clamp(max=T - 1)
        count = count.scatter_add(1, s["draft"].long()[t], _bits(s["mask"]).float())
    x = s["logits"].float()
    rep = s["repetition"][r][:, None]
    x = torch.where(seen | (count > 0), torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][r][:, None] * count - s["presence"][r][:, None] * (count > 0)
    if s["bias"] is not None:
        b = s["bias_token"].numel() // n
        at = torch.arange(n, device=DEV)[:, None].expand(n, b).flatten()
        x = x + torch.zeros((n, V), device=DEV).index_put((at, s["bias_token"].long()), s["bias"])[r]
    if s["allowed"] is not None:
        v = torch.arange(V, device=DEV)
        a = s["allowed_row"].long()
        ok = ((s["allowed"][a.clamp(min=0)].repeat_interleave(32, 1)[:, :V] >> (v % 32)) & 1).bool()
        x = torch.where(ok | (a < 0)[:, None], x, -math.inf)
    return x.to(s["logits"].dtype)


# ---------------------------------------------------------------------------
# one pass: the library's calls
# ---------------------------------------------------------------------------

def _plan(s):
    """The descriptors and the workspace that a program makes once for its buffers."""
    from paper_2502_10940_amd import cola
    c, kind = s["case"], s["case"]["kind"]
    s["cola"] = cola
    if kind == "tree_map":
        s["d"] = cola.tree_map_desc(c["n_req"], s["T"], c["max_nodes"], c["pos0"])
    elif kind == "tree_attn":
        s["c"] = cola.cache_desc(s["n_pages"], c["page"], c["hk"], c["hd"])
        s["d"] = cola.prefix_attn_desc(c["n_req"], s["T"], c["hq"], c["prefix"], s["max_kv"], c["max_nodes"],
                                       s["table"].shape[1])
        s["ws"] = torch.empty(max(1, cola.tree_attn_workspace_bytes(s["d"], s["c"])), dtype=torch.uint8, device=DEV)
    elif kind == "logits":
        s["d"] = cola.logits_desc(s["T"], c["V"], c["n_req"], c["max_hist"], c["max_nodes"], c["dtype"],
                                  n_bias=0 if s["bias"] is None else s["bias"].numel(),
                                  n_allowed=0 if s["allowed"] is None else s["allowed"].shape[0],
                                  ldl=s["logits"].stride(0), ldo=s["out"].stride(0))
        s["rules"] = cola.logits_rules(**{k: s[k] for k in (
            "history", "prompt_len", "hist_len", "draft", "mask", "repetition", "presence", "frequency", "bias_start",
            "bias_token", "bias", "allowed", "allowed_row")})
    else:
        q, k, qo, ko = (s[n].stride(0) for n in ("q", "k", "q_out", "k_out"))
        s["d"] = cola.rope_desc(c["T"], c["hq"], c["hk"], c["hd"], c["rot"], c["dtype"], c["layout"], c["scaling"],
                                c["base"], c["factor"], c["orig"], c["low"], c["high"], seq_len=c["seq_len"], ldq=q, ldk=k,
                                ldqo=qo, ldko=ko)
        if kind == "norm_append":
            s["c"] = cola.cache_desc(s["n_pages"], c["page"], c["hk"], c["hd"], c["dtype"])
        if kind == "norm_bwd":
            s["ws"] = torch.empty(max(1, cola.norm_rope_workspace_bytes(s["d"])), dtype=torch.uint8, device=DEV)
    return cola


def _own(s):
    cola, kind = s.get("cola") or _plan(s), s["case"]["kind"]
    if kind == "tree_map":
        cola.tree_map(s["d"], s["parent"], s["kv_len"], s["start"], s["mask"], s["positions"])
        return {"mask": s["mask"], "positions": s["positions"]}
    if kind == "tree_attn":
        cola.tree_attn(s["d"], s["c"], s["q"], s["K"], s["V"], s["prefix_table"], s["table"], s["kv_len"], s["start"],
                       s["mask"], s["out"], s["lse"], s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if kind == "logits":
        cola.logits_adjust(s["d"], s["rules"], s["logits"], s["start"], s["out"])
        return s["out"]
    if kind == "norm_append":
        cola.norm_append(s["d"], s["c"], s["q"], s["k"], s["v"], s["gq"], s["gk"], s["positions"], s["slots"], s["q_out"],
                         s["K"], s["V"], eps=EPS)
        return {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    if kind == "norm_bwd":
        cola.norm_rope_bwd(s["d"], s["dq_out"], s["dk_out"], s["q"], s["k"], s["gq"], s["gk"], s["positions"], s["q_out"],
                           s["k_out"], s["dgq"], s["dgk"], s["ws"], eps=EPS)
        return {"dq": s["q_out"], "dk": s["k_out"], "dgq": s["dgq"], "dgk": s["dgk"]}
    cola.norm_rope_fwd(s["d"], s["q"], s["k"], s["gq"], s["gk"], s["positions"], s["q_out"], s["k_out"], eps=EPS)
    return {"q": s["q_out"], "k": s["k_out"]}


def run(state):
    if own:
        return _own(state)
    return {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "norm_append": _plain_append, "tree_map": _plain_map,
            "tree_attn": _plain_attn, "logits": _plain_logits}[state["case"]["kind"]](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "tree_map":
        # a parent in, the words and a position out for each row; lengths and starts
        return {"bytes": (8 + 8 * _words(case)) * _tokens(case) + 8 * case["n_req"] + 4, "flops": 8 * _tokens(case)}
    if kind == "tree_attn":
        old, nodes = _lengths(case)
        hq, hk, hd, L = case["hq"], case["hk"], case["hd"], case["prefix"]
        T = sum(nodes)
        # of its tree a row sees about as many nodes as the logarithm of its size
        pairs = T * L + sum(w * (o + 1 + math.log(w)) for o, w in zip(old, nodes))
        return {"bytes": 2 * (2 * T * hq * hd + 2 * (L + sum(old) + T) * hk * hd) + (4 * hq + 8 * _words(case)) * T,
                "flops": int(4 * pairs * hq * hd)}
    if kind == "logits":
        hist, rows = _logit_lengths(case)
        T, V, es = sum(rows), case["V"], 4 if case["dtype"] == "f32" else 2
        states = min(T, T // 2 + 1) if case["grammar"] else 0
        return {"bytes": 2 * es * T * V + 4 * sum(hist) + (12 * T if case["max_nodes"] else 0) +
                8 * case["n_bias"] * case["n_req"] + states * 4 * -(-V // 32), "flops": 4 * T * V}
    es = 4 if case["dtype"] == "f32" else 2
    T, hq, hk, hd = (case[k] for k in ("T", "hq", "hk", "hd"))
    n = T * (hq + hk) * hd
    elements = {"norm_fwd": 2 * n, "norm_bwd": 3 * n, "norm_append": T * hq * hd * 2 + (T - case.get("idle", 0)) * hk * hd * 4}
    return {"bytes": es * elements[kind] + (4 * T if case["far"] else 0) + (4 * T if kind == "norm_append" else 0),
            "flops": (20 if kind == "norm_bwd" else 7) * n}


# ---------------------------------------------------------------------------
# the same results in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _exact_turns(case, positions):
    """exp(i angle) for each row and pair: the pairs' frequencies one by one."""
    freq = []
    for i in range(case["rot"] // 2):
        f = math.exp(-2.0 * i / case["rot"] * math.log(case["base"]))
        if case["scaling"] == "linear":
            f /= case["factor"]
        elif case["scaling"] == "wavelength":
            wave = 2 * math.pi / f
            if wave > case["orig"] / case["low"]:
                f /= case["factor"]
            elif wave > case["orig"] / case["high"]:
                w = (case["orig"] / wave - case["low"]) / (case["high"] - case["low"])
                f *= w + (1.0 - w) / case["factor"]
        freq.append(f)
    if positions is None:
        positions = torch.arange(case["T"], device=DEV).remainder(case["seq_len"] or case["T"])
    angle = torch.outer(positions.double(), torch.tensor(freq, dtype=torch.float64, device=DEV))
    return torch.polar(torch.ones_like(angle), angle)


def _exact_normed(case, x, gain, turns):
    rot = case["rot"]
    y = x.unflatten(1, (-1, case["hd"]))
    y = y / torch.sqrt(y.square().sum(-1, keepdim=True) / case["hd"] + EPS) * gain
    part = y[..., :rot]
    pairs = part.unflatten(-1, (2, rot // 2)).transpose(-1, -2) if case["layout"] == "half" else part.unflatten(-1, (-1, 2))
    z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turns[:, None])
    z = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
    return torch.cat([z, y[..., rot:]], -1).flatten(1)


def _exact_norm(case, seed):
    s = _prepare_norm(case, seed)
    turns, out = _exact_turns(case, s["positions"]), {}
    for name in ("q", "k"):
        x, gain = s[name].double(), s["g" + name].double()
        if case["kind"] == "norm_fwd":
            out[name] = _exact_normed(case, x, gain, turns)
            continue
        x.requires_grad_(), gain.requires_grad_()
        out["d" + name], out["dg" + name] = torch.autograd.grad(_exact_normed(case, x, gain, turns), (x, gain),
                                                                s["d" + name + "_out"].double())
    return out


def _exact_append(case, seed):
    s = _prepare_append(case, seed)
    turns = _exact_turns(case, s["positions"])
    k = _exact_normed(case, s["k"].double(), s["gk"].double(), turns)
    out = {"q": _exact_normed(case, s["q"].double(), s["gq"].double(), turns)}
    at = s["slots"].long()[:s["used"]]
    for name, rows in (("K", k), ("V", s["v"].double())):
        c = s[name].double().transpose(1, 2).flatten(0, 1)                # a row for each slot
        c[at] = rows[:s["used"]].view(-1, case["hk"], case["hd"])
        out[name] = c.unflatten(0, (-1, case["page"])).transpose(1, 2).contiguous()
    return out


def _exact_attn(case, seed):
    s = _prepare_attn(case, seed)
    L, hq, hk, hd, page = (case[k] for k in ("prefix", "hq", "hk", "hd", "page"))
    out, lse = torch.zeros((s["T"], hq, hd), dtype=torch.float64, device=DEV), s["lse"].double()
    q = s["q"].double().view(s["T"], hk, hq // hk, hd) / math.sqrt(hd)
    start, total = s["start"].tolist(), s["kv_len"].tolist()

    def keys(pages, n):
        return [c[pages.long()].transpose(0, 1).flatten(1, 2)[:, :n].double() for c in (s["K"], s["V"])]

    Kp, Vp = keys(s["prefix_table"], L)
    for r in range(case["n_req"]):
        lo, hi, n = start[r], start[r + 1], total[r]
        K, V = keys(s["table"][r, :-(-n // page)], n)
        x = q[lo:hi].permute(1, 2, 0, 3).flatten(1, 2)                      # [hk][g rows][hd]
        w = torch.cat([x @ Kp.mT.contiguous(), x @ K.mT.contiguous()], -1).unflatten(1, (-1, hi - lo))
        for i in range(hi - lo):
            words = s["mask"][lo + i].tolist()
            hidden = [L + n - (hi - lo) + j for j in range(hi - lo) if not words[j // 64] >> (j % 64) & 1]
            w[:, :, i, hidden] = -math.inf
        total_weight = torch.logsumexp(w, -1)
        p = torch.exp(w - total_weight[..., None]).flatten(1, 2)
        y = p[..., :L] @ Vp + p[..., L:] @ V
        out[lo:hi] = y.unflatten(1, (-1, hi - lo)).permute(2, 0, 1, 3).flatten(1, 2)
        lse[:, lo:hi] = total_weight.flatten(0, 1)
    return {"out": out.flatten(1), "lse": lse}


def _exact_logits(case, seed):
    s = _prepare_logits(case, seed)
    V, n, start = case["V"], case["n_req"], s["start"].tolist()
    out = s["logits"].double().clone()
    value = lambda name, r: s[name][r].double()
    for r in range(n):
        rows = out[start[r]:start[r + 1]]
        past, end = int(s["prompt_len"][r]), int(s["hist_len"][r])
        prompt = torch.bincount(s["history"][r, :past], minlength=V)
        times = torch.bincount(s["history"][r, past:end], minlength=V).double().repeat(len(rows), 1)
        if s["draft"] is not None:
            words = s["mask"][start[r]:start[r + 1]].tolist()
            for i in range(len(rows)):
                ancestors = [j for j in range(len(rows)) if words[i][j // 64] >> (j % 64) & 1]
                times[i] += torch.bincount(s["draft"][start[r]:start[r + 1]][ancestors], minlength=V)
        shrink = torch.where(rows > 0, 1.0 / value("repetition", r), value("repetition", r))
        rows.mul_(torch.where((times > 0) | (prompt > 0), shrink, 1.0))
        rows.sub_(times * value("frequency", r)).sub_((times > 0) * value("presence", r))
        if s["bias"] is not None:
            lo, hi = s["bias_start"][r:r + 2].tolist()
            rows[:, s["bias_token"][lo:hi].long()] += s["bias"][lo:hi].double()
    if s["allowed"] is not None:
        states = s["allowed"].cpu().numpy().view("uint8")
        import numpy as np
        ok = torch.from_numpy(np.unpackbits(states, axis=1, bitorder="little")[:, :V].astype(bool)).to(DEV)
        a = s["allowed_row"].long()
        out[(a >= 0)[:, None] & ~ok[a.clamp(min=0)]] = -math.inf
    return out


def exact(case, seed):
    if case["kind"] == "tree_map":
        return None                                                        # whole numbers
    make = {"norm_append": _exact_append, "tree_attn": _exact_attn, "logits": _exact_logits}
    return make.get(case["kind"], _exact_norm)(case, seed)
