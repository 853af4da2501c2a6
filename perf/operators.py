"""Performance cases of the operators on a cache that is in use: what a program does with a layer's compact cache after the prefill.

Four operators, each on one layer's cache (sequence b has a region of slots of which the first lens[b] are in use):
  attend  fresh tokens, the last ones in the cache, attend to it: single tokens, which may add their attention weights to the
          mass that is kept for each slot, or trees of drafted tokens
  append  rows of keys and values into the free slots behind those in use
  accept  the verified path of a drafted tree stays, with its attention weights added to the mass, and the other drafts go
  evict   a cache over its budget keeps the slots of largest mass and the most recent ones

Where `own` is false, `run` computes them in plain torch operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _case(kind, name=None, *, heads=32, kv_heads=8, head_dim=128, dtype="bf16", batch=1, slots=2080, fill=1.0, tokens=1, planes=1,
          softcap=0.0, slopes=False, decay=0.0, budget=0, tail=0):
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, batch=batch, slots=slots, fill=fill,
             tokens=tokens, planes=planes, softcap=softcap, slopes=slopes, decay=decay, budget=budget, tail=tail)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest configuration, full precision, one KV head per query head: seven drafted tokens, a bias by distance
        _case("attend", "attend_f32_1k_tree7", heads=8, kv_heads=8, head_dim=64, dtype="f32", slots=1031, tokens=7, slopes=True),
        # a token after a 32K prefill that kept 2048 tokens and its window of 32; its weights go on the one mass of all heads
        _case("attend", "attend_2k_token", slots=2081, decay=0.9),
        # tokens of sixteen sequences with caches of 5 % of up to 128K, a mass for each KV head
        _case("attend", "attend_6k_batch16", batch=16, slots=6586, fill=0.15, planes=8, decay=0.9),
        # trees of 64 drafts over caches of the longest configuration's budget, capped scores
        _case("attend", "attend_16k_tree64", batch=4, slots=16512, fill=0.5, tokens=64, softcap=30.0),
        # tokens over caches that were not compacted, the longest
        _case("attend", "attend_128k_batch8", batch=8, slots=131073, fill=0.5, planes=8, decay=0.98),
        # a token of each of 64 sequences
        _case("append", "append_token_b64", batch=64, slots=2112, fill=0.9),
        # eight compact caches stored after their prefill
        _case("append", "append_prompt_b8", batch=8, slots=8192, fill=0.0, tokens=5715),
        # one verified tree of 26 drafts
        _case("accept", "accept_2k_tree26", slots=2106, tokens=26, decay=0.9),
        # eight of 64 drafts, a mass for each KV head
        _case("accept", "accept_16k_tree64", batch=8, slots=16512, fill=0.5, tokens=64, planes=8, decay=0.9),
        # every step of a cache that is full evicts one token
        _case("evict", "evict_one", slots=2081, budget=2080, tail=32),
        # sixteen caches are halved, each head by its own mass
        _case("evict", "evict_8k_batch16", batch=16, slots=8192, fill=0.75, planes=8, budget=4096, tail=64),
        # a cache that was not compacted comes down to the longest configuration's budget
        _case("evict", "evict_128k", slots=131072, budget=16448, tail=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("attend", "append", "accept", "evict"), (6, 2, 3, 3))[0]
    heads, kv_heads, head_dim = rng.choice(((32, 8, 128), (32, 8, 128), (8, 2, 128), (16, 2, 128), (32, 32, 128), (8, 8, 64), (32, 8, 64)))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    batch = rng.choice((1, 1, 2, 4, 7, 16, 33, 64))
    planes = rng.choice((1, kv_heads))
    fill = 1.0 if batch == 1 else rng.choice((0.1, 0.5, 0.9))
    decay = rng.choice((0.5, 0.9, 1.0))
    softcap, slopes = rng.choice((0.0, 0.0, 30.0, 50.0)), rng.random() < 0.25
    row = kv_heads * head_dim * (4 if dtype == "f32" else 2)
    most = max(256, min(131072, (3 << 29) // (row * batch)))   # slots whose keys and values cost less than the largest listed ones
    like = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, batch=batch, planes=planes)
    if kind == "append":
        tokens = rng.choice((1, 1, 5, _log(rng, 16, most // 4)))
        return _case(kind, **like, slots=_log(rng, 2 * tokens, most) + tokens, fill=0.5, tokens=tokens)
    if kind == "evict":
        slots = _log(rng, 128, most)
        budget = min(slots - 1, max(16, int(slots * rng.choice((0.1, 0.5, 0.9, 0.99)))))
        return _case(kind, **like, slots=slots, fill=max(fill, 0.5), budget=budget, tail=min(budget // 2, rng.choice((0, 8, 32, 64))))
    tokens = 1 if kind == "attend" and rng.random() < 0.5 else rng.choice((2, 5, 8, 13, 26, 32, 48, 64))
    most = max(256, min(most, (1 << 27) // (heads * tokens * batch)))   # ... and the plain form's scores
    c = _case(kind, **like, slots=_log(rng, 64, most) + tokens, fill=fill, tokens=tokens, softcap=softcap, slopes=slopes, decay=decay)
    return dict(c, decay=0.0) if kind == "attend" and (tokens > 1 or rng.random() < 0.3) else c


def _trees(batch, tokens, r):
    """Random trees of drafts, parents first: which drafts each one sees (bits, itself among them), its depth, a path to verify."""
    masks, depths, paths = np.zeros((batch, tokens), np.uint64), np.zeros((batch, tokens), np.int64), []
    for b in range(batch):
        for t in range(tokens):
            parent = r.randint(-1, t) if t and r.rand() > 0.1 else -1
            masks[b, t] = (masks[b, parent] if parent >= 0 else np.uint64(0)) | np.uint64(1 << t)
            depths[b, t] = depths[b, parent] + 1 if parent >= 0 else 0
        last = int(masks[b, r.randint(0, tokens)])
        paths.append([t for t in range(tokens) if last >> t & 1])
    return masks, depths, paths


def prepare(case, seed):
    H, G, d, dt = case["heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    batch, slots, T, P = case["batch"], case["slots"], case["tokens"], case["planes"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    r = np.random.RandomState(seed % (1 << 32))
    new = 0 if case["kind"] == "evict" else T          # tokens that are fresh, or come
    old = slots - new
    before = np.array([r.randint(int(case["fill"] * old), old + 1) for _ in range(batch)])
    held = before if case["kind"] in ("append", "evict") else before + T
    cuda = lambda x, t: torch.as_tensor(np.ascontiguousarray(x), dtype=t).cuda()  # noqa: E731
    s = dict(case, cu_slots=[slots * b for b in range(batch + 1)], cu_new=[new * b for b in range(batch + 1)], lens=cuda(held, torch.int32),
             lens_out=torch.empty(batch, dtype=torch.int32, device="cuda"))
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda", dtype=dt)  # noqa: E731
    s["k"], s["v"] = normal(G, batch * slots, d), normal(G, batch * slots, d)
    # as the weights that tokens have gathered: skewed, and different everywhere
    s["mass"] = torch.exp(0.5 * torch.randn(P, batch * slots, generator=g, device="cuda"))
    # positions of kept tokens: ascending, with gaps
    s["pos"] = torch.randint(1, 8, (P, batch, slots), generator=g, device="cuda").cumsum(2).int().view(P, batch * slots)
    if case["kind"] == "append":
        s["k_new"], s["v_new"] = normal(G, batch * T, d), normal(G, batch * T, d)
        s["pos_new"] = (1 << 20) + torch.arange(T, device="cuda", dtype=torch.int32).repeat(batch)
        s["mass_new"] = torch.rand(batch * T, generator=g, device="cuda")
    elif case["kind"] == "evict":
        s["scores"] = s["mass"].clone()   # what is ranked: the mass as the last step left it
        s["budgets"] = [case["budget"]] * batch
    else:
        s["q"] = normal(batch * T, H, d)
        # heavy hitters, as a compact cache holds them: a sixteenth of the slots along their KV head's mean query
        mean = s["q"].float().view(batch, T, G, H // G, d).mean(dim=(1, 3))
        along = 4.0 * math.sqrt(d) * mean / mean.norm(dim=2, keepdim=True)
        hit = (torch.rand(batch, slots, generator=g, device="cuda") < 1 / 16).to(dt)
        s["k"].view(G, batch, slots, d).addcmul_(hit[None, :, :, None], along.transpose(0, 1)[:, :, None, :].to(dt))
        masks, depths, paths = _trees(batch, T, r)
        s["tree"] = cuda(masks.view(np.int64).reshape(-1), torch.int64)
        # the drafts lie behind what they follow, by their depth
        at = cuda((np.arange(batch) * slots + before)[:, None] + np.arange(T), torch.int64)
        s["pos"][:, at] = 8 * slots + cuda(depths, torch.int32)
        s["slopes_t"] = torch.exp2(-8.0 * torch.arange(1, H + 1, device="cuda") / H) / 64 if case["slopes"] else None
        s["scale"] = 1.0 / math.sqrt(d)
        s["out"] = torch.empty(batch * T, H, d, dtype=dt, device="cuda")
        s["lse"] = torch.empty(batch * T, H, device="cuda")
        if case["kind"] == "accept":
            s["lse"].copy_(_scores(s, torch.float32)[0].logsumexp(-1).view(G, batch, T, H // G).permute(1, 2, 0, 3).reshape(batch * T, H))
            path = np.zeros((batch, T), np.int32)
            for b, p in enumerate(paths):
                path[b, : len(p)] = p
            s["path"], s["n_accept"] = cuda(path.reshape(-1), torch.int32), cuda([len(p) for p in paths], torch.int32)
    if own:   # the cache's handle and the calls' workspace, which a program makes once
        from paper_2604_06746_amd import binding as B
        s["B"], s["cache"] = B, B.make_cache(s["k"], s["v"], s["cu_slots"], s["lens"], mass=s["mass"], pos=s["pos"])
        s["workspace"] = torch.empty(B.structkv_cache_workspace_bytes(s["cache"], H, batch * new), dtype=torch.uint8, device="cuda")
    return s


def _scores(s, t):
    """Scores of the fresh tokens, [KV head, sequence, token and head, slot], -inf where a token does not see a slot."""
    G, B, T, n, d = s["kv_heads"], s["batch"], s["tokens"], s["slots"], s["head_dim"]
    gs = s["heads"] // G
    q = s["q"].to(t).view(B, T, G, gs, d).permute(2, 0, 1, 3, 4).reshape(G, B, T * gs, d)
    x = torch.matmul(q, s["k"].to(t).view(G, B, n, d).transpose(2, 3)).view(G, B, T, gs, n) * s["scale"]
    if s["softcap"]:
        x = s["softcap"] * torch.tanh(x / s["softcap"])
    slot = torch.arange(n, device="cuda")
    first = s["lens"].long() - T                                                            # the first fresh slot
    if s["slopes_t"] is not None:
        pos = s["pos"].view(-1, B, n).expand(G, B, n)
        at = (first[:, None] + torch.arange(T, device="cuda")).expand(G, B, T)
        far = (pos.gather(2, at)[:, :, :, None] - pos[:, :, None, :]).to(t)                 # [KV head, sequence, token, slot]
        x = x - s["slopes_t"].to(t).view(G, 1, 1, gs, 1) * far[:, :, :, None, :]
    rank = (slot - first[:, None]).clamp(0, 63)[:, None, :]                                  # of a fresh slot among the fresh
    sees = (s["tree"].view(B, T, 1) >> rank & 1).bool() | (slot < first[:, None])[:, None, :]
    sees &= (slot < s["lens"][:, None])[:, None, :]
    return x.masked_fill(~sees[None, :, :, None, :], -math.inf).view(G, B, T * gs, n), first


def _add_to_mass(s, weights):
    """mass <- decay mass + weights [KV head, sequence, slot], in the slots in use."""
    if s["planes"] == 1:
        weights = weights.sum(0, keepdim=True)
    mass = s["mass"].view(-1, s["batch"], s["slots"])
    used = torch.arange(s["slots"], device="cuda") < s["lens"][:, None]
    mass.copy_(torch.where(used, s["decay"] * mass + weights, mass))


def _attend(s):
    if own:
        s["B"].structkv_cache_attend(s["cache"], s["heads"], s["q"], s["cu_new"], s["out"], s["lse"], s["workspace"],
                                     tree_mask=s["tree"], scale=s["scale"], softcap=s["softcap"], slopes=s["slopes_t"], lam=s["decay"])
        return [s["out"], s["lse"], s["mass"]]
    G, B, T, H, d = s["kv_heads"], s["batch"], s["tokens"], s["heads"], s["head_dim"]
    x, _ = _scores(s, torch.float32)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    a = e / total
    back = lambda y, w: y.view(G, B, T, H // G, w).permute(1, 2, 0, 3, 4).reshape(B * T, H, w)  # noqa: E731
    out = torch.matmul(a, s["v"].float().view(G, B, -1, d))
    s["out"].copy_(back(out, d))
    s["lse"].copy_(back(top + torch.log(total), 1)[:, :, 0])
    if s["decay"]:
        _add_to_mass(s, a.sum(2))
    return [s["out"], s["lse"], s["mass"]]


def _append(s):
    if own:
        s["B"].structkv_cache_append(s["cache"], s["k_new"], s["v_new"], s["cu_new"], s["lens_out"], pos_new=s["pos_new"],
                                     mass_new=s["mass_new"])
        return [s["k"], s["v"], s["pos"], s["mass"], s["lens_out"]]
    first = torch.arange(s["batch"], device="cuda") * s["slots"] + s["lens"]
    at = (first[:, None] + torch.arange(s["tokens"], device="cuda")).view(-1)
    s["k"][:, at], s["v"][:, at] = s["k_new"], s["v_new"]
    s["pos"][:, at], s["mass"][:, at] = s["pos_new"], s["mass_new"]
    s["lens_out"].copy_(s["lens"] + s["tokens"])
    return [s["k"], s["v"], s["pos"], s["mass"], s["lens_out"]]


def _accept(s):
    if own:
        s["B"].structkv_cache_accept(s["cache"], s["heads"], s["q"], s["lse"], s["cu_new"], s["lens_out"], path=s["path"],
                                     n_accept=s["n_accept"], tree_mask=s["tree"], scale=s["scale"], softcap=s["softcap"],
                                     slopes=s["slopes_t"], lam=s["decay"])
        return [s["k"], s["v"], s["pos"], s["mass"], s["lens_out"]]
    G, B, T, H = s["kv_heads"], s["batch"], s["tokens"], s["heads"]
    x, first = _scores(s, torch.float32)
    lse = s["lse"].view(B, T, G, H // G).permute(2, 0, 1, 3).reshape(G, B, -1, 1)
    nth, path = torch.arange(T, device="cuda"), s["path"].view(B, T).long()
    taken = nth < s["n_accept"][:, None]                                                    # entries of the paths that count
    counts = torch.zeros(B, T, device="cuda").scatter_add_(1, path, taken.float())          # drafts that were accepted
    a = torch.exp(x - lse).view(G, B, T, H // G, -1) * counts.view(1, B, T, 1, 1)
    _add_to_mass(s, a.sum((2, 3)))
    base = torch.arange(B, device="cuda") * s["slots"] + first
    to, came = (base[:, None] + nth)[taken], (base[:, None] + path)[taken]
    s["k"][:, to], s["v"][:, to] = s["k"][:, came], s["v"][:, came]
    s["pos"][:, to], s["mass"][:, to] = s["pos"][:, came], s["mass"][:, came]
    s["lens_out"].copy_(first + s["n_accept"])
    return [s["k"], s["v"], s["pos"], s["mass"], s["lens_out"]]


def _evict(s):
    if own:
        s["B"].structkv_cache_evict(s["cache"], s["scores"], s["budgets"], s["tail"], s["lens_out"], s["workspace"])
        return [s["k"], s["v"], s["pos"], s["mass"], s["lens_out"]]
    G, P, B, n, budget = s["kv_heads"], s["planes"], s["batch"], s["slots"], s["budget"]
    slot = torch.arange(n, device="cuda")
    used = slot < s["lens"][:, None]
    pos = s["pos"].view(P, B, n).masked_fill(~used, -1)
    recent = pos > pos.amax(-1, keepdim=True) - s["tail"]
    rank = s["scores"].view(P, B, n).masked_fill(recent, math.inf).masked_fill(~used, -math.inf)
    order = rank.sort(dim=-1, descending=True, stable=True)[1]                             # ties: the lower slot first
    kept = torch.zeros(P, B, n, dtype=torch.bool, device="cuda").scatter_(2, order[:, :, :budget], True) & used
    holes, moved = ~kept & used & (slot < budget), kept & (slot >= budget)
    hole, move = holes.view(P, -1), moved.view(P, -1)
    s["mass"][hole], s["pos"][hole] = s["mass"][move], s["pos"][move]
    hole, move = hole.expand(G, -1), move.expand(G, -1)
    s["k"][hole], s["v"][hole] = s["k"][move], s["v"][move]
    s["lens_out"].copy_(s["lens"].clamp(max=budget))
    return [s["k"], s["v"], s["pos"], s["mass"], s["lens_out"]]


RUN = {"attend": _attend, "append": _append, "accept": _accept, "evict": _evict}


def run(s):
    return RUN[s["kind"]](s)


def work(case):
    H, G, d, e = case["heads"], case["kv_heads"], case["head_dim"], 4 if case["dtype"] == "f32" else 2
    B, n, T, P = case["batch"], case["slots"], case["tokens"], case["planes"]
    row = G * d * e                                       # one slot's keys, or values, of all heads
    if case["kind"] == "append":                          # the rows, their positions and masses in and out; lengths
        return {"bytes": B * T * (4 * row + 2 * 4 * (1 + P)) + 8 * B, "flops": 0}
    if case["kind"] == "evict":
        used = max(case["budget"], 0.5 * (1 + case["fill"]) * n)
        moved = case["budget"] * (used - case["budget"]) / used   # kept slots behind the budget, where all are alike
        # scores and positions in; keys, values, masses and positions of the moved slots in and out
        return {"bytes": B * (8 * P * used + moved * (4 * row + 16 * P)) + 8 * B, "flops": 0}
    used = 0.5 * (1 + case["fill"]) * (n - T) + T
    bias = 4 * P * used * B if case["slopes"] else 0
    if case["kind"] == "attend":                          # the cache; queries in and results out; masses in and out
        moved = B * (2 * used * row + T * H * (2 * d * e + 4)) + (8 * P * used * B if case["decay"] else 0) + bias
        return {"bytes": moved, "flops": 4 * B * T * H * d * used}
    rows = min(T, 1 + math.log(T))                        # a path's length in a random tree
    # keys, masses in and out, the accepted tokens' queries; their slots' rows in and out
    moved = B * (used * row + 8 * P * used + rows * (H * (d * e + 4) + 4 * row + 16 * P)) + bias
    return {"bytes": moved, "flops": 2 * B * rows * H * d * used}


def exact(case, seed):
    """The definitions in 64 bits, one sequence and KV head at a time.  Copies and lengths have no such value."""
    if case["kind"] in ("append", "evict"):
        return None
    s = prepare(case, seed)
    H, G, T, n, P = case["heads"], case["kv_heads"], case["tokens"], case["slots"], case["planes"]
    gs = H // G
    out = torch.zeros(case["batch"], T, H, case["head_dim"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["batch"], T, H, dtype=torch.float64, device="cuda")
    mass = s["mass"].double().view(P, case["batch"], n)
    for b in range(case["batch"]):
        used = int(s["lens"][b])
        lo, base = b * n, used - T
        bits = [int(m) & (2**64 - 1) for m in s["tree"][b * T:(b + 1) * T].tolist()]
        sees = torch.ones(T, used, dtype=torch.bool)
        sees[:, base:] = torch.tensor([[bool(m >> j & 1) for j in range(T)] for m in bits])
        sees = sees.cuda()
        weight = torch.zeros(G, used, dtype=torch.float64, device="cuda")
        accepted = s["path"][b * T: b * T + int(s["n_accept"][b])].long() if case["kind"] == "accept" else slice(None)
        for g in range(G):
            k, v = s["k"][g, lo:lo + used].double(), s["v"][g, lo:lo + used].double()
            pos = s["pos"][g if P > 1 else 0, lo:lo + used].double()
            for h in range(g * gs, (g + 1) * gs):
                x = s["q"][b * T:(b + 1) * T, h].double() @ k.T * s["scale"]
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                if case["slopes"]:
                    x -= s["slopes_t"][h].double() * (pos[base:, None] - pos[None, :])
                x[~sees] = -math.inf
                lse[b, :, h] = torch.logsumexp(x, 1)
                if case["kind"] == "attend":
                    out[b, :, h] = torch.softmax(x, 1) @ v
                a = torch.softmax(x, 1) if case["kind"] == "attend" else torch.exp(x - s["lse"][b * T:(b + 1) * T, h, None].double())
                weight[g] += a[accepted].sum(0)
        if case["decay"]:
            mass[:, b, :used] = case["decay"] * mass[:, b, :used] + (weight if P > 1 else weight.sum(0, keepdim=True))
        if case["kind"] == "accept":
            mass[:, b, base:base + len(accepted)] = mass[:, b, base + accepted]
    mass = mass.view(P, -1)
    if case["kind"] == "accept":
        return [None, None, None, mass, None]
    return [out.view(-1, H, case["head_dim"]), lse.view(-1, H), mass]
