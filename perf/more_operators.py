"""Performance cases of a cache held in 8 bits in pages, of the attention over it, and of the rotation by position that its keys carry.

Three operators:
  rotate  rows of queries or keys turned by their positions: halves or neighbours as pairs, all of the head or a part of it, frequencies
          as they are or scaled for long contexts; forwards, or backwards as for gradients
  append  rows of keys and values into the pages of sequences, the keys rotated on the way and the queries beside them; each page and
          KV head has a scale, the least power of two that brings what it holds within the range of an 8-bit float (e4m3: 448)
  attend  fresh tokens, the last ones in the cache, attend to it: single tokens, which may add their weights to the mass kept for each
          page, chains of drafted tokens, or chunks of a prompt.  Pages that were dropped are not in the pool: nobody sees their tokens

Where `own` is false, `run` computes them in plain torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E4M3, TOP = torch.float8_e4m3fn, 448.0


def _case(kind, name=None, *, heads=32, kv_heads=8, head_dim=128, dtype="bf16", batch=1, slots=2080, fill=1.0, tokens=1, page=16,
          softcap=0.0, decay=0.0, dropped=0.0, rot=128, interleaved=False, scaling="none", factor=1.0, inverse=False):
    c = dict(kind=kind, heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, batch=batch, slots=slots, fill=fill, tokens=tokens,
             page=page, softcap=softcap, decay=decay, dropped=dropped, rot=rot, interleaved=interleaved, scaling=scaling, factor=factor,
             inverse=inverse)
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest configuration, full precision, one KV head per query head: a chain of seven drafts
        _case("attend", "attend_f32_1k_chain7", heads=8, kv_heads=8, head_dim=64, dtype="f32", slots=1031, tokens=7),
        # a token after a 32K prefill that kept 2048 tokens and its window of 32; its weights go to the mass of the pages
        _case("attend", "attend_2k_token", slots=2081, decay=0.9),
        # tokens of sixteen sequences with caches of 5 % of up to 128K, a tenth of whose pages were dropped
        _case("attend", "attend_6k_batch16", batch=16, slots=6586, fill=0.15, page=32, decay=0.9, dropped=0.1),
        # chains of eight drafts over caches of the longest configuration's budget, capped scores
        _case("attend", "attend_16k_chain8", batch=4, slots=16512, fill=0.5, tokens=8, page=64, softcap=30.0),
        # tokens over caches that were not compacted, the longest
        _case("attend", "attend_128k_batch8", batch=8, slots=131073, fill=0.5, page=64, decay=0.98),
        # the last chunk of a 32K prompt whose earlier chunks are in the cache
        _case("attend", "attend_32k_chunk512", slots=32768, tokens=512, page=128),
        # a token of each of 64 sequences, queries and keys rotated by halves
        _case("append", "append_token_b64", batch=64, slots=2112, fill=0.9),
        # eight prompts stored, positions scaled four times
        _case("append", "append_prompt_b8", batch=8, slots=8192, fill=0.2, tokens=5715, page=64, scaling="yarn", factor=4.0),
        # the observation window's queries at the end of 128K tokens
        _case("rotate", "rotate_window64", slots=131072, tokens=64),
        # the keys of 128K tokens, bands of frequencies scaled eight times
        _case("rotate", "rotate_k_128k", heads=8, slots=131072, tokens=131072, scaling="bands", factor=8.0),
        # gradients of queries on the way back: part of the head, neighbours as pairs
        _case("rotate", "rotate_grad_f32", head_dim=80, dtype="f32", slots=8191, tokens=8191, rot=20, interleaved=True, inverse=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choices(("attend", "append", "rotate"), (5, 3, 3))[0]
    heads, kv_heads, head_dim = rng.choice(((32, 8, 128), (32, 8, 128), (8, 2, 128), (16, 2, 128), (32, 32, 128), (8, 8, 64), (32, 8, 64),
                                            (32, 4, 80), (16, 8, 256)))
    dtype = "f32" if rng.random() < 0.2 else "bf16"
    rot = rng.choice((head_dim, head_dim, head_dim // 2, 20))
    scaling = rng.choice(("none", "linear", "ntk", "yarn", "bands"))
    like = dict(heads=heads, kv_heads=kv_heads, head_dim=head_dim, dtype=dtype, rot=rot, interleaved=rng.random() < 0.4, scaling=scaling,
                factor=1.0 if scaling == "none" else rng.choice((2.0, 8.0, 32.0)))
    if kind == "rotate":
        most = (1 << 28) // (heads * head_dim * (2 if dtype == "f32" else 1))   # rows that are no more than the largest listed ones
        tokens = _log(rng, 1, min(131072, most))
        return _case(kind, **like, slots=tokens + _log(rng, 1, 1 << 20), tokens=tokens, inverse=rng.random() < 0.4)
    batch = rng.choice((1, 1, 2, 4, 7, 16, 33, 64))
    like.update(batch=batch, page=rng.choice((16, 16, 32, 64, 128, 256)), fill=1.0 if batch == 1 else rng.choice((0.1, 0.5, 0.9)))
    most = max(256, min(131072, (3 << 28) // (kv_heads * head_dim * batch)))      # slots whose codes are no more than the largest listed ones
    if kind == "append":
        tokens = rng.choice((1, 1, 5, _log(rng, 16, max(17, most // 24))))
        return _case(kind, **dict(like, fill=0.3), slots=_log(rng, 2 * tokens + 16, max(most, 2 * tokens + 17)) + tokens, tokens=tokens)
    tokens = rng.choice((1, 1, 1, 2, 5, 13, 32, 64, _log(rng, 65, 1024)))
    most = max(64, min(most, (1 << 36) // (heads * tokens * batch * head_dim)))   # ... and products no more either
    if tokens > 64:
        batch = like["batch"] = min(batch, 2)
    return _case(kind, **like, slots=_log(rng, 64, max(65, most)) + tokens, tokens=tokens, softcap=rng.choice((0.0, 0.0, 30.0)),
                 decay=rng.choice((0.0, 0.5, 0.9, 1.0)) if tokens == 1 else 0.0, dropped=rng.choice((0.0, 0.0, 0.3)))


BASE, ORIGINAL, YARN, BANDS = 500000.0, 8192.0, (32.0, 1.0), (1.0, 4.0)


def _frequencies(case):
    """Radians a position, in 64 bits, and the factor of cosine and sine."""
    rot, factor = case["rot"], case["factor"]
    i = torch.arange(rot // 2, dtype=torch.float64)
    base = BASE * factor ** (rot / (rot - 2)) if case["scaling"] == "ntk" else BASE
    f = base ** (-2.0 * i / rot)
    if case["scaling"] == "linear":
        f = f / factor
    elif case["scaling"] == "yarn":   # pairs that turn often over the original length stay, those that turn less than once are stretched
        at = lambda turns: rot * math.log(ORIGINAL / (turns * 2 * math.pi)) / (2 * math.log(BASE))  # noqa: E731
        lo, hi = max(0, math.floor(at(YARN[0]))), min(rot - 1, math.ceil(at(YARN[1])))
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        f = f * (1 - ramp) + f / factor * ramp
        return f, 0.1 * math.log(factor) + 1.0
    elif case["scaling"] == "bands":
        turns = ORIGINAL * f / (2 * math.pi)
        smooth = ((turns - BANDS[0]) / (BANDS[1] - BANDS[0])).clamp(0, 1)
        f = f * smooth + f / factor * (1 - smooth)
    return f, 1.0


def prepare(case, seed):
    H, G, d, dt = case["heads"], case["kv_heads"], case["head_dim"], DTYPES[case["dtype"]]
    B, T, ps = case["batch"], case["tokens"], case["page"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    normal = lambda *shape, dtype=dt: torch.randn(*shape, generator=g, device="cuda", dtype=dtype)  # noqa: E731
    f, magnitude = _frequencies(case)
    s = dict(case, freq=f.cuda(), magnitude=magnitude)
    if case["kind"] == "rotate":
        s["x"] = normal(T, H, d) if H > 8 else normal(H, T, d).transpose(0, 1)           # queries by token, keys by head
        s["out"] = torch.empty_like(s["x"])
        s["pos"] = torch.arange(case["slots"] - T, case["slots"], device="cuda", dtype=torch.int32)
    else:
        per = -(-case["slots"] // ps)                                                     # pages of a sequence
        n_pages = B * per + 3
        new = 0 if case["kind"] == "attend" else T
        room = case["slots"] - new
        low = min(room, max(T if case["kind"] == "attend" else 0, int(case["fill"] * room)))
        s["lens"] = torch.randint(low, room + 1, (B,), generator=g, device="cuda").int()
        s["pages"] = torch.randperm(n_pages, generator=g, device="cuda")[: B * per].int().view(B, per)
        for name in ("k", "v"):   # normal numbers, a page's and head's in units of a scale of its own
            x = normal(n_pages, G, ps, d, dtype=torch.bfloat16)
            spread = torch.exp2(torch.randint(-1, 2, (n_pages, G), generator=g, device="cuda").float())
            s[name], s[name + "_scale"] = x.mul_(64.0).to(E4M3), spread / 64
        s["cu_new"] = [T * b for b in range(B + 1)]
        s["lens_out"] = torch.empty_like(s["lens"])
        if case["kind"] == "attend":
            s["q"] = normal(B * T, H, d)
            gone = torch.rand(B, per, generator=g, device="cuda") < case["dropped"]
            fresh = (s["lens"].long() - T)[:, None] // ps <= torch.arange(per, device="cuda")  # (those of the fresh tokens stay)
            s["pages"].masked_fill_(gone & ~fresh, -1)
            # heavy hitters along their KV head's mean query, as a compact cache holds them: one slot in sixteen
            mean = s["q"].float().view(B, T, G, H // G, d).mean(dim=(1, 3))
            along = (4.0 * math.sqrt(d) * mean / mean.norm(dim=2, keepdim=True)).to(torch.bfloat16)
            for b in range(B):
                own_pages = s["pages"][b][s["pages"][b] >= 0].long()
                hit = s["k"][own_pages, :, :: 16].float()
                up = along[b][None, :, None, :].float() / s["k_scale"][own_pages][:, :, None, None]
                s["k"][own_pages, :, :: 16] = (hit + up).clamp(-TOP, TOP).to(E4M3)
            s["mass"] = torch.exp(0.5 * torch.randn(B, per, generator=g, device="cuda"))
            s["scale"] = 1.0 / math.sqrt(d)
            s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(B * T, H, device="cuda")
        else:
            qkv = normal(B * T, H + 2 * G, d)                                             # as one projection gives them
            s["q"], s["q_out"] = qkv[:, :H], torch.empty(B * T, H, d, device="cuda", dtype=dt)
            s["k_new"], s["v_new"] = qkv[:, H:H + G].transpose(0, 1), qkv[:, H + G:].transpose(0, 1)
    if own:   # the rotation's plan, the cache's handle and the calls' workspace, which a program makes once
        from paper_2604_06746_amd import binding as lib
        s["lib"] = lib
        low_high = YARN if case["scaling"] == "yarn" else BANDS
        turns, magnitude = lib.structkv_rotary_turns(case["rot"], BASE, case["scaling"], case["factor"], ORIGINAL, *low_high)
        s["rotary"] = lib.make_rotary(turns.cuda(), interleaved=case["interleaved"], magnitude=magnitude)
        if case["kind"] != "rotate":
            s["cache"] = lib.make_paged(s["k"], s["v"], s["k_scale"], s["v_scale"], s["pages"], s["lens"], dt, mass=s.get("mass"))
            size = lib.structkv_paged_workspace_bytes(s["cache"], H, B * T)
            s["workspace"] = torch.empty(size, dtype=torch.uint8, device="cuda")
    return s


def _rotated(s, x, pos):
    """Rows x [tokens, heads, d] in 32 bits, turned by their positions [tokens]."""
    rot = s["rot"]
    angle = pos.double()[:, None] * s["freq"]
    sign = -1.0 if s["inverse"] else 1.0
    cos = (s["magnitude"] * torch.cos(angle)).float()[:, None]
    sin = (sign * s["magnitude"] * torch.sin(angle)).float()[:, None]
    x = x.float()
    y = x.clone()
    first = slice(0, rot, 2) if s["interleaved"] else slice(0, rot // 2)
    second = slice(1, rot, 2) if s["interleaved"] else slice(rot // 2, rot)
    a, b = x[..., first], x[..., second]
    y[..., first], y[..., second] = a * cos - b * sin, b * cos + a * sin
    return y


def _rotate(s):
    if own:
        s["lib"].structkv_rotate(s["rotary"], s["x"], s["pos"], s["out"], inverse=s["inverse"])
    else:
        s["out"].copy_(_rotated(s, s["x"], s["pos"]))
    return [s["out"]]


def _scales(top):
    """The least powers of two s with top <= 448 s, of 2^-64 at least."""
    m, e = torch.frexp(top)
    return torch.exp2((e - 9 + (m > 0.875)).clamp(min=-64).float())


def _append(s):
    if own:
        s["lib"].structkv_paged_append(s["cache"], s["k_new"], s["v_new"], s["cu_new"], s["lens_out"], rotary=s["rotary"], q=s["q"],
                                       q_out=s["q_out"])
        return [s["k"], s["v"], s["k_scale"], s["v_scale"], s["q_out"], s["lens_out"]]
    G, B, T, ps, d = s["kv_heads"], s["batch"], s["tokens"], s["page"], s["head_dim"]
    lens = s["lens"].long()
    pos = (lens[:, None] + torch.arange(T, device="cuda")).view(-1)
    s["q_out"].copy_(_rotated(s, s["q"], pos))
    first, touched = lens // ps, (T + ps - 2) // ps + 1
    nth = first[:, None] + torch.arange(touched, device="cuda")
    there = nth <= ((lens + T - 1) // ps)[:, None]                                # the last page may be one sooner
    pages = s["pages"].gather(1, nth.clamp(max=s["pages"].shape[1] - 1)).long()
    slot = nth[:, :, None] * ps + torch.arange(ps, device="cuda")                 # [sequence, page, row]
    old, fresh = slot < lens[:, None, None], (slot >= lens[:, None, None]) & (slot < (lens + T)[:, None, None])
    row = (slot - lens[:, None, None]).clamp(0, T - 1) + T * torch.arange(B, device="cuda")[:, None, None]
    for name, x in (("k", _rotated(s, s["k_new"].transpose(0, 1), pos)), ("v", s["v_new"].transpose(0, 1).float())):
        pool, scale = s[name], s[name + "_scale"]
        new = x[row].permute(0, 1, 3, 2, 4)                                       # [sequence, page, KV head, row, component]
        keep, was, come = pool[pages], old[:, :, None, :, None], fresh[:, :, None, :, None]
        before = scale[pages]
        top = _scales((new * come).abs().amax((3, 4)))
        now = torch.where(old.any(2)[:, :, None], torch.maximum(top, before), top)
        value = torch.where(was, keep.float() * before[..., None, None], new * come)
        codes = torch.where(was | come, value / now[..., None, None], keep.float()).to(E4M3)
        pool[pages[there]], scale[pages[there]] = codes[there], now[there]
    s["lens_out"].copy_(lens + T)
    return [s["k"], s["v"], s["k_scale"], s["v_scale"], s["q_out"], s["lens_out"]]


def _attend(s):
    if own:
        s["lib"].structkv_paged_attend(s["cache"], s["heads"], s["q"], s["cu_new"], s["out"], s["lse"], s["workspace"], scale=s["scale"],
                                       softcap=s["softcap"], lam=s["decay"])
        return [s["out"], s["lse"], s["mass"]]
    G, B, T, H, d, ps = s["kv_heads"], s["batch"], s["tokens"], s["heads"], s["head_dim"], s["page"]
    per = s["pages"].shape[1]
    n, pages, live = per * ps, s["pages"].clamp(min=0).long(), s["pages"] >= 0
    values = lambda x: (s[x][pages].float() * s[x + "_scale"][pages][..., None, None]).transpose(1, 2).reshape(B, G, n, d)  # noqa: E731
    q = s["q"].float().view(B, T, G, H // G, d).permute(0, 2, 1, 3, 4).reshape(B, G, T * (H // G), d)
    x = torch.matmul(q, values("k").transpose(2, 3)) * s["scale"]
    if s["softcap"]:
        x = s["softcap"] * torch.tanh(x / s["softcap"])
    slot = torch.arange(n, device="cuda")
    last = (s["lens"].long() - T)[:, None] + torch.arange(T, device="cuda")           # the last slot that a token sees
    sees = (slot <= last[:, :, None]) & live.repeat_interleave(ps, 1)[:, None, :]
    x = x.view(B, G, T, H // G, n).masked_fill_(~sees[:, None, :, None, :], -math.inf).view(B, G, -1, n)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - top)
    total = e.sum(-1, keepdim=True)
    back = lambda y, w: y.view(B, G, T, H // G, w).transpose(1, 2).reshape(B * T, H, w)  # noqa: E731
    s["out"].copy_(back(torch.matmul(e, values("v").masked_fill_(~sees.any(1)[:, None, :, None], 0.0)) / total, d))
    s["lse"].copy_(back(top + torch.log(total), 1)[:, :, 0])
    if s["decay"]:
        used = torch.arange(per, device="cuda") * ps < s["lens"][:, None]
        s["mass"].copy_(torch.where(used, s["decay"] * s["mass"] + (e / total).sum((1, 2)).view(B, per, ps).sum(2), s["mass"]))
    return [s["out"], s["lse"], s["mass"]]


RUN = {"rotate": _rotate, "append": _append, "attend": _attend}


def run(s):
    return RUN[s["kind"]](s)


def work(case):
    H, G, d, e = case["heads"], case["kv_heads"], case["head_dim"], 4 if case["dtype"] == "f32" else 2
    B, T, ps = case["batch"], case["tokens"], case["page"]
    if case["kind"] == "rotate":      # rows in and out, their positions; two products and a sum for each component
        return {"bytes": T * (2 * H * d * e + 4), "flops": 3 * T * H * case["rot"]}
    if case["kind"] == "append":      # rows in, codes out; queries in and out; scales, table, lengths
        touched = 1 + (T - 1) / ps
        return {"bytes": B * (T * (2 * G * d * (e + 1) + 2 * H * d * e) + touched * (4 + 8 * G) + 8),
                "flops": 3 * B * T * (H + G) * case["rot"]}
    used = 0.5 * (max(T, case["fill"] * case["slots"]) + case["slots"]) * (1 - case["dropped"])
    # the codes; queries in and results out; scales, table and masses of the pages
    moved = B * (2 * used * G * d + T * H * (2 * d * e + 4) + used / ps * (4 + 8 * G + (8 if case["decay"] else 0)))
    return {"bytes": moved, "flops": 4 * B * T * H * d * (used - 0.5 * (T - 1))}


def _e4m3(v):
    """The 8-bit float next to each value, ties to the even one, as 64-bit numbers; of magnitudes up to 448."""
    exponent = torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6)))
    step = torch.exp2(exponent - 3)
    return torch.round(v / step) * step


def exact(case, seed):
    """The definitions in 64 bits; one sequence, head or page at a time."""
    s = prepare(case, seed)
    H, G, d, T, ps, rot = case["heads"], case["kv_heads"], case["head_dim"], case["tokens"], case["page"], case["rot"]
    f, magnitude = _frequencies(case)

    def turned(x, pos):
        """x [tokens, d] as complex numbers, multiplied by m e^{i pos f}."""
        spin = torch.polar(torch.full((x.shape[0], rot // 2), magnitude, dtype=torch.float64, device="cuda"),
                           pos.double().outer(f.cuda()) * (-1 if case["inverse"] else 1))
        x, part = x.double().clone(), x[:, :rot].double()
        pairs = part.reshape(-1, rot // 2, 2) if case["interleaved"] else part.reshape(-1, 2, rot // 2).transpose(1, 2)
        y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * spin)
        x[:, :rot] = (y if case["interleaved"] else y.transpose(1, 2)).reshape(-1, rot)
        return x

    if case["kind"] == "rotate":
        return [torch.stack([turned(s["x"][:, h], s["pos"]) for h in range(H)], dim=1)]
    lens = s["lens"].tolist()
    if case["kind"] == "append":
        pos = torch.cat([torch.arange(n, n + T, device="cuda") for n in lens])
        q = torch.stack([turned(s["q"][:, h], pos) for h in range(H)], dim=1)
        k = torch.stack([turned(s["k_new"][g], pos) for g in range(G)])
        pools = []
        for name, x in (("k", k), ("v", s["v_new"].double())):
            codes, scale = s[name].double(), s[name + "_scale"].double()
            for b, n in enumerate(lens):
                for j in range(n // ps, (n + T - 1) // ps + 1):
                    p, a, z = int(s["pages"][b, j]), max(0, n - j * ps), min(ps, n + T - j * ps)   # rows a .. z - 1 are new
                    new = x[:, b * T + j * ps + a - n: b * T + j * ps + z - n]
                    least = torch.exp2(torch.ceil(torch.log2(new.abs().amax((1, 2)) / TOP)).clamp(min=-64))
                    now = torch.maximum(least, scale[p]) if a else least
                    codes[p, :, :a] = _e4m3(codes[p, :, :a] * (scale[p] / now)[:, None, None])
                    codes[p, :, a:z] = _e4m3(new / now[:, None, None])
                    scale[p] = now
            pools.append((codes, scale))
        return [pools[0][0], pools[1][0], pools[0][1], pools[1][1], q, None]
    out = torch.zeros(case["batch"], T, H, d, dtype=torch.float64, device="cuda")
    lse = torch.zeros(case["batch"], T, H, dtype=torch.float64, device="cuda")
    mass = s["mass"].double()
    for b, n in enumerate(lens):
        entries = [j for j in range(-(-n // ps)) if int(s["pages"][b, j]) >= 0]
        pages = s["pages"][b, entries].long()
        slot = torch.cat([torch.arange(j * ps, (j + 1) * ps) for j in entries]).cuda()
        unseen = slot[None, :] > torch.arange(n - T, n, device="cuda")[:, None]
        weight = torch.zeros(len(entries), dtype=torch.float64, device="cuda")
        for g in range(G):
            k = (s["k"][pages, g].double() * s["k_scale"][pages, g, None, None]).reshape(-1, d)
            v = (s["v"][pages, g].double() * s["v_scale"][pages, g, None, None]).reshape(-1, d)
            v[slot >= n] = 0.0
            for h in range(g * (H // G), (g + 1) * (H // G)):
                x = s["q"][b * T:(b + 1) * T, h].double() @ k.T * s["scale"]
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                x[unseen] = -math.inf
                lse[b, :, h] = torch.logsumexp(x, 1)
                a = torch.softmax(x, 1)
                out[b, :, h] = a @ v
                weight += a.sum(0).view(-1, ps).sum(1)
        if case["decay"]:
            mass[b, :-(-n // ps)] *= case["decay"]
            mass[b, entries] += weight
    return [out.view(-1, H, d), lse.view(-1, H), mass]
