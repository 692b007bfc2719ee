"""The operators around a paged KV cache's attention whose speed is followed: the
rotation of queries and keys by their positions (one axis, or several for images and
video), the append of rotated keys and of values to the pages, and the attention of
one new token of sequences that share a long prefix, whose rows are read once for all.

Cases have 1 to 32 layers, 1 to 256 sequences, 2 to 8 KV heads with groups of 2 to 8
query heads, head_dim 64 and 128 of which a quarter to all is rotated, in halves or in
neighbouring pairs, bf16 and fp32, pages of 16 to 256 rows, runs of 1 to 16,384 tokens
at positions up to 1,000,000, 1 to 8 prefixes of 64 to 16,384 rows with 1 to 2,048 rows
of a sequence's own behind them, windows of 64 to 16,384 rows with up to 64 sinks.

`run` computes a case in plain torch operations, or, where `own` is set, by the
framework's entry points.
"""
import math

import numpy as np
import torch

own = False


def _rope(name, layers, batch, heads, dim, dtype, lo, hi, pos0, rot, axes=1, pairs=False):
    return {"name": name, "kind": "rope", "layers": layers, "batch": batch, "hq": heads, "dim": dim, "dtype": dtype,
            "new_lo": lo, "new_hi": hi, "pos0": pos0, "rot": rot, "axes": axes, "pairs": pairs}


def _append(name, layers, batch, hq, hkv, dim, dtype, page, lo, hi, new_lo, new_hi, pos0, rot, axes=1, pairs=False):
    return {"name": name, "kind": "append", "layers": layers, "batch": batch, "hq": hq, "hkv": hkv, "dim": dim,
            "dtype": dtype, "page": page, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "pos0": pos0,
            "rot": rot, "axes": axes, "pairs": pairs}


def _shared(name, layers, batch, groups, hq, hkv, dim, dtype, page, lo, hi, own_lo, own_hi, append, sinks=0, window=0):
    return {"name": name, "kind": "shared", "layers": layers, "batch": batch, "groups": groups, "hq": hq, "hkv": hkv,
            "dim": dim, "dtype": dtype, "page": page, "lo": lo, "hi": hi, "own_lo": own_lo, "own_hi": own_hi,
            "append": append, "sinks": sinks, "window": window}


def listed():
    return [
        # The smallest call: one token of one layer of the small fp32 model, queries and keys together.
        _rope("rope_token_f32_small", 1, 1, 10, 64, "f32", 1, 1, 2048, 64),
        # A padded batch of prompts of one layer (8B shape), half of each row rotated in neighbouring pairs.
        _rope("rope_prompts_8b", 1, 8, 40, 128, "bf16", 200, 512, 0, 64, pairs=True),
        # One layer of a 16K prompt of image patches: time, height and width (7B shape).
        _rope("rope_grid_7b_16k", 1, 1, 32, 128, "bf16", 16381, 16381, 5, 128, axes=3),
        # One token of one layer of the small fp32 model into its cache.
        _append("append_token_f32_small", 1, 1, 8, 2, 64, "f32", 16, 2047, 2047, 1, 1, 2047, 64),
        # One layer of a serving batch's step: 32 ragged sequences (7B shape).
        _append("append_step_batch32_7b", 1, 32, 28, 4, 128, "bf16", 16, 4096, 32767, 1, 1, 40000, 128),
        # A drafted run of 5 tokens checked at once, all layers in one call (8B shape).
        _append("append_run_8b", 32, 4, 32, 8, 128, "bf16", 32, 1000, 4225, 5, 5, 300000, 128),
        # One layer of a 16K prompt into an empty cache (7B shape).
        _append("append_prompt_7b_16k", 1, 1, 28, 4, 128, "bf16", 64, 0, 0, 16384, 16384, 0, 128),
        # Four samples of one prompt, the small fp32 model.
        _shared("shared_f32_small", 1, 4, 1, 8, 2, 64, "f32", 16, 2048, 2048, 30, 300, True),
        # One layer of eight samples of one prompt (8B shape).
        _shared("shared_layer_8b", 1, 8, 1, 32, 8, 128, "bf16", 32, 8190, 8190, 200, 1500, True),
        # 32 samples of a 16K prompt, eight layers in one call (7B shape).
        _shared("shared_samples32_7b", 8, 32, 1, 28, 4, 128, "bf16", 64, 16384, 16384, 256, 2048, True),
        # Four prompts with 1 to some samples each, seen through a window with sinks (32B shape).
        _shared("shared_window_32b", 4, 16, 4, 40, 8, 128, "bf16", 16, 2049, 8000, 100, 1000, True, sinks=4, window=4096),
        # Many short answers to one question: as many query rows as a short prompt has (8B shape).
        _shared("shared_wide_8b", 1, 128, 1, 32, 8, 128, "bf16", 32, 4096, 4096, 1, 400, True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "shared", "shared"])
    hkv, group = rng.choice([(2, 4), (4, 7), (8, 4), (8, 5), (4, 8), (8, 2)])
    hq = hkv * group
    dim = 128 if rng.random() < 0.75 else 64
    dtype = "bf16" if rng.random() < 0.8 else "f32"
    page = rng.choice([16, 16, 32, 64, 128, 256])
    if kind == "shared":
        while True:
            layers, batch = _log_int(rng, 1, 8), _log_int(rng, 2, 256)
            groups = 1 if rng.random() < 0.5 else rng.randint(1, min(8, batch))
            hi, own_hi = _log_int(rng, 64, 16384), _log_int(rng, 1, 2048)
            pairs = float(layers) * batch * hq * (hi + own_hi)
            # what the plain form gathers, and what it multiplies at fp32's rate
            if float(layers) * batch * hkv * (hi + own_hi) * dim <= 2.4e9 and pairs <= 1.3e8:
                break
        lo = hi if rng.random() < 0.5 else max(1, int(hi * rng.uniform(0.1, 0.9)))
        own_lo = own_hi if rng.random() < 0.3 else max(1, int(own_hi * rng.uniform(0.1, 0.9)))
        sinks, window = (rng.choice([0, 1, 4, 16, 64]), _log_int(rng, 64, 16384)) if rng.random() < 0.3 else (0, 0)
        c = _shared("", layers, batch, groups, hq, hkv, dim, dtype, page, lo, hi, own_lo, own_hi, rng.random() < 0.75,
                    sinks, window)
    else:
        rot = dim if rng.random() < 0.6 else rng.choice([dim // 4, dim // 2, 3 * dim // 4])
        axes = rng.choice([1, 1, 2, 3])
        pos0 = rng.choice([0, _log_int(rng, 1, 1000000)])
        while True:
            layers, batch, new_hi = _log_int(rng, 1, 32), _log_int(rng, 1, 64), _log_int(rng, 1, 16384)
            if layers * batch * new_hi * (hq + 2 * hkv) * dim <= 7.5e7:
                break
        new_lo = new_hi if rng.random() < 0.5 else max(1, int(new_hi * rng.uniform(0.1, 0.9)))
        if kind == "rope":
            c = _rope("", layers, batch, hq + hkv, dim, dtype, new_lo, new_hi, pos0, rot, axes, rng.random() < 0.3)
        else:
            while True:
                hi = 0 if rng.random() < 0.3 else _log_int(rng, 1, 32768)
                if float(layers) * batch * hkv * (hi + new_hi) * dim <= 4.0e8:
                    break
            lo = hi if rng.random() < 0.5 else int(hi * rng.uniform(0.1, 0.9))
            c = _append("", layers, batch, hq, hkv, dim, dtype, page, lo, hi, new_lo, new_hi, pos0, rot, axes,
                        rng.random() < 0.3)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _spread(lo, hi, n, seed):
    """n whole numbers spread evenly over [lo, hi], in a mixed order."""
    return np.random.RandomState(seed).permutation(np.round(np.linspace(lo, hi, n)).astype(np.int64))


def _firsts(case):
    """The first sequence of every group, and the batch behind them."""
    cuts = np.random.RandomState(7).choice(case["batch"] - 1, case["groups"] - 1, replace=False) + 1
    return np.concatenate([[0], np.sort(cuts), [case["batch"]]]).astype(np.int64)


def _prefixes(case):
    """Shared rows of every group, and the group of every sequence."""
    first = _firsts(case)
    return _spread(case["lo"], case["hi"], case["groups"], 8), np.repeat(np.arange(case["groups"]), np.diff(first))


def _lens(case):
    if case["kind"] == "shared":
        rows, of = _prefixes(case)
        return rows[of] + _spread(case["own_lo"], case["own_hi"], case["batch"], 5)
    return _spread(case["lo"], case["hi"], case["batch"], 5)


def _news(case):
    """New tokens of every sequence."""
    if case["kind"] == "shared":
        return np.full(case["batch"], int(case["append"]), dtype=np.int64)
    return _spread(case["new_lo"], case["new_hi"], case["batch"], 6)


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def _pair_axes(case):
    """The axis of every pair: runs of a quarter for the first axis, the others in equal parts behind it."""
    n = case["rot"] // 2
    if case["axes"] == 1:
        return [0] * n
    head = n // 4
    return [0] * head + [1 + i * (case["axes"] - 1) // (n - head) for i in range(n - head)]


def _pages(s, g, lens, news, lead, rows):
    """Pages of the cache in a random order (page 0 belongs to no unit and stands behind every unit's last page
    in the table) and the table.  lead [batch]: the sequence whose pages hold the first rows [batch] of each."""
    case, dev, dt = s["case"], _device(), _type(s["case"])
    NL, Bs, H, D, page = case["layers"], case["batch"], case["hkv"], case["dim"], case["page"]
    need = np.maximum(1, -(-(lens + news) // page))
    most = int(need.max())
    at = np.arange(most)
    skip = np.where(lead == np.arange(Bs), 0, rows // page)       # whole pages that are another sequence's
    has = torch.from_numpy((at >= skip[:, None]) & (at < need[:, None])).to(dev)
    has = has[None, :, None].expand(NL, Bs, H, most)
    used = int(has.sum())
    table = torch.zeros((NL, Bs, H, most), dtype=torch.int64, device=dev)
    table[has] = torch.randperm(used, generator=g, device=dev) + 1
    theirs = torch.from_numpy(at < skip[:, None]).to(dev)[None, :, None]
    table = torch.where(theirs, table[:, torch.from_numpy(lead).to(dev)], table)
    hit = (torch.rand((used + 1, page, 1), generator=g, device=dev) < 0.02).float()
    u = torch.randn((used + 1, 1, D), generator=g, device=dev)
    u = 4.0 * u / torch.linalg.vector_norm(u, dim=-1, keepdim=True)
    for name in "kv":                                     # ~ N(0, 1), with 2% heavy rows
        x = torch.randn((used + 1, page, D), generator=g, device=dev)
        x += hit * u
        s[name] = x.to(dt)
        del x
    s["pages"] = table.to(torch.int32)
    s["full"] = torch.from_numpy(lens.astype(np.int32)).to(dev)[None, :, None].expand(NL, Bs, H).contiguous()
    s["length"] = s["full"].clone()


def prepare(case, seed):
    dev, dt = _device(), _type(case)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    NL, Bs, Hq, D = case["layers"], case["batch"], case["hq"], case["dim"]
    s = {"case": case}
    if case["kind"] == "shared":
        H = case["hkv"]
        rows, of = _prefixes(case)
        first = _firsts(case)
        _pages(s, g, _lens(case), _news(case), first[of], rows[of])
        s["first"] = torch.from_numpy(first.astype(np.int32)).to(dev)
        s["rows"] = torch.from_numpy(rows.astype(np.int32)).to(dev)
        s["q"] = torch.randn((NL, Bs, Hq, D), generator=g, device=dev).to(dt)
        s["kn"] = s["vn"] = None
        if case["append"]:
            s["kn"], s["vn"] = (torch.randn((NL, Bs, H, D), generator=g, device=dev).to(dt) for _ in "kv")
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((NL, Bs, Hq), device=dev)
    else:
        news = _news(case)
        T = int(news.max())
        H = case.get("hkv", 0)
        # what a projection leaves: the heads of a token beside each other
        x = torch.randn((NL, Bs, T, Hq + 2 * H, D), generator=g, device=dev).to(dt).transpose(2, 3)
        s["q"], s["kn"], s["vn"] = x[:, :, :Hq], x[:, :, Hq:Hq + H], x[:, :, Hq + H:]
        s["out"] = torch.zeros((NL, Bs, Hq, T, D), dtype=dt, device=dev)
        s["new"] = torch.from_numpy(news.astype(np.int32)).to(dev)
        # one axis counts tokens; of several the last two walk over rows of 32 patches and the first over images
        i = torch.arange(T, device=dev)
        by = {1: [i], 2: [i // 32, i % 32], 3: [i // 1024, i // 32 % 32, i % 32]}[case["axes"]]
        start = case["pos0"] + torch.randint(0, 8, (Bs, 1), generator=g, device=dev)
        s["pos"] = torch.stack([start + x for x in by]).to(torch.int32).contiguous()
        n = case["rot"] // 2
        s["freq"] = torch.from_numpy((1e6 ** (-np.arange(n) / n)).astype(np.float32)).to(dev)
        s["axis"] = torch.tensor(_pair_axes(case), device=dev)
        if case["kind"] == "append":
            _pages(s, g, _lens(case), news, np.arange(Bs), np.zeros(Bs, dtype=np.int64))
    if own:
        _handle(s)
    return s


def _handle(s):
    """What a program that calls the framework keeps beside its tensors: handles and a workspace."""
    from paper_2608_04771_amd import binding as B
    case = s["case"]
    s["err"] = torch.zeros(1, dtype=torch.int32, device=s["q"].device)
    if case["kind"] != "rope":
        cache = B.PagedKVCache(s["k"], s["v"], s["pages"], s["length"])
    if case["kind"] == "shared":
        s["call"] = B.PreparedPagedSharedDecode(cache, case["hq"], s["first"], s["rows"], s["out"], s["lse"],
                                                B.paged_shared_decode_workspace(cache, case["hq"], case["groups"]),
                                                s["err"], sinks=case["sinks"], window=case["window"])
        return
    rope = B.Rope(s["freq"], _pair_axes(case) if case["axes"] > 1 else None, interleaved=case["pairs"])
    if case["kind"] == "rope":
        s["call"] = B.PreparedRope(rope, s["pos"], s["out"], n_new=s["new"], dev_err=s["err"])
    else:
        s["call"] = B.PreparedPagedAppend(cache, s["out"].shape[3], rope, s["pos"], s["out"], n_new=s["new"],
                                          dev_err=s["err"])


# ------------------------------------------------------------------ the calls
def run(s):
    case = s["case"]
    if case["kind"] == "rope":
        if own:
            s["call"](s["q"])
        else:
            _plain_rope(s)
        return {"out": s["out"]}
    if s["kn"] is not None:
        s["length"].copy_(s["full"])                      # every pass sees the same cache
    if case["kind"] == "append":
        if own:
            s["call"](s["kn"], s["vn"], s["q"])
        else:
            _plain_append(s)
        return {"out": s["out"], "k": s["k"], "v": s["v"], "length": s["length"]}
    if own:
        s["call"](s["q"], s["kn"], s["vn"])
    else:
        _plain_shared(s)
    return {"out": s["out"], "lse": s["lse"], "k": s["k"], "v": s["v"], "length": s["length"]}


def _turned(s, x):
    """x [NL][B][heads][T][D] rotated, in 32 bits; the angles in 64."""
    case, R = s["case"], s["case"]["rot"]
    a = s["pos"][s["axis"]].permute(1, 2, 0).double() * s["freq"].double()      # [B][T][R / 2]
    c, n = a.cos().float()[:, None], a.sin().float()[:, None]
    x = x.float()
    lo, hi = (x[..., 0:R:2], x[..., 1:R:2]) if case["pairs"] else (x[..., :R // 2], x[..., R // 2:R])
    y = (lo * c - hi * n, lo * n + hi * c)
    y = torch.stack(y, -1).flatten(-2) if case["pairs"] else torch.cat(y, -1)
    return torch.cat([y, x[..., R:]], -1)


def _real(s):
    """Which places hold tokens: [B][1][T][1]."""
    return (torch.arange(s["out"].shape[3], device=s["out"].device) < s["new"][:, None])[:, None, :, None]


def _plain_rope(s):
    s["out"].copy_(torch.where(_real(s), _turned(s, s["q"]).to(s["out"].dtype), s["out"]))


def _flat_rows(s, table, rows):
    """Pool rows of rows [U][n] of the units whose pages the table [U][most] lists."""
    page = s["case"]["page"]
    rows = rows.clamp(max=table.shape[1] * page - 1)
    return torch.gather(table, 1, rows // page) * page + rows % page


def _store(s, kn, vn, real):
    """Rows kn, vn [U][T][D] to the rows behind each unit's own; where not real, page 0's own row to itself."""
    U, T, D = kn.shape
    n0 = s["length"].reshape(U, 1).long()
    to = _flat_rows(s, s["pages"].reshape(U, -1).long(), n0 + torch.arange(T, device=n0.device))
    to = torch.where(real, to, 0).reshape(-1)
    for pool, rows in ((s["k"].view(-1, D), kn), (s["v"].view(-1, D), vn)):
        pool[to] = torch.where(real.reshape(-1, 1), rows.reshape(-1, D), pool[0])


def _plain_append(s):
    _plain_rope(s)
    NL, Bs, H, T, D = s["kn"].shape
    real = _real(s)[None, ..., 0].expand(NL, Bs, H, T).reshape(NL * Bs * H, T)
    kn = _turned(s, s["kn"]).to(s["k"].dtype)
    _store(s, kn.reshape(-1, T, D), s["vn"].reshape(-1, T, D), real)
    s["length"].add_(s["new"][None, :, None])


def _plain_shared(s):
    """Append the new rows, then every sequence attends over its prefix's rows and its own."""
    case = s["case"]
    NL, Bs, Hq, D = s["q"].shape
    H, G, U = case["hkv"], Hq // case["hkv"], NL * Bs * case["hkv"]
    dev = s["q"].device
    if s["kn"] is not None:
        _store(s, s["kn"].reshape(U, 1, D), s["vn"].reshape(U, 1, D), torch.ones((U, 1), dtype=torch.bool, device=dev))
        s["length"].add_(1)
    table = s["pages"].long()
    at = torch.arange(Bs, device=dev)
    group = torch.searchsorted(s["first"][1:].long(), at, right=True)
    lead = s["first"].long()[group]
    cap = table.shape[3] * case["page"]
    j = torch.arange(cap, device=dev)
    rows = j.expand(U, cap)
    ids = torch.where((j < s["rows"].long()[group][:, None])[None, :, None],
                      _flat_rows(s, table[:, lead].reshape(U, -1), rows).view(NL, Bs, H, cap),
                      _flat_rows(s, table.reshape(U, -1), rows).view(NL, Bs, H, cap)).view(U, cap)
    n = s["length"].reshape(U, 1).long()
    vis = j < n
    if case["window"]:
        vis &= (j < case["sinks"]) | (j >= n - case["window"])
    k = s["k"].view(-1, D)[ids].float().transpose(1, 2)
    x = torch.matmul(s["q"].float().reshape(U, G, D), k.contiguous()).mul_(1.0 / math.sqrt(D))
    del k
    x.masked_fill_(~vis[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x, s["v"].view(-1, D)[ids].float()) / z
    s["out"].copy_(o.reshape(NL, Bs, Hq, D))
    s["lse"].copy_((top + z.log()).reshape(NL, Bs, Hq))


# ------------------------------------------------------------------ floors
def work(case):
    e, d, NL = _elem(case), case["dim"], case["layers"]
    news = _news(case)
    if case["kind"] != "shared":
        H = case.get("hkv", 0)
        tokens = int(news.sum())
        rows = NL * tokens * (case["hq"] + 2 * H)
        return {"bytes": rows * 2 * d * e + tokens * 4 * case["axes"] + case["rot"] * 2 + NL * case["batch"] * H * 8,
                "flops": 3.0 * case["rot"] * NL * tokens * (case["hq"] + H)}
    prefix, of = _prefixes(case)
    n = _lens(case) + news                                # rows with the token's own
    lo = np.maximum(0, n - case["window"]) if case["window"] else np.zeros_like(n)
    sinks = np.minimum(lo, case["sinks"])
    pairs = int((n - lo + sinks).sum())
    rows = 0                                              # different rows: a prefix's count once
    for i, p in enumerate(prefix):
        m, a, b = n[of == i], lo[of == i], sinks[of == i]
        start = min(int(a.min()), int(p))
        rows += int(p) - start + min(start, case["sinks"])
        rows += int((m - np.maximum(a, p)).sum() + np.maximum(0, b - p).sum())
    G = case["hq"] // case["hkv"]
    byt = (rows + int(news.sum())) * 2 * d * e + case["batch"] * G * (2 * d * e + 4)
    return {"bytes": NL * case["hkv"] * byt, "flops": 4.0 * d * G * NL * case["hkv"] * pairs}


# ------------------------------------------------------------------ 64 bits
def _exact_turn(s, x):
    """Each pair as a complex number times e^(i angle), in 64 bits."""
    case, R = s["case"], s["case"]["rot"]
    x = x.double()
    of = torch.arange(R // 2, device=x.device)
    ends = (2 * of, 2 * of + 1) if case["pairs"] else (of, of + R // 2)
    y = x.clone()
    for i in range(R // 2):
        axis = _pair_axes(case)[i]
        angle = s["pos"][axis].double() * s["freq"][i].double()                 # [B][T]
        z = torch.complex(x[..., ends[0][i]], x[..., ends[1][i]]) * torch.polar(torch.ones_like(angle), angle)[:, None]
        y[..., ends[0][i]], y[..., ends[1][i]] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    NL, Bs = case["layers"], case["batch"]
    news = _news(case)
    if case["kind"] != "shared":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["q"].device)
        turned = _exact_turn(s, s["q"])
        for b in range(Bs):
            out[:, b, :, :news[b]] = turned[:, b, :, :news[b]]
        if case["kind"] == "rope":
            return {"out": out}
        del turned
        k, kn, page = s["k"].double(), _exact_turn(s, s["kn"]), case["page"]
        lens = _lens(case)
        for b in range(Bs):
            row = torch.arange(int(lens[b]), int(lens[b] + news[b]), device=k.device)
            where = s["pages"][:, b][..., row // page].long()                   # [NL][H][n]
            k[where, row % page] = kn[:, b, :, :news[b]]
        return {"out": out, "k": k, "v": None, "length": None}
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=s["q"].device)
    H, page, D = case["hkv"], case["page"], case["dim"]
    G = case["hq"] // H
    lens, first = _lens(case), _firsts(case)
    prefix, of = _prefixes(case)
    for l in range(NL):
        for b in range(Bs):
            row = torch.arange(int(lens[b]), device=out.device)
            p, lead = int(prefix[of[b]]), int(first[of[b]])
            n = int(lens[b]) + int(news[b])
            seen = torch.arange(n, device=out.device)
            if case["window"]:
                seen = seen[(seen < case["sinks"]) | (seen >= n - case["window"])]
            for h in range(H):
                where = torch.where(row < p, s["pages"][l, lead, h].long()[row // page],
                                    s["pages"][l, b, h].long()[row // page])
                k, v = (x[where, row % page].double() for x in (s["k"], s["v"]))
                if news[b]:
                    k, v = (torch.cat([x, y[l, b, h, None].double()]) for x, y in ((k, s["kn"]), (v, s["vn"])))
                k, v = k[seen], v[seen]
                x = torch.matmul(s["q"][l, b, h * G:(h + 1) * G].double(), k.T.contiguous()) / math.sqrt(D)
                total = torch.logsumexp(x, -1)
                out[l, b, h * G:(h + 1) * G] = torch.matmul(torch.exp(x - total[:, None]), v)
                lse[l, b, h * G:(h + 1) * G] = total
    return {"out": out, "lse": lse, "k": None, "v": None, "length": None}
