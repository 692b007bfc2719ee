"""The operators over a paged KV cache whose speed is followed: attention of one
new token, attention of a run of new tokens (causal, with an optional sliding
window and sinks) and eviction by accumulated attention weight, each at the calls
that a program which serves or compresses a reasoning model makes.

A page holds `page` rows of one unit (layer, sequence, KV head); a table gives every
unit its pages in order.  Cases have 1 to 32 layers, 1 to 32 sequences of up to
32,768 cached rows (even or ragged), 2 to 8 KV heads with groups of 2 to 8 query
heads, head_dim 64 and 128, bf16 and fp32, pages of 16 to 256 rows, runs of 1 to
16,384 new tokens, windows of 64 to 4,096 rows with up to 64 sinks, and budgets of
a fifth to all of a cache.

`run` computes a case in plain torch operations, or, where `own` is set, by the
framework's entry points.
"""
import math

import numpy as np
import torch

own = False


def _decode(name, layers, batch, hq, hkv, dim, dtype, page, lo, hi, append, weights=False, sinks=0, window=0):
    return {"name": name, "kind": "decode", "layers": layers, "batch": batch, "hq": hq, "hkv": hkv, "dim": dim,
            "dtype": dtype, "page": page, "lo": lo, "hi": hi, "append": append, "weights": weights, "sinks": sinks,
            "window": window}


def _prefill(name, layers, batch, hq, hkv, dim, dtype, page, lo, hi, new_lo, new_hi, weights=False, sinks=0, window=0):
    return {"name": name, "kind": "prefill", "layers": layers, "batch": batch, "hq": hq, "hkv": hkv, "dim": dim,
            "dtype": dtype, "page": page, "lo": lo, "hi": hi, "new_lo": new_lo, "new_hi": new_hi, "weights": weights,
            "sinks": sinks, "window": window}


def _evict(name, layers, batch, hkv, dim, dtype, page, lo, hi, budget, sinks, recent):
    return {"name": name, "kind": "evict", "layers": layers, "batch": batch, "hkv": hkv, "dim": dim, "dtype": dtype,
            "page": page, "lo": lo, "hi": hi, "budget": budget, "sinks": sinks, "recent": recent}


def listed():
    return [
        # The smallest call, where latency counts: one layer of a small fp32 model over 2,048 rows.
        _decode("decode_f32_small", 1, 1, 8, 2, 64, "f32", 16, 2048, 2048, False),
        # A 7B-shaped sequence after compression, all layers in one call.
        _decode("decode_all_layers_7b", 28, 1, 28, 4, 128, "bf16", 64, 9645, 9645, True),
        # One layer of a serving batch: 32 ragged sequences.
        _decode("decode_layer_batch32_7b", 1, 32, 28, 4, 128, "bf16", 16, 4096, 32768, True),
        # A decoder that keeps each row's accumulated weight for a later eviction (8B shape).
        _decode("decode_weights_8b", 32, 1, 32, 8, 128, "bf16", 32, 4225, 4225, True, weights=True),
        # Long caches seen through a window with four sinks (32B shape, 8 layers, 8 ragged sequences).
        _decode("decode_window_32b", 8, 8, 40, 8, 128, "bf16", 64, 2049, 12289, True, sinks=4, window=4096),
        # A short prompt of the small fp32 model into an empty cache.
        _prefill("prefill_f32_small", 1, 1, 8, 2, 64, "f32", 16, 0, 0, 301, 301),
        # The answer probe: 32 answer tokens over one layer of the compressed 7B-shaped cache.
        _prefill("prefill_probe_7b", 1, 1, 28, 4, 128, "bf16", 64, 9645, 9645, 32, 32),
        # One layer of a padded batch of prompts of 200 to 512 tokens (8B shape), weights kept.
        _prefill("prefill_prompts_8b", 1, 8, 32, 8, 128, "bf16", 32, 0, 0, 200, 512, weights=True),
        # One layer of a 16K prompt through a window of 4,096 with four sinks (7B shape).
        _prefill("prefill_window_7b_16k", 1, 1, 28, 4, 128, "bf16", 64, 0, 0, 16384, 16384, sinks=4, window=4096),
        # A later chunk of four ragged prompts (32B shape).
        _prefill("prefill_chunk_32b", 1, 4, 40, 8, 128, "bf16", 128, 2048, 6144, 1024, 2048),
        # The smallest eviction: one layer of the 8B shape, back to its budget after a step of about 200 tokens.
        _evict("evict_layer_8b", 1, 1, 8, 128, "bf16", 16, 1217, 1217, 1024, 4, 32),
        # The 7B-shaped 16K cache of all layers in one call.
        _evict("evict_7b_16k", 28, 1, 4, 128, "bf16", 64, 16384, 16384, 9516, 4, 64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_shape(rng, max_layers, lo_rows, max_elems):
    """Layers, sequences, heads, page and a row range whose K (or V) holds at most max_elems elements."""
    hkv, group = rng.choice([(2, 4), (4, 7), (8, 4), (8, 5), (4, 8), (8, 2)])
    dim = 128 if rng.random() < 0.75 else 64
    dtype = "bf16" if rng.random() < 0.8 else "f32"
    page = rng.choice([16, 16, 32, 64, 128, 256])
    while True:
        layers, batch = _log_int(rng, 1, max_layers), _log_int(rng, 1, 32)
        hi = _log_int(rng, lo_rows, 32768)
        lo = hi if rng.random() < 0.5 else max(1, int(hi * rng.uniform(0.1, 0.9)))
        if layers * batch * hkv * hi * dim <= max_elems:
            return layers, batch, hkv, group, dim, dtype, page, lo, hi


def draw(rng):
    kind = rng.choice(["decode", "decode", "prefill", "prefill", "evict"])
    sinks, window = (rng.choice([0, 1, 4, 16, 64]), _log_int(rng, 64, 4096)) if rng.random() < 0.4 else (0, 0)
    if kind == "decode":
        layers, batch, hkv, group, dim, dtype, page, lo, hi = _draw_shape(rng, 32, 128, 4.0e8)
        c = _decode("", layers, batch, hkv * group, hkv, dim, dtype, page, lo, hi, rng.random() < 0.75,
                    rng.random() < 0.4, sinks, window)
    elif kind == "prefill":
        while True:
            layers, batch, hkv, group, dim, dtype, page, lo, hi = _draw_shape(rng, 2, 16, 4.0e7)
            if rng.random() < 0.4:
                lo = hi = 0
            new_hi = _log_int(rng, 1, 8192)
            new_lo = new_hi if rng.random() < 0.5 else max(1, int(new_hi * rng.uniform(0.1, 0.9)))
            # what the plain form holds at once, and fp32 products run at a sixteenth of the bf16 rate
            pairs = float(layers) * batch * hkv * group * new_hi * (hi + new_hi)
            if pairs * 4 * dim <= (8.0e11 if dtype == "bf16" else 1.0e11) and pairs <= 4.0e9:
                break
        c = _prefill("", layers, batch, hkv * group, hkv, dim, dtype, page, lo, hi, new_lo, new_hi,
                     rng.random() < 0.3, sinks, window)
    else:
        layers, batch, hkv, group, dim, dtype, page, lo, hi = _draw_shape(rng, 32, 256, 2.5e8)
        keep = rng.choice([0, 1, 4, 16])
        recent = rng.choice([0, 16, 32, 64])
        c = _evict("", layers, batch, hkv, dim, dtype, page, lo, hi,
                   max(keep + recent + 1, int(hi * rng.uniform(0.2, 1.0))), keep, recent)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _device():
    return "cuda" if torch.cuda.is_available() else "cpu"


def _spread(lo, hi, n, seed):
    """n whole numbers spread evenly over [lo, hi], in a mixed order."""
    return np.random.RandomState(seed).permutation(np.round(np.linspace(lo, hi, n)).astype(np.int64))


def _lens(case):
    return _spread(case["lo"], case["hi"], case["batch"], 5)


def _news(case):
    """New rows that a call appends to every unit of each sequence."""
    if case["kind"] == "prefill":
        return _spread(case["new_lo"], case["new_hi"], case["batch"], 6)
    return np.full(case["batch"], 1 if case.get("append") else 0, dtype=np.int64)


def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _elem(case):
    return 4 if case["dtype"] == "f32" else 2


def prepare(case, seed):
    """The cache: pages in a random order (page 0 belongs to no unit and stands behind every unit's last
    page in the table), keys and values ~ N(0, 1) with 2% heavy rows that share a direction per unit."""
    dev, dt = _device(), _type(case)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed))
    NL, Bs, H, D, page = case["layers"], case["batch"], case["hkv"], case["dim"], case["page"]
    lens, news = _lens(case), _news(case)
    need = np.maximum(1, -(-(lens + news) // page))                       # pages of a sequence's units
    max_pages = int(need.max())
    each = torch.from_numpy(np.tile(np.repeat(need, H), NL)).to(dev)      # of every unit
    U = NL * Bs * H
    used = int(each.sum())
    order = torch.randperm(used, generator=g, device=dev) + 1
    taken = torch.arange(max_pages, device=dev)[None, :] < each[:, None]
    table = torch.zeros((U, max_pages), dtype=torch.int64, device=dev)
    table[taken] = order
    owner = torch.zeros(used + 1, dtype=torch.int64, device=dev)
    owner[order] = torch.repeat_interleave(torch.arange(U, device=dev), each)
    u = torch.randn((U, D), generator=g, device=dev)
    u = 4.0 * u / torch.linalg.vector_norm(u, dim=-1, keepdim=True)

    def rows():
        x = torch.randn((used + 1, page, D), generator=g, device=dev)
        x += hit * u[owner][:, None, :]
        return x.to(dt)

    hit = (torch.rand((used + 1, page, 1), generator=g, device=dev) < 0.02).float()
    s = {"case": case, "k": rows(), "v": rows(), "pages": table.to(torch.int32).reshape(NL, Bs, H, max_pages),
         "full": torch.from_numpy(lens.astype(np.int32)).to(dev)[None, :, None].expand(NL, Bs, H).contiguous()}
    s["length"] = s["full"].clone()
    s["weight"] = None
    if case["kind"] == "evict" or case["weights"]:
        # accumulated attention weight is close to lognormal over the rows
        s["weight"] = torch.exp(torch.randn((NL, Bs, H, max_pages * page), generator=g, device=dev)) * 1e-2
    if case["kind"] == "evict":
        s["start"] = s["weight"].clone()
        s["budget"] = torch.full((Bs,), case["budget"], dtype=torch.int32, device=dev)
        s["kept"] = torch.zeros((NL, Bs, H, max_pages * page), dtype=torch.int32, device=dev)
    else:
        Hq, T = case["hq"], int(news.max())
        run_of = (T,) if case["kind"] == "prefill" else ()
        s["q"] = torch.randn((NL, Bs, Hq, *run_of, D), generator=g, device=dev).to(dt)
        s["kn"] = s["vn"] = None
        if T:
            s["kn"], s["vn"] = (torch.randn((NL, Bs, H, *run_of, D), generator=g, device=dev).to(dt) for _ in "kv")
        s["new"] = torch.from_numpy(news.astype(np.int32)).to(dev)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(s["q"].shape[:-1], device=dev)
    if own:
        _handle(s)
    return s


def _handle(s):
    """What a program that calls the framework keeps beside its tensors: the cache's handle and a workspace."""
    from paper_2608_04771_amd import binding as B
    case = s["case"]
    cache = s["cache"] = B.PagedKVCache(s["k"], s["v"], s["pages"], s["length"], s["weight"])
    s["err"] = torch.zeros(1, dtype=torch.int32, device=s["k"].device)
    if case["kind"] == "decode":
        s["call"] = B.PreparedPagedDecode(cache, case["hq"], s["out"], s["lse"],
                                          B.paged_decode_workspace(cache, case["hq"]), s["err"],
                                          sinks=case["sinks"], window=case["window"])
    elif case["kind"] == "prefill":
        size = B.paged_prefill_attn_workspace_size(cache, case["hq"], s["q"].shape[3])
        s["ws"] = torch.empty(size, dtype=torch.uint8, device=s["k"].device)
    else:
        s["ws"] = torch.empty(B.paged_evict_workspace_size(cache), dtype=torch.uint8, device=s["k"].device)


# ------------------------------------------------------------------ the calls
def run(s):
    case = s["case"]
    kind = case["kind"]
    if kind == "evict":
        s["weight"].copy_(s["start"])                     # every pass evicts from the whole cache
        s["length"].copy_(s["full"])
        if own:
            from paper_2608_04771_amd import binding as B
            B.reco_paged_evict(s["cache"], s["budget"], sinks=case["sinks"], recent=case["recent"],
                               kept_idx=s["kept"], ws=s["ws"], dev_err=s["err"])
        else:
            _plain_evict(s)
        return {"k": s["k"], "v": s["v"], "weight": s["weight"], "length": s["length"], "kept": s["kept"]}
    if kind == "decode":
        if own:
            s["call"](s["q"], s["kn"], s["vn"])
        else:
            _plain_attend(s, s["q"].unsqueeze(3), s["out"].unsqueeze(3), s["lse"].unsqueeze(3),
                          None if s["kn"] is None else s["kn"].unsqueeze(3),
                          None if s["vn"] is None else s["vn"].unsqueeze(3))
    elif own:
        from paper_2608_04771_amd import binding as B
        B.reco_paged_prefill_attn(s["cache"], s["q"], s["kn"], s["vn"], n_new=s["new"], sinks=case["sinks"],
                                  window=case["window"], out=s["out"], lse=s["lse"], ws=s["ws"], dev_err=s["err"])
    else:
        _plain_attend(s, s["q"], s["out"], s["lse"], s["kn"], s["vn"])
    got = {"out": s["out"], "lse": s["lse"], "k": s["k"], "v": s["v"]}
    if s["weight"] is not None:
        got["weight"] = s["weight"]
    if s["kn"] is not None:
        got["length"] = s["length"].clone()
        s["length"].copy_(s["full"])                      # take the rows back, so that every pass sees the same cache
    return got


def _row_ids(s):
    """Flat row number [units][capacity] of every row of every unit."""
    page = s["case"]["page"]
    table = s["pages"].reshape(-1, s["pages"].shape[-1]).long()
    return (table[:, :, None] * page + torch.arange(page, device=table.device)).reshape(table.shape[0], -1)


def _plain_attend(s, q, out, lse, kn, vn):
    """Append the new rows, then attend from every new token (or, without new rows, from the last one).
    q, out [NL][B][Hq][T][D]; kn, vn [NL][B][H][T][D] or None."""
    case = s["case"]
    NL, Bs, Hq, T, D = q.shape
    H, G, U = case["hkv"], Hq // case["hkv"], NL * Bs * case["hkv"]
    dev = q.device
    ids = _row_ids(s)
    cap = ids.shape[1]
    kf, vf = s["k"].view(-1, D), s["v"].view(-1, D)
    n0 = s["length"].reshape(U).long()
    at = torch.arange(T, device=dev)
    if kn is not None:
        new = s["new"].long()[None, :, None].expand(NL, Bs, H).reshape(U)
        # a padding token writes the null page's own row back, so that it changes nothing
        real = at[None, :] < new[:, None]
        dst = torch.where(real, torch.gather(ids, 1, (n0[:, None] + at).clamp(max=cap - 1)), 0).reshape(-1)
        keep = real.reshape(-1, 1)
        for pool, row in ((kf, kn), (vf, vn)):
            pool[dst] = torch.where(keep, row.reshape(-1, D), pool[0])
        pos, total = n0[:, None] + at, n0 + new           # a token's own row; rows after the call
        s["length"].add_(s["new"][None, :, None])
    else:
        real, pos, total = torch.ones((U, T), dtype=torch.bool, device=dev), (n0 - 1)[:, None], n0
    j = torch.arange(cap, device=dev)
    vis = j <= pos[:, :, None]                            # [U][T][cap]
    if case["window"]:
        vis &= (j < case["sinks"]) | (j > pos[:, :, None] - case["window"])
    kt = kf[ids].float().transpose(1, 2).contiguous()
    x = torch.matmul(q.float().reshape(U, G * T, D), kt).mul_(1.0 / math.sqrt(D)).reshape(U, G, T, cap)
    del kt
    x.masked_fill_(~vis[:, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    x.sub_(top).exp_()
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x.reshape(U, G * T, cap), vf[ids].float()).reshape(U, G, T, D) / z
    ok = real[:, None, :].expand(U, G, T).reshape(NL, Bs, Hq, T)
    out.copy_(torch.where(ok[..., None], o.reshape(NL, Bs, Hq, T, D).to(out.dtype), out))
    lse.copy_(torch.where(ok, (top + z.log()).reshape(NL, Bs, Hq, T), lse))
    if s["weight"] is None:
        return
    w = s["weight"].view(U, cap)
    fresh = (j >= n0[:, None]) & (j < total[:, None])     # rows that this call appended start at nothing
    w.masked_fill_(fresh, 0.0)
    if case["kind"] == "decode":
        w.add_((x / z).sum((1, 2)))


def _plain_evict(s):
    case = s["case"]
    NL, Bs, H, cap = s["weight"].shape
    U, D = NL * Bs * H, case["dim"]
    ids = _row_ids(s)
    w = s["weight"].view(U, cap)
    n = s["length"].reshape(U, 1).long()
    budget = s["budget"].long()[None, :, None].expand(NL, Bs, H).reshape(U, 1)
    m = torch.minimum(n, budget)
    j = torch.arange(cap, device=w.device)[None, :]
    safe = (j < case["sinks"]) | (j >= n - case["recent"])
    middle = ~safe & (j < n)
    best = torch.sort(torch.where(middle, w, -1.0), dim=1, descending=True, stable=True).indices
    rank = torch.empty_like(best).scatter_(1, best, j.expand(U, cap).contiguous())
    keep = torch.where(n <= budget, j < n, (j < n) & (safe | (rank < budget - case["sinks"] - case["recent"])))
    idx = torch.sort((~keep).to(torch.int8), dim=1, stable=True).indices    # the kept rows first, in order
    idx = torch.where(j < m, idx, j)                                        # rows past m stay as they are
    src = torch.gather(ids, 1, idx).reshape(-1)
    for pool in (s["k"].view(-1, D), s["v"].view(-1, D)):
        pool[ids.reshape(-1)] = pool[src]
    w.copy_(torch.gather(w, 1, idx))
    s["kept"].view(U, cap).copy_(torch.where(j < m, idx, s["kept"].view(U, cap).long()))
    s["length"].view(U, 1).copy_(m)


# ------------------------------------------------------------------ floors
def _seen(case, L, t):
    """Rows that t new tokens behind L rows see: all pairs, and how many different rows."""
    p = np.arange(L, L + t) if t else np.array([L - 1])
    n = p + 1
    if not case["window"]:
        return int(n.sum()), int(n[-1])
    start = np.maximum(0, n - case["window"])
    both = np.minimum(start, case["sinks"])
    pairs = int((n - start + both).sum())
    return pairs, int(n[-1] - start[0] + both[0])


def work(case):
    e, d, units = _elem(case), case["dim"], case["layers"] * case["hkv"]
    if case["kind"] == "evict":
        lens = _lens(case)
        kept = np.minimum(lens, case["budget"])
        moved = int(((kept - case["sinks"]) * (lens > case["budget"])).sum())
        return {"bytes": units * (4 * int(lens.sum()) + 4 * int(kept.sum()) + moved * 2 * (2 * d * e + 4)), "flops": 0}
    pairs = rows = 0
    news = _news(case)
    for L, t in zip(_lens(case), news):
        a, b = _seen(case, int(L), int(t))
        pairs, rows = pairs + a, rows + b
    tokens = int(np.maximum(news, 1).sum())
    G = case["hq"] // case["hkv"]
    byt = (rows + int(news.sum())) * 2 * d * e + tokens * G * (2 * d * e + 4)
    if case["weights"]:
        byt += rows * 8 if case["kind"] == "decode" else int(news.sum()) * 4
    return {"bytes": units * byt, "flops": 4.0 * d * G * units * pairs}


# ------------------------------------------------------------------ 64 bits
def exact(case, seed):
    """Unit by unit from the definition: softmax over the visible rows, gathered row by row."""
    if case["kind"] == "evict":
        return None                                       # whole positions and moved rows: nothing is computed
    s = prepare(case, seed)
    NL, Bs, H, D, page = case["layers"], case["batch"], case["hkv"], case["dim"], case["page"]
    G = case["hq"] // H
    lens, news = _lens(case), _news(case)
    runs = case["kind"] == "prefill"
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["k"].device)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=s["k"].device)
    weight = None if s["weight"] is None else s["weight"].double()
    for l in range(NL):
        for b in range(Bs):
            n, t = int(lens[b]), int(news[b])
            row = torch.arange(n, device=s["k"].device)
            for h in range(H):
                where = s["pages"][l, b, h].long()
                k, v = (x[where[row // page], row % page].double() for x in (s["k"], s["v"]))
                if t:
                    kn, vn = ((x[l, b, h, :t] if runs else x[l, b, h, None]).double() for x in (s["kn"], s["vn"]))
                    k, v = torch.cat([k, kn]), torch.cat([v, vn])
                first = n if t else n - 1
                for g in range(h * G, (h + 1) * G):
                    for a in range(0, max(t, 1), 4096):
                        z = min(max(t, 1), a + 4096)
                        q = (s["q"][l, b, g, a:z] if runs else s["q"][l, b, g, None]).double()
                        p = torch.arange(first + a, first + z, device=q.device)[:, None]
                        key = torch.arange(k.shape[0], device=q.device)[None, :]
                        hidden = key > p
                        if case["window"]:
                            hidden |= (key >= case["sinks"]) & (p - key >= case["window"])
                        x = (torch.matmul(q, k.T.contiguous()) / math.sqrt(D)).masked_fill(hidden, -math.inf)
                        total = torch.logsumexp(x, -1)
                        prob = torch.exp(x - total[:, None])
                        o = torch.matmul(prob, v)
                        if runs:
                            out[l, b, g, a:z], lse[l, b, g, a:z] = o, total
                        else:
                            out[l, b, g], lse[l, b, g] = o[0], total[0]
                        if weight is not None and not runs:
                            if t and g == h * G:
                                weight[l, b, h, n] = 0.0
                            weight[l, b, h, :n + t] += prob[0]
                if weight is not None and runs:
                    weight[l, b, h, n:n + t] = 0.0
    got = {"out": out, "lse": lse, "k": None, "v": None}
    if weight is not None:
        got["weight"] = weight
    if s["kn"] is not None:
        got["length"] = None
    return got
