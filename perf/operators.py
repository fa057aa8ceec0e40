"""Operators of language models that work on one paged cache of keys and values, as a user's program calls them.

A case is a dict with an operation (``op``) and its sizes:

* ``rotary``  rotary positions of a tensor of heads, or their transpose (the gradient);
* ``append``  the new keys (rotated) and values of a batch go into its pages, the queries are rotated beside them;
* ``attend``  attention of every sequence's newest tokens over its pages (one token: decoding; many: a prompt's chunk);
* ``weigh``   the same, and the softmax weights that each cached token received are added to a running total;
* ``evict``   every head keeps the cached tokens of largest total, the first and the last ones, moved up to new pages.

The cache is ``[page, token in page, head, dim]`` for keys and for values; a row of the page table lists a sequence's pages in
order.  ``lengths`` gives every sequence's lengths from the case alone; values, pages and totals come from the seed.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # query heads of a prompt of 8192 tokens, whole heads, halves paired
        dict(name="rotary prompt", op="rotary", tokens=8192, heads=32, dim=128, rot=128, layout="half", scaling="none",
             first=0, inverse=False, dtype="bf16"),
        # gradient of a training batch: part of the head, neighbours paired, frequencies ramped for a long context, odd count
        dict(name="rotary part gradient", op="rotary", tokens=4097, heads=20, dim=64, rot=32, layout="interleaved",
             scaling="ramp", first=120000, inverse=True, dtype="fp16"),
        # one decoding step of 16 sequences: latency
        dict(name="append step", op="append", batch=16, new=1, kv=1024, ragged=True, kv_heads=8, group=4, dim=128, page=16,
             layout="half", dtype="bf16"),
        # prompts of uneven length enter the cache together
        dict(name="append prompts", op="append", batch=6, new=2048, kv=4096, ragged=True, kv_heads=8, group=4, dim=128, page=32,
             layout="interleaved", dtype="fp16"),
        # a single short conversation decodes one token: latency
        dict(name="attend one", op="attend", batch=1, new=1, kv=700, ragged=False, kv_heads=8, group=4, dim=128, page=16,
             window=0, dtype="bf16"),
        # an ordinary decoding step: 64 sequences of uneven length
        dict(name="attend step", op="attend", batch=64, new=1, kv=4096, ragged=True, kv_heads=8, group=4, dim=128, page=16,
             window=0, dtype="bf16"),
        # decoding far into two long contexts, small heads, an odd group
        dict(name="attend far", op="attend", batch=2, new=1, kv=131072, ragged=True, kv_heads=4, group=7, dim=64, page=64,
             window=0, dtype="fp16"),
        # half of a long prompt over all of it: the largest product
        dict(name="attend prompt", op="attend", batch=1, new=8192, kv=16384, ragged=False, kv_heads=8, group=4, dim=128, page=64,
             window=0, dtype="bf16"),
        # a decoding step that keeps the totals
        dict(name="weigh step", op="weigh", batch=24, new=1, kv=4096, ragged=True, kv_heads=8, group=4, dim=128, page=16,
             window=0, dtype="bf16"),
        # a prompt's chunk that keeps the totals
        dict(name="weigh chunk", op="weigh", batch=2, new=2048, kv=8192, ragged=True, kv_heads=8, group=4, dim=128, page=64,
             window=0, dtype="fp16"),
        # a batch of caches shrinks to a quarter
        dict(name="evict", op="evict", batch=8, kv=8192, ragged=True, kv_heads=8, dim=128, page=16, keep=2048, first=4, recent=256,
             dtype="bf16"),
        # one short cache, a few tokens leave: latency
        dict(name="evict few", op="evict", batch=1, kv=1100, ragged=False, kv_heads=4, dim=64, page=32, keep=1000, first=4,
             recent=100, dtype="fp16"),
    ]


def _spread(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("rotary", "append", "attend", "attend", "weigh", "evict"))
    dim = rng.choice((64, 128))
    dtype = rng.choice(("bf16", "fp16"))
    if op == "rotary":
        heads = rng.randint(1, 32)
        return dict(op=op, tokens=_spread(rng, 1, 8192), heads=heads, dim=dim, rot=rng.choice((dim, dim // 2, 32)),
                    layout=rng.choice(("half", "interleaved")), scaling=rng.choice(("none", "linear", "base", "ramp")),
                    first=_spread(rng, 1, 500000), inverse=rng.random() < 0.5, dtype=rng.choice(("bf16", "fp16", "fp32")))
    kv_heads, page = rng.choice((1, 2, 4, 8)), rng.choice((8, 16, 24, 32, 64, 128))
    case = dict(op=op, ragged=rng.random() < 0.7, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype)
    if op == "evict":
        kv = _spread(rng, 200, 8192)
        keep = max(32, int(kv * rng.uniform(0.1, 0.95)))
        return dict(case, batch=_spread(rng, 1, 8), kv=kv, keep=keep, first=rng.choice((0, 4)), recent=rng.randint(0, keep // 2))
    group = rng.choice((1, 2, 3, 4, 5, 7, 8, 16)) if kv_heads < 8 else rng.choice((1, 2, 3, 4))
    if op == "append":
        new = _spread(rng, 1, 2048)
        return dict(case, batch=_spread(rng, 1, 6), new=new, kv=new + _spread(rng, 1, 2048), group=group,
                    layout=rng.choice(("half", "interleaved")))
    window = rng.choice((0, 0, 0, 100, 1024))
    if rng.random() < 0.6:  # decoding, now and then of a few tokens at once
        batch = _spread(rng, 1, 24)
        new = rng.choice((1, 1, 1, 2, 5))
        kv = new + _spread(rng, 1, max(2, (131072 if op == "attend" else 32768) // batch))
    else:
        batch = _spread(rng, 1, 4)
        new = _spread(rng, 8, 2048)
        kv = new + _spread(rng, 1, 6144)
    return dict(case, batch=batch, new=new, kv=kv, group=group, window=window)


def lengths(case):
    """(tokens in the cache, new ones among them) of every sequence: the largest first, uneven ones down to about a third."""
    kv, new = [], []
    for i in range(case["batch"]):
        part = 1.0 - 0.65 * ((i * 0.618034) % 1.0) if case["ragged"] else 1.0
        n = max(1, int(case.get("new", 0) * part)) if case.get("new", 0) > 1 else case.get("new", 0)
        kv.append(max(n, 1, int(case["kv"] * part)))
        new.append(n)
    return kv, new


def angles_per_position(case):
    """(frequencies in 64 bits, factor on cosine and sine) of a case's scaling."""
    r, base, factor, length = case.get("rot", case["dim"]), 10000.0, 8.0, 4096
    f = base ** (-torch.arange(0, r, 2, dtype=torch.float64) / r)
    kind = case.get("scaling", "none")
    if kind == "linear":
        return f / factor, 1.0
    if kind == "base":
        return (base * factor ** (r / (r - 2.0))) ** (-torch.arange(0, r, 2, dtype=torch.float64) / r), 1.0
    if kind == "ramp":  # coordinates that turn less than once in the original length are stretched, those that turn 32 times are not
        keep = ((length * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
        return f / factor * (1 - keep) + f * keep, 0.1 * math.log(factor) + 1.0
    return f, 1.0


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    dt = TYPES[case["dtype"]]
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(dt)  # noqa: E731
    s = dict(case=case)
    if case["op"] in ("rotary", "append"):
        f, s["amp"] = angles_per_position(case)
        s["freqs"] = f.to(dev)
    if case["op"] == "rotary":
        s["x"] = normal(case["tokens"], case["heads"], case["dim"])
        s["pos"] = case["first"] + torch.arange(case["tokens"], device=dev, dtype=torch.int32)
        if own:
            import paper_2609_38198_b200 as fd
            s["fd"] = fd
        return s
    B, H, D, P = case["batch"], case["kv_heads"], case["dim"], case["page"]
    kv, new = lengths(case)
    most = max(kv)
    need = [-(-n // P) for n in kv]
    cols = max(need)
    moved = -(-case["keep"] // P) if case["op"] == "evict" else 0
    pages = sum(need) + B * moved + 3
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    start = np.concatenate([[0], np.cumsum(need)])
    at = torch.from_numpy(np.minimum(start[:-1, None] + np.arange(cols)[None], start[1:, None] - 1)).to(dev)
    s["table"] = order[at].contiguous()
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    s["q_start"] = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev)
    s["kv"], s["new"], s["most"], s["most_new"], s["total"] = kv, new, most, max(new), sum(new)
    s["k_pages"], s["v_pages"] = normal(pages, P, H, D), normal(pages, P, H, D)
    if case["op"] == "evict":
        s["new_table"] = order[sum(need) + torch.arange(B * moved, device=dev)].reshape(B, moved).contiguous()
        s["weights"] = torch.rand(B, H, most, generator=g, device=dev) ** 4 * 10
        s["kept"] = torch.full((B, H, case["keep"]), -1, dtype=torch.int32, device=dev)
        s["new_len"] = torch.zeros(B, dtype=torch.int32, device=dev)
        s["weights_out"] = torch.zeros_like(s["weights"])
    else:
        Hq, T = H * case["group"], s["total"]
        s["q"] = normal(T, Hq, D) if case["op"] == "append" else (2 * normal(T, Hq, D).float()).to(dt)
    if case["op"] == "append":
        s["k"], s["v"] = normal(T, H, D), normal(T, H, D)
        s["pos"] = torch.cat([torch.arange(n - m, n, dtype=torch.int32) for n, m in zip(kv, new)]).to(dev)
    if case["op"] == "weigh":
        s["weights"] = torch.rand(B, H, most, generator=g, device=dev)
        s["weights_out"] = torch.zeros_like(s["weights"])
    if own:
        import paper_2609_38198_b200 as fd
        s["fd"] = fd
        s["cache"] = fd.KVCache(s["k_pages"], s["v_pages"])
        s["batch"] = fd.KVBatch(s["table"], s["kv_len"], s["q_start"], s["total"], s["most_new"], s["most"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _rotate(x, pos, freqs, amp, layout, inverse):
    """Rotary positions of x [tokens, heads, dim] in 32 bits, angles in 64."""
    r = 2 * freqs.numel()
    a = pos.double()[:, None] * freqs
    c, s = (amp * a.cos()).float()[:, None], (amp * a.sin()).float()[:, None]
    s = -s if inverse else s
    y = x.float()
    out = y.clone()
    if layout == "half":
        p, q = y[..., :r // 2], y[..., r // 2:r]
        out[..., :r // 2], out[..., r // 2:r] = p * c - q * s, q * c + p * s
    else:
        p, q = y[..., 0:r:2], y[..., 1:r:2]
        out[..., 0:r:2], out[..., 1:r:2] = p * c - q * s, q * c + p * s
    return out.to(x.dtype)


def _rows(pages, table, most):
    """The cache's rows of every sequence, in order: [batch, slots, heads, dim] in 32 bits."""
    slot = torch.arange(most, device=table.device)
    return pages[table[:, slot // pages.shape[1]].long(), slot % pages.shape[1]].float()


def _attend(s, weigh):
    case = s["case"]
    q, kv_len, start, most, new = s["q"], s["kv_len"].long(), s["q_start"].long(), s["most"], s["most_new"]
    B, H, G, D = case["batch"], case["kv_heads"], case["group"], case["dim"]
    k, v = _rows(s["k_pages"], s["table"], most), _rows(s["v_pages"], s["table"], most)
    i = torch.arange(new, device=q.device)
    n = (start[1:] - start[:-1])[:, None]
    row = torch.where(i < n, start[:-1, None] + i, 0)
    x = q.float()[row].reshape(B, new, H, G, D)
    at = (kv_len[:, None] - n + i)[:, :, None]
    slot = torch.arange(most, device=q.device)
    see = (slot <= at) & (i < n)[:, :, None]
    if case["window"]:
        see &= slot > at - case["window"]
    hide = ~see[:, None, None]
    step = max(1, min(H, (1 << 30) // (B * G * new * most)))
    out = torch.empty(B, new, H, G, D, device=q.device)
    lse = torch.empty(B, new, H, G, device=q.device)
    total = torch.empty(B, H, most, device=q.device)
    for h in range(0, H, step):
        w = torch.einsum("bihgd,bjhd->bhgij", x[:, :, h:h + step], k[:, :, h:h + step])
        w.mul_(1.0 / math.sqrt(D)).masked_fill_(hide, -math.inf)
        top = w.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
        w.sub_(top).exp_()
        norm = w.sum(-1, keepdim=True)
        w.div_(norm.clamp(min=1e-37))
        out[:, :, h:h + step] = torch.einsum("bhgij,bjhd->bihgd", w, v[:, :, h:h + step])
        lse[:, :, h:h + step] = (top + norm.log()).squeeze(-1).permute(0, 3, 1, 2)
        if weigh:
            total[:, h:h + step] = w.sum((2, 3))
    live = (i < n).reshape(-1)
    out = out.reshape(B * new, H * G, D)[live].to(q.dtype)
    lse = lse.reshape(B * new, H * G)[live]
    if not weigh:
        return dict(out=out, lse=lse)
    s["weights_out"].copy_(torch.where(slot < kv_len[:, None, None], s["weights"] + total, s["weights_out"]))
    return dict(out=out, lse=lse, weights=s["weights_out"])


def _append(s):
    case, start = s["case"], s["q_start"].long()
    n = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(case["batch"], device=n.device), n, output_size=s["total"])
    slot = s["kv_len"].long()[seq] - n[seq] + torch.arange(s["total"], device=n.device) - start[seq]
    page, at = s["table"][seq, slot // case["page"]].long(), slot % case["page"]
    s["k_pages"][page, at] = _rotate(s["k"], s["pos"], s["freqs"], s["amp"], case["layout"], False)
    s["v_pages"][page, at] = s["v"]
    return dict(q=_rotate(s["q"], s["pos"], s["freqs"], s["amp"], case["layout"], False), k_pages=s["k_pages"], v_pages=s["v_pages"])


def _evict(s):
    case, w = s["case"], s["weights"]
    keep, most, P = case["keep"], s["most"], case["page"]
    slot, n = torch.arange(most, device=w.device), s["kv_len"].long()[:, None]
    w = torch.where(((slot < case["first"]) | (slot >= n - case["recent"]))[:, None], math.inf, w)
    w = torch.where((slot < n)[:, None], w, -math.inf)
    pick = w.sort(dim=-1, descending=True, stable=True).indices[..., :keep]
    left = n.clamp(max=keep)
    pick = torch.where(torch.arange(pick.shape[-1], device=w.device) < left[..., None], pick, most).sort(-1).values
    fine = pick < most
    s["kept"].fill_(-1)
    s["kept"][..., :pick.shape[-1]] = torch.where(fine, pick, -1)
    b, h, r = fine.nonzero(as_tuple=True)
    src = pick[b, h, r]
    old = s["table"][b, src // P].long(), src % P, h
    to = s["new_table"][b, r // P].long(), r % P, h
    s["k_pages"][to], s["v_pages"][to] = s["k_pages"][old], s["v_pages"][old]
    s["weights_out"].copy_(torch.where((slot < n)[:, None], 0.0, s["weights_out"]))
    s["weights_out"][b, h, r] = s["weights"][b, h, src]
    s["new_len"].copy_(left[:, 0])
    return dict(kept=s["kept"], new_len=s["new_len"], weights=s["weights_out"], k_pages=s["k_pages"], v_pages=s["v_pages"])


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    case, op = s["case"], s["case"]["op"]
    if own:
        if op == "rotary":
            return s["fd"].fd_rotary(s["x"], s["pos"], s["freqs"], layout=case["layout"], scale=s["amp"], inverse=case["inverse"])
        cache, batch = s["cache"], s["batch"]
        if op == "append":
            q = cache.append(batch, s["k"], s["v"], positions=s["pos"], freqs=s["freqs"], layout=case["layout"], scale=s["amp"], q=s["q"])
            return dict(q=q, k_pages=s["k_pages"], v_pages=s["v_pages"])
        if op == "evict":
            cache.evict(batch, s["weights"], case["keep"], first=case["first"], recent=case["recent"], new_table=s["new_table"],
                        kept=s["kept"], new_len=s["new_len"], weights_out=s["weights_out"])
            return dict(kept=s["kept"], new_len=s["new_len"], weights=s["weights_out"], k_pages=s["k_pages"], v_pages=s["v_pages"])
        if op == "weigh":
            out, lse = cache.attend(batch, s["q"], window=case["window"], weights=s["weights"], weights_out=s["weights_out"])
            return dict(out=out, lse=lse, weights=s["weights_out"])
        out, lse = cache.attend(batch, s["q"], window=case["window"])
        return dict(out=out, lse=lse)
    if op == "rotary":
        return _rotate(s["x"], s["pos"], s["freqs"], s["amp"], case["layout"], case["inverse"])
    if op == "append":
        return _append(s)
    if op == "evict":
        return _evict(s)
    return _attend(s, op == "weigh")


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    size = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "rotary":
        n = case["tokens"] * case["heads"]
        return dict(bytes=2 * n * case["dim"] * size + 4 * case["tokens"], flops=3 * n * case["rot"])
    kv, new = lengths(case)
    H, D, T = case["kv_heads"], case["dim"], sum(new)
    if case["op"] == "evict":
        rows = sum(min(n, case["keep"]) for n in kv) * H
        return dict(bytes=rows * (4 * D * size + 8) + 8 * sum(kv) * H, flops=sum(kv) * H)
    G = case["group"]
    if case["op"] == "append":
        return dict(bytes=2 * T * (H * G + 2 * H) * D * size, flops=3 * T * (H * G + H) * D)
    seen, pairs, window = 0, 0, case["window"] or (1 << 40)
    for n, m in zip(kv, new):
        seen += n - max(0, n - m + 1 - window)  # slots that one of the new tokens sees
        first = n - m + 1                       # what the first of them sees, without a window
        if first >= window:
            pairs += m * window
        else:
            short = min(m, window - first)
            pairs += short * first + short * (short - 1) // 2 + (m - short) * window
    flops, total = 4 * pairs * H * G * D, 0
    if case["op"] == "weigh":
        flops, total = flops + pairs * H * G, 8 * sum(kv) * H
    return dict(bytes=2 * seen * H * D * size + 2 * T * H * G * D * size + 4 * T * H * G + total, flops=flops)


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def _turned(x, pos, freqs, amp, layout, inverse):
    """Pairs as complex numbers times amp e^(+-i angle)."""
    r = 2 * freqs.numel()
    z = torch.polar(torch.full_like(pos, amp, dtype=torch.float64)[:, None].expand(-1, r // 2), pos.double()[:, None] * freqs)
    z = (z.conj() if inverse else z)[:, None]
    y = x.double()
    t = y[..., :r]
    if layout == "half":
        u = torch.complex(t[..., :r // 2].contiguous(), t[..., r // 2:].contiguous()) * z
        t = torch.cat([u.real, u.imag], -1)
    else:
        t = torch.view_as_real(torch.view_as_complex(t.reshape(*t.shape[:-1], r // 2, 2).contiguous()) * z).flatten(-2)
    return torch.cat([t, y[..., r:]], -1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rotary":
        return _turned(s["x"], s["pos"], s["freqs"], s["amp"], case["layout"], case["inverse"])
    P, H, D = case["page"], case["kv_heads"], case["dim"]
    if case["op"] == "append":
        k, v, t = s["k_pages"].double(), s["v_pages"].double(), 0
        turned = _turned(s["k"], s["pos"], s["freqs"], s["amp"], case["layout"], False)
        for b, (n, m) in enumerate(zip(s["kv"], s["new"])):
            for page in range((n - m) // P, -(-n // P)):
                lo, hi = max(n - m, page * P), min(n, (page + 1) * P)
                at = int(s["table"][b, page])
                k[at, lo - page * P:hi - page * P] = turned[t + lo - (n - m):t + hi - (n - m)]
                v[at, lo - page * P:hi - page * P] = s["v"][t + lo - (n - m):t + hi - (n - m)].double()
            t += m
        return dict(q=_turned(s["q"], s["pos"], s["freqs"], s["amp"], case["layout"], False), k_pages=k, v_pages=v)
    if case["op"] == "evict":
        w, k, v = s["weights"].double(), s["k_pages"].clone(), s["v_pages"].clone()
        new_w = torch.zeros_like(w)
        for b, n in enumerate(s["kv"]):
            for h in range(H):
                left = torch.ones(n, dtype=torch.bool, device="cuda")
                middle = torch.arange(min(case["first"], n), max(case["first"], n - case["recent"]), device="cuda")
                if n > case["keep"]:  # the lightest of the middle leave, of equal ones the later
                    by = torch.stack([w[b, h, middle], -middle.double()]).cpu().numpy()
                    light = np.lexsort((by[1], by[0]))[:n - case["keep"]]
                    left[middle[torch.from_numpy(light).to("cuda")]] = False
                src = left.nonzero()[:, 0]
                new_w[b, h, :src.numel()] = w[b, h, src]
                for r0 in range(0, src.numel(), P):
                    part, to = src[r0:r0 + P], int(s["new_table"][b, r0 // P])
                    old = s["table"][b, part // P].long(), part % P, h
                    k[to, :part.numel(), h], v[to, :part.numel(), h] = s["k_pages"][old], s["v_pages"][old]
        return dict(kept=None, new_len=None, weights=new_w, k_pages=k.double(), v_pages=v.double())
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    total = s["weights"].double() if case["op"] == "weigh" else None
    G, t = case["group"], 0
    for b, (n, m) in enumerate(zip(s["kv"], s["new"])):
        used = s["table"][b, :-(-n // P)].long()
        k, v = (s[x][used].reshape(-1, H, D)[:n].double() for x in ("k_pages", "v_pages"))
        dist = torch.arange(n - m, n, device="cuda")[:, None] - torch.arange(n, device="cuda")[None]  # slots back
        ok = (dist >= 0) & (dist < case["window"]) if case["window"] else dist >= 0
        for head in range(H * G):
            x = s["q"][t:t + m, head].double() @ k[:, head // G].T / math.sqrt(D)
            x = torch.where(ok, x, -math.inf)
            lse[t:t + m, head] = torch.logsumexp(x, -1)
            p = torch.softmax(x, -1)
            out[t:t + m, head] = p @ v[:, head // G]
            if total is not None:
                total[b, head // G, :n] += p.sum(0)
        t += m
    if total is None:
        return dict(out=out, lse=lse)
    live = torch.arange(s["most"], device="cuda") < s["kv_len"].long()[:, None, None]
    return dict(out=out, lse=lse, weights=torch.where(live, total, 0.0))
