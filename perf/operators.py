"""The paged-cache operators: what they compute, in plain form, and the calls they are timed on.

Before a prompt's keys and values are evicted they live in a paged cache: a pool of pages of a few
rows each, [pages, KV heads, rows, 128], and per sequence a table of the pages that hold its rows.

  rope     rotary positions of query or key rows (ebd_rope)
  append   new tokens' keys and values into their pages, the keys rotated on the way, and the new
           queries rotated by the same launch (ebd_append_paged)
  attend   attention of a chunk of new tokens (one token per sequence: a decode step) over the
           paged cache (ebd_attend_paged)
  gather   the pages of every sequence read out as units, one contiguous run of rows per KV head,
           which the scores and the sampler take (ebd_gather_paged)

With a = amplitude, (x1, x2) a pair of elements and f its frequency in radians per position:
  y1 = a (x1 cos(pos f) - x2 sin(pos f)),  y2 = a (x2 cos(pos f) + x1 sin(pos f))
and, for a query whose row limits are lo .. hi:
  y = sum_{i = lo..hi} softmax_i(q.k_i / sqrt(128)) v_i,  lse = ln sum exp(q.k_i / sqrt(128))
(y = 0, lse = -inf where it sees no row).
"""
import math

import torch

own = False
D = 128


def _case(name, kind, **kw):
    c = dict(kind=kind, **kw)
    if name:
        c["name"] = name
    return c


def _rope(name, rows, heads, rot=D, layout="half", base=1e4, factor=1.0, far=32768, fused=False):
    return _case(name, "rope", rows=rows, heads=heads, rot=rot, layout=layout, base=base,
                 factor=factor, far=far, fused=fused)


def _paged(name, kind, seqs, new, context, kv=8, group=4, page=16, order="heads", ragged=False,
           rot=D, layout="half", base=5e5, factor=1.0, shift=0, fused=True, window=0, padded=False):
    return _case(name, kind, seqs=seqs, new=new, context=context, kv=kv, group=group, page=page,
                 order=order, ragged=ragged, rot=rot, layout=layout, base=base, factor=factor,
                 shift=shift, fused=fused, window=window, padded=padded)


def listed():
    return [
        # the query rows of one decode step of 16 sequences, 32 heads: latency
        _rope("rope_decode_b16", 16, 32, base=5e5, far=131072),
        # a long prompt's query rows as slices of a fused projection, interleaved pairs, half of
        # each head rotated, positions scaled for a context four times as long
        _rope("rope_prompt_partial", 8191, 32, rot=64, layout="pairs", factor=4.0, far=131072,
              fused=True),
        # one layer's append of a decode step: 64 sequences of different lengths
        _paged("append_decode_b64", "append", 64, 1, 4096, ragged=True),
        # one Qwen2.5-7B-shaped layer's append of a batch of prompt chunks (4 KV, 28 query heads),
        # slices of a fused projection
        _paged("append_chunk_ragged", "append", 5, 4096, 6144, kv=4, group=7, page=64, ragged=True,
               base=1e6),
        # one layer's decode step of one sequence, 8 KV heads = 8 query heads: latency
        _paged("attend_decode_b1_4k", "attend", 1, 1, 4096, group=1),
        # one Llama-3-8B-shaped layer's decode step before any eviction, batch 32, 16384 tokens
        _paged("attend_decode_b32_16k", "attend", 32, 1, 16384, page=64),
        # a step of one to eight tokens per sequence (drafted tokens, short turns), 4 KV heads of 7
        # query heads, some tokens padding, pages in token-major order
        _paged("attend_short_b16_6k", "attend", 16, 8, 6144, kv=4, group=7, order="tokens",
               ragged=True, padded=True),
        # a batch of prompt chunks of different lengths with a sliding window
        _paged("attend_chunk_window", "attend", 4, 1000, 8192, page=32, ragged=True, window=2048),
        # a whole prompt of one sequence
        _paged("attend_prompt_8k", "attend", 1, 8192, 8192, page=64),
        # a chunk near the end of a long context
        _paged("attend_chunk_1k_128k", "attend", 1, 1024, 131072, page=256),
        # the units of one layer of one short sequence, before its eviction
        _paged("gather_b1_4k", "gather", 1, 0, 4096),
        # ... of one layer of a batch of 32 prompts of different lengths
        _paged("gather_b32_16k", "gather", 32, 0, 16384, page=64, order="tokens", ragged=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attend", "attend", "attend", "gather"])
    base, factor = rng.choice([1e4, 5e5, 1e6]), rng.choice([1.0, 1.0, 4.0, 8.0])
    layout, rot = rng.choice(["half", "pairs"]), rng.choice([D, D, 2 * rng.randint(1, 64)])
    if kind == "rope":
        return _rope(None, _log(rng, 1, 8191), rng.choice([1, 4, 8, 28, 32]), rot, layout, base,
                     factor, _log(rng, 64, 1 << 20), rng.random() < 0.5)
    kv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 3, 4, 5, 7, 8])
    page, order = rng.choice([16, 32, 64, 128, 256]), rng.choice(["heads", "tokens"])
    context = _log(rng, 1, 131072)
    seqs = min(_log(rng, 1, 64), max(1, 32 * 16384 // context))
    new = 1
    if kind == "append":
        new = min(context, _log(rng, 1, 4096), max(1, 16384 // seqs))
    elif kind == "attend" and rng.random() < 0.7:
        # logits of a padded batch: no more than the largest listed case's
        new = min(context, _log(rng, 1, 8192), max(1, 2 ** 32 // (seqs * kv * group * context)))
    return _paged(None, kind, seqs, 0 if kind == "gather" else new, context, kv, group, page, order,
                  rng.random() < 0.6, rot, layout, base, factor,
                  rng.choice([0, 0, _log(rng, 1, 1 << 20)]), rng.random() < 0.5,
                  _log(rng, 1, context) if rng.random() < 0.3 else 0, rng.random() < 0.3)


# ---- sizes -------------------------------------------------------------------------------------

def _spread(n, count, least, turn):
    """`count` sizes spread over [least, n] in odd steps, the first of them n."""
    return [n] + [least + int((n - least) * ((0.618033988749895 * (i + turn)) % 1.0))
                  for i in range(1, count)]


def _lengths(c):
    """Rows each sequence holds and its new tokens among them."""
    S, n, new = c["seqs"], c["context"], c["new"]
    if not c["ragged"]:
        return [n] * S, [new] * S
    lens = _spread(n, S, max(1, n // 8), 0.3)
    news = _spread(new, S, min(1, new), 0.7)
    return lens, [min(a, b) for a, b in zip(news, lens)]


def _padding(c, s, j, new):
    """Whether token j of sequence s is padding, which sees no row."""
    return c["padded"] and new > 1 and j == new - 1 and s % 2 == 0


def work(c):
    if c["kind"] == "rope":
        n = float(c["rows"] * c["heads"])
        return {"bytes": n * 4 * D + 4 * c["rows"], "flops": n * 3 * c["rot"]}
    lens, news = _lengths(c)
    T, Hq = float(sum(news)), c["kv"] * c["group"]
    if c["kind"] == "append":
        return {"bytes": T * (2 * c["kv"] + Hq) * 4 * D, "flops": T * (c["kv"] + Hq) * 3 * c["rot"]}
    if c["kind"] == "gather":
        return {"bytes": float(sum(lens)) * c["kv"] * 8 * D, "flops": 0.0}
    rows = pairs = 0.0
    for s, (n, m) in enumerate(zip(lens, news)):
        w = c["window"] or n
        real = m - (1 if _padding(c, s, m - 1, m) else 0)
        first, last = n - m, n - m + real - 1
        rows += last + 1 - max(0, first - w + 1) if real else 0
        # sum over hi = first .. last of min(hi + 1, w)
        cut = min(max(w - 1, first), last + 1)
        pairs += (first + 1 + cut) * (cut - first) / 2 + (last + 1 - cut) * w if real else 0
    return {"bytes": rows * c["kv"] * 4 * D + T * Hq * (4 * D + 4), "flops": pairs * Hq * 4 * D}


# ---- inputs ------------------------------------------------------------------------------------

def _frequencies(c):
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    return c["base"] ** (-2.0 * i / c["rot"]) / c["factor"]


def _amplitude(c):
    return 1.0 if c["factor"] == 1.0 else 0.1 * math.log(c["factor"]) + 1.0


def _rows(gen, T, heads, fused):
    """[T, heads, 128]: of its own, or the middle of rows that hold as many heads before and behind."""
    x = torch.randn((T, 3 * heads if fused else heads, D), generator=gen, device="cuda")
    x = x.to(torch.bfloat16)
    return x[:, heads:2 * heads] if fused else x


def _keys(shape, gen):
    """Keys of a cache: N(0, 1), one in fifty of them four times as long."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)
    big = torch.rand(shape[:-1], generator=gen, device="cuda") < 0.02
    return (x * torch.where(big, 4.0, 1.0)[..., None]).to(torch.bfloat16)


def prepare(c, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": c}
    if c["kind"] == "rope":
        st["x"] = _rows(gen, c["rows"], c["heads"], c["fused"])
        st["y"] = torch.empty((c["rows"], c["heads"], D), dtype=torch.bfloat16, device="cuda")
        st["pos"] = torch.randint(0, c["far"], (c["rows"],), generator=gen, device="cuda",
                                  dtype=torch.int32)
        st["freq"], st["amp"] = _frequencies(c), _amplitude(c)
        return st
    lens, news = _lengths(c)
    S, kv, page, T = c["seqs"], c["kv"], c["page"], sum(news)
    used = [-(-n // page) for n in lens]
    perm = torch.randperm(sum(used) + 3, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((S, max(used) + 1), -1, dtype=torch.int32, device="cuda")
    at = 0
    for s, n in enumerate(used):
        table[s, :n] = perm[at:at + n]
        at += n
    pool = (perm.numel(), kv, page, D) if c["order"] == "heads" else (perm.numel(), page, kv, D)
    K = _keys(pool, gen)
    V = torch.randn(pool, generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    if c["order"] == "tokens":
        K, V = K.permute(0, 2, 1, 3), V.permute(0, 2, 1, 3)
    off = [0]
    for n in news:
        off.append(off[-1] + n)
    seq = [s for s, m in enumerate(news) for _ in range(m)]
    row = [n - m + j for n, m in zip(lens, news) for j in range(m)]
    dev = dict(device="cuda")
    st |= {"K": K, "V": V, "table": table, "len": torch.tensor(lens, dtype=torch.int32, **dev),
           "new_off": torch.tensor(off, dtype=torch.int64, **dev),
           "seq": torch.tensor(seq, dtype=torch.int64, **dev),
           "row": torch.tensor(row, dtype=torch.int64, **dev), "max_new": max(news), "max_len": max(lens)}
    if c["kind"] == "gather":
        sizes = [n for n in lens for _ in range(kv)]
        o = [0]
        for n in sizes:
            o.append(o[-1] + n)
        st["seq_off"] = torch.tensor(o, dtype=torch.int64, **dev)
        st["Ku"] = torch.empty((o[-1], D), dtype=torch.bfloat16, **dev)
        st["Vu"] = torch.empty_like(st["Ku"])
        st["unit_row"] = torch.cat([torch.arange(n, **dev) for n in sizes])
        st["unit"] = torch.repeat_interleave(torch.arange(S * kv, **dev), torch.tensor(sizes, **dev))
        return st
    st["q"] = _rows(gen, T, kv * c["group"], c["fused"])
    st["y"] = torch.empty((T, kv * c["group"], D), dtype=torch.bfloat16, **dev)
    if c["kind"] == "append":
        st["k"], st["v"] = _rows(gen, T, kv, c["fused"]), _rows(gen, T, kv, c["fused"])
        st["freq"], st["amp"] = _frequencies(c), _amplitude(c)
        # positions that run on from rows dropped earlier; without a shift they are the cache rows
        st["pos"] = (st["row"] + c["shift"]).to(torch.int32) if c["shift"] else None
        return st
    st["lse"] = torch.empty((T, kv * c["group"]), dtype=torch.float32, **dev)
    hi = [-1 if _padding(c, s, j, m) else n - m + j
          for s, (n, m) in enumerate(zip(lens, news)) for j in range(m)]
    st["hi"] = torch.tensor(hi, dtype=torch.int32, **dev)
    st["token"] = torch.tensor([j for m in news for j in range(m)], dtype=torch.int64, **dev)
    return st


# ---- the framework's calls ---------------------------------------------------------------------

def _plan(st):
    """What a serving program keeps beside its buffers: the call's parameters and its workspace."""
    import paper_2607_21475_amd as ebd

    c = st["case"]
    if c["kind"] in ("rope", "append"):
        rot = ebd.rotary(st["freq"], ebd.EBD_ROPE_PAIRS if c["layout"] == "pairs" else ebd.EBD_ROPE_HALF,
                         amplitude=st["amp"])
    if c["kind"] == "rope":
        return ebd, ebd.rope_params(st["x"], st["y"], st["pos"], rot), None
    pages = ebd.pages(st["K"], st["V"], st["table"])
    if c["kind"] == "append":
        return ebd, ebd.append_paged_params(pages, st["k"], st["v"], st["new_off"], st["len"],
                                            rot, pos=st["pos"], q=st["q"], q_out=st["y"]), None
    if c["kind"] == "gather":
        return ebd, ebd.gather_paged_params(pages, st["seq_off"], st["max_len"]), None
    p = ebd.attend_paged_params(pages, st["q"], st["y"], st["new_off"], st["len"], st["max_new"],
                                st["max_len"], qpos=st["hi"] if c["padded"] else None,
                                window=c["window"])
    return ebd, p, ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_ATTEND_PAGED, p))


def _call(st):
    if "plan" not in st:
        st["plan"] = _plan(st)
    ebd, p, ws = st["plan"]
    kind = st["case"]["kind"]
    if kind == "rope":
        ebd.ebd_rope(p, st["x"], st["y"])
        return st["y"]
    if kind == "append":
        ebd.ebd_append_paged(p, st["k"], st["v"], st["K"], st["V"], st["q"], st["y"])
        return [st["K"], st["V"], st["y"]]
    if kind == "gather":
        ebd.ebd_gather_paged(p, st["K"], st["V"], st["Ku"], st["Vu"])
        return [st["Ku"], st["Vu"]]
    ebd.ebd_attend_paged(p, st["q"], st["K"], st["V"], st["y"], ws, lse=st["lse"])
    return [st["y"], st["lse"]]


# ---- the plain forms ---------------------------------------------------------------------------

def _rotated(x, pos, freq, amp, layout):
    angle = pos.double()[:, None] * freq  # far positions: 64 bits
    cos, sin = (amp * angle.cos()).float()[:, None], (amp * angle.sin()).float()[:, None]
    x = x.float()
    n = freq.numel()
    if layout == "pairs":
        a, b = x[..., 0:2 * n:2], x[..., 1:2 * n:2]
    else:
        a, b = x[..., :n], x[..., n:2 * n]
    u, w = a * cos - b * sin, b * cos + a * sin
    y = torch.stack([u, w], -1).flatten(-2) if layout == "pairs" else torch.cat([u, w], -1)
    return torch.cat([y, x[..., 2 * n:]], -1).to(torch.bfloat16)


def _plain_attend(st):
    c = st["case"]
    S, kv, G, page, N, L = c["seqs"], c["kv"], c["group"], c["page"], st["max_new"], st["max_len"]
    rows = torch.arange(L, device="cuda")
    pg = st["table"][:, rows // page].long().clamp_min(0)  # rows past a sequence's are masked below
    held = (rows < st["len"][:, None])[:, None, :, None]
    # [S, kv, L, D]
    k = torch.where(held, st["K"][pg, :, rows % page].transpose(1, 2), 0).float()
    v = torch.where(held, st["V"][pg, :, rows % page].transpose(1, 2), 0).float()
    q = torch.zeros((S, N, kv, G, D), device="cuda")
    q[st["seq"], st["token"]] = st["q"].float().unflatten(1, (kv, G))
    hi = torch.full((S, N), -1, dtype=torch.int32, device="cuda")
    hi[st["seq"], st["token"]] = st["hi"]
    l = torch.matmul(q.permute(0, 2, 1, 3, 4).reshape(S, kv, N * G, D), k.transpose(2, 3))
    l = l.mul_(1.0 / math.sqrt(D)).view(S, kv, N, G, L)
    hi = hi[:, None, :, None, None]
    seen = rows <= hi
    if c["window"]:
        seen &= rows > hi - c["window"]
    l.masked_fill_(~seen, -math.inf)
    m = l.amax(-1, keepdim=True).clamp_min(-3e38)
    z = l.sub_(m).exp_().sum(-1, keepdim=True)
    o = torch.matmul(l.view(S, kv, N * G, L), v).view(S, kv, N, G, D)
    y = torch.where(z > 0, o / z, 0.0).permute(0, 2, 1, 3, 4)[st["seq"], st["token"]]
    lse = torch.where(z > 0, m + z.log(), -math.inf)[..., 0].permute(0, 2, 1, 3)[st["seq"], st["token"]]
    return [y.flatten(1, 2).to(torch.bfloat16), lse.flatten(1, 2)]


def run(st):
    if own:
        return _call(st)
    c = st["case"]
    if c["kind"] == "rope":
        return _rotated(st["x"], st["pos"], st["freq"], st["amp"], c["layout"])
    if c["kind"] == "attend":
        return _plain_attend(st)
    page = c["page"]
    if c["kind"] == "append":
        pos = st["row"] if st["pos"] is None else st["pos"]
        pg, slot = st["table"][st["seq"], st["row"] // page].long(), st["row"] % page
        st["K"][pg, :, slot] = _rotated(st["k"], pos, st["freq"], st["amp"], c["layout"])
        st["V"][pg, :, slot] = st["v"]
        return [st["K"], st["V"], _rotated(st["q"], pos, st["freq"], st["amp"], c["layout"])]
    s, h = st["unit"] // c["kv"], st["unit"] % c["kv"]
    pg, slot = st["table"][s, st["unit_row"] // page].long(), st["unit_row"] % page
    return [st["K"][pg, h, slot], st["V"][pg, h, slot]]


# ---- the definitions in 64 bits ----------------------------------------------------------------

def _turned(x, pos, freq, amp, layout):
    """Each pair of elements as a complex number, times amp e^(i pos f)."""
    x, n = x.double(), freq.numel()
    y = x.clone()
    turn = torch.polar(torch.full_like(freq, amp).expand(pos.numel(), n), torch.outer(pos.double(), freq))
    first = torch.arange(n, device=x.device) * (2 if layout == "pairs" else 1)
    second = first + (1 if layout == "pairs" else n)
    z = torch.complex(x[..., first], x[..., second]) * turn[:, None, :]
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(c, seed):
    st = prepare(c, seed)
    if c["kind"] == "rope":
        return _turned(st["x"], st["pos"], st["freq"], st["amp"], c["layout"])
    lens, news = _lengths(c)
    page, kv, G = c["page"], c["kv"], c["group"]
    if c["kind"] == "append":
        K, V = st["K"].double(), st["V"].double()
        pos = st["row"] if st["pos"] is None else st["pos"].long()
        k, v, t = _turned(st["k"], pos, st["freq"], st["amp"], c["layout"]), st["v"].double(), 0
        for s, (n, m) in enumerate(zip(lens, news)):
            i = torch.arange(n - m, n, device="cuda")
            p = st["table"][s][i // page].long()
            for h in range(kv):
                K[p, h, i % page], V[p, h, i % page] = k[t:t + m, h], v[t:t + m, h]
            t += m
        return [K, V, _turned(st["q"], pos, st["freq"], st["amp"], c["layout"])]
    if c["kind"] == "gather":
        out = []
        for x in (st["K"], st["V"]):
            out.append(torch.cat([x[st["table"][s, :-(-n // page)].long(), h].reshape(-1, D)[:n].double()
                                  for s, n in enumerate(lens) for h in range(kv)]))
        return out
    y = torch.zeros((sum(news), kv * G, D), dtype=torch.float64, device="cuda")
    lse = torch.full((sum(news), kv * G), -math.inf, dtype=torch.float64, device="cuda")
    t0 = 0
    for s, (n, m) in enumerate(zip(lens, news)):
        p = st["table"][s, :-(-n // page)].long()
        i = torch.arange(n, device="cuda")
        for h in range(kv):
            k, v = (x[p, h].reshape(-1, D)[:n].double() for x in (st["K"], st["V"]))
            for t in range(t0, t0 + m, 512):
                u = min(t + 512, t0 + m)
                hi = st["hi"][t:u].long()[:, None]
                hidden = (i > hi) | (i <= hi - (c["window"] or n + 1))
                for g in range(G):
                    l = (st["q"][t:u, h * G + g].double() @ k.t()) / math.sqrt(D)
                    l = l.masked_fill(hidden, -math.inf)
                    z = torch.logsumexp(l, 1)
                    lse[t:u, h * G + g] = z
                    w = torch.exp(l - torch.where(z.isinf(), 0.0, z)[:, None])
                    y[t:u, h * G + g] = w @ v
        t0 += m
    return [y, lse]
