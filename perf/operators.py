"""The operators on the cache's own tokens, as they are measured: appending a layer's new keys and values to
the paged cache with the position rotation on the way (``gk_append``), and the attention of the new tokens
over that cache (``gk_attention``), in bf16 and in 8 bits with a scale per page and head.

``own`` false: elementary torch operations in 32 bits.  ``own`` true: the library's calls.
"""
import math

import torch

own = False

_contexts = {}  # one context per geometry, as a serving program keeps it


def _case(name, op, **kw):
    c = {"name": name, "op": op, "fp8": False, "scale_kv": 2, "head_major": False, "kv_heads": 8, "group": 4,
         "head_dim": 128, "page_tokens": 16, "seqs": 1, "past_min": 0, "past_max": 0, "new_min": 1, "new_max": 1}
    if op == "append":
        c |= {"rotary_dim": c["head_dim"], "interleaved": False, "axes": 1}
    else:
        c |= {"causal": True, "window": 0, "lse": False}
    c |= kw
    return c


def listed():
    return [
        # one conversation, the next token of a 5,200-token prompt: the smallest append there is
        _case("append one token", "append", past_min=5200, past_max=5200),
        # one decoding step of 96 conversations over the 8-bit cache: most pages are partly filled
        _case("append step fp8", "append", fp8=True, kv_heads=16, page_tokens=32, seqs=96, past_min=40, past_max=6000),
        # a 5,200-token prompt of a 32-head model with 8 key heads
        _case("append prompt", "append", new_min=5200, new_max=5200),
        # image and text tokens of several requests at once, positions with three axes, 8-bit cache
        _case("append three axes fp8", "append", fp8=True, kv_heads=16, page_tokens=32, seqs=7, past_min=9, past_max=4000,
              new_min=333, new_max=3100, axes=3),
        # a small model's first tokens after a short restored block: latency is all there is
        _case("attend short", "attention", kv_heads=2, group=4, head_dim=64, past_min=270, past_max=270),
        # one decoding step of 8 requests, each over two restored blocks of 4,096 tokens
        _case("attend step", "attention", seqs=8, past_min=8192, past_max=8192),
        # one decoding step over the 8-bit cache: 32 restored blocks of about 2,048 tokens
        _case("attend step fp8", "attention", fp8=True, kv_heads=16, page_tokens=32, seqs=32, past_min=1900, past_max=2300),
        # one decoding step behind a restored corpus: one request, a very long cache
        _case("attend corpus", "attention", past_min=97560, past_max=97560),
        # one decoding step of a large ragged batch: 17 to 9,000 tokens, 7 query heads to a key head
        _case("attend ragged", "attention", kv_heads=4, group=7, seqs=128, past_min=17, past_max=9000),
        # a 61-token question behind the same corpus, 8-bit cache: few rows, a very long cache
        _case("attend question fp8", "attention", fp8=True, page_tokens=32, past_min=97560, past_max=97560, new_min=61,
              new_max=61),
        # whole prompts of several lengths, nothing restored; the log-sum-exp is kept for a later join
        _case("attend prompts", "attention", seqs=3, new_min=700, new_max=5200, lse=True),
        # a 4,096-token chunk of a long prompt behind 16,384 restored tokens
        _case("attend chunk", "attention", past_min=16384, past_max=16384, new_min=4096, new_max=4096),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention"])
    fp8 = rng.random() < 0.5
    head_dim = rng.choice([64, 128, 128, 128])
    c = _case("", op, fp8=fp8, scale_kv=rng.choice([1, 2, 2]), head_major=rng.random() < 0.3,
              kv_heads=rng.choice([4, 8, 8, 16]), group=rng.choice([1, 2, 4, 4, 7, 8]), head_dim=head_dim,
              page_tokens=rng.choice([16, 16, 24, 32, 64]))
    del c["name"]
    kind = rng.choice(["step", "step", "prompt", "chunk"])
    tokens = _log(rng, 16, 8000)
    if kind == "step":
        c["seqs"] = _log(rng, 1, 128)
        c["past_max"] = max(1, min(_log(rng, 16, 100000), 500000 // c["seqs"]))
        c["past_min"] = max(1, c["past_max"] // rng.choice([1, 4, 100]))
    elif kind == "prompt":
        c["seqs"] = rng.randint(1, 4)
        c["new_max"] = max(1, tokens // c["seqs"])
        c["new_min"] = max(1, c["new_max"] // rng.choice([1, 3]))
    else:
        c["seqs"] = rng.randint(1, 3)
        c["new_max"] = max(1, tokens // (2 * c["seqs"]))
        c["new_min"] = max(1, c["new_max"] // rng.choice([1, 3]))
        c["past_max"] = _log(rng, 16, max(17, min(60000, 30_000_000 // (c["new_max"] * c["seqs"]))))
        c["past_min"] = max(1, c["past_max"] // rng.choice([1, 2]))
    if op == "append":
        c["axes"] = rng.choice([1, 1, 3])
        c["rotary_dim"] = rng.choice([head_dim, head_dim, head_dim // 2])
        c["interleaved"] = rng.random() < 0.3
    else:
        c["window"] = rng.choice([0, 0, 0, 1000])
        c["causal"] = rng.random() < 0.9 or c["window"] > 0
        c["lse"] = rng.random() < 0.3
        while c["kv_heads"] * c["group"] > 64:
            c["group"] //= 2
    return c


def _spread(lo, hi, n, step):
    """n whole numbers from lo to hi, evenly spread over their logarithm, in a mixed order."""
    v = [int(round((lo + 1) * ((hi + 1) / (lo + 1)) ** (i / max(1, n - 1)))) - 1 for i in range(n)]
    return [v[i * step % n] for i in range(n)]


def _lengths(case):
    """(tokens in the cache, the new ones among them) of every sequence."""
    n = case["seqs"]
    step = next(p for p in (37, 41, 43, 47) if n % p or n == 1)
    past = _spread(case["past_min"], case["past_max"], n, step)
    new = _spread(case["new_min"], case["new_max"], n, 1)
    return [p + q for p, q in zip(past, new)], new


def _sections(case):
    pairs = case["rotary_dim"] // 2
    if case["axes"] == 1:
        return (pairs,)
    third = pairs * 3 // 8
    return (pairs - 2 * third, third, third)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dev = {"device": "cuda"}
    H, D, T, G, n = case["kv_heads"], case["head_dim"], case["page_tokens"], case["group"], case["seqs"]
    total, new = _lengths(case)
    pages_of = [-(-t // T) for t in total]
    width = max(pages_of)
    pages = sum(pages_of) + 8
    layers = 2
    N = sum(new)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    st = {"case": case, "total": total, "new": new, "pages": pages, "N": N,
          "units": sum((t - 1) // T - (t - q) // T + 1 for t, q in zip(total, new))}
    perm = torch.randperm(pages, generator=g, **dev).to(torch.int32)
    table = torch.zeros(n, width, dtype=torch.int32, **dev)
    at = 0
    for s, p in enumerate(pages_of):
        table[s, :p] = perm[at:at + p]
        at += p
    st["table"] = table
    st["kv_len"] = torch.tensor(total, dtype=torch.int32, **dev)
    st["q_start"] = torch.tensor([sum(new[:i]) for i in range(n + 1)], dtype=torch.int32, **dev)
    # the cache: layers x K/V x pages x one page, a page token-major or head-major; this path works on layer 1
    page = (H, T, D) if case["head_major"] else (T, H, D)
    # keys have channels of their own strength, as they have in earnest
    channel = torch.exp(0.4 * randn(H, D))
    st["data"] = torch.empty(layers, 2, pages, *page, dtype=torch.float8_e4m3fn if case["fp8"] else torch.bfloat16, **dev)
    if case["fp8"]:
        st["scales"] = torch.ones(layers, case["scale_kv"], pages, H, **dev)
    for a in range(0, pages, 2048):
        b = min(pages, a + 2048)
        x = randn(2, b - a, T, H, D)
        x[0] *= channel
        if case["fp8"]:  # one scale per page and head from the largest value there
            big = x.abs().amax(dim=(2, 4))
            if case["scale_kv"] == 1:
                big = big.amax(dim=0, keepdim=True)
            s = big / 448.0
            st["scales"][1, :, a:b] = s
            x = x / s[:, :, None, :, None]
        if case["head_major"]:
            x = x.transpose(2, 3)
        st["data"][1, :, a:b] = x.to(st["data"].dtype)
        del x
    st["data"][0] = st["data"][1, :, :1]
    bf = torch.bfloat16
    if case["op"] == "append":
        # q, k and v are views of one projection's output
        qkv = randn(N, (G + 2) * H, D)
        qkv[:, G * H:(G + 1) * H] *= channel
        qkv = qkv.to(bf)
        st["q"], st["k"], st["v"] = qkv[:, :G * H], qkv[:, G * H:(G + 1) * H], qkv[:, (G + 1) * H:]
        st["q_out"] = torch.zeros(N, G * H, D, dtype=bf, **dev)
        R = case["rotary_dim"]
        far = max(total) + 64
        inv = torch.exp(torch.arange(R // 2, dtype=torch.float64, **dev) * (-2.0 * math.log(1e6) / R))
        ang = torch.arange(far, dtype=torch.float64, **dev)[:, None] * inv
        st["cos_sin"] = torch.cat([ang.cos(), ang.sin()], dim=1).to(torch.float32)
        if case["axes"] > 1:
            # text runs along all axes together; rows of an image share a time and differ in height and width
            run = torch.cat([torch.arange(t - q, t, **dev) for t, q in zip(total, new)])
            st["positions"] = torch.stack([run // 7, run // 5 % far, run * 3 % 61]).to(torch.int32)
    else:
        st["q"] = (1.5 * randn(N, G * H, D)).to(bf)
        st["out"] = torch.zeros(N, G * H, D, dtype=bf, **dev)
        if case["lse"]:
            st["lse"] = torch.zeros(N, G * H, dtype=torch.float32, **dev)
    if own:
        import paper_2609_39358_b200 as gk
        geom = gk.Geom(layers, H, D, T, gk.GK_FP8_E4M3 if case["fp8"] else gk.GK_BF16, case["scale_kv"] if case["fp8"] else 0,
                       gk.GK_FLAG_HEAD_MAJOR if case["head_major"] else 0)
        if geom not in _contexts:
            _contexts[geom] = gk.Context(geom, 0)
        st["ctx"] = _contexts[geom]
        slab = T * H * D * st["data"].element_size()
        sc = st.get("scales")
        st["cache"] = gk.Cache(st["data"].view(torch.uint8).view(-1), pages, 2 * pages * slab, pages * slab, slab, sc,
                               0 if sc is None else case["scale_kv"] * pages * H * 4, 0 if sc is None else pages * H * 4,
                               H * 4)
        step = case["new_max"] == 1
        st["batch"] = gk.Batch(table, st["kv_len"], None if step else st["q_start"], N, max(new))
        if case["op"] == "append":
            st["rope"] = gk.Rope(st["cos_sin"], case["interleaved"], _sections(case), st.get("positions"))
    return st


# ---- plain forms ----------------------------------------------------------------------------------------

def _layer_view(st):
    """The layer's K and V as [2, pages, T, H, D]."""
    x = st["data"][1]
    return x.transpose(2, 3) if st["case"]["head_major"] else x


def _token_places(st):
    """Sequence, position, and index within its sequence of every new token."""
    n = st["table"].shape[0]
    q_len = st["q_start"][1:] - st["q_start"][:-1]
    seq = torch.repeat_interleave(torch.arange(n, device="cuda"), q_len, output_size=st["N"])
    j = torch.arange(st["N"], device="cuda") - st["q_start"].long()[seq]
    return seq, (st["kv_len"] - q_len).long()[seq] + j, j


def _rotate(x, cos, sin, interleaved):
    R = 2 * cos.shape[1]
    x = x.to(torch.float32)
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    c, s = cos[:, None], sin[:, None]
    y, z = a * c - b * s, b * c + a * s
    y = torch.stack([y, z], dim=-1).flatten(-2) if interleaved else torch.cat([y, z], dim=-1)
    return torch.cat([y, x[..., R:]], dim=-1)


def _plain_append(st):
    case = st["case"]
    T, fp8 = case["page_tokens"], case["fp8"]
    seq, pos, _ = _token_places(st)
    sec = _sections(case)
    pairs = sum(sec)
    where = st["positions"].long() if "positions" in st else pos[None]
    axis = torch.repeat_interleave(torch.arange(len(sec), device="cuda"), torch.tensor(sec).to("cuda"), output_size=pairs)
    row = where[axis].t()  # [N, pairs]
    at = torch.arange(pairs, device="cuda")
    cos, sin = st["cos_sin"][row, at], st["cos_sin"][row, pairs + at]
    st["q_out"].copy_(_rotate(st["q"], cos, sin, case["interleaved"]))
    new = torch.stack([_rotate(st["k"], cos, sin, case["interleaved"]), st["v"].to(torch.float32)])
    page, slot = st["table"].long()[seq, pos // T], pos % T
    kv = _layer_view(st)
    if not fp8:
        kv[:, page, slot] = new.to(torch.bfloat16)
        return [st["q_out"], st["data"][1]]
    # the pages that the call writes to, one after the other, and which of them each token goes to
    n = st["table"].shape[0]
    q_len = (st["q_start"][1:] - st["q_start"][:-1]).long()
    start, end = st["kv_len"].long() - q_len, st["kv_len"].long()
    first = start // T
    count = torch.where(q_len > 0, (end - 1) // T - first + 1, 0)
    unit0 = count.cumsum(0) - count
    useq = torch.repeat_interleave(torch.arange(n, device="cuda"), count, output_size=st["units"])
    upage = first[useq] + torch.arange(st["units"], device="cuda") - unit0[useq]
    fill = (start[useq] - upage * T).clamp(0, T)  # rows that older tokens hold
    upage = st["table"].long()[useq, upage]
    unit = unit0[seq] + pos // T - first[seq]
    H = case["kv_heads"]
    size = torch.where(torch.isfinite(new), new.abs(), 0.0).amax(-1)  # [2, N, H]
    big = torch.zeros(2, st["units"], H, device="cuda")
    big.scatter_reduce_(1, unit[None, :, None].expand(2, -1, H), size, "amax")
    scales = st["scales"][1]
    if case["scale_kv"] == 1:
        big = big.amax(0, keepdim=True)
    old = scales[:, upage]
    kept = (fill[None, :, None] > 0) & (old > 0) & torch.isfinite(old)
    base = torch.where(kept, old, 1.0)
    m, e = torch.frexp(big / (448.0 * base))
    k = torch.where(m == 0.5, e - 1, e)
    k = torch.where(big > 0, k, 0)
    k = torch.where(kept, k.clamp(min=0), k)
    scale = base * ((k + 127) << 23).to(torch.int32).view(torch.float32)
    scales[:, upage] = scale
    # older rows of a page whose scale has grown
    rows = torch.arange(T, device="cuda")[None, :] < fill[:, None]
    shrink = torch.where(kept, ((127 - k) << 23).to(torch.int32).view(torch.float32), 0.0)
    was = kv[:, upage].to(torch.float32)
    now = was * shrink[:, :, None, :, None]
    kv[:, upage] = torch.where(rows[None, :, :, None, None], now, was).to(torch.float8_e4m3fn)
    kv[:, page, slot] = (new * (1.0 / scale)[:, unit][..., None]).to(torch.float8_e4m3fn)
    return [st["q_out"], st["data"][1], scales]


def _plain_attention(st):
    case = st["case"]
    H, G, D, T = case["kv_heads"], case["group"], case["head_dim"], case["page_tokens"]
    n, width = st["table"].shape
    qm, span = max(st["new"]), width * T
    seq, _, j = _token_places(st)
    q = torch.zeros(n, qm, H, G, D, device="cuda")
    q[seq, j] = st["q"].to(torch.float32).view(-1, H, G, D)
    q = q.permute(0, 2, 1, 3, 4).reshape(n * H, qm * G, D)
    pages = st["table"].long()
    kv = _layer_view(st)

    def states(which):
        x = kv[which][pages].to(torch.float32)  # [n, width, T, H, D]
        if case["fp8"]:
            x *= st["scales"][1][min(which, case["scale_kv"] - 1)][pages][:, :, None, :, None]
        return x.reshape(n, span, H, D).permute(0, 2, 1, 3).reshape(n * H, span, D)

    s = torch.bmm(q, states(0).transpose(1, 2))
    s *= 1.0 / math.sqrt(D)
    total, q_len = st["kv_len"].long(), (st["q_start"][1:] - st["q_start"][:-1]).long()
    at = (total - q_len)[:, None] + torch.arange(qm, device="cuda")  # [n, qm]
    t = torch.arange(span, device="cuda")
    seen = (t < total[:, None])[:, None, :]
    if case["causal"]:
        seen = seen & (t <= at[:, :, None])
    if case["window"]:
        seen = seen & (t > at[:, :, None] - case["window"])
    s = s.view(n, H, qm, G, span).masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = s.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = s.sub_(top).exp_()
    mass = p.sum(-1, keepdim=True)
    o = torch.bmm(p.view(n * H, qm * G, span), states(1)).view(n, H, qm, G, D)
    o = torch.where(mass > 0, o / mass, 0.0).permute(0, 2, 1, 3, 4)[seq, j]
    st["out"].copy_(o.reshape(-1, H * G, D))
    if not case["lse"]:
        return [st["out"]]
    lse = (mass.log() + top).squeeze(-1).permute(0, 2, 1, 3)[seq, j]
    st["lse"].copy_(lse.reshape(-1, H * G))
    return [st["out"], st["lse"]]


def run(st):
    case = st["case"]
    if not own:
        return _plain_append(st) if case["op"] == "append" else _plain_attention(st)
    if case["op"] == "append":
        st["ctx"].gk_append(st["cache"], 1, st["batch"], st["k"], st["v"], st["q"], st["q_out"], st["rope"])
        return [st["q_out"], st["data"][1], st["scales"][1]] if case["fp8"] else [st["q_out"], st["data"][1]]
    lse = st.get("lse")
    st["ctx"].gk_attention(st["cache"], 1, st["batch"], st["q"], st["out"], lse, window=case["window"], causal=case["causal"])
    return [st["out"]] if lse is None else [st["out"], lse]


def work(case):
    H, G, D, T = case["kv_heads"], case["group"], case["head_dim"], case["page_tokens"]
    E = 1 if case["fp8"] else 2
    total, new = _lengths(case)
    N = sum(new)
    if case["op"] == "append":
        units = sum((t - 1) // T - (t - q) // T + 1 for t, q in zip(total, new))
        scales = units * H * 4 * case["scale_kv"] * 2 if case["fp8"] else 0
        moved = N * D * (2 * 2 * G * H + 2 * H * (2 + E)) + N * case["rotary_dim"] * 4 + units * 4 + scales
        return {"bytes": moved, "flops": N * (G + 1) * H * case["rotary_dim"] * 3}
    pairs = kept = pages = 0
    for t, q in zip(total, new):
        w = case["window"] or t
        for i in range(q) if case["causal"] or case["window"] else ():
            hi = t - q + i + 1 if case["causal"] else t
            pairs += hi - max(0, t - q + i + 1 - w)
        if not (case["causal"] or case["window"]):
            pairs += t * q
        first = max(0, t - q + 1 - w)
        kept += t - first
        pages += (t - 1) // T - first // T + 1
    scales = pages * H * 4 * case["scale_kv"] if case["fp8"] else 0
    moved = kept * H * D * 2 * E + N * H * G * D * 2 * 2 + pages * 4 + scales + (N * H * G * 4 if case["lse"] else 0)
    return {"bytes": moved, "flops": 4 * pairs * H * G * D}


# ---- the definitions in 64 bits -------------------------------------------------------------------------

def _e4m3(x):
    """The nearest value of 4 exponent and 3 mantissa bits (ties to even), for |x| <= 448."""
    _, e = torch.frexp(x)
    quantum = torch.exp2((e - 4).clamp(min=-9).to(torch.float64))
    return torch.round(x / quantum) * quantum


def _exact_append(case, st):
    T, R = case["page_tokens"], case["rotary_dim"]
    f8 = torch.float64
    data = st["data"][1].to(f8)
    view = data.transpose(2, 3) if case["head_major"] else data
    scales = st["scales"][1].to(f8) if case["fp8"] else None
    axis = [a for a, m in enumerate(_sections(case)) for _ in range(m)]
    q_out, at = [], 0
    for s, (t, q) in enumerate(zip(st["total"], st["new"])):
        pos = torch.arange(t - q, t, device="cuda")
        where = st["positions"][:, at:at + q].long() if "positions" in st else pos[None]
        angle = torch.stack([where[a] for a in axis])  # [pairs, q]
        pair = torch.arange(R // 2, device="cuda")[:, None]
        z = torch.complex(st["cos_sin"][angle, pair].to(f8), st["cos_sin"][angle, R // 2 + pair].to(f8)).t()[:, None]

        def turn(x):
            x = x[at:at + q].to(f8)
            lo, hi = (x[..., 0:R:2], x[..., 1:R:2]) if case["interleaved"] else (x[..., :R // 2], x[..., R // 2:R])
            y = torch.complex(lo.contiguous(), hi.contiguous()) * z
            y = torch.view_as_real(y)
            y = y.flatten(-2) if case["interleaved"] else torch.cat([y[..., 0], y[..., 1]], -1)
            return torch.cat([y, x[..., R:]], -1)

        q_out.append(turn(st["q"]))
        fresh = torch.stack([turn(st["k"]), st["v"][at:at + q].to(f8)])
        at += q
        if not case["fp8"]:
            view[:, st["table"][s].long()[pos // T], pos % T] = fresh
            continue
        for p in range((t - q) // T, (t - 1) // T + 1):
            g = int(st["table"][s, p])
            a, b = max(t - q, p * T), min(t, p * T + T)
            x = fresh[:, a - (t - q):b - (t - q)]
            held = a - p * T
            big = x.abs().amax(dim=(1, 3))  # [2, H]
            if case["scale_kv"] == 1:
                big = big.amax(0, keepdim=True)
            base = scales[:, g].clone() if held else torch.ones_like(scales[:, g])
            k = torch.ceil(torch.log2(big / (448 * base)))
            if held:
                k = k.clamp(min=0)
            sc = base * torch.exp2(k)
            scales[:, g] = sc
            view[:, g, :held] = _e4m3(view[:, g, :held] * torch.exp2(-k)[:, None, :, None])
            view[:, g, held:held + b - a] = _e4m3((x / sc[:, None, :, None]).clamp(-448, 448))
    out = [torch.cat(q_out), data]
    return out + [scales] if case["fp8"] else out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "append":
        return _exact_append(case, st)
    H, G, D, T = case["kv_heads"], case["group"], case["head_dim"], case["page_tokens"]
    view = st["data"][1].transpose(2, 3) if case["head_major"] else st["data"][1]
    out = torch.empty(st["N"], H, G, D, dtype=torch.float64, device="cuda")
    lse = torch.empty(st["N"], H, G, dtype=torch.float64, device="cuda")
    at = 0
    for s, (t, q) in enumerate(zip(st["total"], st["new"])):
        pages = st["table"][s, :-(-t // T)].long()
        i = torch.arange(t - q, t, device="cuda")[:, None, None]
        u = torch.arange(t, device="cuda")
        hide = torch.zeros(q, 1, t, dtype=torch.bool, device="cuda")
        if case["causal"]:
            hide = hide | (u > i)
        if case["window"]:
            hide = hide | (u <= i - case["window"])
        for h in range(H):
            k, v = (view[w, pages, :, h].to(torch.float64) for w in (0, 1))
            if case["fp8"]:
                k = k * st["scales"][1, 0, pages, h].to(torch.float64)[:, None, None]
                v = v * st["scales"][1, case["scale_kv"] - 1, pages, h].to(torch.float64)[:, None, None]
            k, v = k.reshape(-1, D)[:t], v.reshape(-1, D)[:t]
            x = st["q"][at:at + q, h * G:(h + 1) * G].to(torch.float64)
            w = (x @ k.t() / math.sqrt(D)).masked_fill(hide, -math.inf)
            lse[at:at + q, h] = torch.logsumexp(w, -1)
            out[at:at + q, h] = torch.softmax(w, -1) @ v
        at += q
    out = out.view(st["N"], H * G, D)
    return [out, lse.view(st["N"], H * G)] if case["lse"] else [out]
