"""gk_append against a 64-bit definition: types, layouts, page and head sizes, rotations of one to three axes, partly filled
pages, scales that grow, values that are no numbers, faults, and the bytes that must not change.

A rotated value is two products and a sum in fp32 (each rounded by at most 2^-24 of its size) and one rounding to bf16 (at
most 2^-8 of the result) or e4m3 (at most 2^-4 of it, or 2^-10 of the scale for the smallest values)."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2609_39358_b200 as gk
from seq_reference import F8, Layout, Paged, batch_of, e4m3_round64, make_seqs, rotate64


def table_of(R, far, seed=2):
    inv = torch.exp(torch.arange(R // 2, dtype=torch.float64) * (-math.log(1e4) / (R // 2)))
    a = torch.arange(far, dtype=torch.float64)[:, None] * inv
    return torch.cat([a.cos(), a.sin()], 1).to(torch.float32).cuda()


def reference(lay, p, layer, sq, k, v, rows, cos_sin, interleaved):
    """What the layer holds after the call, in 64 bits: [K, V] stored values, scales; and by how much each may differ."""
    kr = k.to(torch.float64) if cos_sin is None else rotate64(k, cos_sin, rows, interleaved)
    slack_k = torch.zeros_like(kr)
    if cos_sin is not None:
        # three roundings, each of at most 2^-24 of |a c| + |b s| (first of a pair) or |b c| + |a s| (second): with the
        # sines' sign turned the first comes out as that sum, without it the second
        size = cos_sin.abs()
        minus = torch.cat([size[:, :size.shape[1] // 2], -size[:, size.shape[1] // 2:]], 1)
        slack_k = 3 * 2.0 ** -24 * torch.maximum(rotate64(k.abs(), minus, rows, interleaved).abs(),
                                                 rotate64(k.abs(), size, rows, interleaved).abs())
    new = [kr, v.to(torch.float64)]
    slack = [slack_k, torch.zeros_like(kr)]
    stored = [x.to(torch.float64).clone() for x in p.layer(layer)]
    tol = [torch.zeros_like(x) for x in stored]
    scales = [p.scale(layer, kv).to(torch.float64).clone() for kv in range(2)] if lay.fp8 else None
    i = 0
    for s, (t, n) in enumerate(zip(sq.kv, sq.new)):
        lo = max(t - n, 0)
        i += lo - (t - n)
        for page in range(lo // lay.T, (t - 1) // lay.T + 1) if t > lo else ():
            a, b = max(lo, page * lay.T), min(t, (page + 1) * lay.T)
            g = int(sq.table[s, page])
            r = slice(a - page * lay.T, b - page * lay.T)
            x = [y[i:i + b - a] for y in new]
            sl = [y[i:i + b - a] for y in slack]
            i += b - a
            if not lay.fp8:
                for kv in range(2):
                    stored[kv][g, r] = x[kv]
                    tol[kv][g, r] = x[kv].abs() * 2.0 ** -8 + sl[kv]
                continue
            top = [torch.where(torch.isfinite(y), y, 0.0).abs().amax((0, 2)) for y in x]
            if lay.scale_kv == 1:
                top = [torch.maximum(*top)] * 2
            for kv in range(2):
                old = scales[kv][g].clone()
                kept = (old > 0) & torch.isfinite(old) & (r.start > 0)
                base = torch.where(kept, old, 1.0)
                e = torch.ceil(torch.log2(top[kv] / (448 * base)))
                e = torch.where(top[kv] > 0, e, 0.0)
                e = torch.where(kept, e.clamp(min=0), e)
                sc = base * torch.exp2(e)
                shrink = torch.where(kept, torch.exp2(-e), 0.0)
                was = stored[kv][g, :r.start]
                stored[kv][g, :r.start] = torch.where(shrink[:, None] == 1, was, e4m3_round64(was * shrink[:, None]))
                y = x[kv] / sc[:, None]
                stored[kv][g, r] = torch.where(torch.isfinite(y), y, math.nan)
                tol[kv][g, r] = torch.maximum(y.abs() * 2.0 ** -4, torch.full_like(y, 2.0 ** -10)) + (sl[kv] + x[kv].abs() * 2.0 ** -22) / sc[:, None]
                if kv == 1 or lay.scale_kv == 2:
                    scales[kv][g] = sc
                    if lay.scale_kv == 1:
                        scales[0][g] = sc
    return kr, stored, tol, scales


def run(lay, kv, new, G=2, R=None, axes=1, interleaved=False, positions=False, spread=1.0, seed=1, step_form=False, queries=True,
        in_place=False, mend=None):
    R = lay.D if R is None else R
    sq = make_seqs(lay, kv, new, seed)
    p = Paged(lay, sq.pages, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 9)
    N = sq.n
    qkv = torch.randn(N, (G + 2) * lay.H, lay.D, device="cuda", generator=g) * spread
    qkv = qkv.to(torch.bfloat16)
    q, k, v = qkv[:, :G * lay.H], qkv[:, G * lay.H:(G + 1) * lay.H], qkv[:, (G + 1) * lay.H:]
    if mend:
        mend(p, sq, q, k, v)
    far = max(kv + [1]) + 50
    cos_sin = table_of(R, far) if R else None
    pos = torch.cat([torch.arange(t - n, t) for t, n in zip(kv, new)]).clamp(min=0).cuda()
    where, rope, rows = None, None, None
    if R:
        sections = (R // 2,) if axes == 1 else (R // 2 - 5, 5) if axes == 2 else (R // 2 - 7, 3, 4)
        if positions or axes > 1:
            where = torch.randint(0, far, (axes, N), dtype=torch.int32, device="cuda", generator=g)
        axis = torch.cat([torch.full((m,), a) for a, m in enumerate(sections)]).cuda()
        rows = (where.long() if where is not None else pos[None].expand(axes, -1))[axis]
        rope = gk.Rope(cos_sin, interleaved, sections, where)
    kr, stored, tol, scales = reference(lay, p, 1, sq, k, v, rows, cos_sin, interleaved)
    qr = q.to(torch.float64) if not R else rotate64(q, cos_sin, rows, interleaved)
    before = p.bytes.clone()
    s_before = p.scales.clone() if lay.fp8 else None
    q_abs = q.to(torch.float64).abs()
    out = q if in_place else torch.full((N, G * lay.H, lay.D), 9.0, dtype=torch.bfloat16, device="cuda")
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_append(p.cache(), 1, batch_of(sq, step_form=step_form), k, v, q if queries else None,
                      out if queries else None, rope)
        torch.cuda.synchronize()
    if queries and N:
        err = (out.to(torch.float64) - qr).abs()
        assert float((err - qr.abs() * 2.0 ** -8 - 2.0 ** -20 * q_abs.amax()).nan_to_num(0).max()) <= 0
    for which in range(2):
        got = p.layer(1)[which].to(torch.float64)
        assert torch.equal(torch.isnan(got), torch.isnan(stored[which])), "NaN in other places"
        over = ((got - stored[which]).abs() - tol[which]).nan_to_num(-1.0)
        assert float(over.max()) <= 0, f"{'KV'[which]} off at {int(over.argmax())}"
        if lay.fp8:
            assert torch.equal(p.scale(1, which).to(torch.float64), scales[which]), "scales"
    # every other byte as before: the other layer, other pages, other rows, the room between
    changed = p.bytes.clone()
    p.bytes.copy_(before)
    untouched = [x.clone().view(torch.uint8) for x in p.layer(1)]
    p.bytes.copy_(changed)
    i = 0
    mask = torch.zeros(2, sq.pages, lay.T, dtype=torch.bool, device="cuda")
    for s, (t, n) in enumerate(zip(kv, new)):
        for a in range(max(t - n, 0), t):
            mask[:, sq.table[s, a // lay.T].long(), a % lay.T] = True
        if lay.fp8 and t > max(t - n, 0):
            a = max(t - n, 0)
            mask[:, sq.table[s, a // lay.T].long(), :a % lay.T] = True     # may have been rescaled: checked above
    for which in range(2):
        same = (p.layer(1)[which].view(torch.uint8) == untouched[which]).flatten(2).all(-1)
        assert bool((same | mask[which]).all())
        p.layer(1)[which].view(torch.uint8).copy_(untouched[which])
    assert torch.equal(p.bytes, before)
    if lay.fp8:
        for which in range(lay.scale_kv):
            p.scale(1, which).copy_(torch.as_strided(s_before, p.scale(1, which).shape, p.scale(1, which).stride(),
                                                     p.scale(1, which).storage_offset()))
        assert torch.equal(p.scales.view(torch.int32), s_before.view(torch.int32))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [16, 48, 64, 80, 128, 192, 256])
@pytest.mark.parametrize("head_major", [False, True])
def test_head_sizes(fp8, D, head_major):
    run(Layout(3, D, 16, fp8, head_major=head_major, gap=32, scale_gap=1) if D % 16 == 0 and (3 * D) % 16 == 0 else Layout(2, D, 16, fp8),
        [1, 40, 100], [1, 3, 100])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 2, 7, 16, 32, 100, 256])
@pytest.mark.parametrize("scale_kv", [1, 2])
def test_page_sizes(fp8, T, scale_kv):
    run(Layout(4, 64, T, fp8, scale_kv), [500, 33, 64, 300], [1, 33, 20, 299])
    run(Layout(4, 64, T, fp8, scale_kv), [500, 33, 64, 1], [1] * 4, step_form=True)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("axes,interleaved,R,positions", [(1, False, 64, True), (1, True, 64, False), (2, False, 64, True),
                                                          (3, False, 128, True), (3, True, 128, True), (3, False, 32, True),
                                                          (1, False, 16, False), (1, True, 48, True), (1, False, 0, False)])
def test_rotations(fp8, axes, interleaved, R, positions):
    run(Layout(2, 128, 16, fp8), [300, 20, 64], [60, 20, 1], R=R, axes=axes, interleaved=interleaved, positions=positions)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("spread", [1e-30, 1e-3, 30.0, 3e4, 1e30])
def test_sizes_of_values(fp8, spread):
    run(Layout(2, 64, 16, fp8), [50, 37, 16], [1, 37, 5], spread=spread)


@pytest.mark.parametrize("fp8", [False, True])
def test_empty_sequences_and_no_queries(fp8):
    lay = Layout(2, 64, 16, fp8)
    run(lay, [0, 30, 40, 9], [0, 0, 7, 9])
    run(lay, [0, 30, 40, 9], [0, 0, 7, 9], queries=False)
    run(lay, [10, 30], [25, 3])                 # 15 rows before position 0 are not appended
    run(lay, [200, 30], [150, 3], in_place=True)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("n_seqs", [40, 300])
def test_many_sequences(fp8, n_seqs):
    kv = [1 + (i * 37) % 90 for i in range(n_seqs)]
    run(Layout(2, 64, 16, fp8), kv, [1 + (i * 11) % k for i, k in enumerate(kv)])
    run(Layout(2, 64, 16, fp8), kv, [1] * n_seqs, step_form=True)


@pytest.mark.parametrize("fp8", [False, True])
def test_values_that_are_no_numbers(fp8):
    def mend(p, sq, q, k, v):
        k[3, 0, 5], k[4, 1, 6], v[5, 0, 7], v[6, 1, 8] = math.nan, math.inf, -math.inf, math.nan
    run(Layout(2, 64, 16, fp8), [40, 20], [40, 1], R=0, mend=mend)


@pytest.mark.parametrize("value", [0.0, -1.0, math.nan, math.inf])
def test_scales_that_are_none(value):
    """A page with older rows and a scale that is zero, negative or no number: the rows become zeros (or stay NaN) and the page
    starts over."""
    def mend(p, sq, q, k, v):
        p.scale(1, 0)[sq.table[0, 1].long()] = value
    run(Layout(2, 64, 16, True), [25, 20], [3, 1], mend=mend)


def test_all_zero_rows():
    def mend(p, sq, q, k, v):
        k.zero_(), v.zero_()
    run(Layout(2, 64, 16, True), [25, 20, 48], [3, 20, 16], mend=mend)


def test_a_page_filled_token_by_token_does_not_wear_out():
    """Growing values, one token a call: what is stored in the end is within one rounding of every value, and (but for the
    smallest values) the same as if the page had been appended at once."""
    lay = Layout(2, 64, 32, True)
    sq = make_seqs(lay, [32], [1], 3)
    one, all_at_once = Paged(lay, sq.pages, 3), Paged(lay, sq.pages, 3)
    x = torch.randn(32, 2, 64, device="cuda") * torch.exp2(torch.arange(32, device="cuda") / 3.0)[:, None, None]
    x = x.to(torch.bfloat16)
    with gk.Context(lay.geom(), 0) as ctx:
        kv = torch.zeros(1, dtype=torch.int32, device="cuda")
        b = gk.Batch(sq.table, kv)
        for i in range(32):
            kv.fill_(i + 1)
            ctx.gk_append(one.cache(), 1, b, x[i:i + 1], x[i:i + 1])
        sq.kv, sq.new = [32], [32]
        ctx.gk_append(all_at_once.cache(), 1, batch_of(sq), x, x)
        torch.cuda.synchronize()
    g = int(sq.table[0, 0])
    assert torch.equal(one.scale(1, 0)[g], all_at_once.scale(1, 0)[g])
    a, b = (p.values(1, 0)[g] for p in (one, all_at_once))
    top = all_at_once.scale(1, 0)[g].to(torch.float64)[None, :, None]
    assert float(((a - b).abs() - top * 2.0 ** -9).max()) <= 0          # one subnormal step
    assert float(((a - x.to(torch.float64)).abs() - torch.maximum(x.abs().to(torch.float64) * 2.0 ** -4, top * 2.0 ** -9)).max()) <= 0


@pytest.mark.parametrize("fp8", [False, True])
def test_faults(fp8):
    """Bad page ids, lengths beyond the table and rotation indexes outside the angle table: nothing is written where the page is not
    known, NaN where the angle is not, the codes in the status, other sequences as ever."""
    lay = Layout(2, 64, 16, fp8)
    sq = make_seqs(lay, [30, 40, 50, 20], [20, 20, 20, 20], 3, extra_columns=0)
    p = Paged(lay, sq.pages, 3)
    sq.table[0, 1] = sq.pages
    status = torch.zeros(4, dtype=torch.uint8, device="cuda")
    b = batch_of(sq, status)
    b.kv_len[1] = 16 * sq.table.shape[1] + 3
    where = torch.arange(80, dtype=torch.int32, device="cuda")
    where[45] = 5000
    where[65] = -1
    cos_sin = table_of(64, 100)
    k = torch.randn(80, 2, 64, device="cuda").to(torch.bfloat16)
    q = k.clone()
    first = p.bytes.clone()
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_append(p.cache(), 1, b, k, k, q, q, gk.Rope(cos_sin, positions=where[None]))
        torch.cuda.synchronize()
    assert status.tolist() == [2, 2, 5, 5]
    bad = torch.isnan(q).flatten(1).any(1)
    assert bad.nonzero().flatten().tolist() == [45, 65]
    K = p.layer(1)[0].to(torch.float64)
    at = sq.table[2, (30 + 5) // 16].long(), (30 + 5) % 16
    assert bool(torch.isnan(K[at]).all())
    # rows 10..15 of sequence 0 went to its good page, the others nowhere
    good = p.layer(1)[0][sq.table[0, 0].long(), 10:]
    was = first.view(torch.uint8)
    assert int((p.bytes != was).sum()) > 0 and bool(torch.isfinite(good.float()).all())


def test_refusals():
    lay = Layout(2, 64, 16)
    sq = make_seqs(lay, [40, 50], [1, 1], 3)
    p = Paged(lay, sq.pages, 3)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device="cuda")
    table = table_of(64, 100)
    b = batch_of(sq)

    def refused(code, layer=1, k=x, v=x, q=None, q_out=None, rope=None, batch=b):
        with pytest.raises(gk.GkError) as e:
            ctx.gk_append(p.cache(), layer, batch, k, v, q, q_out, rope)
        assert e.value.code == code

    with gk.Context(lay.geom(), 0) as ctx:
        refused(-1, layer=2)
        refused(-1, k=x.float())
        refused(-1, v=x[:, :1])
        refused(-1, k=x[:1])
        refused(-2, k=torch.zeros(2, 2, 68, dtype=torch.bfloat16, device="cuda")[..., :64])
        refused(-1, rope=gk.Rope(table, sections=(16, 8, 4), positions=torch.zeros(3, 2, dtype=torch.int32, device="cuda")))
        refused(-1, rope=gk.Rope(table, sections=(16, 8, 8)))
        refused(-1, rope=gk.Rope(table, positions=torch.zeros(1, 5, dtype=torch.int32, device="cuda")))
        refused(-1, rope=gk.Rope(table_of(80, 100)))
        refused(-2, rope=gk.Rope(table_of(40, 100)))
        refused(-1, q=x, q_out=x[:, :1])
        with pytest.raises(gk.GkError):
            gk.Rope(table.double())
        ctx.gk_append(p.cache(), 1, gk.Batch(sq.table, b.kv_len, torch.zeros(3, dtype=torch.int32, device="cuda"), 0), x[:0], x[:0])
        torch.cuda.synchronize()
    odd = Layout(2, 24, 16)
    with gk.Context(odd.geom(), 0) as ctx:
        p = Paged(odd, 8, 3)
        y = torch.zeros(2, 2, 24, dtype=torch.bfloat16, device="cuda")
        refused(-2, k=y, v=y)
