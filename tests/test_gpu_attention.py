"""gk_attention against a 64-bit definition: every type, layout, head size and group, lengths from none to long, masks
that leave rows empty, foreign values in masked places, page tables with faults, strides, streams, graphs.

Tolerance of an output element: the result is rounded to bf16 once (at most 2^-8 of its size), the weights may be rounded
to bf16 (at most 2^-8 each, so 2^-8 of sum w|V| / sum w together), and scores carry the rounding of fp32 sums of D
products, D * 2^-23 * sum |q k| * scale, below 2^-11 for the sizes and values here, as does the exponential.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

import paper_2609_39358_b200 as gk
from seq_reference import F8, Layout, Paged, Seqs, attention64, batch_of, make_seqs


def check(out, lse, ref, tag=""):
    want, want_lse, spread = ref
    got = out.to(torch.float64)
    tol = want.abs() * (2.0 ** -8 + 2.0 ** -11) + spread * (2.0 ** -8 + 2.0 ** -11) + 1e-30
    assert torch.equal(torch.isnan(got), torch.isnan(want)), tag
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), tag
    over = torch.where(fine, (got - want).abs() - tol, -1.0)
    assert float(over.max()) <= 0 if over.numel() else True, f"{tag}: {float(over.max())} at {int(over.argmax())}"
    if lse is not None:
        g = lse.to(torch.float64)
        inf = torch.isinf(want_lse)
        assert torch.equal(g[inf], want_lse[inf]), tag
        err = torch.where(inf | torch.isnan(want_lse), 0.0, (g - want_lse).abs())
        assert float(err.max()) <= 2.0 ** -11, f"{tag}: lse off by {float(err.max())}"


def run(lay, kv, new, G=4, window=0, causal=True, scale=None, seed=1, step_form=False, lse=True, layer=1, tune=None):
    sq = make_seqs(lay, kv, new, seed)
    p = Paged(lay, sq.pages, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 5)
    q = torch.randn(sq.n, G * lay.H, lay.D, device="cuda", generator=g).to(torch.bfloat16)
    out = torch.full_like(q, 7.0)
    ls = torch.full((sq.n, G * lay.H), 7.0, device="cuda") if lse else None
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_attention(p.cache(), layer, batch_of(sq, step_form=step_form), q, out, ls, scale, window, causal)
        torch.cuda.synchronize()
        assert ctx.gk_get_stats()["device_wait_expired"] == 0
    check(out, ls, attention64(p, layer, sq, q, scale, window, causal), f"{lay} {kv} {new}")
    return out


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [16, 48, 64, 96, 128, 160, 256])
def test_head_sizes(fp8, D):
    run(Layout(2, D, 16, fp8), [1, 77, 300], [1, 1, 1], G=3)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 2, 5, 7, 8, 16, 17, 40])
def test_groups(fp8, G):
    run(Layout(2, 64, 16, fp8), [129, 64], [1, 1], G=G, step_form=True)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("T", [1, 3, 8, 16, 24, 32, 64, 100, 128, 200, 256])
@pytest.mark.parametrize("head_major", [False, True])
def test_page_sizes_and_layouts(fp8, T, head_major):
    run(Layout(2, 64, T, fp8, head_major=head_major, gap=48, scale_gap=3), [1, 333, 200, 640], [1, 1, 150, 1])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 257, 1000, 5003])
def test_one_token_lengths(fp8, D, length):
    run(Layout(4, D, 16, fp8), [length], [1], step_form=True)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("scale_kv", [1, 2])
def test_a_ragged_step(fp8, scale_kv):
    kv = [1 + (i * 7919) % 2500 for i in range(200)]
    run(Layout(2, 128, 16, fp8, scale_kv if fp8 else 2), kv, [1] * 200, G=7, step_form=True)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 128, 96])
@pytest.mark.parametrize("new", [2, 5, 31, 32, 33, 64, 127, 128, 129, 300, 700])
def test_prompts(fp8, D, new):
    run(Layout(2, D, 16, fp8), [new], [new])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("G", [1, 3, 4, 7, 8, 16, 32])
def test_prompts_with_groups(fp8, G):
    run(Layout(2, 128, 32, fp8), [290, 1100, 64], [290, 100, 7], G=G)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("D", [64, 128])
def test_chunks_behind_a_long_cache(fp8, causal, D):
    run(Layout(2, D, 16, fp8), [9000, 4096, 130], [61, 128, 129], causal=causal)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("window", [1, 2, 64, 100, 128, 1000, 100000])
@pytest.mark.parametrize("causal", [True, False])
def test_windows(fp8, window, causal):
    run(Layout(2, 64, 16, fp8), [400, 1500, 33, 1], [400, 70, 1, 1], window=window, causal=causal)
    run(Layout(2, 64, 16, fp8), [400, 1500, 33, 1], [1, 1, 1, 1], window=window, causal=causal, step_form=True)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 96, 128])
def test_empty_rows_and_sequences(fp8, D):
    """No tokens in the cache, no rows, more rows than tokens: zeros and a log-sum-exp of -infinity."""
    lay = Layout(2, D, 16, fp8)
    run(lay, [0, 5, 0, 40, 0], [1, 0, 3, 1, 0])
    run(lay, [10, 100, 3], [30, 200, 300])
    run(lay, [10, 100, 3], [30, 200, 300], causal=False)
    run(lay, [0], [1], step_form=True)
    run(lay, [0, 0], [0, 200])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("scale", [0.0, -0.3, 2.5, 1e-3])
def test_scales(fp8, scale):
    run(Layout(2, 64, 16, fp8), [300, 200], [1, 1], scale=scale)
    run(Layout(2, 64, 16, fp8), [300, 200], [100, 130], scale=scale)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("D", [64, 96, 128])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_foreign_values_in_masked_places(fp8, D, bad):
    """What a row does not attend to must not reach it: values behind a sequence's end in its last page, tokens of
    the same call that come later, and tokens before the window, all infinite or NaN."""
    lay = Layout(2, D, 16, fp8)
    if fp8:
        bad = math.nan   # e4m3 has no infinities
    for kv, new, window in (([37, 300], [1, 1], 0), ([37, 300], [37, 200], 0), ([37, 700], [1, 150], 64)):
        sq = make_seqs(lay, kv, new, 3)
        p = Paged(lay, sq.pages, 3)
        K, V = p.layer(1)
        for s, t in enumerate(kv):
            for x in (K, V):
                x[sq.table[s, (t - 1) // 16].long(), (t - 1) % 16 + 1:] = bad      # behind the end
                if new[s] > 8:
                    x[sq.table[s, (t - 4) // 16].long(), (t - 4) % 16] = bad       # a late token of the call
        q = torch.randn(sq.n, 8, D, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)).to(torch.bfloat16)
        out, lse = torch.full_like(q, 7.0), torch.full((sq.n, 8), 7.0, device="cuda")
        with gk.Context(lay.geom(), 0) as ctx:
            ctx.gk_attention(p.cache(), 1, batch_of(sq), q, out, lse, window=window)
        torch.cuda.synchronize()
        ref = attention64(p, 1, sq, q, window=window)
        fine = torch.isfinite(ref[0]).all(-1)
        # rows that attend to none of them are as if they were not there; the others are no numbers
        assert torch.equal(torch.isfinite(out.float()).all(-1), fine)
        assert bool(fine.any())
        ref = tuple(torch.where(fine.reshape(fine.shape + (1,) * (r.dim() - 2)), r, 0.0) for r in ref)
        check(torch.where(fine[..., None], out, 0.0), torch.where(fine, lse, 0.0), ref)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new", [1, 90])
def test_infinite_values_in_seen_places(D, new):
    """+inf or -inf in V gives that infinity; both give NaN; a score of +inf gives NaN, one of -inf no weight."""
    lay = Layout(1, D, 16)
    sq = make_seqs(lay, [200], [new], 3)
    p = Paged(lay, sq.pages, 3)
    V = p.layer(1)[1]
    def at(t):
        return sq.table[0, t // 16].long(), t % 16
    V[at(5)[0], at(5)[1], 0, 3] = math.inf
    V[at(60)[0], at(60)[1], 0, 4] = -math.inf
    V[at(7)[0], at(7)[1], 0, 5] = math.inf
    V[at(100)[0], at(100)[1], 0, 5] = -math.inf
    q = torch.randn(sq.n, 4, D, device="cuda").to(torch.bfloat16)
    out = torch.zeros_like(q)
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_attention(p.cache(), 1, batch_of(sq), q, out)
    torch.cuda.synchronize()
    assert bool((out[..., 3] == math.inf).all()) and bool((out[..., 4] == -math.inf).all())
    assert bool(torch.isnan(out[..., 5]).all()) and bool(torch.isfinite(out[..., 6:].float()).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [1, 100])
def test_faults_in_the_page_table(fp8, new):
    """An id that is no page, or a length beyond the table: NaN for the rows that would have read it, the code in the
    status, and the other sequences as ever."""
    lay = Layout(2, 128, 16, fp8)
    sq = make_seqs(lay, [400, 500, 300, 600], [new] * 4, 3, extra_columns=0)
    good = sq.table.clone()
    p = Paged(lay, sq.pages, 3)
    q = torch.randn(sq.n, 8, lay.D, device="cuda").to(torch.bfloat16)
    ref = attention64(p, 1, sq, q)
    out, lse = torch.full_like(q, 7.0), torch.full((sq.n, 8), 7.0, device="cuda")
    status = torch.zeros(4, dtype=torch.uint8, device="cuda")
    sq.table[1, 3] = sq.pages
    sq.table[2, 0] = -1
    b = batch_of(sq, status)
    b.kv_len[3] = 16 * sq.table.shape[1] + 1
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_attention(p.cache(), 1, b, q, out, lse)
        torch.cuda.synchronize()
        assert status.tolist() == [0, 2, 2, 2]
        rows = out.view(4, new, 8, lay.D)
        assert bool(torch.isnan(rows[1:]).all()) and bool(torch.isnan(lse.view(4, new, 8)[1:]).all())
        check(out[:new], lse[:new], tuple(r[:new] for r in ref))
        # the context is as good as new
        sq.table.copy_(good)
        b.kv_len[3] = 600
        ctx.gk_attention(p.cache(), 1, b, q, out, lse)
        torch.cuda.synchronize()
    check(out, lse, ref)


@pytest.mark.parametrize("fp8", [False, True])
def test_value_scales_far_apart(fp8):
    """Pages whose value scales differ by factors of up to 2^40: small pages keep their precision where they decide."""
    lay = Layout(2, 128, 16, True)
    for order in (1, -1):
        sq = make_seqs(lay, [600, 600], [1, 40], 3)
        p = Paged(lay, sq.pages, 3)
        for kv in range(2):
            p.scale(1, 1)[sq.table[kv, :38].long()] = torch.exp2(torch.arange(38, device="cuda") * 1.0 * order - 20)[:, None]
        q = torch.randn(sq.n, 8, lay.D, device="cuda").to(torch.bfloat16)
        out, lse = torch.zeros_like(q), torch.zeros(sq.n, 8, device="cuda")
        with gk.Context(lay.geom(), 0) as ctx:
            ctx.gk_attention(p.cache(), 1, batch_of(sq), q, out, lse)
        torch.cuda.synchronize()
        check(out, lse, attention64(p, 1, sq, q))


def test_large_queries_and_keys_in_8_bits():
    """Queries whose squares leave the range of f16, and tiny ones."""
    lay = Layout(2, 64, 16, True)
    sq = make_seqs(lay, [100, 90], [1, 60], 3)
    p = Paged(lay, sq.pages, 3)
    for f in (3e30, 1e-30):
        q = torch.randn(sq.n, 8, lay.D, device="cuda").to(torch.bfloat16) * f
        out, lse = torch.zeros_like(q), torch.zeros(sq.n, 8, device="cuda")
        with gk.Context(lay.geom(), 0) as ctx:
            ctx.gk_attention(p.cache(), 1, batch_of(sq), q, out, lse, scale=0.1 / f)
        torch.cuda.synchronize()
        check(out, lse, attention64(p, 1, sq, q, scale=0.1 / f))


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [1, 80])
def test_strides_and_the_same_bits_again(fp8, new):
    """q and out as slices of larger tensors, a table with long rows; two calls give the same bits, on a stream too."""
    lay = Layout(3, 128, 16, fp8)
    sq = make_seqs(lay, [700, 333, 90], [new] * 3, 3)
    wide = torch.full((3, 300), -1, dtype=torch.int32, device="cuda")
    wide[:, 8:8 + sq.table.shape[1]] = sq.table
    sq.table = wide[:, 8:8 + sq.table.shape[1]]
    p = Paged(lay, sq.pages, 3)
    big = torch.randn(sq.n, 40, lay.D + 8, device="cuda").to(torch.bfloat16)
    q = big[:, 5:17, 8:]
    room = torch.full((12, sq.n + 2, lay.D + 16), 7.0, device="cuda", dtype=torch.bfloat16)
    out = room.transpose(0, 1)[1:-1, :, 8:-8]
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_attention(p.cache(), 1, batch_of(sq), q, out)
        torch.cuda.synchronize()
        check(out, None, attention64(p, 1, sq, q))
        first = out.clone()
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        out.fill_(0)
        st.wait_stream(torch.cuda.current_stream())
        ctx.gk_attention(p.cache(), 1, batch_of(sq), q, out, stream=st)
        torch.cuda.synchronize()
    assert torch.equal(first, out)
    edge = room.clone()
    edge.transpose(0, 1)[1:-1, :, 8:-8] = 7.0
    assert bool((edge == 7.0).all())        # nothing outside the slice was written


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("new", [1, 70])
def test_captured_calls_follow_lengths_and_tables(fp8, new):
    lay = Layout(2, 128, 16, fp8)
    sq = make_seqs(lay, [900, 400], [new, new], 3)
    p = Paged(lay, sq.pages, 3)
    q = torch.randn(sq.n, 8, lay.D, device="cuda").to(torch.bfloat16)
    out = torch.zeros_like(q)
    b = batch_of(sq)
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_attention(p.cache(), 1, b, q, out)       # allocates
        torch.cuda.synchronize()
        before = ctx.gk_get_stats()["allocations"]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            ctx.gk_attention(p.cache(), 1, b, q, out)
        for kv in ([900, 400], [123, 399], [77, 80]):
            b.kv_len.copy_(torch.tensor(kv, dtype=torch.int32))
            sq.kv = kv
            graph.replay()
            torch.cuda.synchronize()
            check(out, None, attention64(p, 1, sq, q))
        assert ctx.gk_get_stats()["allocations"] == before


@pytest.mark.parametrize("fp8", [False, True])
def test_offsets_beyond_32_bits(fp8):
    """A cache of more than 4 GiB, its last pages in use."""
    lay = Layout(8, 128, 64, fp8, layers=1)
    slab = 64 * 8 * 128 * (1 if fp8 else 2)
    pages = (5 << 30) // slab
    cache = torch.zeros(2 * pages * slab, dtype=torch.uint8, device="cuda")
    scales = torch.ones(2 * pages * 8, device="cuda") if fp8 else None
    small = make_seqs(lay, [500, 200], [1, 100], 3, spare=0)
    p = Paged(lay, small.pages, 3)
    el = cache.view(lay.elem).view(2, pages, 64, 8, 128)
    for kv in range(2):
        el[kv, pages - small.pages:].copy_(p.layer(0)[kv])
        if fp8:
            scales.view(2, pages, 8)[kv, pages - small.pages:] = p.scale(0, kv)
    q = torch.randn(small.n, 16, 128, device="cuda").to(torch.bfloat16)
    ref = attention64(p, 0, small, q)
    small.table = torch.where(small.table >= 0, small.table + (pages - small.pages), small.table)
    out = torch.zeros_like(q)
    big = gk.Cache(cache, pages, 0, pages * slab, slab, scales, 0, pages * 32 if fp8 else 0, 32 if fp8 else 0)
    with gk.Context(lay.geom(), 0) as ctx:
        ctx.gk_attention(big, 0, batch_of(small), q, out)
    torch.cuda.synchronize()
    check(out, None, ref)


def test_refusals():
    lay = Layout(2, 64, 16)
    sq = make_seqs(lay, [40, 50], [1, 1], 3)
    p = Paged(lay, sq.pages, 3)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device="cuda")
    b = batch_of(sq)

    def refused(code, ctx=None, cache=None, layer=1, batch=b, q=q, out=None, **kw):
        with pytest.raises(gk.GkError) as e:
            ctx.gk_attention(cache or p.cache(), layer, batch, q, torch.zeros_like(q) if out is None else out, **kw)
        assert e.value.code == code

    with gk.Context(lay.geom(), 0) as ctx:
        refused(-1, ctx, layer=2)
        refused(-1, ctx, scale=math.nan)
        refused(-1, ctx, q=torch.zeros(2, 3, 64, dtype=torch.bfloat16, device="cuda"))
        refused(-1, ctx, q=q.float())
        refused(-1, ctx, q=q[:1])
        refused(-1, ctx, out=torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda")[..., ::2])
        refused(-2, ctx, q=torch.zeros(2, 4, 72, dtype=torch.bfloat16, device="cuda")[..., 1:65])
        refused(-1, ctx, lse=torch.zeros(2, 3, device="cuda"))
        with pytest.raises(gk.GkError):
            gk.Batch(sq.table.long(), b.kv_len)
        with pytest.raises(gk.GkError):
            gk.Batch(sq.table, b.kv_len, n_tokens=3)
        with pytest.raises(gk.GkError):
            gk.Batch(sq.table, b.kv_len, b.q_start)
        # no rows at all: nothing to do
        ctx.gk_attention(p.cache(), 1, gk.Batch(sq.table, b.kv_len, torch.zeros(3, dtype=torch.int32, device="cuda"), 0),
                         q[:0], q[:0].clone())
        torch.cuda.synchronize()
    odd = Layout(2, 24, 16)
    with gk.Context(odd.geom(), 0) as ctx:
        refused(-2, ctx, cache=Paged(odd, 8, 3).cache(), q=torch.zeros(2, 4, 24, dtype=torch.bfloat16, device="cuda"))
    far = Layout(1, 272, 16)
    with gk.Context(far.geom(), 0) as ctx:
        refused(-2, ctx, cache=Paged(far, 8, 3).cache(), q=torch.zeros(2, 4, 272, dtype=torch.bfloat16, device="cuda"))
