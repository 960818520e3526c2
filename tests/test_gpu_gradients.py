"""Norm, clipping, gather and scatter of many tensors on the GPU against the definition in 64 bits.

Tolerances.  An L2 norm is summed in fp64 (n terms: relative error below n 2^-53, at most 2^-20 of what follows), its
root is rounded once to fp32: half a step, 2^-24 of the value, or 2^-150 below the normal range.  A maximum is exact.  The
factor c = limit / N is a quotient of fp32 numbers whose divisor is off by 2^-24: 2 * 2^-24; the product adds 2^-24, and the
destination's type half a step: 2^-8 (bf16), 2^-11 (fp16).  Besides, given the norm that the call reports, every output
is one fp32 product and one rounding, which torch's own conversions reproduce bit for bit.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

from test_gpu_parity import dq  # noqa: E402,F401

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_STEP = {F32: 0.0, BF16: 2.0 ** -8, F16: 2.0 ** -11}                  # beyond the product's own rounding
SMALLEST = {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}         # half a step below the normal range
SLACK = 1.0 + 2.0 ** -19
FILL = 0.3125                       # what lies around the tensors; must stay

# (sizes, ...): one launch by one cluster; the whole GPU; more tensors than a table of each size holds
LISTS = {
    "one": [1],
    "few": [1, 2, 7, 8, 9, 31, 255, 256, 257],
    "tiles": [1023, 1024, 1025, 2047, 2048, 2049, 3 * 1024 + 5],
    "empties": [0, 5, 0, 0, 4097, 0],
    "short_most": [(1 << 19) - 8000] + [50] * 159,
    "short_norm": [(1 << 19) - 50 * 127] + [50] * 127,          # the most that one launch takes
    "short_scale": [50] * 100 + [(3 << 17) - 50 * 100],
    "past_short": [3 << 17, 1],
    "tensors_161": [50 + 13 * i % 701 for i in range(161)],
    "tensors_700": [1 + 37 * i % 1500 for i in range(700)],
    "tensors_1900": [1 + 101 * i % 900 if i % 50 else 0 for i in range(1900)],
    "long": [3_000_001, 17, 1_200_000, 333, 2_097_152 + 1],
    "long_one": [5_000_003],
}
ALIGNS = ["own", "side_by_side"]


class Bucket:
    """Tensors in one buffer with sentinel values around each (side by side: only around all), to see what is left alone."""

    def __init__(self, sizes, dtypes, how, offset=0):
        self.parts, self.buffers, at = [], {}, dict.fromkeys(set(dtypes), 16 + offset)
        places = []
        for n, t in zip(sizes, dtypes):
            places.append(at[t])
            at[t] += n if how == "side_by_side" else (n + 16 + 7) // 8 * 8
        self.buffers = {t: torch.full((at[t] + 32,), FILL, dtype=t, device="cuda") for t in at}
        self.mask = {t: torch.ones_like(b, dtype=torch.bool) for t, b in self.buffers.items()}
        for n, t, p in zip(sizes, dtypes, places):
            self.parts.append(self.buffers[t][p:p + n])
            self.mask[t][p:p + n] = False

    def check(self):
        for t, b in self.buffers.items():
            assert bool((b[self.mask[t]] == FILL).all()), f"{t}: something around the tensors was overwritten"


def _dtypes(sizes, which):
    if which == "mixed":
        return [(F32, BF16, F16)[i % 3] for i in range(len(sizes))]
    return [which] * len(sizes)


def _gradients(sizes, dtypes, how="own", seed=0, scale=1.0, offset=0):
    b = Bucket(sizes, dtypes, how, offset)
    g = torch.Generator(device="cuda").manual_seed(seed)
    for i, p in enumerate(b.parts):
        p.copy_(torch.randn(p.numel(), device="cuda", generator=g) * (scale * (0.1 + (i % 7))))
    return b


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy().reshape(-1)


def _norms(arrays, kind):
    if kind == "max":
        each = [float(np.abs(a).max()) if a.size else 0.0 for a in arrays]
        return each, max(each, default=0.0)
    sums = [math.fsum((a * a).tolist()) if a.size < 100_000 else float(np.sum(a.astype(np.longdouble) ** 2)) for a in arrays]
    return [math.sqrt(s) for s in sums], math.sqrt(math.fsum(sums))


def _kind(dq, kind):
    return dq.DQ_NORM_MAX if kind == "max" else dq.DQ_NORM_L2


def _assert_norm(got, want, kind):
    got = float(got)
    if kind == "max":
        assert got == want
    else:
        assert abs(got - want) <= want * 2.0 ** -24 * SLACK + 2.0 ** -150, (got, want)


def _factor(norm, limit):
    """c in fp32 from the reported norm, as the definition has it."""
    norm = np.float32(float(norm))
    limit = np.float32(limit)
    with np.errstate(divide="ignore", invalid="ignore"):
        return np.float32(1.0) if norm <= limit else limit / norm


def _assert_clipped(out, src, norm, limit, want_norm):
    """out: tensors, src: what they were clipped from (copies)."""
    c32 = _factor(norm, limit)
    c64 = 1.0 if want_norm <= limit else float(np.float32(limit)) / want_norm
    for o, s in zip(out, src):
        exactly = (s.float().reshape(-1) * torch.tensor(c32, device=s.device)).to(o.dtype)
        assert torch.equal(o.reshape(-1), exactly)
        x, y = _f64(s) * c64, _f64(o)
        tol = np.abs(x) * (HALF_STEP[o.dtype] + 3 * 2.0 ** -24) * SLACK + SMALLEST[o.dtype] * SLACK + 2.0 ** -149
        assert (np.abs(y - x) <= tol).all()


# ------------------------------------------------------------------------------------------------------ norm
@pytest.mark.parametrize("how", ALIGNS)
@pytest.mark.parametrize("kind", ["l2", "max"])
@pytest.mark.parametrize("which", [F32, BF16, F16, "mixed"], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", LISTS)
def test_norm(dq, name, which, kind, how):
    sizes = LISTS[name]
    b = _gradients(sizes, _dtypes(sizes, which), how, seed=3)
    each, total = _norms([_f64(p) for p in b.parts], kind)
    for with_each in (False, True):
        norms = dq.binding.new_output(len(sizes), F32, "cuda") if with_each else None
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = dq.grad_norm(b.parts, _kind(dq, kind), out_norms=norms, status_word=status)
        _assert_norm(got, total, kind)
        assert int(status) == 0
        if with_each:
            for i, v in enumerate(norms.tolist()):
                _assert_norm(v, each[i], kind)


@pytest.mark.parametrize("offset", range(1, 8))
@pytest.mark.parametrize("which", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
def test_norm_at_every_alignment(dq, which, offset):
    sizes = [1, 7, 8, 9, 100, 1024, 1500]
    for how in ALIGNS:
        b = _gradients(sizes, _dtypes(sizes, which), how, seed=offset, offset=offset)
        for kind in ("l2", "max"):
            _assert_norm(dq.grad_norm(b.parts, _kind(dq, kind)), _norms([_f64(p) for p in b.parts], kind)[1], kind)


@pytest.mark.parametrize("n", [100, 2_000_000])
@pytest.mark.parametrize("scale", [1e-36, 1e-25, 1e18, 1e30, 3e38])
def test_norm_keeps_the_whole_range_of_fp32(dq, n, scale):
    x = torch.rand(n, device="cuda").add_(1e-3).clamp_(max=1.0).mul_(scale)
    each, total = _norms([_f64(x)], "l2")
    norms = torch.empty(1, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = dq.grad_norm([x], out_norms=norms, status_word=status)
    if total > float(np.finfo(np.float32).max):
        assert float(got) == math.inf and float(norms) == math.inf and int(status) == dq.DQ_WARN_NONFINITE_NORM
    else:
        _assert_norm(got, total, "l2")
        _assert_norm(norms, total, "l2")
        assert int(status) == 0


def test_norm_of_subnormal_gradients(dq):
    for t, tiny in ((F32, 2.0 ** -149), (BF16, 2.0 ** -133), (F16, 2.0 ** -24)):
        x = torch.full((5000,), tiny, dtype=t, device="cuda")
        _assert_norm(dq.grad_norm([x]), math.sqrt(5000.0) * tiny, "l2")
        assert float(dq.grad_norm([x], dq.DQ_NORM_MAX)) == tiny


@pytest.mark.parametrize("n", [300, 3_000_000])
@pytest.mark.parametrize("which", [F32, BF16, F16], ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("kind", ["l2", "max"])
def test_nonfinite_gradients(dq, kind, which, n):
    """One Inf or NaN anywhere: the norm is Inf or NaN, the status says so, and only that tensor's own norm is affected."""
    for bad in (math.inf, -math.inf, math.nan):
        for at in (0, n // 2, n - 1):
            g = [torch.ones(50, dtype=which, device="cuda"), torch.ones(n, dtype=which, device="cuda")]
            g[1][at] = bad
            norms = torch.empty(2, device="cuda")
            status = torch.zeros(1, dtype=torch.int32, device="cuda")
            got = float(dq.grad_norm(g, _kind(dq, kind), out_norms=norms, status_word=status))
            assert math.isnan(got) if math.isnan(bad) else got == math.inf
            assert int(status) == dq.DQ_WARN_NONFINITE_NORM
            assert float(norms[0]) == (1.0 if kind == "max" else float(np.float32(math.sqrt(50.0))))
            status.zero_()
            again = float(dq.grad_norm(g, _kind(dq, kind), status_word=status))
            assert again == got or math.isnan(got) and math.isnan(again)
            assert int(status) == dq.DQ_WARN_NONFINITE_NORM
            # NaN poisons what is clipped by it; Inf scales finite elements to 0
            out = [torch.empty_like(x) for x in g]
            status.zero_()
            dq.grad_clip(g, 1.0, out=out, kind=_kind(dq, kind), status_word=status)
            assert int(status) == dq.DQ_WARN_NONFINITE_NORM
            if math.isnan(bad):
                assert all(bool(o.isnan().all()) for o in out)
            else:
                assert bool((out[0] == 0).all()) and bool(out[1][at].isnan())
                assert int(out[1].isnan().sum()) == 1


def test_norms_of_empty_lists(dq):
    for out, call in ((torch.full((1,), 9.0, device="cuda"), dq.grad_norm),):
        call([], out_norm=out)
        assert float(out) == 0.0
    e = torch.empty(0, device="cuda")
    norms = torch.full((3,), 9.0, device="cuda")
    assert float(dq.grad_norm([e, e, e], out_norms=norms)) == 0.0
    assert norms.tolist() == [0.0, 0.0, 0.0]
    assert float(dq.grad_norm([e, e])) == 0.0
    out = torch.full((1,), 9.0, device="cuda")
    dq.grad_clip([e], 1.0, out_norm=out)
    assert float(out) == 0.0
    dq.grad_clip([], 1.0, out_norm=out.fill_(9.0))
    assert float(out) == 0.0
    flat = torch.full((1,), 9.0, device="cuda")
    dq.grad_gather([e], flat, max_norm=1.0, out_norm=out.fill_(9.0))
    assert float(out) == 0.0 and float(flat) == 9.0
    many = [e] * 300                                     # more than a short list's tables hold
    for call in (lambda: dq.grad_norm(many, out_norm=out), lambda: dq.grad_clip(many, 1.0, out=many, out_norm=out),
                 lambda: dq.grad_clip(many, 1.0, out_norm=out), lambda: dq.grad_gather(many, flat, max_norm=1.0, out_norm=out),
                 lambda: dq.grad_scatter(e, many, max_norm=1.0, kind=dq.DQ_NORM_MAX, out_norm=out)):
        out.fill_(9.0)
        call()
        assert float(out) == 0.0
    given = torch.full((1,), 4.0, device="cuda")
    assert float(dq.grad_clip([e], 1.0, norm=given, out_norm=out)) == 4.0


def test_a_norm_is_the_same_every_time(dq):
    sizes = LISTS["long"] + LISTS["tensors_161"]
    b = _gradients(sizes, _dtypes(sizes, "mixed"), "side_by_side", seed=9)
    first = dq.grad_norm(b.parts)
    norms = torch.empty(len(sizes), device="cuda")
    dq.grad_norm(b.parts, out_norms=norms)
    for _ in range(5):
        again = torch.empty_like(norms)
        assert torch.equal(dq.grad_norm(b.parts), first)
        dq.grad_norm(b.parts, out_norms=again)
        assert torch.equal(again, norms)


# ------------------------------------------------------------------------------------------------------ clipping
@pytest.mark.parametrize("how", ALIGNS)
@pytest.mark.parametrize("ratio", [0.3, 1.5])
@pytest.mark.parametrize("kind", ["l2", "max"])
@pytest.mark.parametrize("pair", [(F32, F32), (BF16, BF16), (F16, F32), (BF16, F32), (F32, BF16), (F32, F16), (F16, BF16),
                                  (BF16, F16), (F16, F16), ("mixed", "mixed")], ids=str)
@pytest.mark.parametrize("name", LISTS)
def test_clip_into_other_tensors(dq, name, pair, kind, ratio, how):
    sizes = LISTS[name]
    # the two sides differ in alignment: 1, 3 or 5 elements apart
    b = _gradients(sizes, _dtypes(sizes, pair[0]), how, seed=5, offset=len(sizes) % 4)
    out = Bucket(sizes, _dtypes(sizes, pair[1]), how, offset=(1, 3, 5)[len(sizes) % 3])
    src = [p.clone() for p in b.parts]
    _, total = _norms([_f64(p) for p in src], kind)
    limit = float(np.float32(ratio * total))
    norm = dq.grad_clip(b.parts, limit, out=out.parts, kind=_kind(dq, kind))
    _assert_norm(norm, total, kind)
    _assert_clipped(out.parts, src, norm, limit, total)
    assert all(torch.equal(p, s) for p, s in zip(b.parts, src))
    out.check()
    b.check()


@pytest.mark.parametrize("how", ALIGNS)
@pytest.mark.parametrize("which", [F32, BF16, F16, "mixed"], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", LISTS)
def test_clip_in_place(dq, name, which, how):
    sizes = LISTS[name]
    for ratio in (0.3, 1.5):
        b = _gradients(sizes, _dtypes(sizes, which), how, seed=6, offset=len(sizes) % 5)
        src = [p.clone() for p in b.parts]
        _, total = _norms([_f64(p) for p in src], "l2")
        limit = float(np.float32(ratio * total))
        norm = dq.grad_clip(b.parts, limit)
        _assert_norm(norm, total, "l2")
        _assert_clipped(b.parts, src, norm, limit, total)
        b.check()


@pytest.mark.parametrize("src_at", range(8))
@pytest.mark.parametrize("pair", [(F32, F32), (BF16, F32), (F32, BF16), (F16, F16)], ids=str)
def test_clip_at_every_pair_of_alignments(dq, pair, src_at):
    sizes = [1, 8, 9, 24, 1000, 1500]
    b = _gradients(sizes, _dtypes(sizes, pair[0]), "own", seed=src_at, offset=src_at)
    _, total = _norms([_f64(p) for p in b.parts], "l2")
    for dst_at in range(8):
        out = Bucket(sizes, _dtypes(sizes, pair[1]), "own", offset=dst_at)
        norm = dq.grad_clip(b.parts, 0.5, out=out.parts)
        _assert_clipped(out.parts, b.parts, norm, 0.5, total)
        out.check()


@pytest.mark.parametrize("n", [40, 1_000_000])
def test_clip_by_a_given_norm(dq, n):
    x = torch.randn(n, device="cuda")
    for norm, limit in ((10.0, 1.0), (1.0, 10.0), (0.0, 0.0), (2.0, 0.0), (math.inf, 1.0), (math.inf, math.inf),
                        (math.nan, 1.0), (1.0, math.inf)):
        given = torch.tensor([norm], device="cuda")
        out = [torch.full_like(x, FILL)]
        y = x.clone()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        copy = torch.full((1,), 7.0, device="cuda")
        dq.grad_clip([x], limit, out=out, norm=given, out_norm=copy, status_word=status)
        dq.grad_clip([y], limit, norm=given)
        want = x * torch.tensor(_factor(norm, limit), device="cuda")
        for got in (out[0], y):
            assert torch.equal(got, want) or (math.isnan(norm) and bool(got.isnan().all()))
        assert float(copy) == norm or math.isnan(norm) and math.isnan(float(copy))
        assert int(status) == (0 if math.isfinite(norm) else dq.DQ_WARN_NONFINITE_NORM)


def test_limits_at_the_edge(dq):
    """A norm equal to the limit is not clipped; a limit of 0 scales everything to 0, a zero gradient stays."""
    for n in (5, 1_000_000):
        x = torch.full((n,), 0.5, device="cuda")
        limit = float(dq.grad_norm([x]))
        y = x.clone()
        dq.grad_clip([y], limit)
        assert torch.equal(x, y)
        dq.grad_clip([y], 0.0)
        assert bool((y == 0).all())
        dq.grad_clip([y], 0.0)
        assert bool((y == 0).all())
        dq.grad_clip([x], math.inf)
        assert bool((x == 0.5).all())


# ------------------------------------------------------------------------------------------------------ strides
def _blocks(dtype, rows, widths, total, seed=1, lead=()):
    m = torch.randn(*lead, rows, total, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)
    at, out = 0, []
    for w in widths:
        out.append(m[..., at:at + w])
        at += w
    return m, out


@pytest.mark.parametrize("pair", [(F32, F32), (BF16, BF16), (F16, F32), (F32, BF16)], ids=str)
@pytest.mark.parametrize("shape", [(1, [8, 8], 16), (37, [8, 16, 24], 48), (37, [8, 16, 24], 53), (50, [1, 2, 33, 7], 50),
                                   (3000, [1], 700), (700, [512, 512, 512], 1536), (300, [1000, 999], 2000),
                                   (9, [5000], 9000), (2, [200_000], 300_001), (40, [600, 511, 513], 1624),
                                   (60, [511, 512], 1024), (5, [2041, 2042, 4096], 9001), (1200, [5] * 150, 800)], ids=str)
def test_column_blocks(dq, shape, pair):
    rows, widths, total = shape
    m, blocks = _blocks(pair[0], rows, widths, total)
    before = m.clone()
    ref = [b.contiguous().clone() for b in blocks]          # (a block of one row is contiguous itself)
    _, norm64 = _norms([_f64(b) for b in ref], "l2")
    norms = torch.empty(len(blocks), device="cuda")
    _assert_norm(dq.grad_norm(blocks, out_norms=norms), norm64, "l2")
    for v, r in zip(norms.tolist(), ref):
        _assert_norm(v, _norms([_f64(r)], "l2")[1], "l2")
    limit = float(np.float32(0.5 * norm64))
    # into contiguous tensors
    out = [torch.empty(b.shape, dtype=pair[1], device="cuda") for b in blocks]
    norm = dq.grad_clip(blocks, limit, out=out)
    _assert_clipped(out, ref, norm, limit, norm64)
    # into blocks of another matrix
    to, out = _blocks(pair[1], rows, widths, total + 3, seed=2)
    keep = to.clone()
    norm = dq.grad_clip(blocks, limit, out=out)
    _assert_clipped([o.contiguous() for o in out], ref, norm, limit, norm64)
    assert torch.equal(to[:, sum(widths):], keep[:, sum(widths):])
    # from contiguous tensors into blocks
    to2 = torch.full_like(to, FILL)
    norm = dq.grad_clip(ref, limit, out=_split(to2, widths))
    assert torch.equal(to2[:, :sum(widths)], to[:, :sum(widths)]) and bool((to2[:, sum(widths):] == FILL).all())
    # into the flat vector and back
    flat = dq.grad_gather(blocks, max_norm=limit)
    _assert_clipped([flat], [torch.cat([r.reshape(-1).float() for r in ref])], norm, limit, norm64)
    if pair[0] == F32:
        back = torch.full_like(m, FILL)
        dq.grad_scatter(flat, _split(back, widths))
        assert torch.equal(torch.cat([b.reshape(-1) for b in _split(back, widths)]), flat)
        assert bool((back[:, sum(widths):] == FILL).all())
    assert torch.equal(m, before)
    # in place
    norm = dq.grad_clip(blocks, limit)
    _assert_clipped([b.contiguous() for b in blocks], ref, norm, limit, norm64)
    assert torch.equal(m[:, sum(widths):], before[:, sum(widths):])


def _split(m, widths):
    out, at = [], 0
    for w in widths:
        out.append(m[..., at:at + w])
        at += w
    return out


@pytest.mark.parametrize("which", [F32, BF16], ids=["f32", "bf16"])
def test_more_column_blocks_than_a_table_holds(dq, which):
    widths = [8 + i % 40 for i in range(1100)]
    m, blocks = _blocks(which, 12, widths, sum(widths) + 9, seed=3)
    before, ref = m.clone(), [b.contiguous().clone() for b in blocks]
    _, total = _norms([_f64(b) for b in ref], "l2")
    limit = float(np.float32(0.25 * total))
    norms = torch.empty(len(blocks), device="cuda")
    _assert_norm(dq.grad_norm(blocks, out_norms=norms), total, "l2")
    for v, r in zip(norms.tolist(), ref):
        _assert_norm(v, _norms([_f64(r)], "l2")[1], "l2")
    out = [torch.empty(b.shape, device="cuda") for b in blocks]
    norm = dq.grad_clip(blocks, limit, out=out)
    _assert_norm(norm, total, "l2")
    _assert_clipped(out, ref, norm, limit, total)
    norm = dq.grad_clip(blocks, limit)
    _assert_clipped([b.contiguous() for b in blocks], ref, norm, limit, total)
    assert torch.equal(m[:, sum(widths):], before[:, sum(widths):])


def test_other_layouts(dq):
    g = torch.Generator(device="cuda").manual_seed(4)
    dense = torch.randn(6, 5, 8, 8, device="cuda", generator=g).to(memory_format=torch.channels_last)
    turned = torch.randn(300, 200, device="cuda", generator=g).t()
    batch = torch.randn(4, 30, 64, device="cuda", generator=g)[:, :, 16:48]              # rows at one distance over two axes
    column = torch.randn(500, 3, device="cuda", generator=g)[:, 1]
    single = torch.randn(1, 700, device="cuda", generator=g)[:, 100:200]
    everything = [dense, turned, batch, column, single]
    _, want = _norms([_f64(t) for t in everything], "l2")
    _assert_norm(dq.grad_norm(everything), want, "l2")
    # in place, and into tensors of the same strides, order does not matter
    like = [torch.empty_like(dense), torch.empty(300, 200, device="cuda").t()]
    src = [t.clone() for t in everything]
    norm = dq.grad_clip([dense, turned], 1.0, out=like)
    _assert_clipped([t.contiguous() for t in like], [dense.contiguous(), turned.contiguous()], norm, 1.0,
                    _norms([_f64(dense), _f64(turned)], "l2")[1])
    norm = dq.grad_clip(everything, 1.0)
    _assert_clipped([t.contiguous() for t in everything], [t.contiguous() for t in src], norm, 1.0, want)
    # where it matters, only rows at one distance
    for t in (dense, turned):
        with pytest.raises(TypeError, match="strides"):
            dq.grad_clip([t], 1.0, out=[torch.empty(t.shape, device="cuda")])
        with pytest.raises(TypeError, match="strides"):
            dq.grad_gather([t])
        with pytest.raises(TypeError, match="strides"):
            dq.grad_scatter(torch.zeros(t.numel(), device="cuda"), [t])
    holes = torch.zeros(4, 30, 64, device="cuda")[:, ::2, 16:32][:, :7]
    for t in (holes, torch.zeros(1, device="cuda").expand(8), torch.zeros(16, device="cuda")[::2].view(2, 4)[:, :3],
              torch.zeros(3, 1, device="cuda").expand(3, 4)):
        with pytest.raises(TypeError, match="strides"):
            dq.grad_norm([t])
    with pytest.raises(ValueError, match="shape"):
        dq.grad_clip([torch.zeros(4, 6, device="cuda")], 1.0, out=[torch.zeros(6, 4, device="cuda")])
    with pytest.raises(ValueError, match="each"):
        dq.grad_clip([column], 1.0, out=[])
    with pytest.raises(dq.DqError):
        dq.grad_clip([column, column], 1.0)
    with pytest.raises(dq.DqError):
        dq.grad_clip([column], 1.0, out=[column])
    with pytest.raises(dq.DqError):
        dq.grad_clip([column], -1.0)
    with pytest.raises(ValueError, match="elements"):
        dq.grad_gather([column], torch.empty(501, device="cuda"))
    with pytest.raises(ValueError, match="small"):
        dq.grad_gather([column], torch.empty(499, device="cuda"))
    with pytest.raises(ValueError, match="max_norm"):
        dq.grad_gather([column], norm=torch.ones(1, device="cuda"))
    with pytest.raises(TypeError):
        dq.grad_norm([torch.zeros(4)])
    with pytest.raises(TypeError):
        dq.grad_clip([column], None)


# ------------------------------------------------------------------------------------------------------ flat vector
@pytest.mark.parametrize("how", ALIGNS)
@pytest.mark.parametrize("which", [F32, BF16, F16, "mixed"], ids=["f32", "bf16", "f16", "mixed"])
@pytest.mark.parametrize("name", LISTS)
def test_gather_and_scatter(dq, name, which, how):
    sizes = LISTS[name]
    b = _gradients(sizes, _dtypes(sizes, which), how, seed=8, offset=len(sizes) % 3)
    src = torch.cat([p.float() for p in b.parts])
    assert torch.equal(dq.grad_gather(b.parts), src)
    for kind in ("l2", "max"):
        _, total = _norms([_f64(p) for p in b.parts], kind)
        limit = float(np.float32(0.4 * total))
        norm = torch.empty(1, device="cuda")
        flat = dq.grad_gather(b.parts, max_norm=limit, kind=_kind(dq, kind), out_norm=norm)
        _assert_norm(norm, total, kind)
        _assert_clipped([flat], [src], norm, limit, total)
        out = Bucket(sizes, _dtypes(sizes, which), how, offset=2)
        norm2 = torch.empty(1, device="cuda")
        got = dq.grad_scatter(src, out.parts, max_norm=limit, kind=_kind(dq, kind), out_norm=norm2)
        assert got is out.parts
        _assert_norm(norm2, total, kind)
        _assert_clipped(out.parts, src.split(sizes), norm2, limit, total)
        out.check()
    # unclipped, there and back: the same bits
    out = Bucket(sizes, _dtypes(sizes, which), how, offset=1)
    dq.grad_scatter(src, out.parts)
    assert all(torch.equal(p, q) for p, q in zip(out.parts, b.parts))
    out.check()


# ------------------------------------------------------------------------------------------------------ large offsets
def test_offsets_beyond_32_bits(dq):
    """A bf16 tensor of more than 2^32 elements: the last ones count, are scaled, and nothing behind them is touched."""
    n = (1 << 32) + 13
    buf = torch.zeros(n + 64, dtype=BF16, device="cuda")
    x = buf[3:3 + n]
    x[-1], x[-9], x[5], x[1 << 31] = 4.0, 3.0, 2.0, 1.0
    buf[3 + n:] = FILL
    assert float(dq.grad_norm([x], dq.DQ_NORM_MAX)) == 4.0
    norms = torch.empty(1, device="cuda")
    _assert_norm(dq.grad_norm([x], out_norms=norms), math.sqrt(30.0), "l2")
    _assert_norm(norms, math.sqrt(30.0), "l2")
    dq.grad_clip([x], 1.0, kind=dq.DQ_NORM_MAX)
    assert [float(x[-1]), float(x[-9]), float(x[5]), float(x[1 << 31])] == [1.0, 0.75, 0.5, 0.25]
    assert int(torch.count_nonzero(x)) == 4
    assert bool((buf[3 + n:] == FILL).all()) and bool((buf[:3] == 0).all())
    # column blocks of a matrix whose rows lie further apart than 2^32 elements together
    m = buf[:1 << 32].view(1 << 16, 1 << 16)
    m.zero_()
    block = m[:, 100:108]
    block[-1, 7], block[0, 0] = 3.0, 4.0
    _assert_norm(dq.grad_norm([block]), 5.0, "l2")
    flat = dq.grad_gather([block], max_norm=2.5)
    assert float(flat[-1]) == 1.5 and float(flat[0]) == 2.0 and int(torch.count_nonzero(flat)) == 2


# ------------------------------------------------------------------------------------------------------ streams, graphs
def test_a_call_on_a_side_stream(dq):
    sizes = LISTS["long"]
    b = _gradients(sizes, _dtypes(sizes, F32), seed=11)
    want = dq.grad_gather(b.parts, max_norm=1.0).clone()
    norm = dq.grad_norm(b.parts).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)                       # the current stream is busy; the calls do not wait for it
    flat = dq.grad_gather(b.parts, max_norm=1.0, stream=side)
    got = dq.grad_norm(b.parts, stream=side)
    with torch.cuda.stream(side):
        early = flat.cpu(), got.cpu()
    torch.cuda.synchronize()
    assert torch.equal(early[0], want.cpu()) and torch.equal(early[1], norm.cpu())


def test_two_streams_at_once(dq):
    """Calls that overlap in time have a workspace each."""
    sizes = LISTS["long"]
    lists = [_gradients(sizes, _dtypes(sizes, F32), seed=20 + i).parts for i in range(2)]
    want = [dq.grad_norm(g).clone() for g in lists]
    streams = [torch.cuda.Stream() for _ in lists]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(30):
        for i, (g, s) in enumerate(zip(lists, streams)):
            got[i].append(dq.grad_norm(g, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_captured_calls_replay(dq):
    """Two graphs in turn, on new values each time: nothing is kept from the capture but the addresses."""
    graphs, states = [], []
    side = torch.cuda.Stream()
    for k, name in enumerate(["long", "few", "tensors_700"]):
        sizes = LISTS[name]
        b = _gradients(sizes, _dtypes(sizes, "mixed"), seed=k)
        flat, out = torch.empty(sum(sizes), device="cuda"), Bucket(sizes, _dtypes(sizes, "mixed"), "own")
        norm, norms = torch.empty(1, device="cuda"), torch.empty(len(sizes), device="cuda")

        def step(b=b, flat=flat, out=out, norm=norm, norms=norms):
            dq.grad_norm(b.parts, out_norm=norm, out_norms=norms)
            dq.grad_gather(b.parts, flat, max_norm=1.0)
            dq.grad_scatter(flat, out.parts, max_norm=0.5)

        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        graphs.append(graph)
        states.append((b, flat, out, norm, norms))
    for turn in range(3):
        for b, flat, out, norm, norms in states:
            for p in b.parts:
                p.mul_(1.0 + turn).add_(0.01)
            flat.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for b, flat, out, norm, norms in states:
            each, total = _norms([_f64(p) for p in b.parts], "l2")
            _assert_norm(norm, total, "l2")
            assert torch.equal(flat, dq.grad_gather(b.parts, max_norm=1.0))
            again = Bucket([p.numel() for p in b.parts], [p.dtype for p in b.parts], "own")
            dq.grad_scatter(flat, again.parts, max_norm=0.5)
            assert all(torch.equal(x, y) for x, y in zip(out.parts, again.parts))
            out.check()


def test_calls_back_to_back_see_each_other(dq):
    """A kernel may start while its predecessor drains; it must not read what that one has not written."""
    sizes = [200_000, 3, 65_536, 1001]
    b = _gradients(sizes, _dtypes(sizes, F32), seed=2)
    flat = torch.empty(sum(sizes), device="cuda")
    back = [torch.empty_like(p) for p in b.parts]
    norms = []
    limit = 1.0
    for i in range(40):
        dq.grad_gather(b.parts, flat, max_norm=limit)
        dq.grad_scatter(flat, back, max_norm=limit / 2)
        norms.append(dq.grad_norm(back))
        dq.grad_clip(back, limit / 4)
        norms.append(dq.grad_norm(back))
        for p in b.parts:
            p.add_(0.001)
    for i, n in enumerate(norms):
        want = limit / 2 if i % 2 == 0 else limit / 4
        assert abs(float(n) - want) <= want * 1e-6


def test_autograd_sees_that_a_tensor_was_written(dq):
    w = torch.randn(100, device="cuda", requires_grad=True)
    y = w * w
    z = y.exp()                                         # saves its result
    with torch.no_grad():
        dq.grad_clip([z], 0.5)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.sum().backward()
    flat = torch.zeros(100, device="cuda")
    v = flat._version
    dq.grad_gather([w.detach()], flat)
    assert flat._version > v


# ------------------------------------------------------------------------------------------------------ the whole step
@pytest.mark.parametrize("n_scale", [1, 40])
def test_a_training_step(dq, n_scale):
    """Lists of W workers, gathered and clipped, encoded, decoded to the mean, scattered and clipped into the model's
    tensors: against the same step on vectors that torch prepares."""
    sizes = [n_scale * m for m in (3001, 17, 8192, 40_000, 1)]
    dtypes = _dtypes(sizes, "mixed")
    W, step, bucket = 4, 3, 512
    pd = dq.DqParams(bucket, 3, 5)
    pn = dq.DqParams(bucket, 2, 0, 4, 2.0, 1.0)
    n = sum(sizes)
    msgs, want_msgs, keep = [], [], []
    for w in range(W):
        b = _gradients(sizes, dtypes, "side_by_side", seed=7)
        for p in b.parts:
            p.add_(torch.randn(p.numel(), device="cuda").to(p.dtype) * 0.05)
        encode = dq.dqsg_encode if w == 0 else dq.ndqsg_encode
        params, kind = (pd, dq.DQ_KIND_DQSG) if w == 0 else (pn, dq.DQ_KIND_NDQSG)
        norm = torch.empty(1, device="cuda")
        flat = dq.grad_gather(b.parts, max_norm=1.0, out_norm=norm)
        msgs.append(dq.Message(*encode(flat, 50 + w, w, step, params), 50 + w, w, kind, params))
        plain = torch.cat([p.float() for p in b.parts]) * torch.tensor(_factor(norm, 1.0), device="cuda")
        assert torch.equal(flat, plain)
        want_msgs.append(dq.Message(*encode(plain, 50 + w, w, step, params), 50 + w, w, kind, params))
        keep.append((b, flat, plain))
    mean = dq.ndqsg_decode_aggregate_side_first(msgs, n, step)
    want = dq.ndqsg_decode_aggregate_side_first(want_msgs, n, step)
    assert torch.equal(mean, want)
    model = Bucket(sizes, dtypes, "own")
    norm = torch.empty(1, device="cuda")
    dq.grad_scatter(mean[:n], model.parts, max_norm=0.5, out_norm=norm)
    _, total = _norms([_f64(want[:n])], "l2")
    _assert_norm(norm, total, "l2")
    _assert_clipped(model.parts, want[:n].split(sizes), norm, 0.5, total)
    model.check()


@pytest.mark.parametrize("nested", [False, True])
def test_clipping_a_message_clips_its_gradient(dq, nested):
    """A bucket scale is linear in the gradient.  With a factor that is a power of two no rounding is involved: the
    codes are the same and the scales differ by the factor."""
    p = dq.DqParams(512, 2, 0, 4, 4.0, 1.0) if nested else dq.DqParams(512, 3, 7)
    encode = dq.ndqsg_encode if nested else dq.dqsg_encode
    g = torch.randn(100_003, device="cuda")
    norm = torch.full((1,), 8.0, device="cuda")
    packed, scale = encode(g, 1, 0, 0, p)
    dq.grad_clip([scale], 2.0, norm=norm)
    clipped = g.clone()
    dq.grad_clip([clipped], 2.0, norm=norm)
    want_packed, want_scale = encode(clipped, 1, 0, 0, p)
    assert torch.equal(clipped, g * 0.25)
    assert torch.equal(packed, want_packed) and torch.equal(scale, want_scale)


# ------------------------------------------------------------------------------------------------------ random lists
def _random_tensor(rng, g):
    """(tensor, buffer around it): contiguous at any address, or a block of a matrix."""
    dtype = rng.choice([F32, BF16, F16])
    if rng.random() < 0.6:
        n = rng.choice([0, 1, rng.randint(1, 40), rng.randint(1, 3000), rng.randint(1, 60_000), rng.randint(1, 700_000)])
        at = rng.randint(0, 17)
        buf = torch.randn(at + n + 20, device="cuda", generator=g).to(dtype)
        return buf[at:at + n], buf
    rows, row = rng.randint(1, 60), rng.choice([rng.randint(1, 30), 8 * rng.randint(1, 200), rng.randint(1, 5000)])
    left, right = rng.choice([(0, 0), (8, 16), (rng.randint(0, 9), rng.randint(0, 9))])
    buf = torch.randn(rows, left + row + right, device="cuda", generator=g).to(dtype)
    return buf[:, left:left + row], buf


def _around(t, buf):
    """What of buf is not t's, as one tensor (t is a view of buf)."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask.as_strided(t.shape, t.stride(), t.storage_offset()).fill_(False)
    return buf[mask]


@pytest.mark.parametrize("seed", range(60))
def test_random_lists(dq, seed):
    import random
    rng = random.Random(seed)
    g = torch.Generator(device="cuda").manual_seed(seed)
    pairs = [_random_tensor(rng, g) for _ in range(rng.choice([1, 2, 5, 20, 90]))]
    grads = [t for t, _ in pairs]
    src = [t.contiguous().clone() for t in grads]
    kind = rng.choice(["l2", "max"])
    each, total = _norms([_f64(t) for t in src], kind)
    norms = dq.binding.new_output(len(grads), F32, "cuda")
    got = dq.grad_norm(grads, _kind(dq, kind), out_norms=norms)
    _assert_norm(got, total, kind)
    _assert_norm(dq.grad_norm(grads, _kind(dq, kind)), total, kind)
    for v, w in zip(norms.tolist(), each):
        _assert_norm(v, w, kind)
    limit = float(np.float32(rng.choice([0.2, 0.9, 1.5]) * total))
    # gather, and scatter of what was gathered into tensors of the same layouts
    norm = torch.empty(1, device="cuda")
    flat = dq.grad_gather(grads, max_norm=limit, kind=_kind(dq, kind), out_norm=norm)
    n = sum(t.numel() for t in grads)
    _assert_norm(norm, total, kind)
    _assert_clipped([flat[:n]], [torch.cat([s.float().reshape(-1) for s in src])], norm, limit, total)
    targets = [(b.clone(), t) for t, b in pairs]
    out = [c.as_strided(t.shape, t.stride(), t.storage_offset()) for c, t in targets]
    before = [_around(o, c).clone() for o, (c, _) in zip(out, targets)]
    dq.grad_scatter(flat[:n], out)
    for o, p in zip(out, flat[:n].split([t.numel() for t in grads])):
        assert torch.equal(o.reshape(-1), p.to(o.dtype))
    for o, (c, _), b in zip(out, targets, before):
        assert torch.equal(_around(o, c), b)
    # clipped into contiguous tensors of any type, and in place
    to = [torch.empty(t.shape, dtype=rng.choice([F32, BF16, F16]), device="cuda") for t in grads]
    norm = dq.grad_clip(grads, limit, out=to, kind=_kind(dq, kind))
    _assert_clipped(to, src, norm, limit, total)
    before = [_around(t, b).clone() for t, b in pairs]
    norm = dq.grad_clip(grads, limit, kind=_kind(dq, kind))
    _assert_clipped([t.contiguous() for t in grads], src, norm, limit, total)
    for (t, b), w in zip(pairs, before):
        assert torch.equal(_around(t, b), w)


def test_empty_tensors_gather_into_an_empty_vector_and_back(dq):
    e = [torch.empty(0, device="cuda"), torch.empty(0, 5, dtype=BF16, device="cuda")]
    norm = torch.full((1,), 9.0, device="cuda")
    for kw in ({}, dict(max_norm=1.0, out_norm=norm)):
        flat = dq.grad_gather(e, **kw)
        assert flat.numel() == 0 and flat.dtype == F32 and flat.is_cuda
        dq.grad_scatter(flat, e, **kw)
    assert float(norm) == 0.0


def _described(dq, tensors):
    kinds = {F32: dq.DQ_F32, BF16: dq.DQ_BF16, F16: dq.DQ_F16}
    return (dq.DqTensor * len(tensors))(*[dq.DqTensor(t.data_ptr(), t.numel(), 0, 0, kinds[t.dtype], 0) for t in tensors])


@pytest.mark.parametrize("call", ["norms", "gather_many"])
def test_an_encode_that_stores_early_may_have_the_memory_of_the_workspace(dq, call):
    """The workspace of a call goes back to the allocator when the call returns; an encode whose flags let it store before
    its predecessor is complete may be handed that memory for its message."""
    flags = dq.DQ_FLAG_INPUT_READY | dq.DQ_FLAG_OUTPUT_FREE
    sizes = [1500] * 2000 if call == "gather_many" else [40_000] * 300
    b = _gradients(sizes, _dtypes(sizes, F32), seed=12)
    src = torch.cat(b.parts)
    ws = int(dq.lib().dq_grad_workspace_bytes(_described(dq, b.parts), len(sizes), 1 if call == "norms" else 0))
    assert ws > 0
    n, plain, early = 16 * (ws // 4) - 5, dq.DqParams(512, 2, 3), dq.DqParams(512, 2, 3, 0, 0.0, 0.0, 0, flags)
    g = torch.randn(n, device="cuda")
    packed = torch.empty(dq.packed_words(n, 2), dtype=torch.int32, device="cuda")
    scale = torch.empty(dq.num_buckets(n, 512), device="cuda")
    dq.dqsg_encode(g, 5, 0, 1, plain, packed, scale)
    want_packed, want_scale = packed.clone(), scale.clone()
    norms, flat = torch.empty(len(sizes), device="cuda"), torch.empty(sum(sizes), device="cuda")
    norm = torch.empty(1, device="cuda")
    dq.grad_norm(b.parts, out_norm=norm, out_norms=norms)
    want_norm, want_norms = norm.clone(), norms.clone()
    want_flat = src * torch.tensor(_factor(norm, 1.0), device="cuda")
    shared = 0
    for _ in range(20):
        norms.zero_()
        flat.zero_()
        scale.zero_()
        probe = torch.empty(ws, dtype=torch.uint8, device="cuda")
        at = probe.data_ptr()
        del probe
        if call == "norms":
            dq.grad_norm(b.parts, out_norm=norm, out_norms=norms)
        else:
            dq.grad_gather(b.parts, flat, max_norm=1.0)
        message = torch.empty(ws // 4, dtype=torch.int32, device="cuda")             # (nothing is enqueued by this)
        shared += message.data_ptr() == at
        dq.dqsg_encode(g, 5, 0, 1, early, message, scale)
        torch.cuda.synchronize()
        assert torch.equal(message[:want_packed.numel()], want_packed) and torch.equal(scale, want_scale)
        if call == "norms":
            assert torch.equal(norm, want_norm) and torch.equal(norms, want_norms)
        else:
            assert torch.equal(flat, want_flat)
        del message
    assert shared == 20


def test_every_output_is_marked_as_written_and_none_of_a_refused_call(dq):
    x, y, z = (torch.ones(100, device="cuda") for _ in range(3))
    flat, norms = torch.ones(200, device="cuda"), torch.ones(2, device="cuda")
    norm, status = torch.ones(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    everything = dict(x=x, y=y, z=z, flat=flat, norms=norms, norm=norm, status=status)
    words = dict(out_norm=norm, status_word=status)

    def written(call):
        before = {k: t._version for k, t in everything.items()}
        try:
            call()
        except dq.DqError:
            assert all(t._version == before[k] for k, t in everything.items())
            return "refused"
        return sorted(k for k, t in everything.items() if t._version > before[k])

    assert written(lambda: dq.grad_norm([x, y], out_norms=norms, **words)) == ["norm", "norms", "status"]
    assert written(lambda: dq.grad_norm([x, y], out_norm=norm)) == ["norm"]
    assert written(lambda: dq.grad_clip([x, y], 1.0, **words)) == ["norm", "status", "x", "y"]
    assert written(lambda: dq.grad_clip([x], 1.0, out=[z], norm=norm, status_word=status)) == ["status", "z"]
    assert written(lambda: dq.grad_gather([x, y], flat, max_norm=1.0, **words)) == ["flat", "norm", "status"]
    assert written(lambda: dq.grad_scatter(flat, [x, y], max_norm=1.0, **words)) == ["norm", "status", "x", "y"]
    assert written(lambda: dq.grad_gather([x, y], flat)) == ["flat"]
    assert written(lambda: dq.grad_scatter(flat, [x, y])) == ["x", "y"]
    # refused by the library
    assert written(lambda: dq.grad_norm([x, y], 7, out_norms=norms, **words)) == "refused"
    assert written(lambda: dq.grad_clip([x, x], 1.0, **words)) == "refused"
    assert written(lambda: dq.grad_clip([x, y], -1.0, **words)) == "refused"
    assert written(lambda: dq.grad_clip([x], 1.0, out=[x], **words)) == "refused"
    assert written(lambda: dq.grad_gather([flat[:100], y], flat, **words, max_norm=1.0)) == "refused"
    assert written(lambda: dq.grad_scatter(flat, [flat[:100], y])) == "refused"


def test_inference_tensors_are_written_in_inference_mode_only(dq):
    with torch.inference_mode():
        t = torch.full((4,), 3.0, device="cuda")
        dq.grad_clip([t], 1.0)
        assert t.tolist() == [0.5] * 4
        norm = dq.grad_norm([t])
    flat = dq.grad_gather([t])                          # (read at any time)
    assert flat.tolist() == [0.5] * 4
    for call in (lambda: dq.grad_clip([t], 0.1), lambda: dq.grad_scatter(flat, [t]), lambda: dq.grad_norm([flat], out_norm=norm),
                 lambda: dq.grad_gather([flat], t)):
        with pytest.raises(RuntimeError, match="inference"):
            call()
    assert t.tolist() == [0.5] * 4 and float(norm) == 1.0


# ------------------------------------------------------------------------------------------------------ the largest lists
@pytest.mark.parametrize("count", [8000, 8001, 20_000, 65_536])
def test_lists_of_thousands(dq, count):
    """Up to the most tensors of a call: several launches of every kernel, contiguous tensors and blocks of one matrix."""
    g = torch.Generator(device="cuda").manual_seed(count)
    whole = torch.randn(count, 7, device="cuda", generator=g)
    each = dq.binding.new_output(count, F32, "cuda")

    def check_norms(tensors, values):
        total = dq.grad_norm(tensors, out_norms=each)
        want = values.double().square().sum(1)
        assert bool(((each.double() - want.sqrt()).abs() <= want.sqrt() * 2.0 ** -24 * SLACK).all())
        _assert_norm(total, math.sqrt(math.fsum(want.tolist())), "l2")
        assert torch.equal(dq.grad_norm(tensors, dq.DQ_NORM_MAX, out_norms=each), values.abs().max().reshape(1))
        assert torch.equal(each, values.abs().amax(1))
        return total

    tensors = list(whole.unbind(0))
    total = check_norms(tensors, whole)
    c = torch.tensor(_factor(total, 0.5), device="cuda")
    norm = torch.empty(1, device="cuda")
    flat = dq.grad_gather(tensors, max_norm=0.5, out_norm=norm)
    assert torch.equal(flat, whole.reshape(-1) * torch.tensor(_factor(norm, 0.5), device="cuda"))
    assert torch.equal(dq.grad_gather(tensors, max_norm=0.5, norm=total), whole.reshape(-1) * c)
    half = torch.empty(count, 7, dtype=BF16, device="cuda")
    dq.grad_scatter(flat, list(half.unbind(0)), max_norm=0.25, out_norm=norm)
    assert torch.equal(half.reshape(-1), (flat * torch.tensor(_factor(norm, 0.25), device="cuda")).to(BF16))
    before = whole.clone()
    norm = dq.grad_clip(tensors, 0.125)
    assert torch.equal(whole, before * torch.tensor(_factor(norm, 0.125), device="cuda"))

    matrix = torch.randn(5, count * 9, device="cuda", generator=g)
    blocks = [matrix[:, 9 * i:9 * i + 8] for i in range(count)]
    inside = matrix.clone().view(5, count, 9)[:, :, :8].transpose(0, 1)
    check_norms(blocks, inside.reshape(count, 40))
    assert torch.equal(dq.grad_gather(blocks), inside.reshape(-1))
    want = matrix.clone()
    norm = dq.grad_clip(blocks, 1.0)
    want.view(5, count, 9)[:, :, :8] *= torch.tensor(_factor(norm, 1.0), device="cuda")
    assert torch.equal(matrix, want)


def test_gather_and_scatter_beyond_32_bits(dq):
    n = (1 << 32) + 13
    buf = torch.zeros(n + 64, dtype=BF16, device="cuda")
    x, y = buf[3:3 + n], torch.tensor([9.0, 10.0], device="cuda")
    spots = [0, 5, 1 << 31, (1 << 31) + 1, (1 << 32) - 1, 1 << 32, n - 9, n - 1]
    for i, s in enumerate(spots):
        x[s] = float(i + 1)
    flat = torch.full((n + 2,), FILL, device="cuda")
    norm = torch.empty(1, device="cuda")
    dq.grad_gather([x, y], flat, max_norm=5.0, kind=dq.DQ_NORM_MAX, out_norm=norm)
    assert float(norm) == 10.0
    want = [0.5 * (i + 1) for i in range(8)]
    assert [float(flat[s]) for s in spots] == want and flat[n:].tolist() == [4.5, 5.0]
    assert int(torch.count_nonzero(flat)) == 10
    buf.fill_(FILL)
    back = torch.zeros(2, device="cuda")
    dq.grad_scatter(flat, [x, back])
    assert [float(x[s]) for s in spots] == want and back.tolist() == [4.5, 5.0]
    assert int(torch.count_nonzero(x)) == 8
    assert bool((buf[:3] == FILL).all()) and bool((buf[3 + n:] == FILL).all())
