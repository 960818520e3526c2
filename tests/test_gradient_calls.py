"""Calls on gradients of many tensors, without a GPU: what the C ABI refuses before it launches anything, what the binding
refuses, and the sizes of the workspace."""
import ctypes as C
import os
import subprocess
import sys
from pathlib import Path

import pytest

torch = pytest.importorskip("torch")

OK, INVALID, UNSUPPORTED, ALIGNMENT = 0, 1, 2, 3
BASE = 0x100000                     # never dereferenced: checks come first
MANY = 1 << 20                      # elements: more than one launch takes, so that a workspace is needed


@pytest.fixture(scope="module")
def dq():
    from paper_1904_01197_b200 import build
    build.build()
    import paper_1904_01197_b200 as dq
    return dq


def _list(dq, *tensors):
    return (dq.DqTensor * max(1, len(tensors)))(*tensors)


def _t(dq, data=BASE, n=MANY, row=0, stride=0, dtype=0, reserved=0):
    return dq.DqTensor(data, n, row, stride, dtype, reserved)


def _clip(dq, max_norm=1.0, kind=0, norm=None, out_norm=0x40, status=None):
    return C.byref(dq.DqClip(max_norm, kind, norm, out_norm, status))


WS = dict(ws=0x200, bytes=1 << 30)


def test_struct_layout_matches_header(dq):
    assert C.sizeof(dq.DqTensor) == 40 and dq.DqTensor.dtype.offset == 32
    assert C.sizeof(dq.DqClip) == 32 and dq.DqClip.norm.offset == 8


BAD_TENSORS = [
    (dict(dtype=3), INVALID),
    (dict(dtype=-1), INVALID),
    (dict(reserved=1), INVALID),
    (dict(data=None), INVALID),
    (dict(n=1 << 34), UNSUPPORTED),
    (dict(data=BASE + 2), ALIGNMENT),                       # fp32 at an address of two bytes
    (dict(data=BASE + 1, dtype=1), ALIGNMENT),
    (dict(row=3), INVALID),                                 # no whole number of rows
    (dict(row=1024, stride=1023), INVALID),                 # rows that overlap
    (dict(row=1024, stride=0), INVALID),
    (dict(n=1 << 33, row=1 << 31, stride=(1 << 31) + 1), UNSUPPORTED),
    (dict(row=1024, stride=1 << 32), UNSUPPORTED),
    (dict(n=1 << 33, row=2, stride=(1 << 32) - 1), UNSUPPORTED),     # further apart than addresses go
    (dict(data=1 << 57), UNSUPPORTED),
]


@pytest.mark.parametrize("kw,want", BAD_TENSORS, ids=[str(k) for k, _ in BAD_TENSORS])
def test_a_bad_tensor_is_refused_by_every_call(dq, kw, want):
    L = dq.lib()
    before = L.dq_launch_count()
    bad, good = _list(dq, _t(dq, data=BASE << 8), _t(dq, **kw)), _list(dq, _t(dq, data=BASE << 8), _t(dq, data=BASE << 12))
    flat = BASE << 16
    assert L.dq_grad_norm(bad, 2, 0, 0x40, None, None, WS["ws"], WS["bytes"], None) == want
    assert L.dq_grad_clip(bad, 2, _clip(dq), None, WS["ws"], WS["bytes"], None) == want
    assert L.dq_grad_clip(good, 2, _clip(dq), bad, WS["ws"], WS["bytes"], None) == want
    assert L.dq_grad_gather(bad, 2, _clip(dq), flat, WS["ws"], WS["bytes"], None) == want
    assert L.dq_grad_gather(bad, 2, None, flat, None, 0, None) == want
    assert L.dq_grad_scatter(flat, _clip(dq), bad, 2, WS["ws"], WS["bytes"], None) == want
    assert L.dq_grad_workspace_bytes(bad, 2, 0) == 0
    assert L.dq_launch_count() == before


def test_bad_arguments_are_refused(dq):
    L = dq.lib()
    before = L.dq_launch_count()
    one = _list(dq, _t(dq))
    norm = lambda *a: L.dq_grad_norm(*a, WS["ws"], WS["bytes"], None)                            # noqa: E731
    assert norm(None, 1, 0, 0x40, None, None) == INVALID
    assert norm(one, 1, 2, 0x40, None, None) == INVALID                                         # kind
    assert norm(one, 1, 0, None, None, None) == INVALID                                         # no place for the norm
    assert norm(one, 1, 0, 0x42, None, None) == ALIGNMENT
    assert norm(one, 1, 0, 0x40, 0x42, None) == ALIGNMENT
    assert norm(one, 1, 0, 0x40, None, 0x41) == ALIGNMENT
    assert norm(one, 65537, 0, 0x40, None, None) == UNSUPPORTED
    assert norm(_list(dq, _t(dq, n=(1 << 34) - 4), _t(dq, n=4)), 2, 0, 0x40, None, None) == UNSUPPORTED    # together
    clip = lambda c, out=None: L.dq_grad_clip(one, 1, c, out, WS["ws"], WS["bytes"], None)      # noqa: E731
    assert clip(None) == INVALID
    assert clip(_clip(dq, -1.0)) == INVALID
    assert clip(_clip(dq, float("nan"))) == INVALID
    assert clip(_clip(dq, kind=7)) == INVALID
    assert clip(_clip(dq, norm=0x82)) == ALIGNMENT
    assert clip(_clip(dq, out_norm=0x42)) == ALIGNMENT
    assert clip(_clip(dq), _list(dq, _t(dq, data=BASE << 8, n=MANY - 1))) == INVALID            # another size
    a, b = _list(dq, _t(dq, row=1024, stride=2048)), _list(dq, _t(dq, data=BASE << 8, row=512, stride=2048))
    assert L.dq_grad_clip(a, 1, _clip(dq), b, WS["ws"], WS["bytes"], None) == UNSUPPORTED       # rows of two lengths
    for ws, size, want in ((None, 1 << 30, INVALID), (0x200, 16, INVALID), (0x208, 1 << 30, ALIGNMENT)):
        assert L.dq_grad_norm(one, 1, 0, 0x40, None, None, ws, size, None) == want
        assert L.dq_grad_clip(one, 1, _clip(dq), None, ws, size, None) == want
        assert L.dq_grad_gather(one, 1, _clip(dq), BASE << 8, ws, size, None) == want
        assert L.dq_grad_scatter(BASE << 8, _clip(dq), one, 1, ws, size, None) == want
    assert L.dq_grad_gather(one, 1, None, None, None, 0, None) == INVALID
    assert L.dq_grad_gather(one, 1, None, (BASE << 8) + 4, None, 0, None) == ALIGNMENT
    assert L.dq_grad_scatter(None, None, one, 1, None, 0, None) == INVALID
    assert L.dq_grad_scatter((BASE << 8) + 8, None, one, 1, None, 0, None) == ALIGNMENT
    assert L.dq_launch_count() == before


def _clip_status(dq, tensors, out=None, clip=None):
    """The status of a call whose only fault can be an overlap: a workspace that is too small is found after it."""
    L = dq.lib()
    a = _list(dq, *tensors)
    return L.dq_grad_clip(a, len(tensors), clip or _clip(dq), None if out is None else _list(dq, *out), 0x208, 1 << 30, None)


NO_OVERLAP = ALIGNMENT              # of the workspace, which is checked last


def test_tensors_that_overlap_are_refused(dq):
    t = lambda at, n=MANY, **kw: _t(dq, data=BASE + at, n=n, **kw)                               # noqa: E731
    size = 4 * MANY
    far = 1 << 30
    assert _clip_status(dq, [t(0), t(size)]) == NO_OVERLAP
    assert _clip_status(dq, [t(size), t(0)]) == NO_OVERLAP
    assert _clip_status(dq, [t(0), t(0)]) == INVALID                                             # the same one twice
    assert _clip_status(dq, [t(0), t(size), t(size - 4)]) == INVALID
    assert _clip_status(dq, [t(0, n=0), t(0), t(64, n=0)]) == NO_OVERLAP                         # empty ones overlap nothing
    assert _clip_status(dq, [t(0), t(64, n=16)]) == INVALID                                      # one inside another
    # inputs may overlap each other, outputs nothing
    assert _clip_status(dq, [t(0), t(0)], [t(far), t(far + size)]) == NO_OVERLAP
    assert _clip_status(dq, [t(0), t(0)], [t(far), t(far)]) == INVALID
    assert _clip_status(dq, [t(0)], [t(size - 4)]) == INVALID
    assert _clip_status(dq, [t(0)], [t(0)]) == INVALID
    # an input that reaches over two outputs behind it
    assert _clip_status(dq, [t(0, n=4 * MANY), t(far)], [t(8 * size, n=4 * MANY), t(size)]) == INVALID
    # column blocks of one matrix lie side by side; one that is a column too wide does not
    block = lambda col, row=1024, stride=3000: t(4 * col, row=row, stride=stride)               # noqa: E731
    assert _clip_status(dq, [block(0), block(1024), block(2048, row=512)]) == NO_OVERLAP
    assert _clip_status(dq, [block(0), block(1023)]) == INVALID
    assert _clip_status(dq, [block(1024), block(0, row=2048)]) == INVALID
    assert _clip_status(dq, [block(0), block(2048)]) == INVALID                                  # into the next row
    assert _clip_status(dq, [block(0), block(1024, stride=4096)]) == INVALID                     # interleaved otherwise
    # the words of the norm
    assert _clip_status(dq, [t(0)], clip=_clip(dq, out_norm=BASE + 64)) == INVALID
    assert _clip_status(dq, [t(0)], clip=_clip(dq, status=BASE + size - 4)) == INVALID
    assert _clip_status(dq, [t(0)], clip=_clip(dq, out_norm=0x40, status=0x40)) == INVALID
    assert _clip_status(dq, [t(0)], clip=_clip(dq, norm=BASE, out_norm=0x40)) == INVALID         # clipped by itself
    assert _clip_status(dq, [t(0)], clip=_clip(dq, norm=0x40, out_norm=0x40)) == INVALID
    L = dq.lib()
    flat = _list(dq, t(0), t(size))
    for at in (0, 4 * (MANY - 4), size, 2 * size - 16):
        assert L.dq_grad_gather(flat, 2, None, BASE + at, None, 0, None) == INVALID
        assert L.dq_grad_scatter(BASE + at, None, flat, 2, None, 0, None) == INVALID


@pytest.mark.parametrize("order", ["ascending", "descending", "two_runs", "random"])
@pytest.mark.parametrize("count", [100, 300, 3000])
def test_one_overlap_among_many_tensors_is_found(dq, count, order):
    import random
    rng = random.Random(count)
    spots = list(range(2 * count))
    if order == "descending":
        spots.reverse()
    elif order == "two_runs":
        spots = spots[::2] + spots[1::2]
    elif order == "random":
        rng.shuffle(spots)
    n = 8192                                            # (long lists: the workspace's fault stops a call that has no other)
    tensors = [_t(dq, data=BASE + 4 * n * s, n=n) for s in spots]
    assert count * n > 1 << 19
    assert _clip_status(dq, tensors[:count], tensors[count:]) == NO_OVERLAP
    for _ in range(5):
        k = rng.randrange(count, 2 * count)
        if spots[k] == 2 * count - 1:
            continue
        bad = list(tensors)
        bad[k] = _t(dq, data=BASE + 4 * n * spots[k] + 16, n=n)          # 16 bytes into the next one
        assert _clip_status(dq, bad[:count], bad[count:]) == INVALID


def test_workspace_sizes(dq):
    L = dq.lib()
    short, long = _list(dq, _t(dq, n=4096)), _list(dq, _t(dq))
    assert L.dq_grad_workspace_bytes(short, 1, 0) == 0
    assert L.dq_grad_workspace_bytes(short, 1, 1) > 0
    assert L.dq_grad_workspace_bytes(long, 1, 0) > 0
    for each in (0, 1):
        assert L.dq_grad_workspace_bytes(_list(dq, _t(dq, n=0)), 1, each) == 0
    assert L.dq_grad_workspace_bytes(None, 0, 0) == 0
    many = (dq.DqTensor * 5000)(*[_t(dq, n=7)] * 5000)
    assert L.dq_grad_workspace_bytes(many, 5000, 0) > L.dq_grad_workspace_bytes(long, 1, 0)


class _Stream:
    cuda_stream = 0x1230


class _FakeCalls:
    """In the place of the native calls: every call succeeds without a GPU."""
    grad_norm = grad_clip = grad_gather = grad_scatter = staticmethod(lambda *a: 0)


@pytest.mark.parametrize("given", [True, False])
def test_outputs_are_allocated_on_the_stream_of_the_call(dq, monkeypatch, given):
    import contextlib
    entered, allocated_in = [], []

    @contextlib.contextmanager
    def on(stream):
        entered.append(stream)
        yield
        entered.pop()

    def new_output(numel, dtype, device):
        allocated_in.append((numel, list(entered)))
        return torch.empty(numel, dtype=dtype)

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda ptr, device: ("stream", ptr))
    monkeypatch.setattr(dq.binding, "new_output", new_output)
    monkeypatch.setattr(dq.binding, "_calls_module", _FakeCalls)
    g, s = [torch.zeros(3, 4), torch.zeros(5)], _Stream if given else None
    where = [("stream", 0x1230)] if given else []
    norm = torch.ones(1)
    for call, sizes in ((lambda: dq.grad_norm(g, stream=s), [1]), (lambda: dq.grad_clip(g, 1.0, stream=s), [1]),
                        (lambda: dq.grad_gather(g, stream=s), [17]), (lambda: dq.grad_norm(g, out_norm=norm, stream=s), []),
                        (lambda: dq.grad_clip(g, 1.0, norm=norm, stream=s), [])):
        allocated_in.clear()
        call()
        assert allocated_in == [(n, where) for n in sizes]
    assert dq.grad_clip(g, 1.0, norm=norm, stream=s) is norm


def test_the_binding_refuses_what_is_no_list_of_gradients(dq):
    cpu, out = torch.zeros(8), torch.zeros(1)
    for bad in ([cpu], [None], [3.0], cpu, 7):
        for call in (lambda: dq.grad_norm(bad, out_norm=out, stream=_Stream),
                     lambda: dq.grad_clip(bad, 1.0, out_norm=out, stream=_Stream),
                     lambda: dq.grad_gather(bad, cpu, stream=_Stream),
                     lambda: dq.grad_scatter(cpu, bad, stream=_Stream)):
            with pytest.raises(TypeError):
                call()
    for call in (lambda: dq.grad_norm([]), lambda: dq.grad_clip([], 1.0), lambda: dq.grad_gather([])):
        with pytest.raises(ValueError, match="empty"):
            call()


# Fake tensors stand in for CUDA tensors; their addresses are never asked for.
_FAKES = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
import paper_1904_01197_b200 as dq

class Stream:
    cuda_stream = 0

def refused(name, kind, call):
    try:
        call()
    except kind as e:
        print(name, "refused")
        return
    print(name, "accepted")

with FakeTensorMode(allow_non_fake_inputs=True):
    def new(*shape, dtype=torch.float32, device="cuda:0"):
        return torch.empty(*shape, dtype=dtype, device=device)
    f32, one, other = new(64, 64), new(1), new(64, 64, device="cuda:1")
    S = dict(stream=Stream)
    refused("int", TypeError, lambda: dq.grad_norm([new(8, dtype=torch.int32)], out_norm=one, **S))
    refused("double", TypeError, lambda: dq.grad_norm([new(8, dtype=torch.float64)], out_norm=one, **S))
    refused("sparse", TypeError, lambda: dq.grad_norm([torch.sparse_coo_tensor(size=(4, 4), device="cuda:0")], out_norm=one, **S))
    def body(t):
        try:
            dq.grad_norm([t], out_norm=one, **S)
        except RuntimeError as e:
            print("vmap raised", "storage" in str(e))
        return t
    torch.vmap(body)(f32)
"""


def test_the_binding_refuses_other_kinds_of_tensors(dq):
    r = subprocess.run([sys.executable, "-c", _FAKES, str(Path(__file__).resolve().parent.parent)], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    lines = r.stdout.split("\n")
    assert lines[:3] == ["int refused", "double refused", "sparse refused"], r.stdout
    assert "vmap raised True" in lines, r.stdout


def test_a_list_of_empty_tensors_gathers_into_an_empty_vector(dq, monkeypatch):
    """Not one element, which nothing would have written."""
    monkeypatch.setattr(dq.binding, "_calls_module", _FakeCalls)
    for grads in ([torch.zeros(0)], [torch.zeros(0), torch.zeros(3, 0)]):
        assert dq.grad_gather(grads, stream=None).numel() == 0


def test_the_next_kernel_comes_in_after_the_last_read_of_a_workspace():
    """The last kernel of a call reads the norm's parts, or the norm, from a workspace that is given back when the call
    returns; an encode that stores without waiting may be handed that memory.  So a CTA may let the next kernel in only
    behind a barrier that follows its last read, or by its end.  (grad_norm_kernel, which writes the parts, is followed by a
    kernel of the same call, which waits for it; grad_cluster_kernel has no workspace.)"""
    import re
    source = (Path(__file__).resolve().parent.parent / "paper_1904_01197_b200" / "csrc" / "dq_grad.cuh").read_text()
    source = re.sub(r"//[^\n]*", "", source)
    kernels = {re.search(r"(\w+)\s*\(const __grid_constant__", k).group(1): k[:k.index("\n}\n")]
               for k in source.split("__global__")[1:]}
    assert set(kernels) == {"grad_norm_kernel", "grad_norm_join_kernel", "grad_scale_kernel", "grad_cluster_kernel"}
    assert "launch_next" not in kernels["grad_norm_join_kernel"]
    assert "a.norm" not in kernels["grad_cluster_kernel"] and "slots" not in kernels["grad_cluster_kernel"]
    scale = kernels["grad_scale_kernel"]
    lets_in = scale.index("grid_dependency_launch_next()")
    assert lets_in > scale.index("grid_dependency_wait()") and scale.count("launch_next") == 1
    reads = [m.start() for m in re.finditer(r"joined_norm<|\*a\.norm", scale)]
    assert len(reads) == 3 and all("__syncthreads()" in scale[r:lets_in] for r in reads)


_FAKE_GRAD_MODE = _FAKES.split("    f32, one, other =")[0] + """
    x, out, one, flat = new(8), new(8), new(1), new(8)
    leaf, word, vector = new(8).requires_grad_(), new(1).requires_grad_(), new(8).requires_grad_()
    result = leaf * 2
    S = dict(stream=Stream)
    def outcome(name, call):
        try:
            call()
        except RuntimeError as e:                       # (without a GPU: what else there is to complain of is the missing driver)
            print(name, "refused" if "requires a gradient" in str(e) else "not refused")
    for name, call in (
            ("leaf in place", lambda: dq.grad_clip([x, leaf], 1.0, out_norm=one, **S)),
            ("result in place", lambda: dq.grad_clip([result], 1.0, out_norm=one, **S)),
            ("leaf as out", lambda: dq.grad_clip([x, x], 1.0, out=[out, leaf], out_norm=one, **S)),
            ("view of a leaf", lambda: dq.grad_clip([x[:4]], 1.0, out=[leaf[:4]], out_norm=one, **S)),
            ("scatter", lambda: dq.grad_scatter(flat, [leaf], **S)),
            ("flat", lambda: dq.grad_gather([x], vector, **S)),
            ("norm", lambda: dq.grad_norm([x], out_norm=word, **S)),
            ("norm of a clip", lambda: dq.grad_clip([x], 1.0, out_norm=word, **S)),
            ("norms", lambda: dq.grad_norm([x] * 8, out_norm=one, out_norms=vector, **S))):
        outcome(name, call)
        with torch.no_grad():                           # where nothing is recorded it is an ordinary tensor
            outcome("no_grad " + name, call)
    # what is only read may require a gradient
    for name, call in (("read norm", lambda: dq.grad_norm([leaf, result], out_norm=one, **S)),
                       ("read gather", lambda: dq.grad_gather([leaf], flat, **S)),
                       ("read clip", lambda: dq.grad_clip([leaf], 1.0, out=[out], norm=word, **S))):
        outcome(name, call)
"""


def _without_gpu(script):
    """The output of a script on fake tensors, whose addresses no GPU may see."""
    r = subprocess.run([sys.executable, "-c", script, str(Path(__file__).resolve().parent.parent)], capture_output=True,
                       text=True, timeout=300, env={**os.environ, "CUDA_VISIBLE_DEVICES": ""})
    assert r.returncode == 0, r.stderr[-2000:]
    return [x for x in r.stdout.split("\n") if x]


def test_tensors_that_require_a_gradient_are_written_in_no_grad_only(dq):
    lines = _without_gpu(_FAKE_GRAD_MODE)
    want = ["leaf in place", "result in place", "leaf as out", "view of a leaf", "scatter", "flat", "norm", "norm of a clip",
            "norms"]
    assert lines == [x for w in want for x in (w + " refused", "no_grad " + w + " not refused")] + [
        "read norm not refused", "read gather not refused", "read clip not refused"], lines


_FAKE_DEVICES = _FAKES.split("    f32, one, other =")[0] + """
    def on(d):
        return dict(x=new(8, device=d), y=new(8, device=d), one=new(1, device=d), flat=new(16, device=d),
                    status=new(1, dtype=torch.int32, device=d))
    a, b = on("cuda:0"), on("cuda:1")
    S = dict(stream=Stream)
    def outcome(name, call):
        try:
            call()
        except TypeError as e:
            print(name, "refused" if "on one device" in str(e) else e)
        except RuntimeError as e:                       # (the missing driver)
            print(name, "not refused")
    for p, q, where in ((a, b, "01"), (b, a, "10")):
        outcome("norm list " + where, lambda: dq.grad_norm([p["x"], q["y"]], out_norm=p["one"], **S))
        outcome("norm word " + where, lambda: dq.grad_norm([p["x"]], out_norm=q["one"], **S))
        outcome("norms " + where, lambda: dq.grad_norm([p["x"]], out_norm=p["one"], out_norms=q["flat"], **S))
        outcome("status " + where, lambda: dq.grad_norm([p["x"]], out_norm=p["one"], status_word=q["status"], **S))
        outcome("clip list " + where, lambda: dq.grad_clip([p["x"], q["y"]], 1.0, out_norm=p["one"], **S))
        outcome("clip out " + where, lambda: dq.grad_clip([p["x"]], 1.0, out=[q["y"]], out_norm=p["one"], **S))
        outcome("clip norm " + where, lambda: dq.grad_clip([p["x"]], 1.0, norm=q["one"], **S))
        outcome("clip out_norm " + where, lambda: dq.grad_clip([p["x"]], 1.0, out_norm=q["one"], **S))
        outcome("gather list " + where, lambda: dq.grad_gather([p["x"], q["y"]], p["flat"], **S))
        outcome("gather flat " + where, lambda: dq.grad_gather([p["x"], p["y"]], q["flat"], **S))
        outcome("scatter list " + where, lambda: dq.grad_scatter(p["flat"], [p["x"], q["y"]], **S))
        outcome("scatter flat " + where, lambda: dq.grad_scatter(q["flat"], [p["x"], p["y"]], **S))
        outcome("one device", lambda: dq.grad_norm([p["x"], p["y"]], out_norm=p["one"], out_norms=p["flat"],
                                                   status_word=p["status"], **S))
"""


def test_the_tensors_of_a_call_lie_on_one_device(dq):
    lines = _without_gpu(_FAKE_DEVICES)
    assert len(lines) == 26
    assert all(x == "one device not refused" if x.startswith("one device") else x.endswith(" refused") for x in lines), lines
    assert sum(x.endswith("not refused") for x in lines) == 2, lines


# ------------------------------------------------------------------------------------------ overlap in large groups
def _overlap_by_pairs(extents):
    """The rule, pair by pair: extents are (start, end, width and pitch of a row in bytes (pitch 0: one piece), written)."""
    order = sorted(extents, key=lambda x: x[0])
    for k, (lo, _, width, pitch, out) in enumerate(order):
        for a_lo, a_hi, a_width, a_pitch, a_out in order[:k]:
            if not (out or a_out) or a_hi <= lo:
                continue
            if a_pitch == 0 or (pitch != 0 and pitch != a_pitch):
                return True
            column = (lo - a_lo) % a_pitch
            if column < a_width or column + width > a_pitch:
                return True
    return False


def _extent(t, out):
    size = 4 if t.dtype == 0 else 2
    if t.row and t.row_stride != t.row and t.row != t.n:
        return t.data, t.data + size * ((t.n // t.row - 1) * t.row_stride + t.row), size * t.row, size * t.row_stride, out
    return t.data, t.data + size * t.n, size * t.n, 0, out


def _blocks_beside_each_other(dq, rng, base):
    """Blocks of one matrix, with gaps, in bands of rows, and contiguous tensors in what a row leaves free."""
    pitch, tensors, column = rng.choice([2000, 5000]), [], rng.randrange(0, 40)
    while True:
        width = rng.choice([1, 2, 7, 8, 30, 64])
        if column + width > pitch:
            break
        row = 0
        while row < 12:
            rows = rng.randint(1, 6)
            if rng.random() < 0.8:
                tensors.append((base + 4 * (row * pitch + column), rows * width, width, pitch) if rows > 1
                               else (base + 4 * (row * pitch + column), width, 0, 0))
            row += rows
        column += width + rng.choice([0, 0, 1, 5, 40])
    rng.shuffle(tensors)
    return [_t(dq, data=d, n=n, row=r, stride=s) for d, n, r, s in tensors]


@pytest.mark.parametrize("seed", range(12))
def test_overlap_in_a_large_group_is_found_as_pair_by_pair(dq, seed):
    import random
    rng = random.Random(seed)
    seen = []
    for _ in range(8):
        blocks = _blocks_beside_each_other(dq, rng, BASE << 12)[:500]
        lists = {"in place": (blocks, None)}
        # inputs that overlap each other, in another matrix or in one of another pitch, into those
        sources = [_t(dq, data=(BASE << 16) + 4 * rng.randrange(4000), n=b.n, row=b.row,
                      stride=b.row_stride + rng.choice([0, 0, 3]) if b.row else 0, dtype=rng.choice([0, 1])) for b in blocks]
        lists["overlapping inputs"] = (sources, blocks)
        # inputs among the outputs: every other block is read, into tensors far away, and the rest into itself in place of those
        half = len(blocks) // 2
        far = [_t(dq, data=(BASE << 20) + 8192 * i, n=b.n) for i, b in enumerate(blocks[:half])]
        near = [_t(dq, data=b.data, n=b.n, row=b.row, stride=b.row_stride) for b in blocks[:half]]
        lists["inputs beside outputs"] = (near + [_t(dq, data=(BASE << 24) + 8192 * i, n=b.n)
                                                  for i, b in enumerate(blocks[half:])], far + blocks[half:])
        for name, (src, out) in lists.items():
            assert len(src) > 128                       # (long lists: the workspace's fault stops a call that has no other)
            for move in [0] + [rng.choice([-64, -8, -4, 4, 8, 28, 400, 8000, 20000, 20004]) for _ in range(6)]:
                side = rng.choice([src, out or src])
                k = rng.randrange(len(side))
                side[k].data += move
                extents = [_extent(t, out is None) for t in src] + [_extent(t, True) for t in out or []]
                want = _overlap_by_pairs(extents)
                got = _clip_status(dq, src, out)
                assert got == (INVALID if want else NO_OVERLAP), (name, k, move)
                seen.append(want)
                side[k].data -= move
    assert len(seen) > 100 and 0.2 < sum(seen) / len(seen) < 0.9


@pytest.mark.parametrize("into", [False, True], ids=["in_place", "into_others"])
@pytest.mark.parametrize("count", [1000, 4000, 65536])
def test_many_blocks_of_one_matrix_are_checked_quickly(dq, count, into):
    """Blocks of one matrix all reach over one another.  Pair by pair 65,536 of them took 9 s."""
    import time
    L = dq.lib()
    blocks = [_t(dq, data=BASE + 32 * i, n=64, row=8, stride=8 * count) for i in range(count)]
    others = [_t(dq, data=(BASE << 24) + 32 * i, n=64, row=8, stride=8 * count) for i in range(count)] if into else None
    a, b = _list(dq, *blocks), _list(dq, *others) if into else None
    written = b if into else a

    def call():
        start = time.perf_counter()
        s = L.dq_grad_clip(a, count, _clip(dq), b, 0x208, 1 << 30, None)
        return s, time.perf_counter() - start

    assert call()[0] == NO_OVERLAP
    took = min(call()[1] for _ in range(3))
    assert took < 1e-3 + 4e-6 * count, took             # (measured: 0.3 to 0.5 us each)
    # one block a column too wide or too far left, anywhere among them
    for k, change in ((0, dict(row=9, n=72)), (count // 2, dict(row=9, n=72)), (count - 1, dict(data=-4)), (count // 3, dict(data=4))):
        kept = written[k].data, written[k].n, written[k].row
        written[k].data += change.get("data", 0)
        written[k].row, written[k].n = change.get("row", 8), change.get("n", 64)
        if into:
            a[k].row, a[k].n, a[k].row_stride = 0, written[k].n, 0
            a[k].data = BASE << 34
        assert call()[0] == INVALID
        written[k].data, written[k].n, written[k].row = kept
        if into:
            a[k].data, a[k].n, a[k].row, a[k].row_stride = BASE + 32 * k, 64, 8, 8 * count
    assert call()[0] == NO_OVERLAP


def test_many_inputs_that_overlap_each_other_are_checked_quickly(dq):
    """They may; only outputs are compared with anything."""
    import time
    L = dq.lib()
    count = 20_000
    a = _list(dq, *[_t(dq, data=BASE + 4 * i, n=64, row=8, stride=4096 + (i % 3)) for i in range(count)])
    start = time.perf_counter()
    s = L.dq_grad_gather(a, count, _clip(dq), BASE << 24, 0x208, 1 << 30, None)
    assert s == NO_OVERLAP and time.perf_counter() - start < 0.1
