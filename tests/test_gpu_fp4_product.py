"""The product of MXFP4 rows with their group's MXFP4 weights (mxfp4_product) against
64 bits: groups of every size (empty ones too), odd channel counts and columns,
output types and strides, the layer's own group table; refusals.

Tolerances. Products of elements and scales are exact; sums are fp32. With S the
sum of the absolute values of a result's terms, each of the at most 64 steps of
64 columns (4,096 columns) may lose 2^-22 S (sums of a step aligned and cut at fp32's
last bits): 1.6e-5 S. f32 results: 2e-5 S. bf16 results: one rounding (2^-8 with a
neighbour) more. GELU has a slope of at most 1.13, in bf16 output 3e-4 |v| more, in
f32 output 2e-6 |v| + 2e-7 (erff, and 1 + erff where they cancel)."""
import ctypes as C
import math

import pytest
import torch

LEVELS = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def codes(rows, cols, g, lo=118, hi=130):
    """Random rows in 4 bits, as the operator takes them."""
    from paper_2608_10392_gb300 import Mxfp4
    blocks = (cols + 31) // 32
    c = torch.randint(0, 16, (rows, blocks * 32), generator=g, dtype=torch.uint8)
    c[:, cols:] = 0
    s = torch.zeros(rows, (blocks + 7) // 8 * 8, dtype=torch.uint8)
    s[:, :blocks] = torch.randint(lo, hi, (rows, blocks), generator=g, dtype=torch.uint8)
    return Mxfp4((c[:, 0::2] | c[:, 1::2] << 4).cuda(), s.cuda(), cols)


def values(q):
    """What the codes stand for, in 64 bits."""
    c, s = q.codes.cpu(), q.scales.cpu()
    c, s = c.reshape(-1, c.shape[-1]), s.reshape(-1, s.shape[-1])
    table = torch.tensor(LEVELS + [-v for v in LEVELS], dtype=torch.float64)
    v = torch.stack([table[(c & 15).long()], table[(c >> 4).long()]], -1).reshape(len(c), -1)
    size = torch.exp2(s.double() - 127)
    size[s == 255] = math.nan
    return (v * size.repeat_interleave(32, 1)[:, :v.shape[1]])[:, :q.cols]


def reference(a, w, n, offsets, act):
    av, wv = values(a), values(w)
    out = torch.full((len(av), n), math.nan, dtype=torch.float64)
    size = torch.zeros_like(out)
    for g in range(len(offsets) - 1):
        lo, hi = offsets[g], offsets[g + 1]
        m = wv[g * n:(g + 1) * n]
        out[lo:hi] = av[lo:hi] @ m.T
        size[lo:hi] = av[lo:hi].abs() @ m.abs().T
    pre = out.clone()
    if act == "gelu":
        out = out * 0.5 * (1 + torch.erf(out / math.sqrt(2)))
    return out, size, pre


def check(sizes, n, cols, act="none", dtype="bf16", seed=0, out=None, offsets=None):
    from paper_2608_10392_gb300 import Mxfp4, mxfp4_product, mxfp4_status
    g = torch.Generator().manual_seed(seed)
    rows, G = sum(sizes), len(sizes)
    a, w = codes(rows, cols, g), codes(G * n, cols, g)
    off = [0]
    for s in sizes:
        off.append(off[-1] + s)
    wg = Mxfp4(w.codes.view(G, n, -1), w.scales.view(G, n, -1), cols)
    # about unit results: rows come out around sqrt(cols) 2.4^2 2^-6
    got = mxfp4_product(a, wg, torch.tensor(off, dtype=torch.int32, device="cuda"),
                        activation=act, dtype=dtype, out=out)
    assert mxfp4_status() == 0
    want, size, pre = reference(a, w, n, off, act)
    tol = 2e-5 * size
    if act == "gelu":
        tol = 1.13 * tol + (3e-4 * pre.abs() if dtype == "bf16" else 2e-6 * pre.abs() + 2e-7)
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * want.abs()
    err = (got.double().cpu() - want).abs()
    assert got.shape == want.shape and not torch.isnan(got).any()
    assert (err <= tol).all(), (float((err / tol.clamp(min=1e-30)).max()), int((err > tol).sum()))
    return a, wg, got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes,n,cols", [
    ([1], 1, 1), ([1], 128, 256), ([5], 64, 32), ([16], 130, 64), ([17], 257, 96),
    ([31, 1, 0, 33], 128, 384), ([0, 0, 7, 0], 200, 100), ([192, 193, 191], 128, 768),
    ([385, 12], 192, 2048), ([1000], 1000, 1024), ([127, 128, 129, 65, 64, 63], 96, 4096),
    ([3] * 40, 72, 320), ([2, 0, 300], 33, 31), ([500], 7, 257)])
def test_against_64_bits(sizes, n, cols, dtype):
    check(sizes, n, cols, dtype=dtype, seed=n + cols)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gelu(dtype):
    check([70, 0, 200, 3], 160, 640, act="gelu", dtype=dtype, seed=5)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [33, 272, 1100, 4160])
def test_many_groups(G):
    g = torch.Generator().manual_seed(G)
    sizes = torch.randint(0, 9 if G < 4000 else 3, (G,), generator=g).tolist()
    check(sizes, 64, 128, seed=G)


@pytest.mark.gpu
@pytest.mark.parametrize("sizes,n,cols,act,dtype", [
    # rows as the M operand: channels that 128-channel tiles would waste
    ([129, 0, 300, 1, 128], 192, 768, "gelu", "bf16"), ([500, 77], 160, 300, "none", "bf16"),
    ([90] * 20, 144, 512, "gelu", "bf16"), ([1000], 176, 33, "none", "bf16"),
    ([200, 100], 192, 256, "gelu", "f32"),
    # pairs of CTAs: many steps, an even number of 128-channel tiles
    ([385, 0, 3, 192, 193], 512, 2048, "gelu", "bf16"), ([40, 33, 31, 60], 256, 2100, "none", "f32"),
    ([700], 1000, 4096, "gelu", "f32"), ([2100, 1500], 250, 1024, "none", "bf16"),
    ([17, 97, 31, 5, 20, 100, 32, 1], 300, 2304, "none", "bf16")])
def test_other_operand_orders(sizes, n, cols, act, dtype):
    check(sizes, n, cols, act=act, dtype=dtype, seed=n)


@pytest.mark.gpu
def test_more_items_than_sms():
    """Several items per CTA with few and many steps: the ring and the accumulators
    come round, in groups of unequal size."""
    check([700, 0, 1500, 9, 333], 1200, 512, seed=1, dtype="f32")
    check([50] * 30, 1500, 300, seed=2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,pad,shift", [(128, 8, 0), (96, 1, 0), (64, 7, 1), (63, 0, 0), (64, 2, 1)])
def test_strided_output(n, pad, shift, dtype):
    wide = torch.full((150, n + pad + shift), 3.0, device="cuda",
                      dtype=torch.bfloat16 if dtype == "bf16" else torch.float32)
    check([100, 50], n, 256, dtype=dtype, out=wide[:, shift:shift + n])
    assert (wide[:, :shift] == 3).all() and (wide[:, shift + n:] == 3).all()


@pytest.mark.gpu
def test_scales_of_every_size():
    """Scales from 2^-127 to 2^63 and the NaN byte: a NaN spoils its row of the output
    (of its channel, in the weights) and nothing else."""
    from paper_2608_10392_gb300 import Mxfp4, mxfp4_product
    g = torch.Generator().manual_seed(3)
    for lo, hi in ((0, 1), (60, 70), (180, 191)):
        a, w = codes(40, 128, g, lo, hi), codes(64, 128, g, 127, 130)
        got = mxfp4_product(a, w, dtype="f32").double().cpu()
        av, wv = values(a), values(w)
        assert ((got - av @ wv.T).abs() <= 2e-5 * (av.abs() @ wv.abs().T) + 2.0 ** -140).all()
    a, w = codes(40, 128, g), codes(64, 128, g)
    a.scales[7, 2], w.scales[9, 0] = 255, 255
    got = mxfp4_product(a, w, dtype="f32").cpu()
    nan = torch.zeros(40, 64, dtype=torch.bool)
    nan[7], nan[:, 9] = True, True
    assert torch.equal(torch.isnan(got), nan)


@pytest.mark.gpu
def test_offsets_that_leave_rows_out_or_are_out_of_range():
    """Rows of no group keep what the output held; offsets beyond the rows, below 0 or
    falling are taken as the documentation says, and nothing else is written."""
    from paper_2608_10392_gb300 import Mxfp4, mxfp4_product
    g = torch.Generator().manual_seed(4)
    a, w = codes(60, 96, g), codes(3 * 40, 96, g)
    wg = Mxfp4(w.codes.view(3, 40, -1), w.scales.view(3, 40, -1), 96)
    av, wv = values(a), values(w).view(3, 40, 96)

    def run(off, rows_of):
        wide = torch.full((62, 40), 3.0, device="cuda")
        mxfp4_product(a, wg, torch.tensor(off, dtype=torch.int32, device="cuda"), dtype="f32",
                      out=wide[1:61])
        want = torch.full((62, 40), 3.0, dtype=torch.float64)
        for k, (lo, hi) in enumerate(rows_of):
            want[1 + lo:1 + hi] = av[lo:hi] @ wv[k].T
        assert ((wide.double().cpu() - want).abs() <= 1e-4 * (1 + want.abs())).all()

    run([5, 10, 30, 50], [(5, 10), (10, 30), (30, 50)])
    run([-100, 20, 20, 2000000000], [(0, 20), (20, 20), (20, 60)])
    run([40, 60, 20, 30], [(40, 60), (0, 0), (20, 30)])
    run([0, 60, 0, 60], [(0, 60), (0, 0), (0, 0)])  # the third group's rows are over the count


@pytest.mark.gpu
def test_repeatable_streams_and_no_rows():
    from paper_2608_10392_gb300 import mxfp4_product
    a, wg, got = check([300, 200], 256, 1024, seed=8)
    off = torch.tensor([0, 300, 500], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = mxfp4_product(a, wg, off)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, again)
    none = type(a)(a.codes[:0], a.scales[:0], a.cols)
    assert mxfp4_product(none, wg, torch.zeros_like(off)).shape == (0, 256)


@pytest.mark.gpu
def test_graph_capture():
    """The call can be captured and replayed."""
    from paper_2608_10392_gb300 import mxfp4_product
    a, wg, got = check([90, 30], 128, 512, seed=9)
    off = torch.tensor([0, 90, 120], dtype=torch.int32, device="cuda")
    out = torch.zeros_like(got)
    mxfp4_product(a, wg, off, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mxfp4_product(a, wg, off, out=out)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, got)


@pytest.mark.gpu
def test_stream_argument_and_a_capture_first():
    from paper_2608_10392_gb300 import mxfp4_product, mxfp4_quantize, operators
    a, wg, got = check([300, 200], 256, 1024, seed=8)
    off = torch.tensor([0, 300, 500], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    again = [mxfp4_product(a, wg, off, stream=side) for _ in range(5)]
    x = torch.randn(64, 96, device="cuda")
    torch.cuda.synchronize()
    q = mxfp4_quantize(x, stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(got, r) for r in again)
    assert torch.equal(q.codes, mxfp4_quantize(x).codes)
    # the word that products report to is not made inside a capture
    kept = dict(operators._status_words)
    operators._status_words.clear()
    try:
        graph, out = torch.cuda.CUDAGraph(), torch.empty_like(got)
        with pytest.raises(RuntimeError, match="capture"):
            with torch.cuda.graph(graph):
                mxfp4_product(a, wg, off, out=out)
    finally:
        operators._status_words.update(kept)


@pytest.mark.gpu
@pytest.mark.parametrize("G", [309, 310, 311, 320, 323, 324, 325])
def test_group_counts_at_which_the_ring_gets_shorter(G):
    """The table of groups takes shared memory beside the ring of stages: on both sides
    of the count from which the ring has fewer."""
    g = torch.Generator().manual_seed(G)
    sizes = torch.randint(0, 9, (G,), generator=g).tolist()
    check(sizes, 64, 128, seed=G)
    # rows as the M operand: 64 rows a group, channels that 128-channel tiles would waste
    sizes = torch.randint(40, 90, (G,), generator=g).tolist()
    sizes[7] += max(0, 64 * G - sum(sizes))
    check(sizes, 160, 64, act="gelu", seed=G)


class Word:
    """Stands for the word on a device that products report to."""

    def __init__(self, calls, value):
        self.calls, self.value = calls, value

    def item(self):
        self.calls.append("read")
        return self.value

    def zero_(self):
        self.calls.append("clear")
        self.value = 0
        return self


@pytest.fixture
def words(monkeypatch):
    """Calls that touch the words, without a GPU: device 0 has a word that is set."""
    from paper_2608_10392_gb300 import operators
    calls = []

    def made(*args, **kw):
        calls.append("make")
        return Word(calls, 0)

    class Stream:
        def synchronize(self):
            calls.append("wait")

    monkeypatch.setattr(operators, "_status_words", {torch.device("cuda", 0): Word(calls, 1)})
    monkeypatch.setattr(torch, "zeros", made)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    monkeypatch.setattr(torch.cuda, "synchronize", lambda *a: calls.append("wait"))
    return calls


@pytest.mark.parametrize("device", ["cuda", "cuda:0", 0, None])
def test_status_of_a_device_by_any_of_its_names(device, words):
    """The word that a product reports to is found by every name of its device."""
    from paper_2608_10392_gb300 import mxfp4_status
    assert mxfp4_status(device) == -5
    assert mxfp4_status(device) == 0
    assert "make" not in words


def test_status_word_is_cleared_before_a_later_product(words):
    """Making and clearing the word have ended when the call returns: a product on another
    stream does not have its report cleared."""
    from paper_2608_10392_gb300 import mxfp4_status, operators
    mxfp4_status()
    assert words == ["wait", "read", "clear", "wait"]
    del words[:]
    operators._status_word(torch.device("cuda", 1))
    assert words == ["make", "wait"]


def test_refusals():
    from paper_2608_10392_gb300 import build
    build.build()
    import paper_2608_10392_gb300 as pkg
    L = pkg.lib()
    p = C.c_void_p(4096)

    def call(**k):
        v = dict(a=p, sa=p, rows=4, cols=64, w=p, sw=p, n=8, groups=2, off=p, act=0, out=p, dt=1, ld=8,
                 status=p)
        v.update(k)
        return L.unif_moe_mxfp4_product(v["a"], v["sa"], v["rows"], v["cols"], v["w"], v["sw"], v["n"],
                                        v["groups"], v["off"], v["act"], v["out"], v["dt"], v["ld"],
                                        v["status"], None)

    for k in (dict(a=None), dict(sa=None), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(w=None),
              dict(sw=None), dict(n=0), dict(groups=0), dict(off=None), dict(act=2), dict(act=-1),
              dict(out=None), dict(dt=2), dict(ld=7), dict(status=None), dict(a=C.c_void_p(4104)),
              dict(sw=C.c_void_p(4100)), dict(n=1 << 30)):
        assert call(**k) == -1, k
    assert call(groups=4225) == -2
    assert call(rows=0, a=None) == 0
    z = torch.zeros(4, 32, dtype=torch.uint8)
    s = torch.zeros(4, 8, dtype=torch.uint8)
    with pytest.raises(ValueError, match="a.codes"):
        pkg.mxfp4_product(pkg.Mxfp4(z, s, 64), pkg.Mxfp4(z, s, 64))
    with pytest.raises(ValueError, match="codes"):
        pkg.mxfp4_product(pkg.Mxfp4(z, s, 65), pkg.Mxfp4(z, s, 64))
