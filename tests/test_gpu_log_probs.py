"""log_probs and log_probs_backward against their definitions in 64 bits, within the bounds of their roundings."""
import math

import numpy as np
import pytest

from tests import operator_refs as R

pytestmark = pytest.mark.gpu
INF = math.inf


def logits(rows, vocab, dtype, seed=0, std=3.0, masked=0.0, stride=None, offset=0):
    """stride: logits from row to row; offset: logits in front of the first one."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, vocab, generator=gen) * std
    if masked:
        x[torch.rand(x.shape, generator=gen) < masked] = -INF
    stride = stride or vocab
    buf = torch.full((offset + rows * stride,), 1e4, dtype=getattr(torch, dtype), device="cuda")
    y = buf[offset:].view(rows, stride)[:, :vocab]
    y.copy_(x.to(y.dtype))
    return y


def targets(rows, vocab, bits=64, seed=1):
    import torch
    t = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(seed))
    t[1::5] = -100
    t[3::11] = vocab
    return t.to(torch.int64 if bits == 64 else torch.int32).cuda()


def check(x, t, *, scale=1.0, top=0, entropy=True, got=None):
    """x: a tensor on the GPU."""
    import torch
    from paper_2003_11666_amd import log_probs
    r = got or log_probs(x, t, scale=scale, top=top, entropy=entropy)
    torch.cuda.synchronize()
    scale = float(np.float32(scale))
    tn = t.cpu().numpy().astype(np.int64) if t is not None else np.full(x.shape[0], -1)
    ref = R.log_probs(R.f64(x), tn, scale)

    def near(a, b, bound):
        a = R.f64(a)
        with np.errstate(invalid="ignore"):
            same = (a == b) | (np.isnan(a) & np.isnan(b)) | (np.abs(a - b) <= bound)
        assert np.all(same), (a[~same][:5], b[~same][:5], np.broadcast_to(bound, a.shape)[~same][:5])

    assert (r.logp is None) == (t is None) and (r.entropy is not None) == entropy
    near(r.norm[:, 0], ref["norm"][:, 0], ref["b_m"])
    near(r.norm[:, 1], ref["norm"][:, 1], ref["b_ls"])
    if t is not None:
        near(r.logp, ref["logp"], ref["b_logp"])
    if entropy:
        near(r.entropy, ref["entropy"], ref["b_entropy"])
    if top:
        ids = r.top_ids.cpu().numpy()
        assert r.top_ids.dtype == (t.dtype if t is not None else torch.int64)
        assert np.array_equal(ids, ref["order"][:, :top])
        near(r.top_logp, np.take_along_axis(ref["lnp"], ids.astype(np.int64), 1), np.take_along_axis(ref["b_lnp"], ids.astype(np.int64), 1))
    return r, ref


VOCABS = [1, 2, 63, 64, 65, 255, 1000, 2048, 2049, 4099, 32768, 50001]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies(vocab, dtype):
    for rows in (1, 7):
        check(logits(rows, vocab, dtype), targets(rows, vocab), top=min(vocab, 5), scale=0.7)
        check(logits(rows, vocab, dtype, seed=5), targets(rows, vocab, 32))


@pytest.mark.parametrize("rows,vocab", [(1, 200003), (3, 131072), (700, 3000), (5000, 33), (2048, 1001), (1100, 2049), (1100, 4096), (1100, 4097), (3, 16384), (3, 16385)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows(rows, vocab, dtype):
    check(logits(rows, vocab, dtype, std=1.5), targets(rows, vocab, 32), top=8)


@pytest.mark.parametrize("top", [1, 2, 31, 33, 63, 64])
@pytest.mark.parametrize("vocab", [64, 65, 640, 5003, 70001])
def test_alternatives(vocab, top):
    check(logits(6, vocab, "bfloat16", std=0.5), targets(6, vocab), top=top)      # (many equal logits: the lower index first)
    check(logits(6, vocab, "float32"), None, top=top, entropy=False)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset,stride", [(1, 1003), (2, 1001), (3, 1024), (7, 1999), (0, 1008)])
def test_rows_off_16_byte_boundaries(offset, stride, dtype):
    check(logits(9, 1001, dtype, offset=offset, stride=stride), targets(9, 1001), top=3)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("order", ["rising", "falling", "equal", "zeros of both signs", "two values"])
def test_orders_and_ties(order, dtype):
    x = logits(3, 9000, dtype)
    y = np.linspace(-5, 5, 9000)
    y = {"rising": y, "falling": -y, "equal": 0 * y + 2, "zeros of both signs": np.where(np.arange(9000) % 3, -0.0, 0.0), "two values": np.round(y / 5) + 0.0}[order]
    import torch
    x.copy_(torch.from_numpy(np.broadcast_to(y, (3, 9000)).copy()))
    for top in (1, 20, 64):
        check(x, targets(3, 9000), top=top)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [100, 70000])
def test_masked_logits(vocab, dtype):
    import torch
    x = logits(8, vocab, dtype, masked=0.9)
    t = torch.arange(8, device="cuda")
    low = torch.finfo(x.dtype).min
    x[0] = -INF                      # nothing left
    x[1] = -INF
    x[1, vocab - 3] = 1.5            # one left
    x[2] = low                       # all of the type's lowest value: uniform
    x[3] = torch.where(torch.isinf(x[3]), low, x[3].float()).to(x.dtype)
    x[4, : vocab // 2] = -INF
    r, ref = check(x, t, top=9)
    assert r.logp[0] == -INF and r.entropy[0] == 0 and r.norm[0, 0] == -INF and r.norm[0, 1] == 0
    assert r.top_ids[0].tolist() == list(range(9)) and torch.isinf(r.top_logp[0]).all()
    assert r.entropy[1] == 0 and r.top_logp[1, 0] == 0
    check(x, t, top=2, scale=3.0)    # (the lowest value times 3 is -inf)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", [50, 40000])
def test_values_that_are_not_finite(vocab, dtype):
    import torch
    x = logits(6, vocab, dtype)
    x[0, vocab - 1] = math.nan
    x[1, 3] = INF
    x[2, 7], x[2, 9] = INF, math.nan
    x[3] = math.nan
    x[4] = -INF
    x[4, 5] = math.nan
    from paper_2003_11666_amd import log_probs
    t = torch.zeros(6, dtype=torch.int64, device="cuda")
    r = log_probs(x, t, top=4)
    for row in range(5):
        assert torch.isnan(r.logp[row]) and torch.isnan(r.entropy[row]) and torch.isnan(r.norm[row]).any() and torch.isnan(r.top_logp[row]).all()
    order = R.log_probs(R.f64(x), np.zeros(6, np.int64), 1.0)["order"]
    assert np.array_equal(r.top_ids.cpu().numpy(), order[:, :4])
    check(x[5:], t[5:], top=4)
    g = _backward(x, t, r, 1.0, True)
    assert torch.isnan(g[:5]).all() and torch.isfinite(g[5]).all()


def test_large_and_small_logits():
    x = logits(6, 3000, "float32", std=1.0)
    x[0] *= 1e4
    x[1] *= 1e-20
    x[2] += 1e6
    x[3, 5] = 200.0
    check(x, targets(6, 3000), top=3)
    check(x, targets(6, 3000), top=3, scale=1e-3)


def test_leading_dimensions_and_rows_of_nothing():
    import torch
    from paper_2003_11666_amd import log_probs, log_probs_backward
    x, t = logits(6, 50, "float32"), targets(6, 50)
    a, b = log_probs(x.view(2, 3, 50), t.view(2, 3), top=4), log_probs(x, t, top=4)
    for p, q in zip(a, b):
        assert torch.equal(p.reshape(q.shape), q)
    assert a.logp.shape == (2, 3) and a.norm.shape == (2, 3, 2) and a.top_ids.shape == (2, 3, 4)
    one = log_probs(x[0], t[0], top=4)
    assert one.logp.shape == () and torch.equal(one.top_ids, b.top_ids[0]) and torch.equal(one.logp, b.logp[0])
    none = log_probs(x[:0], t[:0], top=4)
    assert none.logp.shape == (0,) and none.top_ids.shape == (0, 4)
    assert log_probs_backward(x[:0], t[:0], none.norm, none.logp).shape == (0, 50)


def _backward(x, t, r, scale, both, out=None, seed=3, only_entropy=False):
    import torch
    from paper_2003_11666_amd import log_probs_backward
    gen = torch.Generator().manual_seed(seed)
    gl, ge = (torch.randn(x.shape[0], generator=gen).cuda() for _ in range(2))
    _backward.grads = (None if only_entropy else gl, ge if both or only_entropy else None)
    return log_probs_backward(x, None if only_entropy else t, r.norm, _backward.grads[0], entropy=r.entropy if both or only_entropy else None,
                              g_entropy=_backward.grads[1], scale=scale, out=out)


def check_backward(x, t, *, scale=1.0, both=True, out=None, **kw):
    import torch
    from paper_2003_11666_amd import log_probs
    r = log_probs(x, t, scale=scale)
    before = R.f64(x)
    d = _backward(x, t, r, scale, both, out, **kw)
    torch.cuda.synchronize()
    gl, ge = (None if g is None else R.f64(g) for g in _backward.grads)
    tn = t.cpu().numpy().astype(np.int64)
    if gl is None:
        gl, tn = np.zeros(len(tn)), np.full(len(tn), -1)
    ref, bound = R.log_probs_grad(before, tn, R.f64(r.norm), R.f64(r.entropy), gl, ge, float(np.float32(scale)),
                                  R.HALF[str(x.dtype).split(".")[1]])
    got = R.f64(d)
    assert np.all(np.isfinite(got) == np.isfinite(ref))
    assert np.all(np.abs(got - ref) <= bound), np.max(np.abs(got - ref) / bound)
    return d


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("vocab", VOCABS)
def test_gradient(vocab, dtype):
    for rows in (1, 6):
        check_backward(logits(rows, vocab, dtype), targets(rows, vocab), scale=0.7)
        check_backward(logits(rows, vocab, dtype), targets(rows, vocab, 32), both=False)
    check_backward(logits(3, vocab, dtype), targets(3, vocab), only_entropy=True)


@pytest.mark.parametrize("rows,vocab", [(1, 200003), (3000, 65), (40000, 3)])
def test_gradient_of_many_and_of_long_rows(rows, vocab):
    check_backward(logits(rows, vocab, "bfloat16"), targets(rows, vocab), scale=1.5)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("offset,stride,d_offset,d_stride", [(1, 1003, 0, 1001), (0, 1001, 3, 1002), (2, 1024, 2, 1024), (5, 1999, 4, 1007)])
def test_gradient_off_16_byte_boundaries(offset, stride, d_offset, d_stride, dtype):
    import torch
    out = logits(9, 1001, dtype, offset=d_offset, stride=d_stride)
    whole = out.as_strided((9, d_stride), (d_stride, 1)) if d_offset == 0 else None
    check_backward(logits(9, 1001, dtype, offset=offset, stride=stride), targets(9, 1001), out=out)
    if whole is not None and d_stride > 1001:
        assert torch.all(whole[:, 1001:] == 1e4)          # what lies between two rows is left alone


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradient_in_place_of_the_logits(dtype):
    import torch
    x = logits(33, 2003, dtype, stride=2005)
    copy = x.clone()
    t = targets(33, 2003)
    d = check_backward(x, t, out=x)
    assert d is x
    assert torch.equal(check_backward(copy, t), d)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_gradient_of_masked_rows(dtype):
    import torch
    x = logits(6, 700, dtype, masked=0.8)
    x[0] = -INF
    x[1] = torch.finfo(x.dtype).min
    x[2] = -INF
    x[2, 9] = 3.0
    t = torch.tensor([4, 4, 9, 3, 600, -1], device="cuda")
    d = check_backward(x, t)
    assert torch.all(d[0] == 0)
    masked = torch.isinf(x)
    masked[torch.arange(5, device="cuda"), t[:5]] = False
    assert torch.all(d[masked] == 0)


def test_gradient_against_differences():
    """Differences of the definition in 64 bits: central ones of 2^-10, their error the third derivative's 2^-20 / 6 * (a few) and
    the rounding of 64-bit values, below 1e-5."""
    x, t = logits(4, 37, "float32", std=1.0), targets(4, 37)
    scale = 1.25
    d = R.f64(check_backward(x, t, scale=scale))
    gl, ge = (R.f64(g) for g in _backward.grads)
    x0, tn, h = R.f64(x), t.cpu().numpy(), 2.0 ** -10

    def loss(y):
        r = R.log_probs(y, tn, scale)
        return r["logp"] * gl + r["entropy"] * ge

    for j in range(37):
        e = np.zeros((1, 37))
        e[0, j] = h
        diff = (loss(x0 + e) - loss(x0 - e)) / (2 * h)
        assert np.all(np.abs(diff - d[:, j]) < 1e-5)


def test_same_bits_again_and_on_another_stream():
    import torch
    from paper_2003_11666_amd import log_probs
    x, t = logits(3, 150001, "bfloat16"), targets(3, 150001)
    first = log_probs(x, t, top=64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = log_probs(x, t, top=64)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_replayed_calls_are_the_eager_ones():
    import torch
    from paper_2003_11666_amd import log_probs, log_probs_backward
    x, t = logits(5, 70001, "bfloat16"), targets(5, 70001)
    g = torch.randn(5, device="cuda")
    log_probs(x, t, top=16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r = log_probs(x, t, top=16)
        d = log_probs_backward(x, t, r.norm, g, entropy=r.entropy, g_entropy=g)
    for k in range(4):
        x.copy_(logits(5, 70001, "bfloat16", seed=20 + k))
        graph.replay()
        e = log_probs(x, t, top=16)
        f = log_probs_backward(x, t, e.norm, g, entropy=e.entropy, g_entropy=g)
        torch.cuda.synchronize()
        for a, b in zip((*r, d), (*e, f)):
            assert torch.equal(a, b), k
        check(x, t, top=16, got=r)


def test_more_rows_than_a_launch_has_workgroups():
    """2^24 + 5 rows of 3 logits: their rows repeat, and so must the results."""
    import torch
    from paper_2003_11666_amd import log_probs, log_probs_backward
    n = (1 << 24) + 5
    few = logits(1 << 12, 3, "bfloat16")
    x, t = few.repeat(n // len(few) + 1, 1)[:n], targets(1 << 12, 3).repeat(n // len(few) + 1)[:n]
    a, b = log_probs(x, t, top=1), log_probs(few, t[: len(few)], top=1)
    g = torch.ones(n, device="cuda")
    da, db = log_probs_backward(x, t, a.norm, g), log_probs_backward(few, t[: len(few)], b.norm, g[: len(few)])
    for p, q in zip((*a, da), (*b, db)):
        for at in range(0, n, 1 << 22):
            part = p[at:at + (1 << 22)]
            assert torch.equal(part, q.repeat(*([len(part) // len(q) + 1] + [1] * (q.dim() - 1)))[: len(part)]), at


def test_a_row_beyond_32_bit_offsets():
    """Rows 2^30 bf16 elements apart: the third starts at 4 GiB."""
    import torch
    from paper_2003_11666_amd import log_probs, log_probs_backward
    stride = 1 << 30
    buf = torch.empty(2 * stride + 300, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((3, 300), (stride, 1))
    src = logits(3, 300, "bfloat16")
    x.copy_(src)
    t = targets(3, 300)
    check(x, t, top=5)
    r = log_probs(src, t)
    g = torch.ones(3, device="cuda")
    ref = log_probs_backward(src, t, r.norm, g)
    assert torch.equal(log_probs_backward(x, t, r.norm, g, out=x), ref)
