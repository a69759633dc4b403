"""adamw_step against its definition: 32-bit moments within the bounds of their roundings, 8-bit moments bit for bit (their
codes are defined on 32-bit operations), weights and predicted weights within theirs."""
import numpy as np
import pytest

from tests import operator_refs as R

pytestmark = pytest.mark.gpu

SIZES = [(1,), (127, 128, 129), (5, 0, 1023, 4096, 4097, 0), (3, 70000, 333), tuple(range(1, 140)), (1 << 20,)]


def make(sizes, *, w="float32", g="float32", bits=32, hat=None, seed=0, offset=0):
    """offset: elements by which the tensors miss the boundaries they would lie on."""
    import torch
    gen = torch.Generator().manual_seed(seed)
    total = sum(R.padded(n) for n in sizes)

    def tensors(dtype, std):
        ts = []
        for k, n in enumerate(sizes):
            buf = torch.empty(n + offset, dtype=getattr(torch, dtype), device="cuda")
            buf[offset:] = (torch.randn(n, generator=gen) * std * 10.0 ** -(k % 3)).to(buf.dtype)
            ts.append(buf[offset:])
        return ts

    s = dict(sizes=sizes, w=tensors(w, 0.5), g=tensors(g, 0.1), hat=tensors(hat, 1.0) if hat else None, m_exp=None, v_exp=None)
    m, v = torch.randn(total, generator=gen) * 0.05, torch.rand(total, generator=gen) * 0.01
    v[::17] = 0
    m[::17] = 0
    if bits == 8:
        none = np.full(total, 1 << 19)
        at = 0
        for n in sizes:                 # (what lies between two tensors is zero)
            m[at + n:at + R.padded(n)] = 0
            v[at + n:at + R.padded(n)] = 0
            at += R.padded(n)
        for key, x, top in (("m", m, 15), ("v", v, 31)):
            c, e = R.encode(x.numpy(), none, top) if total else (np.zeros(0, np.uint8),) * 2
            s[key], s[key + "_exp"] = torch.from_numpy(c).cuda(), torch.from_numpy(e).cuda()
    else:
        s["m"], s["v"] = m.cuda(), v.cuda()
    return s


def flat(ts, sizes):
    out = np.zeros(sum(R.padded(n) for n in sizes))
    at = 0
    for t, n in zip(ts, sizes):
        out[at:at + n] = R.f64(t)
        at += R.padded(n)
    return out


def mask(sizes):
    return np.concatenate([np.arange(R.padded(n)) < n for n in sizes]) if sizes else np.zeros(0, bool)


def check(s, *, step, lr=1e-2, betas=(0.9, 0.999), eps=1e-8, decay=0.05, horizon=0.0, scale=None, seed=0, call=None, step_arg=None):
    import torch
    from paper_2003_11666_amd import adamw_step
    sizes, real = s["sizes"], mask(s["sizes"])
    eight = s["m_exp"] is not None
    w, g = flat(s["w"], sizes), flat(s["g"], sizes)
    decay_of = decay if isinstance(decay, list) else [decay] * len(sizes)
    dec = np.concatenate([np.full(R.padded(n), x) for n, x in zip(sizes, decay_of)])
    if scale is not None:
        g = g * float(np.float32(scale))
    if eight:
        m, v = (R.decode(s[k].cpu().numpy(), s[k + "_exp"].cpu().numpy(), top).astype(np.float64) for k, top in (("m", 15), ("v", 31)))
    else:
        m, v = R.f64(s["m"]), R.f64(s["v"])
    m0, v0 = m.copy(), v.copy()
    gs = torch.full((1,), scale, device="cuda") if scale is not None else None

    def run():
        adamw_step(s["w"], s["g"], s["m"], s["v"], step=step if step_arg is None else step_arg, lr=lr, betas=betas, eps=eps, weight_decay=decay, m_exp=s["m_exp"],
                   v_exp=s["v_exp"], seed=seed, grad_scale=gs, predicted=s["hat"], horizon=horizon)
    (call or (lambda f: f()))(run)
    torch.cuda.synchronize()
    w_half = R.HALF[str(s["w"][0].dtype).split(".")[1]]
    h_half = R.HALF[str(s["hat"][0].dtype).split(".")[1]] if s["hat"] else 0
    (w2, m2, v2, h2), (bw, bm, bv, bh) = R.adamw(w, g, m, v, step=step, lr=lr, b1=betas[0], b2=betas[1], eps=eps, decay=dec, horizon=horizon,
                                                 w_half=w_half, hat_half=h_half)
    assert np.all(np.abs(flat(s["w"], sizes) - w2)[real] <= bw[real])
    if s["hat"]:
        assert np.all(np.abs(flat(s["hat"], sizes) - h2)[real] <= bh[real])
    if eight:
        g32 = flat(s["g"], sizes).astype(np.float32)
        if scale is not None:
            g32 = g32 * np.float32(scale)
        m32, v32 = R.moments32(m.astype(np.float32), v.astype(np.float32), g32, *betas)
        dm, dv = R.dither(len(m32), seed, step)
        for key, x, d, top in (("m", m32, dm, 15), ("v", v32, dv, 31)):
            c, e = R.encode(np.where(real, x, np.float32(0)), d, top)
            assert np.array_equal(s[key + "_exp"].cpu().numpy(), e), key
            assert np.array_equal(s[key].cpu().numpy(), c), key
    else:
        assert np.all(np.abs(R.f64(s["m"]) - m2)[real] <= bm[real]) and np.all(np.abs(R.f64(s["v"]) - v2)[real] <= bv[real])
        assert np.array_equal(R.f64(s["m"])[~real], m0[~real]) and np.array_equal(R.f64(s["v"])[~real], v0[~real])


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
def test_sizes(sizes, bits):
    s = make(sizes, bits=bits, hat="float32")
    for t in (1, 2, 1000):
        check(s, step=t, horizon=3.0)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("w", ["float32", "bfloat16"])
@pytest.mark.parametrize("g", ["float32", "bfloat16"])
@pytest.mark.parametrize("hat", [None, "float32", "bfloat16"])
def test_types(w, g, hat, bits):
    s = make((300, 8192, 77, 5000), w=w, g=g, hat=hat, bits=bits, seed=3)
    check(s, step=7, scale=0.3, decay=[0.0, 0.1, 0.0, -0.2], horizon=5.5 if hat else 0.0, seed=2 ** 63 + 5)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 2, 3, 5])
@pytest.mark.parametrize("w", ["float32", "bfloat16"])
def test_tensors_off_16_byte_boundaries(offset, w, bits):
    check(make((1000, 4096, 3, 9000), w=w, g="bfloat16", hat="float32", bits=bits, offset=offset), step=3)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kw", [dict(betas=(0.0, 0.0)), dict(betas=(0.999, 0.5), lr=0.0), dict(eps=1e-3, decay=0.0), dict(step=2 ** 40, betas=(0.9, 1 - 2.0 ** -20))])
def test_hyperparameters(kw, bits):
    check(make((2000, 50), bits=bits, hat="bfloat16"), **{"step": 5, **kw})


@pytest.mark.parametrize("bits", [32, 8])
def test_values_over_the_whole_range(bits):
    """Blocks of very different size, gradients of zero and of 1e-30 beside those of 1: in 8 bits what falls off a block's end."""
    import torch
    s = make((4096, 300), bits=bits)
    gen = torch.Generator().manual_seed(9)
    for g in s["g"]:
        e = torch.rand(g.shape, generator=gen) * 34 - 32
        g.copy_(torch.where(torch.rand(g.shape, generator=gen) < 0.2, torch.zeros(()), torch.randn(g.shape, generator=gen) * 10.0 ** e))
    for t in (1, 2, 3):
        check(s, step=t, seed=t)


def test_eight_bit_moments_from_zero_and_of_weights_without_gradients():
    """Where training starts, and rows of a table that no token named: blocks of zeros beside others, and blocks that empty out."""
    s = make((128 * 40, 700), bits=8, hat="float32")
    for key in ("m", "v", "m_exp", "v_exp"):
        s[key].zero_()
    for t in range(1, 6):
        g = s["g"][0].view(40, 128)
        g.copy_(make((128 * 40,), seed=t)["w"][0].view(40, 128))
        g[t::3] = 0
        s["g"][1].mul_(-0.0 if t == 3 else 1.0)
        check(s, step=t, seed=t, horizon=1.0)


def test_eight_bit_second_moment_decays():
    """With gradients gone, v shrinks by beta2 a step on average though one step is far less than a code."""
    import torch
    from paper_2003_11666_amd import adamw_moments, adamw_step
    n = 1 << 16
    w, g = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
    m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2))
    em, ev = (torch.zeros(n // 128, dtype=torch.uint8, device="cuda") for _ in range(2))
    adamw_step([w], [g], m, v, m_exp=em, v_exp=ev, step=1, lr=0.0)
    before = adamw_moments(m, v, em, ev)[1].double().mean().item()
    g.zero_()
    for t in range(2, 302):
        adamw_step([w], [g], m, v, m_exp=em, v_exp=ev, step=t, lr=0.0, seed=1)
    after = adamw_moments(m, v, em, ev)[1].double().mean().item()
    # a code's step is at most 1/8 of its value, so one rounding's error has a standard deviation of at most 1/16 of it, and the
    # mean over 65536 independent elements after 300 of them sqrt(300) / 16 / 256 = 0.43 %: 5 of these
    assert abs(after / before / 0.999 ** 300 - 1) < 0.022


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_gradient_that_is_not_finite(bad, bits):
    """It spoils its own weight in 32 bits; in 8 bits its block's moments read as NaN from then on, and other blocks are as ever."""
    import torch
    from paper_2003_11666_amd import adamw_moments, adamw_step
    s, clean = make((1000,), bits=bits), make((1000,), bits=bits)
    s["g"][0][300] = bad
    for x in (s, clean):
        adamw_step(x["w"], x["g"], x["m"], x["v"], m_exp=x["m_exp"], v_exp=x["v_exp"], step=1, lr=0.1)
    torch.cuda.synchronize()
    w, good = s["w"][0].cpu().numpy(), clean["w"][0].cpu().numpy()
    others = np.arange(1000) != 300
    assert np.isnan(w[300]) and np.array_equal(w[others], good[others])
    if bits == 8:
        m, v = (t.cpu().numpy() for t in adamw_moments(s["m"], s["v"], s["m_exp"], s["v_exp"]))
        block = np.arange(1024) // 128 == 2
        assert np.isnan(m[block]).all() and np.isnan(v[block]).all()
        ref = [t.cpu().numpy() for t in adamw_moments(clean["m"], clean["v"], clean["m_exp"], clean["v_exp"])]
        assert np.array_equal(m[~block], ref[0][~block]) and np.array_equal(v[~block], ref[1][~block])


def test_moments_of_every_code_and_exponent():
    import torch
    from paper_2003_11666_amd import adamw_moments
    codes = np.tile(np.arange(256, dtype=np.uint8), 256)
    e = np.repeat(np.arange(256, dtype=np.uint8), 2)
    m, v = adamw_moments(*(torch.from_numpy(x).cuda() for x in (codes, codes, e, e)))
    assert np.array_equal(m.cpu().numpy(), R.decode(codes, e, 15), equal_nan=True)
    assert np.array_equal(v.cpu().numpy(), R.decode(codes, e, 31), equal_nan=True)


@pytest.mark.parametrize("bits", [32, 8])
def test_on_another_stream_and_with_the_step_on_the_gpu(bits):
    import torch
    side = torch.cuda.Stream()
    t = torch.full((1,), 12, dtype=torch.int64, device="cuda")

    def call(f):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            f()
        torch.cuda.current_stream().wait_stream(side)

    check(make((5000, 77), bits=bits, hat="bfloat16"), step=12, step_arg=t, call=call, horizon=1.0)


def test_step_on_the_gpu_below_one_gives_nan():
    import torch
    from paper_2003_11666_amd import adamw_step
    s = make((10,))
    adamw_step(s["w"], s["g"], s["m"], s["v"], step=torch.zeros(1, dtype=torch.int64, device="cuda"), lr=0.1)
    assert torch.isnan(s["w"][0]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_replayed_steps_are_the_eager_ones(bits):
    """A captured step whose number is counted on the GPU, replayed with other work between, against eager steps: the same bits."""
    import torch
    from paper_2003_11666_amd import adamw_step
    a, b = (make((3000, 129, 40000), bits=bits, hat="bfloat16") for _ in range(2))
    t = torch.zeros(1, dtype=torch.int64, device="cuda")

    def step(s, n):
        adamw_step(s["w"], s["g"], s["m"], s["v"], m_exp=s["m_exp"], v_exp=s["v_exp"], step=n, lr=0.01, seed=4, predicted=s["hat"], horizon=2.0)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.add_(1)
        step(a, t)
    for n in range(1, 6):
        graph.replay()
        step(b, torch.full((1,), n, dtype=torch.int64, device="cuda"))
        torch.cuda.synchronize()
        for x, y in zip(a["w"] + a["hat"] + [a["m"], a["v"]], b["w"] + b["hat"] + [b["m"], b["v"]]):
            assert torch.equal(x, y), n


@pytest.mark.parametrize("bits", [32, 8])
def test_step_number_of_the_host_and_of_the_gpu_agree(bits):
    """The corrections 1 - beta^t are computed in 64 bits on both: the results of the two are within one rounding of each."""
    import torch
    from paper_2003_11666_amd import adamw_step
    for n in (1, 17, 100000):
        a, b = (make((3000,), bits=bits) for _ in range(2))
        adamw_step(a["w"], a["g"], a["m"], a["v"], m_exp=a["m_exp"], v_exp=a["v_exp"], step=n, lr=0.01)
        adamw_step(b["w"], b["g"], b["m"], b["v"], m_exp=b["m_exp"], v_exp=b["v_exp"], step=torch.full((1,), n, dtype=torch.int64, device="cuda"), lr=0.01)
        assert torch.equal(a["m"], b["m"]) and torch.equal(a["v"], b["v"])
        # corrections one 32-bit rounding apart move the direction by 2 EPS of it, |d| <= 0.011 * |m| / sqrt(v): weights of 0.5 by less than their own rounding
        assert torch.allclose(a["w"][0], b["w"][0], rtol=4 * 2.0 ** -24, atol=4 * 2.0 ** -24)


def test_forms_of_weight_decay():
    from paper_2003_11666_amd import adamw_step
    ref = None
    for wd in (0.25, np.float32(0.25), [0.25, 0.25], (0.25, 0.25), np.array([0.25, 0.25])):
        s = make((300, 77))
        adamw_step(s["w"], s["g"], s["m"], s["v"], step=1, lr=0.5, weight_decay=wd)
        got = flat(s["w"], s["sizes"])
        assert ref is None or np.array_equal(got, ref)
        ref = got


def test_refusals_of_tensors_on_the_gpu():
    import torch
    from paper_2003_11666_amd import PBError, adamw_step
    w, m = torch.zeros(64, 4, device="cuda"), torch.zeros(256, device="cuda")
    for kw in (dict(params=[w.t()]), dict(grads=[w[:3]]), dict(m=m[:128]), dict(v=m.double()), dict(m=m.byte()), dict(m_exp=torch.zeros(2, dtype=torch.uint8, device="cuda")),
               dict(params=[w.half()]), dict(params=[w, w.bfloat16()], grads=[w, w]), dict(grads=[w.cpu()]), dict(weight_decay=[0.1, 0.2]), dict(predicted=[w]), dict(params=[w, w], grads=[w, w], m=m.new_zeros(512), v=m.new_zeros(512)), dict(step=0), dict(betas=(1.0, 0.9)), dict(eps=0.0)):
        a = {**dict(params=[w], grads=[w], m=m, v=m.clone(), step=1, lr=0.1), **kw}
        with pytest.raises(PBError):
            adamw_step(a.pop("params"), a.pop("grads"), a.pop("m"), a.pop("v"), **a)


@pytest.mark.parametrize("bits", ["32", "8"])
def test_update_bench_measures_it(bits, monkeypatch, capsys):
    import json
    import sys
    from paper_2003_11666_amd import update_bench
    monkeypatch.setattr(sys, "argv", ["update_bench", "--elements", str(1 << 16), "--reps", "2", "--adamw", bits])
    update_bench.main()
    out = json.loads(capsys.readouterr().out)
    assert out["adamw_moment_bits"] == int(bits) and out["adamw_us"] > 0 and out["update_us"] > 0


def test_predicted_weights_of_some_tensors_only():
    """The C entry takes w_hat tensor by tensor."""
    import ctypes as C
    import torch
    from paper_2003_11666_amd import operators as P
    lib = P._library()
    w, g = [torch.randn(300, device="cuda") for _ in range(3)], [torch.randn(300, device="cuda") for _ in range(3)]
    hat = torch.full((300,), 5.0, device="cuda")
    m, v = torch.zeros(3 * 384, device="cuda"), torch.zeros(3 * 384, device="cuda")
    rec = np.zeros(3, dtype=P._TENSOR)
    rec["w"], rec["g"], rec["n"] = [t.data_ptr() for t in w], [t.data_ptr() for t in g], 300
    rec["w_hat"][1] = hat.data_ptr()
    d = P._AdamWDesc(moment_bits=32, lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    torch.cuda.synchronize()
    assert lib.pb_adamw_step(rec.ctypes.data, 3, C.byref(d), m.data_ptr(), v.data_ptr(), None, None, None) == 0
    torch.cuda.synchronize()
    assert torch.equal(hat, w[1])
