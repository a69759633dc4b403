"""The operators over plain arrays where sizes pass a limit of their kernels: chunks of large models, offsets beyond 32 bits, more
work than a launch has workgroups, more parts than a wavefront has lanes."""
import numpy as np
import pytest

from tests import operator_refs as R

pytestmark = pytest.mark.gpu


def test_chunks_of_large_models_give_the_codes_of_small_ones():
    """8-bit moments of 2^26 elements and more are taken in larger chunks: the first half of the tensor as in a call of its own (in
    smaller ones), bit for bit, and a ragged tensor behind it by the definition."""
    import torch
    from paper_2003_11666_amd import adamw_elements, adamw_step
    n, half = (1 << 26) + 77, 1 << 25
    gen = torch.Generator(device="cuda").manual_seed(0)
    w, g = (torch.randn(n, device="cuda", generator=gen) * 0.1 for _ in range(2))
    small = [torch.randn(1000, device="cuda", generator=gen) for _ in range(2)]
    total = adamw_elements([w, small[0]])

    def moments(k):
        return [torch.zeros(k, dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.zeros(k // 128, dtype=torch.uint8, device="cuda") for _ in range(2)]

    a, b = moments(total), moments(half)
    wa, wb = w.clone(), w[:half].clone()
    before = R.f64(small[0])
    for t in (1, 2):
        adamw_step([wa, small[0]], [g, small[1]], a[0], a[1], m_exp=a[2], v_exp=a[3], step=t, lr=0.01, seed=5)
        adamw_step([wb], [g[:half]], b[0], b[1], m_exp=b[2], v_exp=b[3], step=t, lr=0.01, seed=5)
    assert torch.equal(wa[:half], wb)
    for x, y in zip(a, b):
        assert torch.equal(x[:len(y)], y)
    # the ragged tensor, two steps by the definition
    start, m, v = total - 1024, np.zeros(1024, np.float32), np.zeros(1024, np.float32)
    grad = np.zeros(1024, np.float32)
    grad[:1000] = small[1].cpu().numpy()
    for t in (1, 2):
        m2, v2 = R.moments32(m, v, grad, 0.9, 0.999)
        dm, dv = R.dither(1024, 5, t, start)
        (cm, em), (cv, ev) = R.encode(m2, dm, 15), R.encode(v2, dv, 31)
        m, v = R.decode(cm, em, 15), R.decode(cv, ev, 31)
    for x, y in zip(a, (cm, cv, em, ev)):
        assert np.array_equal(x[-len(y):].cpu().numpy(), y)
    assert np.all(R.f64(small[0]) != before)


@pytest.mark.parametrize("bits", [8, 32])
def test_moments_beyond_32_bit_places(bits):
    """2^32 + 1000 weights without a gradient but for the last 1000, whose places do not fit 32 bits."""
    import torch
    from paper_2003_11666_amd import adamw_step
    n, last = (1 << 32) + 1000, 1000
    total = R.padded(n)
    w, g = (torch.zeros(n, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g[-last:] = torch.randn(last, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    kind = torch.uint8 if bits == 8 else torch.float32
    m, v = (torch.zeros(total, dtype=kind, device="cuda") for _ in range(2))
    em, ev = (torch.zeros(total // 128, dtype=torch.uint8, device="cuda") if bits == 8 else None for _ in range(2))
    adamw_step([w], [g], m, v, m_exp=em, v_exp=ev, step=1, lr=0.01, weight_decay=0.0, seed=9)
    grad = np.zeros(1024, np.float32)
    grad[:last] = g[-last:].float().cpu().numpy()
    m2, v2 = R.moments32(np.zeros(1024, np.float32), np.zeros(1024, np.float32), grad, 0.9, 0.999)
    if bits == 8:
        dm, dv = R.dither(1024, 9, 1, total - 1024)
        for x, e, ref, d, top in ((m, em, m2, dm, 15), (v, ev, v2, dv, 31)):
            c, exps = R.encode(ref, d, top)
            assert np.array_equal(x[-1024:].cpu().numpy(), c) and np.array_equal(e[-8:].cpu().numpy(), exps)
    else:
        # (of zero moments one product and one sum with 0: no rounding that the definition does not have)
        assert np.array_equal(m[-1024:-24].cpu().numpy(), m2[:last]) and np.array_equal(v[-1024:-24].cpu().numpy(), v2[:last])
    zero = np.zeros(last)
    (w2, *_), (bw, *_) = R.adamw(zero, R.f64(g[-last:]), zero, zero, step=1, lr=0.01, b1=0.9, b2=0.999, eps=1e-8, decay=0.0, horizon=0, w_half=2.0 ** -8, hat_half=0)
    assert np.all(np.abs(R.f64(w[-last:]) - w2) <= bw)
    assert int(torch.count_nonzero(w[:1 << 31])) + int(torch.count_nonzero(w[1 << 31:n - last])) == 0


def test_a_row_in_more_parts_than_a_workgroup_has_lanes():
    import torch
    from tests.test_gpu_log_probs import check, logits
    for top in (0, 1, 64):
        check(logits(1, 3000001, "bfloat16", seed=top), torch.tensor([2999999], device="cuda"), top=top)
    check(logits(2, 1200007, "float32", masked=0.5), torch.tensor([5, 1200006], device="cuda"), top=7)


@pytest.mark.parametrize("vocab", [3001, 4101])
def test_more_long_rows_than_a_launch_has_workgroups(vocab):
    """2^20 + 3 rows, which repeat after 2048 (enough for them to be taken in the same way): so must their results."""
    import torch
    from paper_2003_11666_amd import log_probs
    from tests.test_gpu_log_probs import logits
    n, m = (1 << 20) + 3, 2048
    few = logits(m, vocab, "bfloat16")
    x = few.repeat(n // m + 1, 1)[:n]
    t = torch.arange(n, device="cuda") % m
    a, b = log_probs(x, t, top=2), log_probs(few, t[:m], top=2)
    for p, q in zip(a, b):
        assert torch.equal(p[: n // m * m].view(-1, *q.shape), q.expand(n // m, *q.shape))
        assert torch.equal(p[n // m * m:], q[: n % m])


def test_more_tokens_than_a_launch_has_workgroups():
    import torch
    from paper_2003_11666_amd import embed
    n = 4300007
    w = torch.randn(7, 512, device="cuda", generator=torch.Generator(device="cuda").manual_seed(0))
    ids = (torch.arange(n, device="cuda") * 5 + 3) % 8 - 1                          # (-1 among them)
    got = embed(w, ids, dtype=torch.bfloat16)
    ref = torch.cat([w.bfloat16(), torch.zeros(1, 512, dtype=torch.bfloat16, device="cuda")])
    for at in range(0, n, 1 << 20):
        assert torch.equal(got[at:at + (1 << 20)], ref[ids[at:at + (1 << 20)]]), at


@pytest.mark.parametrize("n,vocab", [(600001, 1000), (600001, 300000), (9000, 300000), (300000, 1)])
def test_gradient_of_many_tokens(n, vocab):
    """Tiles and chunks beyond those of smaller batches, and three passes of the sort.  (Small whole numbers: sums are exact.)"""
    import torch
    from paper_2003_11666_amd import embed_backward
    gen = torch.Generator().manual_seed(n + vocab)
    ids = torch.randint(-1, vocab + 1, (n,), generator=gen).cuda()
    g = torch.randint(-4, 5, (n, 9), generator=gen).float().cuda()
    for add in (False, True):
        d = torch.full((vocab, 9), 2.0, device="cuda")
        there = (ids >= 0) & (ids < vocab)
        ref = torch.zeros(vocab, 9, dtype=torch.float64, device="cuda").index_add_(0, ids[there], g[there].double()) + (2.0 if add else 0.0)
        assert torch.equal(embed_backward(g, ids, d, add=add).double(), ref)
