"""The operators together, as a model of tokens uses them: lookup, a product with the same table for the logits, loss, its
gradient, the table's gradient from both ends, an AdamW step -- three steps against autograd and the definition in 64 bits."""
import numpy as np
import pytest

from tests import operator_refs as R

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
def test_training_steps_of_a_tied_model(bits):
    import torch
    from paper_2003_11666_amd import adamw_elements, adamw_step, embed, embed_backward, log_probs, log_probs_backward
    vocab, dim, n, scale = 211, 36, 90, 36 ** 0.5
    gen = torch.Generator().manual_seed(0)
    E = (torch.randn(vocab, dim, generator=gen) * 0.1).cuda()
    W = (torch.randn(dim, dim, generator=gen) * 0.1).cuda()
    total = adamw_elements([E, W])
    kind = torch.uint8 if bits == 8 else torch.float32
    m, v = (torch.zeros(total, dtype=kind, device="cuda") for _ in range(2))
    em, ev = (torch.zeros(total // 128, dtype=torch.uint8, device="cuda") if bits == 8 else None for _ in range(2))
    ids = torch.randint(0, vocab, (n,), generator=gen).cuda()
    ids[80:] = -1
    nxt = torch.randint(0, vocab, (n,), generator=gen).cuda()
    nxt[80:] = -100
    for step in range(1, 4):
        E64, W64 = (t.double().cpu().requires_grad_() for t in (E, W))
        # the framework's calls and torch's 32-bit products between them
        h = embed(E, ids, scale=scale)
        z = h @ W
        logits = z @ E.t().contiguous()
        r = log_probs(logits, nxt)
        g = torch.full((n,), -1.0 / 80, device="cuda")
        ge = torch.full((n,), -0.01, device="cuda") * (nxt >= 0)
        dl = log_probs_backward(logits, nxt, r.norm, g, entropy=r.entropy, g_entropy=ge)
        dz = dl @ E
        dE = dl.t().contiguous() @ z
        dW = h.t().contiguous() @ dz
        embed_backward(dz @ W.t().contiguous(), ids, dE, scale=scale, add=True)
        # the same in 64 bits by autograd
        i, t = ids.cpu(), nxt.cpu()
        h64 = torch.where((i >= 0)[:, None], E64[i.clamp(min=0)] * float(np.float32(scale)), 0.0)
        lp = torch.log_softmax(h64 @ W64 @ E64.t(), 1)
        ent = -(lp.exp() * lp).sum(1)
        real = (t >= 0).double()
        loss = -(lp[torch.arange(n), t.clamp(min=0)] * real).sum() / 80 - 0.01 * (ent * real).sum()
        loss.backward()
        assert abs(float((r.logp.double() * g.double()).sum() + (r.entropy.double() * ge.double()).sum()) - float(loss.detach())) < 1e-5
        for a, b in ((dE, E64.grad), (dW, W64.grad)):
            # sums of up to 211 products of 32-bit values through four layers of them: some hundred roundings of the largest terms
            assert (a.double().cpu() - b).abs().max() <= 500 * R.EPS * max(1.0, float(b.abs().max()))
        before = [t.double().cpu().numpy().ravel() for t in (E, W)]
        adamw_step([E, W], [dE, dW], m, v, step=step, lr=0.01, weight_decay=[0.0, 0.1], m_exp=em, v_exp=ev, seed=3)
        torch.cuda.synchronize()
        if step == 1:       # moments of zero before: the definition on the gradients that the call was given, whatever the moments' bits
            for t, w0, grad, wd in ((E, before[0], dE, 0.0), (W, before[1], dW, 0.1)):
                zero = np.zeros(t.numel())
                (w2, *_), (bw, *_) = R.adamw(w0, R.f64(grad).ravel(), zero, zero, step=1, lr=0.01, b1=0.9, b2=0.999, eps=1e-8, decay=wd, horizon=0, w_half=R.EPS, hat_half=0)
                assert np.all(np.abs(R.f64(t).ravel() - w2) <= bw)
        assert all(torch.isfinite(t).all() for t in (E, W))


def test_calls_at_once_on_two_streams():
    """The calls that take workspaces, on two streams with nothing between them, against the same calls one after the other."""
    import torch
    from paper_2003_11666_amd import embed_backward, log_probs
    gen = torch.Generator().manual_seed(1)
    work = []
    for k in range(2):
        x = torch.randn(3, 90001, generator=gen).cuda()
        ids = torch.randint(0, 900, (9000 + k,), generator=gen).cuda()
        work.append((x, ids, torch.randn(len(ids), 40, generator=gen).cuda()))

    def calls(x, ids, g):
        out = []
        for _ in range(5):
            out += [*log_probs(x, torch.zeros(3, dtype=torch.int64, device="cuda"), top=33), embed_backward(g, ids, torch.empty(900, 40, device="cuda"))]
        return out

    alone = [calls(*w) for w in work]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    both = []
    for s, w in zip(streams, work):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            both.append(calls(*w))
    torch.cuda.synchronize()
    for a, b in zip(alone, both):
        assert all(torch.equal(p, q) for p, q in zip(a, b))
