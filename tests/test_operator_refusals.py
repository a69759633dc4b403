"""What the operators over plain arrays refuse, before anything is launched: the C entries with addresses that are never
followed, and the checks of the Python calls (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

from paper_2003_11666_amd import operators as P
from paper_2003_11666_amd.binding import PBError

A = 1 << 20            # an address on every boundary that is asked for


def lib():
    return P._library()


def refused(rc, text):
    assert rc == -1
    assert text in lib().pb_last_error().decode(), lib().pb_last_error()


def tensors(**kw):
    rec = np.zeros(2, dtype=P._TENSOR)
    rec["w"], rec["g"], rec["n"] = A, A, 5
    for k, v in kw.items():
        rec[k][1] = v
    return rec


def step(rec=None, m=A, v=A, m_exp=None, v_exp=None, **kw):
    rec = tensors() if rec is None else rec
    d = P._AdamWDesc(moment_bits=32, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    for k, x in kw.items():
        setattr(d, k, x)
    return lib().pb_adamw_step(rec.ctypes.data, len(rec), C.byref(d), m, v, m_exp, v_exp, None)


@pytest.mark.parametrize("kw,text", [
    (dict(w_type=2), "types"), (dict(g_type=-1), "types"), (dict(w_hat_type=7), "types"), (dict(moment_bits=16), "moment_bits"),
    (dict(lr=-1.0), "lr"), (dict(lr=float("nan")), "lr"), (dict(lr=float("inf")), "lr"), (dict(horizon=float("inf")), "horizon"),
    (dict(beta1=1.0), "betas"), (dict(beta2=-0.1), "betas"), (dict(beta2=float("nan")), "betas"), (dict(beta2=1 - 1e-12), "betas"),
    (dict(eps=0.0), "eps"), (dict(eps=1e-60), "eps"), (dict(eps=float("inf")), "eps"), (dict(step=0), "counted from 1"),
    (dict(step_dev=A + 4), "step_dev"), (dict(grad_scale=A + 2), "grad_scale"),
    (dict(m=None), "m and v"), (dict(v=A + 8), "m and v"), (dict(m_exp=A), "8-bit"), (dict(moment_bits=8), "8-bit"),
    (dict(moment_bits=8, m_exp=A), "8-bit"),
    (dict(rec=dict(w=0)), "tensor 1"), (dict(rec=dict(g=0)), "tensor 1"), (dict(rec=dict(n=-1)), "tensor 1"),
    (dict(rec=dict(n=1 << 43)), "tensor 1"), (dict(rec=dict(w=A + 2)), "tensor 1"), (dict(rec=dict(w_hat=A + 1)), "tensor 1"),
    (dict(rec=dict(weight_decay=float("nan"))), "tensor 1"),
])
def test_adamw_step_refuses(kw, text):
    if "rec" in kw:
        kw = dict(rec=tensors(**kw["rec"]))
    refused(step(**kw), text)


def test_adamw_with_nothing_to_do():
    empty = tensors(n=0)
    empty["n"] = 0
    empty["w"] = empty["g"] = 0
    assert step(rec=empty, m=None, v=None) == 0
    assert step(rec=tensors()[:0], m=None, v=None) == 0
    assert lib().pb_adamw_moments(None, None, None, None, 0, None, None, None) == 0


def test_adamw_elements():
    n = np.array([1, 0, 128, 129, 1000], dtype=np.int64)
    assert lib().pb_adamw_elements(n.ctypes.data, 5) == 128 + 0 + 128 + 256 + 1024
    assert lib().pb_adamw_elements(None, 0) == 0
    n[1] = -1
    refused(lib().pb_adamw_elements(n.ctypes.data, 5), "tensor 1")
    refused(lib().pb_adamw_elements(None, 1), "no sizes")


def test_adamw_moments_refuses():
    f = lib().pb_adamw_moments
    refused(f(A, A, A, A, 100, A, A, None), "multiple")
    refused(f(A, A, A, A, -128, A, A, None), "multiple")
    refused(f(A, A, A, None, 128, A, A, None), "NULL")
    refused(f(A, A, A, A, 128, A + 4, A, None), "16-byte")


LOGP = dict(logits=A, dtype=0, rows=4, vocab=100, stride=100, targets=A, id_bits=64, scale=1.0, logp=A, entropy=A, norm=A, top=0, top_logp=None,
            top_ids=None, ws=A, ws_bytes=1 << 40)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=2), "dtype"), (dict(rows=-1), "bad sizes"), (dict(vocab=0, stride=0), "bad sizes"), (dict(stride=99), "bad sizes"),
    (dict(vocab=1 << 31, stride=1 << 31), "bad sizes"), (dict(rows=1 << 40, stride=1 << 20), "bad sizes"), (dict(rows=1 << 31), "too many rows"),
    (dict(scale=0.0), "scale"), (dict(scale=-1.0), "scale"), (dict(scale=float("nan")), "scale"), (dict(scale=float("inf")), "scale"),
    (dict(top=65, top_logp=A, top_ids=A), "top"), (dict(top=-1), "top"), (dict(top=8, vocab=7, top_logp=A, top_ids=A), "top"),
    (dict(top=1), "top_ids"), (dict(top=1, top_logp=A), "top_ids"), (dict(id_bits=16), "32 or 64"), (dict(targets=A + 4), "boundaries"),
    (dict(logits=None), "no logits"), (dict(norm=None), "norm"), (dict(targets=None), "belong together"), (dict(logp=None), "belong together"),
    (dict(logits=A + 2), "boundaries"), (dict(entropy=A + 2), "boundaries"), (dict(top=1, top_logp=A, top_ids=A + 4), "boundaries"),
])
def test_log_probs_refuses(kw, text):
    a = {**LOGP, **kw}
    refused(lib().pb_log_probs(a["logits"], a["dtype"], a["rows"], a["vocab"], a["stride"], a["targets"], a["id_bits"], a["scale"], a["logp"], a["entropy"],
                               a["norm"], a["top"], a["top_logp"], a["top_ids"], a["ws"], a["ws_bytes"], None), text)


def test_log_probs_workspace():
    f = lib().pb_log_probs_workspace
    assert f(0, 10, 0) >= 0 and f(1, 1, 1) >= 0
    refused(f(1, 10, 11), "bad sizes")
    refused(f(1, 0, 0), "bad sizes")
    refused(f(-1, 10, 0), "bad sizes")
    need = f(1, 200000, 64)
    if need:
        for ws, n in ((None, need), (A, need - 1), (A + 8, need)):
            refused(lib().pb_log_probs(A, 0, 1, 200000, 200000, None, 64, 1.0, None, None, A, 64, A, A, ws, n, None), "workspace")


GRAD = dict(logits=A, dtype=0, rows=4, vocab=100, stride=100, targets=A, id_bits=32, scale=1.0, norm=A, entropy=A, g_logp=A, g_entropy=A, d=A, d_stride=100)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=3), "dtype"), (dict(stride=50), "bad sizes"), (dict(d_stride=50), "bad sizes"), (dict(vocab=0), "bad sizes"),
    (dict(scale=0.0), "scale"), (dict(id_bits=8), "32 or 64"), (dict(targets=A + 2), "boundaries"), (dict(logits=None), "NULL"), (dict(norm=None), "NULL"),
    (dict(d=None), "NULL"), (dict(targets=None), "g_logp"), (dict(entropy=None), "g_entropy"), (dict(d=A + 1), "boundaries"), (dict(norm=A + 2), "boundaries"),
    (dict(d=A + 400), "overlaps"), (dict(d_stride=200), "overlaps"), (dict(d=A - 4 * 399), "overlaps"),
])
def test_log_probs_backward_refuses(kw, text):
    a = {**GRAD, **kw}
    refused(lib().pb_log_probs_backward(a["logits"], a["dtype"], a["rows"], a["vocab"], a["stride"], a["targets"], a["id_bits"], a["scale"], a["norm"],
                                        a["entropy"], a["g_logp"], a["g_entropy"], a["d"], a["d_stride"], None), text)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=2), "types"), (dict(out_dtype=2), "types"), (dict(vocab=0), "bad sizes"), (dict(dim=0), "bad sizes"), (dict(n=-1), "bad sizes"),
    (dict(n=1 << 40, dim=1 << 20), "bad sizes"), (dict(dim=1 << 31), "bad sizes"), (dict(id_bits=0), "32 or 64"), (dict(ids=A + 4), "boundaries"), (dict(table=None), "NULL"),
    (dict(ids=None), "NULL"), (dict(out=None), "NULL"), (dict(out=A + 2), "boundaries"),
])
def test_embed_refuses(kw, text):
    a = {**dict(table=A, dtype=0, vocab=10, dim=4, ids=A, id_bits=64, n=3, scale=1.0, out=A, out_dtype=0), **kw}
    refused(lib().pb_embed(a["table"], a["dtype"], a["vocab"], a["dim"], a["ids"], a["id_bits"], a["n"], a["scale"], a["out"], a["out_dtype"], None), text)


@pytest.mark.parametrize("kw,text", [
    (dict(dtype=2), "types"), (dict(table_dtype=2), "types"), (dict(add=2), "add"), (dict(vocab=0), "bad sizes"), (dict(vocab=(1 << 31) + 1), "bad sizes"),
    (dict(n=(1 << 30) + 1), "bad sizes"), (dict(dim=0), "bad sizes"), (dict(dim=1 << 31), "bad sizes"), (dict(id_bits=1), "32 or 64"), (dict(ids=A + 4), "boundaries"), (dict(d_out=None), "NULL"),
    (dict(ids=None), "NULL"), (dict(d_table=None), "NULL"), (dict(d_table=A + 2), "boundaries"), (dict(ws=None), "workspace"), (dict(ws_bytes=1), "workspace"),
    (dict(ws=A + 8), "workspace"),
])
def test_embed_backward_refuses(kw, text):
    a = {**dict(d_out=A, dtype=0, ids=A, id_bits=64, n=3000, vocab=10, dim=4, scale=1.0, d_table=A, table_dtype=0, add=0, ws=A, ws_bytes=1 << 40), **kw}
    refused(lib().pb_embed_backward(a["d_out"], a["dtype"], a["ids"], a["id_bits"], a["n"], a["vocab"], a["dim"], a["scale"], a["d_table"],
                                    a["table_dtype"], a["add"], a["ws"], a["ws_bytes"], None), text)


def test_nothing_to_do_is_no_failure():
    L = lib()
    assert L.pb_log_probs(None, 0, 0, 10, 10, None, 64, 1.0, None, None, None, 0, None, None, None, 0, None) == 0
    assert L.pb_log_probs_backward(None, 0, 0, 10, 10, None, 64, 1.0, None, None, None, None, None, 10, None) == 0
    assert L.pb_embed(None, 0, 10, 4, None, 64, 0, 1.0, None, 0, None) == 0
    assert L.pb_embed_backward(None, 0, None, 64, 0, 10, 4, 1.0, None, 0, 1, None, 0, None) == 0


def test_python_calls_refuse():
    import torch
    f, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    bad = [
        lambda: P.log_probs(f, i),                                            # not on a GPU
        lambda: P.log_probs(f.half(), i), lambda: P.log_probs(f, i.short()), lambda: P.log_probs(f, i[:3]),
        lambda: P.log_probs(f.t(), None), lambda: P.log_probs(f[None].expand(2, 4, 8), None),
        lambda: P.log_probs_backward(f, i, torch.zeros(4, 2), torch.zeros(3)),
        lambda: P.log_probs_backward(f, i, torch.zeros(4), torch.zeros(4)),
        lambda: P.log_probs_backward(f, i, torch.zeros(4, 2), torch.zeros(4), out=f.bfloat16()),
        lambda: P.log_probs_backward(f, i, torch.zeros(4, 2), torch.zeros(4)),
        lambda: P.embed(f, i), lambda: P.embed(f.t(), i), lambda: P.embed(f, i.float()), lambda: P.embed(f.double(), i),
        lambda: P.embed_backward(f, i, f), lambda: P.embed_backward(f, i[:3], f), lambda: P.embed_backward(f, i, f.t()),
        lambda: P.adamw_step([f], [f], torch.zeros(128), torch.zeros(128), step=1, lr=0.1),
        lambda: P.adamw_step([f], [], torch.zeros(128), torch.zeros(128), step=1, lr=0.1),
        lambda: P.adamw_step([f], [f], torch.zeros(128), torch.zeros(128), step=1, lr=0.1, predicted=[]),
        lambda: P.adamw_step([f], [f], torch.zeros(128), torch.zeros(128), step=torch.zeros(1), lr=0.1),
        lambda: P.adamw_step([f], [f], torch.zeros(128), torch.zeros(128), step=1, lr=0.1, grad_scale=torch.zeros(2)),
        lambda: P.adamw_moments(f, f, f, f), lambda: P.adamw_moments(*[torch.zeros(128, dtype=torch.uint8)] * 4),
    ]
    for k, call in enumerate(bad):
        with pytest.raises(PBError):
            call()
            print("accepted:", k)
    assert P.adamw_elements([f, torch.zeros(0), torch.zeros(129)]) == 128 + 256


def test_adamw_refuses_what_it_would_write_twice():
    """Weights, predicted weights and moments, each on its own 4096 bytes here, then two of them on the same."""
    def rec(**kw):
        r = np.zeros(2, dtype=P._TENSOR)
        r["w"], r["w_hat"], r["g"], r["n"] = [A, A + 4096], [A + 8192, A + 12288], A, 1024
        for k, x in kw.items():
            r[k] = x
        return r
    m, v = A + 16384, A + 16384 + 2 * 4096
    for r, m_, v_ in ((rec(w=A), m, v), (rec(w=[A, A + 4092]), m, v), (rec(w_hat=[A, A + 12288]), m, v), (rec(), A, v), (rec(), m, m + 8188 // 16 * 16),
                      (rec(), A + 12288 + 4080, v)):
        refused(step(rec=r, m=m_, v=v_), "overlap")
