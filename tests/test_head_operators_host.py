"""Host-only checks of the norms', the rotary embedding's and the vocabulary head's entry points: what they
refuse, the plans, the frequencies.  No call here reaches a device."""
import math

import pytest

from paper_2502_19864_amd import binding as B

BASE = 1 << 24  # addresses that no call gets to
GIB = 1 << 30


def rows(at, row, off=0):
    return B.Rows(BASE * at + off, row)


def refused(status, call, *args):
    with pytest.raises(B.RingadaError) as e:
        call(*args)
    assert e.value.status == status and str(e.value), str(e.value)


# ---------------------------------------------------------------- norms
def norm_desc(**kw):
    return B.NormDesc(**dict(dict(dtype=B.BF16, kind=B.NORM_LAYER, rows=10, d=64, eps=1e-5), **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), B.RINGADA_E_INVALID), (dict(kind=2), B.RINGADA_E_INVALID), (dict(rows=0), B.RINGADA_E_INVALID),
    (dict(d=0), B.RINGADA_E_INVALID), (dict(eps=-1.0), B.RINGADA_E_INVALID), (dict(eps=math.nan), B.RINGADA_E_INVALID),
    (dict(eps=math.inf), B.RINGADA_E_INVALID), (dict(d=16385), B.RINGADA_E_UNSUPPORTED),
    (dict(rows=1 << 31), B.RINGADA_E_UNSUPPORTED)])
def test_norm_descriptor_is_checked(kw, status):
    refused(status, B.ringada_norm_plan, norm_desc(**kw))


def norm_forward(desc=None, **kw):
    a = dict(x=rows(1, 64), res=rows(2, 64), sum_=rows(3, 64), gain=BASE * 4, shift=BASE * 5, y=rows(6, 64), stats=BASE * 7)
    a.update(kw)
    B.ringada_norm_forward(None, desc or norm_desc(), a["x"], a["res"], a["sum_"], a["gain"], a["shift"], a["y"], a["stats"])


@pytest.mark.parametrize("kw", [
    dict(x=None), dict(y=None), dict(gain=None), dict(res=None), dict(sum_=None), dict(x=B.Rows(0, 64)), dict(x=rows(1, -64)),
    dict(x=rows(1, 64, 1)), dict(y=rows(6, 63)), dict(sum_=rows(3, 0)), dict(x=rows(1, 1 << 40)), dict(gain=BASE * 4 + 1),
    dict(shift=BASE * 5 + 1), dict(stats=BASE * 7 + 4),
    dict(y=rows(1, 64, 2)), dict(y=rows(1, 128)), dict(y=rows(3, 64)), dict(sum_=rows(2, 64, 128)), dict(y=rows(4, 64)),
    dict(stats=BASE * 6 + 8 * 64), dict(stats=BASE * 1), dict(y=rows(5, 64, -128 * 9))])
def test_norm_forward_arguments_are_checked(kw):
    refused(B.RINGADA_E_INVALID, lambda: norm_forward(**kw))


def norm_backward(desc=None, **kw):
    a = dict(dy=rows(1, 64), dskip=rows(2, 64), sum_=rows(3, 64), gain=BASE * 4, stats=BASE * 5, dx=rows(6, 64), dgain=BASE * 7,
             dshift=BASE * 8, ws=BASE * 9, have=0)
    a.update(kw)
    B.ringada_norm_backward(None, desc or norm_desc(), a["dy"], a["dskip"], a["sum_"], a["gain"], a["stats"], a["dx"], a["dgain"],
                            a["dshift"], a["ws"], a["have"])


@pytest.mark.parametrize("kw", [
    dict(dy=None), dict(sum_=None), dict(gain=None), dict(stats=None), dict(dx=None), dict(dx=rows(6, 63)), dict(dgain=BASE * 7 + 2),
    dict(stats=BASE * 5 + 4), dict(dx=rows(1, 64, 128)), dict(dx=rows(3, 72)), dict(dgain=BASE * 8 + 252), dict(dshift=BASE * 5),
    dict(dgain=BASE * 6 + 1280 - 4), dict(ws=BASE * 9 + 16, have=GIB), dict(ws=BASE * 6, have=GIB)])
def test_norm_backward_arguments_are_checked(kw):
    refused(B.RINGADA_E_INVALID, lambda: norm_backward(**kw))


@pytest.mark.parametrize("kw", [dict(), dict(dx=rows(1, 64)), dict(dx=rows(2, 64)), dict(dx=rows(3, 64)),
                                dict(dy=rows(1, 0)), dict(dskip=None), dict(dskip=rows(1, 64)), dict(sum_=rows(1, 7)),
                                dict(dgain=None), dict(dy=rows(10, 128), dx=rows(10, 128, 128))])
def test_norm_backward_takes(kw):
    """Past the tensors' checks: the missing workspace is what is left."""
    refused(B.RINGADA_E_WORKSPACE, lambda: norm_backward(**kw))


def test_norm_plan():
    for n, d in ((1, 64), (10 ** 6, 4096), (3000, 768), (2 ** 31 - 1, 16384)):
        size = B.ringada_norm_plan(norm_desc(rows=n, d=d))
        assert 8 * d <= size <= 2 * 4 * d * 1024


# ---------------------------------------------------------------- rotary
def rotary_desc(**kw):
    d = dict(dtype=B.BF16, batch=2, rows=10, n_heads=4, n_kv_heads=2, d_head=64, n_axes=2, section=(8, 24), inverse=0)
    d.update(kw)
    s = tuple(d.pop("section"))
    out = B.RotaryDesc(**d)
    for i, m in enumerate(s):
        out.section[i] = m
    return out


def view(at, n, heads, dh=64, off=0):
    return B.View(BASE * at + off, n * heads * dh, heads * dh, dh)


def rotary(desc=None, **kw):
    a = dict(q=view(1, 10, 4), k=view(2, 10, 2), pos=BASE * 3, freq=BASE * 4, oq=view(5, 10, 4), ok=view(6, 10, 2))
    a.update(kw)
    B.ringada_rotary(None, desc or rotary_desc(), a["q"], a["k"], a["pos"], a["freq"], a["oq"], a["ok"])


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), B.RINGADA_E_INVALID), (dict(batch=0), B.RINGADA_E_INVALID), (dict(rows=0), B.RINGADA_E_INVALID),
    (dict(n_heads=0), B.RINGADA_E_INVALID), (dict(n_kv_heads=-1), B.RINGADA_E_INVALID), (dict(d_head=1), B.RINGADA_E_INVALID),
    (dict(n_axes=0), B.RINGADA_E_INVALID), (dict(n_axes=5), B.RINGADA_E_INVALID), (dict(section=(8, 0)), B.RINGADA_E_INVALID),
    (dict(section=(8, 25)), B.RINGADA_E_INVALID), (dict(section=(2 ** 31 - 1, 2 ** 31 - 1)), B.RINGADA_E_INVALID),
    (dict(d_head=1026), B.RINGADA_E_UNSUPPORTED), (dict(n_heads=2049), B.RINGADA_E_UNSUPPORTED),
    (dict(n_kv_heads=2049), B.RINGADA_E_UNSUPPORTED), (dict(batch=1 << 12, rows=1 << 12), B.RINGADA_E_UNSUPPORTED)])
def test_rotary_descriptor_is_checked(kw, status):
    refused(status, lambda: rotary(rotary_desc(**kw)))


@pytest.mark.parametrize("kw,dk", [
    (dict(q=None), {}), (dict(oq=None), {}), (dict(pos=None), {}), (dict(freq=None), {}), (dict(k=None), {}), (dict(ok=None), {}),
    ({}, dict(n_kv_heads=0)), (dict(pos=BASE * 3 + 2), {}), (dict(freq=BASE * 4 + 4), {}), (dict(q=view(1, 10, 4, off=8)), {}),
    (dict(q=B.View(BASE, 2560, 260, 64)), {}), (dict(oq=B.View(BASE * 5, 2560, 128, 64)), {}), (dict(q=B.View(BASE, 2560, -256, 64)), {}),
    (dict(oq=view(1, 10, 4, off=128)), {}), (dict(oq=B.View(BASE, 2560, 64, 640)), {}), (dict(ok=view(1, 10, 2)), {}),
    (dict(ok=view(5, 10, 2)), {}), (dict(oq=view(2, 10, 4)), {}), (dict(ok=B.View(BASE * 3, 1280, 128, 64)), {}),
    (dict(oq=view(4, 10, 4)), {})])
def test_rotary_arguments_are_checked(kw, dk):
    refused(B.RINGADA_E_INVALID, lambda: rotary(rotary_desc(**dk), **kw))


def test_rotary_frequencies():
    for sections, shared in (((32,), False), ((16, 24, 24), False), ((16, 24, 24), True), ((1, 1, 1, 1), False), ((512,), True)):
        got = B.ringada_rotary_frequencies(sections, 500000.0, shared)
        p = sum(sections)
        want = [500000.0 ** (-i / p) for i in range(p)] if shared else [500000.0 ** (-j / m) for m in sections for j in range(m)]
        assert all(abs(a - b) <= 1e-15 * b for a, b in zip(got, want)) and len(got) == p
    for sections, theta in (((0,), 1e4), ((513,), 1e4), ((400, 400), 1e4), ((4,), 0.0), ((4,), math.nan), ((4,), math.inf),
                            ((), 1e4), ((1,) * 5, 1e4), ((-1,), 1e4), ((1 << 31,), 1e4)):
        with pytest.raises((B.RingadaError, ValueError)):
            B.ringada_rotary_frequencies(sections, theta, False)


# ---------------------------------------------------------------- vocabulary head
def vocab_desc(**kw):
    return B.VocabDesc(**dict(dict(dtype=B.BF16, rows=10, d=64, vocab=100), **kw))


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=-1), B.RINGADA_E_INVALID), (dict(rows=0), B.RINGADA_E_INVALID), (dict(d=0), B.RINGADA_E_INVALID),
    (dict(vocab=0), B.RINGADA_E_INVALID), (dict(d=60), B.RINGADA_E_UNSUPPORTED), (dict(d=16392), B.RINGADA_E_UNSUPPORTED),
    (dict(vocab=(1 << 22) + 1), B.RINGADA_E_UNSUPPORTED), (dict(rows=(1 << 23) + 1), B.RINGADA_E_UNSUPPORTED)])
def test_vocab_descriptor_is_checked(kw, status):
    refused(status, B.ringada_vocab_plan, vocab_desc(**kw))


def vocab_ce(desc=None, ws=BASE * 20, have=0, **kw):
    a = dict(h=rows(1, 64), w=rows(2, 64), labels=BASE * 3, loss=BASE * 4, lse=BASE * 5, dloss=BASE * 6, dh=rows(7, 64), dw=rows(8, 64))
    a.update(kw)
    B.ringada_vocab_ce(None, desc or vocab_desc(), B.VocabTensors(**a), ws, have)


NONE = B.Rows(0, 0)


@pytest.mark.parametrize("kw", [
    dict(h=NONE), dict(w=NONE), dict(labels=None), dict(loss=None), dict(lse=None), dict(dloss=None), dict(dh=NONE, dw=NONE),
    dict(h=rows(1, 56)), dict(h=rows(1, 68)), dict(h=rows(1, 64, 8)), dict(w=rows(2, -64)), dict(dh=rows(7, 32)), dict(dw=rows(8, 0)),
    dict(labels=BASE * 3 + 1), dict(lse=BASE * 5 + 2), dict(dh=rows(1, 64)), dict(dw=rows(2, 64)), dict(dw=rows(7, 64, 128)),
    dict(lse=BASE * 4 + 36), dict(loss=BASE * 3 + 36), dict(lse=BASE * 6), dict(loss=BASE * 8 + 12796), dict(ws=BASE * 20 + 128, have=GIB),
    dict(ws=BASE * 8 - 256, have=GIB)])
def test_vocab_arguments_are_checked(kw):
    refused(B.RINGADA_E_INVALID, lambda: vocab_ce(**kw))


@pytest.mark.parametrize("kw", [dict(), dict(dh=NONE), dict(dw=NONE), dict(dh=NONE, dw=NONE, dloss=None), dict(ws=None, have=GIB),
                                dict(h=rows(1, 128)), dict(h=rows(1, 128), dh=rows(1, 128, 128))])
def test_vocab_takes(kw):
    refused(B.RINGADA_E_WORKSPACE, lambda: vocab_ce(**kw))


def test_vocab_row_strides_are_bounded():
    refused(B.RINGADA_E_UNSUPPORTED, lambda: vocab_ce(w=rows(2, (1 << 22) + 8)))


@pytest.mark.parametrize("kw", [dict(h=None), dict(w=None), dict(token=None), dict(logprob=None), dict(token=BASE * 3 + 2),
                                dict(logprob=BASE * 3 + 4), dict(token=BASE * 2 + 128 * 99), dict(h=rows(1, 60))])
def test_vocab_next_arguments_are_checked(kw):
    a = dict(h=rows(1, 64), w=rows(2, 64), token=BASE * 3, logprob=BASE * 4)
    a.update(kw)
    call = lambda: B.ringada_vocab_next(None, vocab_desc(), a["h"], a["w"], a["token"], a["logprob"], BASE * 20, 0)
    refused(B.RINGADA_E_INVALID, call)


def test_vocab_plan():
    """Logits of a piece of the rows: the workspace does not grow with rows x vocab."""
    for dtype, es in ((B.BF16, 2), (B.F32, 4)):
        for n, d, V in ((1, 64, 100), (4096, 768, 30011), (1 << 16, 4096, 131072), (1 << 23, 64, 50), (300, 16384, 1 << 22)):
            f, t, x = B.ringada_vocab_plan(vocab_desc(dtype=dtype, rows=n, d=d, vocab=V))
            copy = (n + 63) * (d + 63) * es + 32 * (n + 64) + 12 * 32 * 512
            held = es * max((1 << 31) // es, 256 * (V + 64)) * 5 // 4
            assert 0 < f <= copy + (1 << 28) and x <= copy + (1 << 28)
            cut = 4 * (min(n, held // V) + 255) * (d + 255) * (1 + (V >> 18))  # dh over more than 2^18 classes, in shares
            assert f <= t + (1 << 20) and t <= copy + held + 4 * V * d + cut + (1 << 28)


# ---------------------------------------------------------------- the Python front end
def test_python_front_end_refuses():
    import torch

    from paper_2502_19864_amd import operators as ops
    x, g = torch.zeros(3, 8), torch.zeros(8)
    q = torch.zeros(1, 2, 3, 8)
    lab = torch.zeros(3, dtype=torch.int32)
    pos, freq = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.float64)
    for call in (lambda: ops.norm_forward(x, g), lambda: ops.norm_backward(x, x, g, x), lambda: ops.rotary(q, positions=pos, freq=freq),
                 lambda: ops.vocab_ce_forward(x, x, lab), lambda: ops.vocab_ce_train(x, x, lab, g), lambda: ops.vocab_next(x, x)):
        with pytest.raises(ValueError, match="on a GPU"):
            call()
    with pytest.raises(ValueError):
        ops.vocab_ce_train(x, x, lab, None)
    with pytest.raises(ValueError):
        ops.vocab_ce_train(x, x, lab, g, frozen=True, dw=x)


def test_python_front_end_refuses_what_autograd_would_miss():
    import torch

    from paper_2502_19864_amd import operators as ops
    x, g = torch.zeros(3, 8), torch.zeros(8)
    lx, lg = x.clone().requires_grad_(), g.clone().requires_grad_()
    q = torch.zeros(1, 2, 3, 8)
    lab = torch.zeros(3, dtype=torch.int32)
    pos, freq = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(4, dtype=torch.float64)
    lq = q.clone().requires_grad_()
    for call in (lambda: ops.norm_forward(lx, g), lambda: ops.norm_forward(x, lg), lambda: ops.norm_forward(x, g, lg),
                 lambda: ops.norm_forward(x, g, res=lx), lambda: ops.norm_backward(lx, x, g, x), lambda: ops.norm_backward(x, x, lg, x),
                 lambda: ops.rotary(lq, positions=pos, freq=freq), lambda: ops.rotary(q, lq, positions=pos, freq=freq),
                 lambda: ops.vocab_ce_forward(lx, x, lab), lambda: ops.vocab_ce_train(x, lx, lab, g), lambda: ops.vocab_next(x, lx)):
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on cpu"):
            call()
