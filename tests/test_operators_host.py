"""Host-only checks of the block operators' entry points: what they refuse, the plans,
the bucket map.  No call here reaches a device."""
import ctypes
from fractions import Fraction

import pytest

from paper_2502_19864_amd import binding as B


def desc(**kw):
    d = dict(dtype=B.BF16, batch=2, n_heads=4, n_kv_heads=2, d_head=64, seq_q=10, seq_k=20, causal=1, window=0,
             sinks=0, scale=0.125, n_buckets=0, max_distance=0)
    d.update(kw)
    return B.AttnDesc(**d)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=7), B.RINGADA_E_INVALID),
    (dict(batch=0), B.RINGADA_E_INVALID),
    (dict(n_kv_heads=3), B.RINGADA_E_INVALID),
    (dict(seq_q=0), B.RINGADA_E_INVALID),
    (dict(window=-1), B.RINGADA_E_INVALID),
    (dict(sinks=-1), B.RINGADA_E_INVALID),
    (dict(scale=0.0), B.RINGADA_E_INVALID),
    (dict(scale=float("nan")), B.RINGADA_E_INVALID),
    (dict(scale=float("inf")), B.RINGADA_E_INVALID),
    (dict(n_buckets=-1), B.RINGADA_E_INVALID),
    (dict(n_buckets=4, max_distance=1025), B.RINGADA_E_UNSUPPORTED),
    (dict(d_head=96), B.RINGADA_E_UNSUPPORTED),
    (dict(dtype=B.F32, d_head=129), B.RINGADA_E_UNSUPPORTED),
    (dict(seq_k=1 << 25), B.RINGADA_E_UNSUPPORTED),
    (dict(batch=1 << 20, seq_k=1 << 20), B.RINGADA_E_UNSUPPORTED),
])
def test_attention_descriptor_is_checked(kw, status):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_plan(desc(**kw), False)
    assert e.value.status == status and B.ringada_last_error()


@pytest.mark.parametrize("kw", [dict(), dict(dtype=B.F32, d_head=16), dict(seq_q=128, seq_k=128),
                                dict(n_kv_heads=1, seq_q=200, seq_k=200)])
def test_launches_are_bounded_by_their_threads(kw):
    """A launch holds fewer than 2^32 threads, 256 to a workgroup: refused before anything is enqueued."""
    d = dict(dict(n_heads=16, n_kv_heads=16, seq_q=1, seq_k=1), **kw)
    blocks = 16 * ((d["seq_q"] + 127) // 128)  # workgroups of a batch row, one per 128 queries of a head
    most = ((1 << 24) - 1) // blocks
    assert B.ringada_attn_plan(desc(batch=most, **d), False)[1] > 0
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_plan(desc(batch=most + 1, **d), False)
    assert e.value.status == B.RINGADA_E_UNSUPPORTED


def test_a_stage_refuses_what_no_launch_holds():
    d = stage_desc(dtype="f32", d_model=64, n_heads=32, d_ffn=64, d_adapter=16, batch=1 << 19, seq=1)
    opt = B.StageAttention(window=4)
    assert B.ringada_stage_plan_attention(d, opt, (1 << 19) - 1, 1) > 0
    with pytest.raises(B.RingadaError) as e:
        B.ringada_stage_plan_attention(d, opt, 1 << 19, 1)
    assert e.value.status == B.RINGADA_E_UNSUPPORTED


def test_attention_plan():
    f, b = B.ringada_attn_plan(desc(), False)
    assert b >= 2 * 4 * 10 * 4
    _, b2 = B.ringada_attn_plan(desc(n_buckets=8, max_distance=16), True)
    _, b3 = B.ringada_attn_plan(desc(n_buckets=8, max_distance=16), False)
    assert b3 == b and b2 >= b + 2 * 4 * 33 * 4


@pytest.mark.parametrize("kw", [dict(batch=1, n_heads=32, n_kv_heads=8, window=16, sinks=1 << 20),
                                dict(batch=500, window=16, sinks=4), dict(batch=500, window=1000, sinks=4),
                                dict(batch=64, n_heads=16, n_kv_heads=1, window=0), dict(batch=1, window=0)])
def test_split_backward_stays_within_its_workspace(kw):
    """At most some 4096 workgroups of 128 KB of partial sums, beside 8 bytes a row."""
    d = desc(d_head=128, seq_q=8192, seq_k=8192, **kw)
    _, b = B.ringada_attn_plan(d, False)
    assert b <= 8 * d.batch * d.n_heads * 8192 + (4096 << 17) + 512


@pytest.mark.parametrize("kw", [
    dict(dtype=B.F32, n_heads=8, n_kv_heads=1, seq_q=512, seq_k=512),
    dict(dtype=B.F32, n_heads=4, n_kv_heads=1, seq_q=600, seq_k=600),
    dict(dtype=B.F32, d_head=16, n_heads=16, n_kv_heads=2, seq_q=305, seq_k=305),
    dict(dtype=B.F32, d_head=16, n_heads=16, n_kv_heads=2, seq_q=305, seq_k=305, window=100),
    dict(dtype=B.F32, n_heads=16, n_kv_heads=1, seq_q=600, seq_k=600, window=80, sinks=3),
    dict(d_head=128, n_heads=32, n_kv_heads=1, seq_q=768, seq_k=768),
    dict(n_heads=8, n_kv_heads=1, seq_q=4096, seq_k=128, causal=0)])
def test_few_key_blocks_are_split(kw):
    """A backward of a few key blocks, each met by many query tiles, has partial sums of 16 workgroups at least."""
    d = desc(batch=1, **kw)
    rows = 8 * d.n_heads * d.seq_q
    assert B.ringada_attn_plan(d, False)[1] - rows >= 16 * 4 * 2 * 32 * 64 * 4


BASE = 1 << 20  # addresses that no call gets to


def view(at, rows, heads, dh=64):
    return B.View(BASE * at, rows * heads * dh, heads * dh, dh)


def tensors(**kw):
    t = dict(q=view(1, 10, 4), k=view(2, 20, 2), v=view(3, 20, 2), o=view(4, 10, 4), lse=BASE * 5)
    t.update(kw)
    return B.AttnTensors(**t)


def grads(**kw):
    g = dict(dout=view(6, 10, 4), dq=view(7, 10, 4), dk=view(8, 20, 2), dv=view(9, 20, 2))
    g.update(kw)
    return B.AttnGrads(**g)


@pytest.mark.parametrize("kw,dk", [
    (dict(q=B.View(0, 1, 1, 1)), {}),                                # no data
    (dict(k=B.View(BASE * 2 + 8, 2560, 128, 64)), {}),               # misaligned
    (dict(k=B.View(BASE * 2, 2560, 100, 64)), {}),                   # a stride that is no multiple of 8
    (dict(v=B.View(BASE * 3, 2560, -128, 64)), {}),                  # backwards
    (dict(o=B.View(BASE * 4, 2560, 128, 64)), {}),                   # rows of the output overlap
    (dict(o=B.View(BASE * 4, 64, 256, 64)), {}),                     # and its sequences
    (dict(o=view(1, 10, 4)), {}),                                    # the output is an input
    (dict(table=BASE * 10, bucket=BASE * 11), {}),                   # a table without buckets
    ({}, dict(n_buckets=4, max_distance=3)),                         # and the other way round
    (dict(table=BASE * 10), dict(n_buckets=4, max_distance=3)),      # no map
])
def test_attention_tensors_are_checked(kw, dk):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_forward(None, desc(**dk), tensors(**kw), BASE * 12, 0)
    assert e.value.status == B.RINGADA_E_INVALID


def test_row_strides_are_bounded():
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_forward(None, desc(), tensors(k=B.View(BASE * 2, 64, 1 << 24, 64)), BASE * 12, 0)
    assert e.value.status == B.RINGADA_E_UNSUPPORTED


@pytest.mark.parametrize("kw,gkw", [
    (dict(lse=None), {}),
    ({}, dict(dq=view(1, 10, 4))),
    ({}, dict(dq=view(6, 10, 4))),
    ({}, dict(dv=view(8, 20, 2))),
    ({}, dict(dtable=BASE * 10)),
    ({}, dict(dk=B.View(BASE * 8, 2560, 64, 64))),
])
def test_gradients_are_checked(kw, gkw):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_backward(None, desc(), tensors(**kw), grads(**gkw), BASE * 12, 1 << 20)
    assert e.value.status == B.RINGADA_E_INVALID


def test_workspaces_are_checked():
    _, n = B.ringada_attn_plan(desc(), False)
    for ws, have, status in ((None, n, B.RINGADA_E_WORKSPACE), (BASE * 12, n - 1, B.RINGADA_E_WORKSPACE),
                             (BASE * 12 + 16, n, B.RINGADA_E_INVALID)):
        with pytest.raises(B.RingadaError) as e:
            B.ringada_attn_backward(None, desc(), tensors(), grads(), ws, have)
        assert e.value.status == status
    L = B.lib()
    assert L.ringada_attn_plan(None, 0, None, None) == B.RINGADA_E_INVALID
    assert L.ringada_attn_forward(None, ctypes.byref(desc()), None, None, 0) == B.RINGADA_E_INVALID
    assert L.ringada_attn_backward(None, ctypes.byref(desc()), ctypes.byref(tensors()), None, None, 0) == \
        B.RINGADA_E_INVALID


def dec(**kw):
    """A call whose forward needs a workspace: without one it gets past the checks of its tensors, and no further."""
    return desc(batch=1, seq_q=1, seq_k=4096, **kw)


def packed(at, heads, first=0, width=8, rows=4096, off=0):
    """Heads first .. of a [1, rows, width, 64] buffer."""
    return B.View(BASE * at + 2 * (64 * first + off), rows * width * 64, width * 64, 64)


def decode(**kw):
    t = dict(q=packed(1, 4, rows=1), k=packed(8, 2, 4), v=packed(8, 2, 6), o=packed(2, 4, rows=1), lse=BASE * 5)
    t.update(kw)
    return B.AttnTensors(**t)


@pytest.mark.parametrize("kw", [
    dict(),
    dict(o=packed(8, 4)),                                    # the first four heads of the keys' and values' buffer
    dict(o=packed(8, 4, off=8 * 64 * 4095)),                 # of its last row
    dict(q=packed(1, 4, 0, 8), o=packed(1, 4, 4, 8)),        # side by side in one row
    dict(lse=BASE * 8 + 2 * 64 * 8 * 4096),                  # right behind the keys' buffer
    dict(lse=BASE * 8),                                      # in a hole of it
])
def test_tensors_woven_into_each_other_are_taken(kw):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_forward(None, dec(), decode(**kw), BASE * 100, 0)
    assert e.value.status == B.RINGADA_E_WORKSPACE, str(e.value)


@pytest.mark.parametrize("kw", [
    dict(o=packed(8, 4, 1)),                                 # its last head is k's first, in the first row
    dict(o=packed(8, 4, 2, off=8 * 64 * 4095)),              # and in the last
    dict(o=packed(1, 4, 3, rows=1)),                         # the last head of q
    dict(o=B.View(BASE * 1 + 16, 256, 256, 64)),             # q, 16 bytes on
    dict(lse=BASE * 2 + 4 * 64 * 2 - 8),                     # the end of o
    dict(lse=BASE * 8 + 2 * 64 * 6),                         # v's first row
    dict(len_k=BASE * 5 + 12),                               # lse's last entry
])
def test_partly_overlapping_tensors_are_refused(kw):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_forward(None, dec(), decode(**kw), BASE * 100, 0)
    assert e.value.status == B.RINGADA_E_INVALID and "overlaps" in str(e.value)


@pytest.mark.parametrize("kw,gkw,ok", [
    ({}, {}, True),
    ({}, dict(dq=packed(7, 4, 0, rows=10), dk=packed(8, 2, 4, rows=20), dv=packed(8, 2, 6, rows=20)), True),
    ({}, dict(dk=packed(8, 2, 4, rows=20), dv=packed(8, 2, 5, rows=20)), False),    # one head of two gradients
    ({}, dict(dk=B.View(BASE * 8, 2560, 128, 64), dv=B.View(BASE * 8 + 2560, 2560, 128, 64)), False),
    ({}, dict(dk=B.View(BASE * 8, 5120, 128, 64), dv=B.View(BASE * 8 + 5120, 5120, 128, 64)), True),  # batch by batch
    ({}, dict(dq=B.View(BASE * 6 + 2 * 64, 2560, 256, 64)), False),                 # dout, a head on
    ({}, dict(dv=B.View(BASE * 5 - 2 * 64, 2560, 128, 64)), False),                 # into lse
    (dict(len_q=BASE * 8 + 16), {}, False),
])
def test_gradients_overlap_nothing(kw, gkw, ok):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_backward(None, desc(), tensors(**kw), grads(**gkw), BASE * 12, 0)
    assert e.value.status == (B.RINGADA_E_WORKSPACE if ok else B.RINGADA_E_INVALID), str(e.value)


def test_overlaps_against_the_addresses_themselves():
    """Small random views of one stretch of memory: dq refused exactly where it shares an element with q."""
    import itertools
    import random

    rng = random.Random(5)
    met = 0
    for _ in range(600):
        b, h, sq, dh = (rng.randint(1, 3) for _ in range(4))
        d = desc(dtype=B.F32, batch=b, n_heads=h, n_kv_heads=h, d_head=dh, seq_q=sq, seq_k=sq)

        def some():
            out, extent = {}, dh
            for name, n in rng.sample([("batch", b), ("row", sq), ("head", h)], 3):  # nested, with gaps
                out[name] = extent + rng.randint(0, 4)
                extent += out[name] * (n - 1)
            return out, extent

        (sq_, eq), (sd, ed) = some(), some()
        if rng.random() < 0.5:  # slices of one tensor
            sd, ed = sq_, eq
        at = rng.randint(-ed, eq)
        el = lambda s, o: {o + i * s["batch"] + j * s["row"] + k * s["head"] + x for i, j, k, x in
                           itertools.product(range(b), range(sq), range(h), range(dh))}
        far = lambda i: B.View(BASE * i, 1000, 100, 10)
        q, dq = B.View(BASE * 30, sq_["batch"], sq_["row"], sq_["head"]), \
            B.View(BASE * 30 + 4 * at, sd["batch"], sd["row"], sd["head"])
        with pytest.raises(B.RingadaError) as e:
            B.ringada_attn_backward(None, d, B.AttnTensors(q=q, k=far(2), v=far(3), o=far(4), lse=BASE * 5),
                                    B.AttnGrads(dout=far(6), dq=dq, dk=far(8), dv=far(9)), BASE * 12, 0)
        meet = bool(el(sq_, 0) & el(sd, at))
        assert e.value.status == (B.RINGADA_E_INVALID if meet else B.RINGADA_E_WORKSPACE), str(e.value)
        met += meet
    assert 100 < met < 500


def test_the_table_and_the_workspace_overlap_nothing():
    d = desc(n_buckets=4, max_distance=3)
    _, n = B.ringada_attn_plan(d, True)
    t = dict(table=BASE * 10, bucket=BASE * 11)
    for kw, gkw, ws, have in ((t, dict(dtable=BASE * 10 + 60), BASE * 12, 0), (t, dict(dtable=BASE * 11 + 24), BASE * 12, 0),
                              (t, dict(dtable=BASE * 13), BASE * 10 - n + 256, n),
                              (t, dict(dtable=BASE * 13), BASE * 9 + 256, n)):
        with pytest.raises(B.RingadaError) as e:
            B.ringada_attn_backward(None, d, tensors(**kw), grads(**gkw), ws, have)
        assert e.value.status == B.RINGADA_E_INVALID and "overlaps" in str(e.value)


def test_strides_of_single_entries_do_not_count():
    """A dimension of one entry may have any stride, as torch gives it."""
    one = dict(q=B.View(BASE, -5, 3, 64), k=B.View(BASE * 8, 1 << 50, 512, 64), o=B.View(BASE * 2, 0, 1 << 30, 64))
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_forward(None, dec(), decode(**one), BASE * 100, 0)
    assert e.value.status == B.RINGADA_E_WORKSPACE, str(e.value)


def test_numbers_out_of_range_are_refused():
    """ctypes alone would cut them to their low bits."""
    import torch

    from paper_2502_19864_amd import operators as ops
    from paper_2502_19864_amd.stage import Stage
    st = object.__new__(Stage)  # the numbers are looked at before the handle is
    st.torch, st.handle, st.dev = torch, None, torch.device("cpu")
    st.w = type("W", (), dict(n_heads=2))
    for call in (lambda: st.set_attention(window=1 << 32), lambda: st.set_attention(window=4, sinks=(1 << 32) + 1),
                 lambda: st.set_dropout(0.1, None, 1 << 32), lambda: st.set_dropout(0.1, None, -1),
                 lambda: ops.relpos_buckets((1 << 32) + 32, 128, True),
                 lambda: ops.relpos_buckets(32, (1 << 32) + 128, True),
                 lambda: B.ringada_dropout(None, B.BF16, BASE, None, BASE * 3, 1000, 0.0, BASE * 9 + 1, 1 << 32),
                 lambda: B.ringada_dropout(None, B.BF16, BASE, None, BASE * 3, (1 << 64) + 8, 0.0, BASE * 9 + 1, 0)):
        with pytest.raises(ValueError):
            call()


def test_strides_beyond_any_memory_are_refused():
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_forward(None, dec(), decode(k=B.View(BASE * 8, 0, 512, 1 << 39), v=packed(9, 2)), BASE * 100, 0)
    assert e.value.status == B.RINGADA_E_WORKSPACE  # 2^39 elements on, but within 2^46
    with pytest.raises(B.RingadaError) as e:
        B.ringada_attn_backward(None, desc(batch=200), tensors(q=B.View(BASE * 1, 1 << 39, 256, 64)), grads(), BASE * 12, 0)
    assert e.value.status == B.RINGADA_E_INVALID


@pytest.mark.parametrize("kw", [
    dict(dtype=3), dict(x=None), dict(y=None), dict(rng=None), dict(n=0), dict(n=(1 << 35) + 1), dict(p=-0.1),
    dict(p=1.0), dict(p=float("nan")), dict(p=0.999999), dict(y=BASE + 16), dict(res=BASE * 3 + 4), dict(x=BASE + 1),
    dict(rng=BASE * 9 + 4)])
def test_dropout_arguments_are_checked(kw):
    a = dict(dtype=B.BF16, x=BASE, res=None, y=BASE * 3, n=1000, p=0.1, rng=BASE * 9)
    a.update(kw)
    with pytest.raises(B.RingadaError) as e:
        B.ringada_dropout(None, a["dtype"], a["x"], a["res"], a["y"], a["n"], a["p"], a["rng"], 0)
    assert e.value.status == B.RINGADA_E_INVALID


def test_the_tests_generator_gives_the_published_vectors():
    import operator_reference as R
    import philox_vectors as P

    for counter, key, out in P.VECTORS:
        assert P.words(counter, key) == out
    seed, offset, site = 0x0123456789abcdef, 0xfedcba9876543210, 0x13579bdf
    assert R.philox(40, seed, offset, site) == [h for c in range(5) for h in P.halves(c, seed, offset, site)]


@pytest.mark.parametrize("n,dist,bidi", [(32, 128, True), (32, 128, False), (16, 20, True), (64, 512, False),
                                         (4, 2, True), (2, 2, False), (2, 1024, False), (64, 1024, True),
                                         (8, 16, True), (320, 500, True), (1000, 1024, False)])
def test_bucket_map(n, dist, bidi):
    """Against the rule in whole numbers: d >= one (dist / one)^(k / m) as powers of m."""
    got = B.ringada_relpos_buckets(n, dist, bidi)
    per = n // 2 if bidi else n
    one = per // 2
    m = per - one
    for rel in range(-dist, dist + 1):
        d = abs(rel) if bidi else max(-rel, 0)
        t = d
        if d >= one:
            k = 0
            while k < m and Fraction(d, one) ** m >= Fraction(dist, one) ** (k + 1):
                k += 1
            t = min(per - 1, one + k)
        assert got[rel + dist] == t + (per if bidi and rel > 0 else 0), rel


@pytest.mark.parametrize("n,dist,rel,bucket", [(73, 905, 347, 61), (222, 316, 245, 194), (226, 188, 157, 185),
                                               (281, 527, 297, 219)])
def test_bucket_map_next_to_a_border(n, dist, rel, bucket):
    """Distances 3e-11 to 6e-10 of themselves below a border that is no whole number."""
    one = n // 2
    m, k = n - one, bucket + 1 - one
    assert rel ** m < dist ** k * one ** (m - k) and (rel + 1) ** m > dist ** k * one ** (m - k)
    assert B.ringada_relpos_buckets(n, dist, False)[dist - rel] == bucket
    assert B.ringada_relpos_buckets(2 * n, dist, True)[dist - rel] == bucket


@pytest.mark.parametrize("n,dist,bidi", [(1, 8, False), (0, 8, False), (3, 8, True), (2, 8, True), (32, 8, True),
                                         (32, 16, False), (32, 1025, True), (8, -1, False)])
def test_bucket_map_refuses(n, dist, bidi):
    with pytest.raises(B.RingadaError) as e:
        B.ringada_relpos_buckets(n, dist, bidi)
    assert e.value.status == B.RINGADA_E_INVALID


def test_python_front_end_refuses():
    import torch

    from paper_2502_19864_amd import operators as ops
    q = torch.zeros(1, 2, 3, 64)
    with pytest.raises(ValueError):  # not on a GPU
        ops.attention_forward(q, q, q)
    with pytest.raises(ValueError):
        ops.attention_forward(q[0], q, q)
    with pytest.raises(ValueError):
        ops.dropout(q, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError):
        ops.attention_backward(q, q, q, q, q, None)


def test_python_front_end_refuses_what_autograd_would_miss():
    import torch

    from paper_2502_19864_amd import operators as ops
    q = torch.zeros(1, 2, 3, 64)
    leaf, rng = q.clone().requires_grad_(), torch.zeros(2, dtype=torch.int64)
    table = torch.zeros(4, 3, requires_grad=True)
    calls = [lambda: ops.attention_forward(leaf, q, q), lambda: ops.attention_forward(q, q, leaf),
             lambda: ops.attention_forward(q, q, q, table=table, bucket=torch.zeros(3, dtype=torch.int32)),
             lambda: ops.attention_backward(q, q, leaf, q, q, q), lambda: ops.dropout(leaf, 0.1, rng),
             lambda: ops.dropout(q, 0.1, rng, res=leaf)]
    for call in calls:
        with pytest.raises(ValueError, match="requires a gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="on cpu"):  # the next check
            call()


def stage_desc(**kw):
    from paper_2502_19864_amd.stage import make_desc
    from paper_2502_19864_amd.workloads import WORKLOADS
    return make_desc(WORKLOADS["bert_base"].replace(**kw))


def test_stage_attention_plan():
    d = stage_desc()
    assert B.ringada_stage_plan_attention(d, B.StageAttention(), 32, 128) == 0
    n = B.ringada_stage_plan_attention(d, B.StageAttention(window=40), 32, 128)
    assert n >= 32 * 12 * 128 * 4
    t = B.StageAttention(n_buckets=8, max_distance=20, g_table=BASE)
    assert B.ringada_stage_plan_attention(d, t, 32, 128) >= 32 * 12 * 128 * 4 + 32 * 12 * 41 * 4
    for bad, status in ((B.StageAttention(window=-1), B.RINGADA_E_INVALID),
                        (B.StageAttention(sinks=-1), B.RINGADA_E_INVALID),
                        (B.StageAttention(n_buckets=4, max_distance=2000), B.RINGADA_E_UNSUPPORTED)):
        with pytest.raises(B.RingadaError) as e:
            B.ringada_stage_plan_attention(d, bad, 32, 128)
        assert e.value.status == status
    with pytest.raises(B.RingadaError):
        B.ringada_stage_plan_attention(d, B.StageAttention(window=4), 33, 128)


def test_stage_options_are_checked():
    h = B.ringada_stage_create(stage_desc(), None, 0)
    try:
        for bad in (B.StageAttention(window=-1), B.StageAttention(n_buckets=4, max_distance=3),
                    B.StageAttention(table=BASE, bucket=BASE), B.StageAttention(window=1, g_table=BASE),
                    B.StageAttention(n_buckets=4, max_distance=3, table=BASE),
                    B.StageAttention(window=4, workspace=BASE + 16, workspace_bytes=1 << 20)):
            with pytest.raises(B.RingadaError) as e:
                B.ringada_stage_set_attention(h, bad)
            assert e.value.status == B.RINGADA_E_INVALID
        for p, rng in ((-0.1, BASE), (1.0, BASE), (0.1, None), (0.1, BASE + 4), (float("nan"), BASE)):
            with pytest.raises(B.RingadaError) as e:
                B.ringada_stage_set_dropout(h, p, rng, 0)
            assert e.value.status == B.RINGADA_E_INVALID
        B.ringada_stage_set_attention(h, B.StageAttention(window=4))
        B.ringada_stage_set_attention(h, None)
        B.ringada_stage_set_dropout(h, 0.0, None, 0)
    finally:
        B.ringada_stage_destroy(h)
