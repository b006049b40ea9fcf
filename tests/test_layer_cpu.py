"""Host logic of the layer operators that needs no GPU: refusals before any launch, geometry, frequencies."""
import math

import pytest
import torch

import paper_2506_08520_gb300 as pn
from paper_2506_08520_gb300 import build as nbuild
from paper_2506_08520_gb300 import layer


@pytest.fixture(scope="module", autouse=True)
def lib():
    nbuild.build()


def sig(*shape, dtype=torch.bfloat16, stride=None):
    t = torch.empty(shape, dtype=dtype, device="meta")
    return (t.shape, t.stride() if stride is None else stride, t.dtype)


def test_cpu_tensors_are_refused():
    x = torch.zeros(2, 3, 4, 8)
    ld, inv = torch.zeros(3), torch.zeros(4, dtype=torch.float64)
    for call in (lambda: pn.layer_norm(x), lambda: pn.rotary(x, inv), lambda: pn.rotary_qk(x, x, inv),
                 lambda: pn.linear_attention(x, x, x, ld), lambda: pn.linear_attention_backward(x, x, x, x, ld),
                 lambda: pn.linear_attention_step(x[:, :, 0], x[:, :, 0], x[:, :, 0], ld, torch.zeros(2, 3, 8, 8)),
                 lambda: pn.layer_norm_backward(x, x, x[..., 0], x[..., 0])):
        with pytest.raises(ValueError, match="no CPU path"):
            call()


def test_rotary_plan():
    q, k, inv = sig(2, 6, 50, 30), sig(2, 3, 50, 30), sig(15, dtype=torch.float64)
    plan = lambda *a: layer._rotary_plan(*a)  # noqa: E731
    rows, r, bits, step, n, N, d, lay, dt = plan(q, k, inv, None, None, None, "half")
    assert (r, bits, n, N, d, lay) == (30, 0, 2, 50, 30, 0) and [x[2] for x in rows] == [6, 3]
    assert list(rows[1][0]) == [3 * 1500, 1500, 30]
    pos = sig(2, 50, dtype=torch.int32)
    assert plan(q, k, inv, pos, None, None, "interleaved")[2:4] == (32, 50)
    assert plan(q, k, inv, sig(50, dtype=torch.int64), None, None, "half")[2:4] == (64, 0)
    for bad in ((q, sig(2, 3, 49, 30), inv, None, None, None, "half"), (sig(2, 6, 50), None, inv, None, None, None, "half"),
                (q, k, sig(15), None, None, None, "half"), (q, k, inv, None, None, None, "spiral"),
                (q, k, inv, sig(49, dtype=torch.int64), None, None, "half"),
                (q, k, inv, sig(2, 50, dtype=torch.int16), None, None, "half"),
                (q, k, inv, sig(2, 50, dtype=torch.int32, stride=(100, 2)), None, None, "half"),
                (q, k, inv, None, sig(2, 6, 50, 32), None, "half"), (q, sig(2, 3, 50, 30, dtype=torch.float16), inv, None, None, None, "half"),
                (sig(2, 6, 50, 30, stride=(18000, 3000, 60, 2)), None, inv, None, None, None, "half"),
                (sig(2, 6, 50, 30, dtype=torch.int32), None, inv, None, None, None, "half")):
        with pytest.raises(ValueError):
            plan(*bad)


def test_linear_plan():
    q, v, ld = sig(2, 3, 40, 16), sig(2, 3, 40, 24), sig(3, dtype=torch.float32)
    st = sig(2, 3, 16, 24, dtype=torch.float32)
    good = dict(q=q, k=q, v=v, dout=None, log_decay=ld, state=st, lengths=sig(2, dtype=torch.int32), dstate=None, out=v,
                backward=0)

    def plan(**kw):
        return layer._linear_plan(*{**good, **kw}.values())

    assert plan()[1:7] == (2, 3, 40, 16, 24, 0)
    assert plan(q=sig(1, 1, 9000, 64), k=sig(1, 1, 9000, 64), v=sig(1, 1, 9000, 64), log_decay=sig(1, dtype=torch.float32),
                state=None, lengths=None, out=None)[6] > 0
    for bad in (dict(k=v), dict(v=sig(2, 3, 41, 24)), dict(log_decay=sig(3)), dict(log_decay=sig(2, dtype=torch.float32)),
                dict(state=sig(2, 3, 24, 16, dtype=torch.float32)), dict(state=sig(2, 3, 16, 24)),
                dict(state=sig(2, 3, 16, 24, dtype=torch.float32, stride=(1152, 384, 1, 16))),
                dict(lengths=sig(2, dtype=torch.int64)), dict(lengths=sig(3, dtype=torch.int32)), dict(out=q),
                dict(q=sig(2, 3, 40, 129), k=sig(2, 3, 40, 129)), dict(q=sig(2, 3, 40), k=sig(2, 3, 40)),
                dict(dout=sig(2, 3, 40, 24, dtype=torch.float32))):
        with pytest.raises(ValueError):
            plan(**bad)
    with pytest.raises(pn.NystraError):
        big = sig(1, 1, (1 << 24) + 1, 8)
        plan(q=big, k=big, v=big, log_decay=sig(1, dtype=torch.float32), state=None, lengths=None, out=None)


def test_rows_of_a_norm():
    def rows(x):
        return layer._rows(x.shape, x.stride())

    t = torch.empty(4, 6, 32, device="meta")
    assert rows(t) == (24, 32) and rows(t[0, 0]) == (1, 32)
    assert rows(t[..., 8:24]) == (24, 32) and rows(t[:, 0]) == (4, 192)
    assert rows(t.transpose(0, 1)[:1]) == (4, 192)
    assert rows(torch.empty(32, device="meta").expand(5, 32)) == (5, 0)
    assert rows(torch.empty(0, 32, device="meta"))[0] == 0
    for bad in (t[:, :5], t.transpose(0, 1), t.transpose(1, 2), t[0, 0, ::2], t[..., ::2]):
        with pytest.raises(ValueError):
            rows(bad)


def test_norm_plan():
    x, w = sig(4, 6, 32), sig(32, dtype=torch.float32)
    dt, wdt, rows, C, xs, ys, ds, need = layer._norm_plan(x, w, None, None, x)
    assert (dt, wdt, rows, C, xs, ys, ds) == (1, 0, 24, 32, 32, 32, 32) and need > 0
    for bad in ((x, sig(31), None, None, None), (x, sig(32, dtype=torch.float16), None, None, None),
                (x, w, sig(32), None, None), (x, sig(32, stride=(2,)), None, None, None), (x, None, None, sig(24, 32), None),
                (x, None, None, None, sig(4, 6, 32, dtype=torch.float32)), (sig(4, 6, 32, dtype=torch.int8), None, None, None, None)):
        with pytest.raises(ValueError):
            layer._norm_plan(*bad)


def test_rotary_frequencies():
    plain, one = pn.rotary_frequencies(8, base=100.0, device="cpu")
    assert plain.dtype == torch.float64 and one == 1.0
    assert torch.allclose(plain, torch.tensor([1, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64))
    assert torch.allclose(pn.rotary_frequencies(8, base=100.0, scaling="linear", factor=4, device="cpu")[0], plain / 4)
    yarn, amp = pn.rotary_frequencies(64, scaling="yarn", factor=8, original_length=2048, device="cpu")
    assert amp == pytest.approx(0.1 * math.log(8) + 1) and yarn.shape == (32,)
    assert pn.rotary_frequencies(0, device="cpu")[0].shape == (0,)
    for bad in (dict(rotary_dim=7), dict(rotary_dim=-2), dict(rotary_dim=258), dict(rotary_dim=8, base=1.0),
                dict(rotary_dim=8, factor=0.5), dict(rotary_dim=8, factor=math.inf), dict(rotary_dim=8, scaling="other"),
                dict(rotary_dim=8, scaling="yarn", factor=2)):
        with pytest.raises(ValueError):
            pn.rotary_frequencies(**bad, device="cpu")


@pytest.mark.parametrize("big", [2 ** 31, 2 ** 32 + 8])
def test_sizes_beyond_32_bits_are_refused(big):
    """The C entries take sizes of 32 bits: a larger one must not reach them, where only its low bits would count."""
    ld, inv = sig(1, dtype=torch.float32), sig(1, dtype=torch.float64)
    long, many, wide = sig(1, 1, big, 2), sig(big, 1, 1, 2), sig(1, big, 1, 2)
    for x in (long, many, wide):
        heads = sig(x[0][1], dtype=torch.float32)
        with pytest.raises(ValueError, match="at most"):
            layer._linear_plan(x, x, x, None, heads, None, None, None, None, 0)
        with pytest.raises(ValueError, match="at most"):
            layer._linear_plan(x, x, x, x, heads, None, None, None, None, 1)
        for k in (None, x):
            with pytest.raises(ValueError, match="at most"):
                layer._rotary_plan(x, k, inv, None, None, None, "half")
    with pytest.raises(ValueError, match="at most"):  # the keys' heads alone
        layer._rotary_plan(sig(1, 1, 1, 2), wide, inv, None, None, None, "half")
    with pytest.raises(ValueError, match="at most"):  # a table as long as the head of 2 that its low bits would fit
        layer._rotary_plan(sig(1, 1, 1, 2), None, sig(big, dtype=torch.float64), None, None, None, "half")
    for x in (sig(big, 1, 2), sig(1, big, 2)):
        heads = sig(x[0][1], dtype=torch.float32)
        state = sig(*x[0][:2], 2, 2, dtype=torch.float32)
        with pytest.raises(ValueError, match="at most"):
            layer._step_plan(x, x, x, heads, state, state, None)
    for w in (None, sig(big)):
        with pytest.raises(ValueError, match="at most"):
            layer._norm_plan(sig(1, big), w, None, None, None)
    assert layer._norm_plan(sig(big, 1), None, None, None, None)[2] == big  # rows are 64 bits there


def test_norm_rows_too_long():
    with pytest.raises(pn.NystraError):
        layer._norm_plan(sig(1, 2 ** 30 + 1), None, None, None, None)


def test_gradients_that_would_be_cut_off():
    """Both kinds: a graph to record, and a tangent that goes along forward."""
    x = torch.ones(3)
    assert not layer._recorded(x)
    g = x.clone().requires_grad_()
    assert layer._recorded(g)
    with torch.no_grad():
        assert not layer._recorded(g)
    import torch.autograd.forward_ad as fw
    with fw.dual_level():
        dual = fw.make_dual(x, x)
        assert layer._recorded(dual) and not layer._recorded(x)
        with torch.no_grad():  # which does not stop a tangent
            assert layer._recorded(dual) == (fw.unpack_dual(dual * 2).tangent is not None)
        primal = fw.unpack_dual(dual).primal
        assert not layer._recorded(primal)

        class Twice(torch.autograd.Function):  # of one's own, with its derivatives: fine inside
            @staticmethod
            def forward(x):
                assert not layer._recorded(x)
                return x * 2

            @staticmethod
            def setup_context(ctx, inputs, output):
                pass

            @staticmethod
            def jvp(ctx, t):
                return t * 2

        assert fw.unpack_dual(Twice.apply(dual)).tangent.tolist() == [2, 2, 2]
