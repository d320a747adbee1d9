"""Calls on rotary positions and growing sets whose tensors lie elsewhere than they say: of more tokens than there are positions where the layout
depends on their number, or on another device."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

from paper_2506_19225_amd import vxl

from test_binding_native import streams  # noqa: F401
from test_mixed_refusals import B, BF, D, HKV, HQ, I32, T, Typed, append, attend, evict, launches, refused, rotate  # noqa: F401

HEADS_FIRST = vxl.make_desc(HQ, HKV, D, "bf16")


def of(heads, tokens):
    return Typed((heads, tokens, D), BF)


def good(n=B * T):
    return dict(q=of(HQ, n), k=of(HKV, n), qo=of(HQ, n), ko=of(HKV, n))


def test_rotation_of_heads_of_more_tokens_than_positions():
    """[heads, tokens, D] without strides: rows of a head after the first lie where the number of positions says."""
    n = B * T
    assert refused(rotate, desc=HEADS_FIRST, **good()) == vxl.VXL_ERR_HIP
    assert refused(rotate, desc=HEADS_FIRST, **dict(good(), k=None, ko=None)) == vxl.VXL_ERR_HIP
    for less in (n - 1, 1, 0):
        at = Typed((less,), I32)
        assert refused(rotate, desc=HEADS_FIRST, at=at, **good()) == vxl.VXL_ERR_INVALID_ARG, less
        for name, x in good().items():
            assert refused(rotate, desc=HEADS_FIRST, at=at, **dict(good(less), **{name: x})) == vxl.VXL_ERR_INVALID_ARG, (less, name)
    for name, x in good().items():
        more = Typed((x.shape[0], n + 1, D), BF)
        assert refused(rotate, desc=HEADS_FIRST, **dict(good(), **{name: more})) == vxl.VXL_ERR_INVALID_ARG, name
    # token after token fewer positions are the first tokens, as before
    assert refused(rotate, at=Typed((n - 1,), I32)) == refused(rotate, at=Typed((1,), I32)) == vxl.VXL_ERR_HIP
    one = vxl.make_desc(1, 1, D, "bf16")                                      # (one head: the same)
    assert refused(rotate, desc=one, q=of(1, n + 3), k=of(1, n + 2), qo=of(1, n), ko=of(1, n + 1)) == vxl.VXL_ERR_HIP
    empty = {name: Typed((x.shape[0], 0, D), BF, 0) for name, x in good().items()}
    rotate(desc=HEADS_FIRST, at=Typed((0,), I32, 0), **empty)                # (nothing to do)
    rotate(at=Typed((0,), I32, 0))


def test_append_of_heads_of_more_tokens_than_positions():
    n = B * T
    fit = dict(q=of(HQ, n), k=of(HKV, n), v=of(HKV, n))
    assert refused(append, desc=HEADS_FIRST, **fit) == vxl.VXL_ERR_HIP
    for name, x in fit.items():
        for tokens in (n + 1, 2 * n):
            assert refused(append, desc=HEADS_FIRST, **dict(fit, **{name: of(x.shape[0], tokens)})) == vxl.VXL_ERR_INVALID_ARG, name
    assert refused(append, q=Typed((n + 5, HQ, D), BF), k=Typed((n + 1, HKV, D), BF)) == vxl.VXL_ERR_HIP


def test_rotation_without_positions():
    """Not a call of no tokens, which would leave the results unwritten without a word."""
    for kw in (dict(), dict(k=None, ko=None), dict(desc=HEADS_FIRST, **good())):
        assert refused(rotate, at=None, **kw) == vxl.VXL_ERR_INVALID_ARG


@pytest.mark.parametrize("call,optional", [(rotate, "k ko"), (append, "pos w"), (attend, "lse w w2"), (attend, "at pos"), (evict, "new")])
def test_tensors_of_nothing_are_not_none(call, optional):
    """A tensor without elements in the place of one that may be None: refused, not left out."""
    import inspect
    have = {k: p.default for k, p in inspect.signature(call).parameters.items()}
    rest = {rotate: {}, append: {}, attend: dict(rule=None), evict: dict(recent=0)}[call]
    names = optional.split()
    assert refused(call, **rest, **{name: None for name in names}) == vxl.VXL_ERR_HIP
    for some in [names] + [[name] for name in names]:
        for shape in ((0,), have[some[0]].shape[:-1] + (0,)):
            with pytest.raises((vxl.VxlError, IndexError)) as e:
                call(**rest, **{name: Typed(shape, have[name].dtype, 0) for name in some})
            assert not isinstance(e.value, vxl.VxlError) or e.value.status == vxl.VXL_ERR_INVALID_ARG, some


def test_slopes_of_no_head():
    with pytest.raises(ValueError, match="slope per query head"):
        attend(rule=vxl.ScoreRule(slopes=Typed((0,), torch.float32, 0)))


@pytest.mark.filterwarnings("ignore:Accessing the data pointer of FakeTensor")
@pytest.mark.parametrize("call", [attend, evict])
def test_a_workspace_of_another_device(call, monkeypatch):
    """Tensors that say where they are and have no memory: of the current device for the library to refuse, of another one refused here."""
    def on(device):
        with FakeTensorMode():
            return torch.empty(1 << 20, dtype=torch.uint8, device=device)
    monkeypatch.setattr(vxl, "_native", None)                                # (a binding that asks for the device as it is set here)
    assert refused(call, ws=on("cuda:0")) == vxl.VXL_ERR_WORKSPACE
    with pytest.raises(ValueError, match="another device than the current one"):
        call(ws=on("cuda:1"))
    monkeypatch.setattr(vxl, "_current_device", lambda: 1)
    monkeypatch.setattr(vxl, "_native", None)
    assert refused(call, ws=on("cuda:1")) == vxl.VXL_ERR_WORKSPACE
    with FakeTensorMode():
        weight = torch.empty(2, 2, 20, device="cuda:1")
    with pytest.raises(ValueError, match="several devices"):
        call(w=weight, ws=on("cuda:0"))
