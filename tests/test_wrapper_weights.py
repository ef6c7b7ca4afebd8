"""The wrappers take e2m1 weights of the very size that the shape says, in rows of the right length (no GPU)."""
import pytest
import torch

from paper_2607_18631_amd import moe
from test_abi_serving import BASE, _Pretend

U8 = torch.uint8
SH = BASE.replace(T=4, F=96, F_shared=32)
# rows and values per row
SIZES = dict(w13=(8 * 2 * 96, 64), w2=(8 * 64, 96), ws13=(2 * 32, 64), ws2=(64, 32))


@pytest.fixture(autouse=True)
def calls(monkeypatch):
    """No call of the library is made: those that pass the wrapper's checks are listed."""
    seen = []
    monkeypatch.setattr(moe, "_on", lambda device, stream, call, *args: seen.append(call))
    return seen


def p(*shape, dtype=torch.bfloat16):
    return _Pretend(torch.zeros(shape, dtype=dtype))


def wrong(rows, n):
    """Tensors of other sizes, or of other rows."""
    yield "longer", p(rows + 1, n, dtype=U8)
    yield "longer and flat", p(rows * n + 16, dtype=U8)
    yield "shorter", p(rows - 1, n, dtype=U8)
    yield "another type", p(rows, n)
    if rows != n:
        yield "transposed", p(n, rows, dtype=U8)
    yield "not contiguous", _Pretend(torch.zeros((rows, 2 * n), dtype=U8)[:, :n])


def decode(**change):
    q = {n: p(rows, K // 2, dtype=U8) for n, (rows, K) in SIZES.items()}
    s = {n: p(rows, K // 32, dtype=U8) for n, (rows, K) in SIZES.items()}
    for name, t in change.items():
        (s if name.endswith("_scales") else q)[name.replace("_scales", "")] = t
    moe.moe_layer_decode(SH, p(4, 64), p(8, 64), None, q["w13"], q["w2"], q["ws13"], q["ws2"], p(4, 64), p(1 << 20, dtype=U8),
                         tuple(s[n] for n in SIZES))


def mlp(**change):
    cap = SH.capacity
    args = dict(x_q=p(cap, 64, dtype=U8), x_scales=p(cap, 2, dtype=U8), offsets=p(9, dtype=torch.int32),
                y_perm=p(cap, 64), ws=p(1 << 20, dtype=U8))
    for n in ("w13", "w2"):
        rows, K = SIZES[n]
        args.update({n + "_q": p(rows, K // 2, dtype=U8), n + "_scales": p(rows, K // 32, dtype=U8)})
    moe.moe_mx_grouped_ffn(SH, moe.MOE_MX_E4M3, **{**args, **change})


@pytest.mark.parametrize("name", list(SIZES))
@pytest.mark.parametrize("scales", [False, True])
def test_few_token_layer(name, scales):
    rows, K = SIZES[name]
    arg = name + "_scales" if scales else name
    for what, t in wrong(rows, K // 32 if scales else K // 2):
        with pytest.raises(moe.MoEError, match=f"{arg} is .* expected contiguous"):
            decode(**{arg: t})
            pytest.fail(what)


@pytest.mark.parametrize("name", ["w13", "w2"])
@pytest.mark.parametrize("scales", [False, True])
def test_expert_mlp(name, scales):
    rows, K = SIZES[name]
    arg = name + ("_scales" if scales else "_q")
    for what, t in wrong(rows, K // 32 if scales else K // 2):
        with pytest.raises(moe.MoEError, match=f"{arg} is .* expected contiguous"):
            mlp(**{arg: t})
            pytest.fail(what)


def test_forms_that_fit(calls):
    """Flat, a matrix of all rows, and a matrix per expert."""
    rows, K = SIZES["w13"]
    for shape in ((rows * K // 2,), (rows, K // 2), (8, rows // 8, K // 2), (8, 2, rows // 16, K // 2)):
        decode(w13=p(*shape, dtype=U8))
        mlp(w13_q=p(*shape, dtype=U8))
    assert len(calls) == 8
