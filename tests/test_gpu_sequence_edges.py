"""Attention over sequences where values are not finite, very large, or cancel: what a pair that is seen, or not seen, gives."""
import math

import pytest
import torch

from tests.test_gpu_sequence_attention import Call

pytestmark = pytest.mark.gpu
N, AT = 300, 150


def pair_of_calls(seed, dtype, n=N, heads=2, kv_heads=1, d=64, causal=True, **change):
    """Two calls of the same inputs; `change` [name: function of the tensor] is made in both, so that it can make scores one-sided."""
    out = []
    for _ in range(2):
        c = Call(seed, dtype, heads, kv_heads, d, n, n, q_offsets=[0, n], k_offsets=[0, n], causal=causal)
        for name, f in change.items():
            c.dev[name].copy_(f(c.dev[name]))
        out.append(c)
    return out


def positive(channel):
    def f(t):
        t = t.clone()
        t[..., channel] = t[..., channel].abs() + 0.5
        return t
    return f


def run(*calls):
    for c in calls:
        c.forward()
        c.backward()


def same(a, b, what):
    assert torch.equal(a, b), (what, float((a.float() - b.float()).abs().nan_to_num(1e30).max()))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_key_without_probability_gets_no_gradient(dtype):
    """Channel 5 of one key is -inf and of all queries positive: its scores are -inf, its probabilities zero, as they are exactly where that channel is -1e5
    (scores thousands below the row's others).  Out, lse, dk and dv keep their bits, also where the queries do not fill their last tile."""
    clean, bad = pair_of_calls(200, dtype, causal=False, q=positive(5))
    clean.dev["k"][AT, :, 5] = -1e5
    bad.dev["k"][AT, :, 5] = -math.inf
    run(clean, bad)
    for n in ("out", "dk", "dv"):
        same(bad.out[n], clean.out[n], n)
    same(bad.lse, clean.lse, "lse")
    assert float(bad.out["dk"][AT].abs().sum()) == 0 and float(bad.out["dv"][AT].abs().sum()) == 0


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_seen_key_with_an_infinite_channel(dtype, causal):
    """As above: everything keeps its bits but channel 5 of dq, which is not finite for the rows that see the key."""
    clean, bad = pair_of_calls(201, dtype, causal=causal, q=positive(5))
    clean.dev["k"][AT, :, 5] = -1e5
    bad.dev["k"][AT, :, 5] = -math.inf
    run(clean, bad)
    first = AT if causal else 0
    dq, want = bad.out["dq"].clone(), clean.out["dq"].clone()
    assert not bool(torch.isfinite(dq[first:, :, 5]).any())
    dq[first:, :, 5] = want[first:, :, 5] = 0
    same(dq, want, "dq")
    for n in ("out", "dk", "dv"):
        same(bad.out[n], clean.out[n], n)
    same(bad.lse, clean.lse, "lse")
    assert bool(torch.isfinite(want.float()).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_gradient_of_a_row(dtype):
    """Channel 3 of one row of dout is +inf and that channel of v positive: the row's dP and delta are +inf, its dS is NaN.  dv gets +inf in that channel from every key that
    the row sees, dk is NaN there, and keys that it does not see keep their bits."""
    clean, bad = pair_of_calls(202, dtype, v=positive(3))
    bad.dev["dout"][AT, 1, 3] = math.inf
    run(clean, bad)
    seen = AT + 1
    assert bool(torch.isnan(bad.out["dk"][:seen]).all())
    dv, want = bad.out["dv"].clone(), clean.out["dv"].clone()
    assert bool((dv[:seen, :, 3] == math.inf).all())
    dv[:seen, :, 3] = want[:seen, :, 3] = 0
    same(dv, want, "dv")
    same(bad.out["dk"][seen:], clean.out["dk"][seen:], "dk")
    assert bool(torch.isnan(bad.out["dq"][AT, 1]).all())
    rest = torch.ones(N, 2, dtype=torch.bool)
    rest[AT, 1] = False
    same(bad.out["dq"][rest], clean.out["dq"][rest], "dq")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_infinite_value_of_a_key_without_probability(dtype):
    """The scores of one key are -inf and a channel of its value +inf: zero times infinity is NaN in that channel of the rows that see it, on the diagonal as elsewhere."""
    clean, bad = pair_of_calls(203, dtype, q=positive(5))
    clean.dev["k"][AT, :, 5] = -1e5
    bad.dev["k"][AT, :, 5] = -math.inf
    bad.dev["v"][AT, :, 3] = math.inf
    clean.forward()
    bad.forward()
    out, want = bad.out["out"].clone(), clean.out["out"].clone()
    assert bool(torch.isnan(out[AT:, :, 3]).all())
    out[AT:, :, 3] = want[AT:, :, 3] = 0
    same(out, want, "out")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_channel_of_an_infinite_key_that_is_seen(dtype):
    """Its probabilities are zero, and zero times infinity is NaN in that channel of dq: of the rows that see the key, in and behind the tile on the diagonal, and of no others."""
    clean, bad = pair_of_calls(208, dtype, q=positive(5))
    bad.dev["k"][AT, :, 5] = -math.inf
    run(clean, bad)
    assert bool(torch.isnan(bad.out["dq"][AT:, :, 5]).all())
    same(bad.out["dq"][:AT], clean.out["dq"][:AT], "dq")
    assert bool(torch.isfinite(bad.out["dq"][..., :5].float()).all())


@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_row_whose_scores_are_all_minus_infinity(dtype, causal):
    """It sees keys, so its softmax is not that of a row that sees none: out and its gradients are NaN, lse -inf; other rows, and keys that it does not see, keep their bits."""
    clean, bad = pair_of_calls(204, dtype, causal=causal, k=positive(5))
    bad.dev["q"][AT, 0, 5] = -math.inf
    run(clean, bad)
    assert bool(torch.isnan(bad.out["out"][AT, 0]).all()) and float(bad.lse[0, AT]) == -math.inf
    assert bool(torch.isnan(bad.out["dq"][AT, 0]).all())
    seen = AT + 1 if causal else N
    rest = torch.ones(N, 2, dtype=torch.bool)
    rest[AT, 0] = False
    for n in ("out", "dq"):
        same(bad.out[n][rest], clean.out[n][rest], n)
    for n in ("dk", "dv"):
        assert bool(torch.isnan(bad.out[n][:seen]).all()), n
        same(bad.out[n][seen:], clean.out[n][seen:], n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_token_whose_scores_are_minus_infinity_over_a_long_cache(dtype):
    """All of them: NaN and lse -inf, from pieces of the keys too.  Those of the first 1500 keys alone: as without these keys.  A cache that holds none: zeros."""
    calls = []
    for _ in range(2):
        c = Call(205, dtype, 4, 2, 64, 1, 5000, batch=3, k_lengths=[5000, 4000, 0], causal=True)
        c.dev["q"].copy_(positive(5)(c.dev["q"]))
        calls.append(c)
    clean, bad = calls
    clean.dev["k"][1, :1500, :, 5] = -1e5
    bad.dev["k"][1, :1500, :, 5] = -math.inf
    bad.dev["k"][0, :, :, 5] = -math.inf
    for c in calls:
        c.forward()
    assert bool(torch.isnan(bad.out["out"][0]).all()) and bool((bad.lse[:, 0] == -math.inf).all())
    same(bad.out["out"][1:], clean.out["out"][1:], "out")
    same(bad.lse[:, 1:], clean.lse[:, 1:], "lse")
    assert float(bad.out["out"][2].abs().sum()) == 0 and bool((bad.lse[:, 2] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [False, True], ids=["full", "causal"])
@pytest.mark.parametrize("rows,keys,batch,heads", [(200, 700, 1, 2), (130, 200, 64, 4), (1, 200, 256, 8)])
def test_values_of_1e30_under_growing_scores(rows, keys, batch, heads, causal, dtype):
    """Scores that grow by some 24 along the keys, and values whose weighted sum is far below the type's largest while e^24 times one of them is above it."""
    d = 64
    c = Call(206, dtype, heads, heads, d, rows, keys, batch=batch, causal=causal, scale=1.0, spread=0.05)
    c.host["q"][..., 0] = 1.0
    c.host["k"][..., 0] = torch.linspace(0.0, 24.0, keys)[None, :, None].to(c.io)
    c.host["v"] = (c.host["v"].double() * 1e30).to(c.io)
    for n in "qkv":
        c.dev[n].copy_(c.host[n])
    c.forward()
    c.check(train=False)
