"""Norm and rotation of queries and keys against the fp64 oracle, through the C ABI.

Tolerance in fp32, relative to the size of the pair (|a| + |b| after the norm): the row's sum of squares passes through at most 13 fp32
roundings (half of their relative error reaches its root: 4e-7), rsqrtf adds 2 ulp (2.4e-7), the products with it and the weight three
roundings (1.8e-7), the angle, reduced in 64 bits and then held in fp32 as a fraction of a turn, 2^-25 x 2 pi / 2 (1e-7), sincospif 2 ulp
(2.4e-7) and the rotation three roundings (1.8e-7): 1.4e-6 in all, 2e-6 allowed.  bf16 adds the last rounding, 2^-8 of the result."""
import numpy as np
import pytest
import torch

from oracle import kv4_oracle as O
from paper_2609_23900_b200 import binding
from synthetic import workload as W
from tests.harness import ctx

pytestmark = pytest.mark.gpu


def dev(a, dt):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dt).cuda()


def freqs(rot):
    return (1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / max(rot, 1))).float().cuda()


def check(got, x, pos, freq, dt, **kw):
    """x: the tensor the kernel read; kw as the oracle's."""
    h = lambda t: t.double().cpu().numpy()                               # noqa: E731
    T = pos.shape[-1]
    xr, fr = h(x).reshape(T, x.shape[-2], x.shape[-1]), h(freq)
    w = kw.pop("weight", None)
    kw["weight"] = h(w) if w is not None else None
    ref = O.norm_rope(xr, pos, fr, **kw)
    plain = O.norm_rope(xr, pos, [], **{**kw, "sections": None, "turns": False})       # the norm alone: sizes of the pairs
    size = np.abs(plain)
    n = len(fr)
    first, second = (slice(0, n), slice(n, 2 * n)) if kw.get("style", "half") == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    both = size[..., first] + size[..., second]
    size[..., first] = size[..., second] = both * max(1.0, abs(kw.get("mscale", 1.0)))
    tol = 2e-6 * size + 1e-30
    if dt == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(ref) + tol)
    err = np.abs(h(got).reshape(ref.shape) - ref)
    assert (err <= tol).all(), f"worst ratio {(err / tol).max():.2f}"


CASES = [
    # T, Hq, Hkv, dh, rot, style, sections, turns
    (1, 32, 8, 128, 128, "half", None, False),
    (1, 1, 1, 64, 64, "pairs", None, False),
    (3, 5, 1, 64, 32, "half", None, False),
    (7, 6, 3, 256, 64, "half", None, False),
    (130, 17, 2, 128, 48, "pairs", None, False),
    (257, 8, 8, 128, 128, "half", [24, 20, 20], False),
    (66, 4, 2, 128, 96, "half", [16, 16, 16], True),
    (65, 4, 2, 256, 256, "pairs", [128, 0, 0], True),
    (33, 2, 1, 64, 16, "half", [3, 3, 2], True),
    (5, 3, 0, 128, 128, "half", None, False),                             # queries alone
    (9, 2, 2, 128, 0, "half", None, False),                               # norm alone
    (1201, 40, 8, 128, 64, "half", [12, 10, 10], True),                   # several tokens a CTA, the last one not full
]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("T,Hq,Hkv,dh,rot,style,sections,turns", CASES)
def test_matches_the_oracle(T, Hq, Hkv, dh, rot, style, sections, turns, dt):
    rs = np.random.default_rng(T * dh + rot)
    row = (Hq + 2 * Hkv) * dh + 16                                        # parts of longer rows
    packed = dev(rs.standard_normal((T, row)) * 3, dt)
    q = packed[:, :Hq * dh].unflatten(1, (Hq, dh))
    k = packed[:, Hq * dh:(Hq + Hkv) * dh].unflatten(1, (Hkv, dh)) if Hkv else None
    wide = torch.full((T, Hq * dh + 32), 5.0, dtype=dt, device="cuda")
    q_out = wide[:, :Hq * dh].unflatten(1, (Hq, dh))
    k_out = torch.empty(T, Hkv, dh, dtype=dt, device="cuda") if Hkv else None
    qw, kw = dev(rs.standard_normal(dh), dt), dev(rs.standard_normal(dh), dt)
    pos = rs.integers(0, 1 << 20, (3 if sections else 1, T)).astype(np.int32)
    freq = freqs(rot)
    layer = binding.QkNormRope(q=q, k=k, q_out=q_out, k_out=k_out, inv_freq=freq if rot else None, q_weight=qw, k_weight=kw if Hkv else None, eps=1e-5,
                               weight_offset=0.5, mscale=1.25, style=style, pos=dev(pos, torch.int32), sections=sections, turns=turns)
    ctx().qk_norm_rope(layer)
    torch.cuda.synchronize()
    opts = dict(offset=0.5, eps=1e-5, style=style, sections=sections, turns=turns, mscale=1.25)
    check(q_out, q, pos, freq, dt, weight=qw, **opts)
    if Hkv:
        check(k_out, k, pos, freq, dt, weight=kw, **opts)
    assert (wide[:, Hq * dh:] == 5.0).all()                               # nothing beyond the heads


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B,N", [(1, 1), (3, 28), (5, 200)])
def test_tree_nodes_stand_behind_their_context(B, N, dt):
    rs = np.random.default_rng(B * N)
    parent = np.array([W.tree_random(W.IntStream(W.stream_key(7, b)), N, 9) if N > 1 else [-1] for b in range(B)], dtype=np.int32)
    desc = ctx().tree_desc(parent, slot=np.array([rs.permutation(N + 3)[:N] for _ in range(B)]), n_slots=N + 3)
    q, k = dev(rs.standard_normal((B, N, 4, 128)), dt), dev(rs.standard_normal((B, N, 2, 128)), dt)
    ctx_len, freq = rs.integers(0, 200000, B).astype(np.int32), freqs(128)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    ctx().qk_norm_rope(binding.QkNormRope(q=q, k=k, q_out=qo, k_out=ko, inv_freq=freq, ctx_len=dev(ctx_len, torch.int32)), desc)
    torch.cuda.synchronize()
    depth = np.zeros((B, N), np.int64)
    for b in range(B):
        for i in range(N):
            depth[b, i] = 0 if parent[b, i] < 0 else depth[b, parent[b, i]] + 1
    pos = (ctx_len[:, None] + depth).reshape(1, -1)
    check(qo, q, pos, freq, dt)
    check(ko, k, pos, freq, dt)


@pytest.mark.parametrize("style", ["half", "pairs"])
def test_in_place_without_norm_and_rows_of_zeros_and_nan(style):
    rs = np.random.default_rng(1)
    x = rs.standard_normal((40, 6, 128))
    x[3, 2], x[5, 1, 9] = 0.0, np.nan
    q = dev(x, torch.bfloat16)
    keep, freq, pos = q.clone(), freqs(128), rs.integers(0, 999, (1, 40)).astype(np.int32)
    ctx().qk_norm_rope(binding.QkNormRope(q=q, q_out=q, inv_freq=freq, pos=dev(pos, torch.int32), normalise=False, style=style))
    torch.cuda.synchronize()
    ref = O.norm_rope(keep.double().cpu().numpy(), pos, freq.double().cpu().numpy(), normalise=False, style=style)
    got = q.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and (got[3, 2] == 0).all()
    ok = ~np.isnan(ref)
    assert (np.abs(got - ref)[ok] <= 2.0 ** -8 * np.abs(ref)[ok] + 2e-5).all()
    # with the norm: zeros stay zeros (eps), a NaN stays in its row
    q2 = torch.empty_like(keep)
    ctx().qk_norm_rope(binding.QkNormRope(q=keep, q_out=q2, inv_freq=freq, pos=dev(pos, torch.int32), style=style))
    torch.cuda.synchronize()
    nan = torch.isnan(q2)
    assert nan[5, 1].all() and nan.sum() == 128 and (q2[3, 2] == 0).all()


def test_the_same_token_alone_and_among_many():
    """One token a CTA and several: bitwise the same rows."""
    rs = np.random.default_rng(3)
    x, pos, freq = dev(rs.standard_normal((4000, 20, 128)), torch.bfloat16), dev(rs.integers(0, 1 << 17, 4000), torch.int32), freqs(128)
    many, few = torch.empty_like(x), torch.empty_like(x[:3])
    ctx().qk_norm_rope(binding.QkNormRope(q=x, q_out=many, inv_freq=freq, pos=pos))
    ctx().qk_norm_rope(binding.QkNormRope(q=x[:3], q_out=few, inv_freq=freq, pos=pos[:3]))
    torch.cuda.synchronize()
    assert torch.equal(many[:3], few)
