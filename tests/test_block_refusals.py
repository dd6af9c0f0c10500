"""CPU-only: what the entry points of the MoE block beside the DTS gate refuse.  Every check is made on the host before anything is
launched, so a context that is never used and addresses that are never read are enough; a call that passes all checks would go on
to the GPU, and none here does."""
import ctypes

import pytest

from paper_2112_14397_amd import binding as B

CTX = ctypes.create_string_buffer(4096)
A = 1 << 20                       # an aligned address, never read
F32, BF16 = "f32", "bf16"
BIG = 1 << 40


def shape(T=64, d=64, E=8, F=96, dtype=BF16, P=128):
    return B.make_shape(T, d, E, F, dtype, "gelu", P)


def topk(**kw):
    o = dict(k=2, score="softmax", groups=4, top_groups=2, group_keys=2, renormalise=True, scale=1.0)
    raw = {n: kw.pop(n) for n in ("score_id", "renormalise_id") if n in kw}
    o.update(kw)
    t = B.make_topk(**o)
    t.score = raw.get("score_id", t.score)
    t.renormalise = raw.get("renormalise_id", t.renormalise)
    return t


def call(name, s, args, ctx=CTX):
    fn = getattr(B.lib(), name)
    return fn(ctx, None if s is None else ctypes.byref(s), *args)


GOOD = {
    "evomoe_gate_logits": [A] * 4,
    "evomoe_gate_logits_bwd": [A] * 8 + [BIG],
    "evomoe_topk_gate": [topk()] + [A] * 8,
    "evomoe_topk_gate_bwd": [topk()] + [A] * 6 + [1.0, A],
    "evomoe_add_rmsnorm": [A, A, A, 1e-5, A, 2 * A, 3 * A, 4 * A, 5 * A],
    "evomoe_add_rmsnorm_bwd": [A] * 8 + [BIG],
    "evomoe_expert_ffn_mx8": [A] * 12 + [BIG],
}
NULLABLE = {"evomoe_gate_logits": {2}, "evomoe_gate_logits_bwd": {3, 5}, "evomoe_topk_gate": {2, 3, 7, 8}, "evomoe_topk_gate_bwd": {6},
            "evomoe_add_rmsnorm": {1, 4, 5, 6}, "evomoe_add_rmsnorm_bwd": {1, 6}, "evomoe_expert_ffn_mx8": {2, 6, 9}}


def marshalled(args):
    return [ctypes.byref(a) if isinstance(a, B.TopK) else a for a in args]


@pytest.mark.parametrize("name", sorted(GOOD))
def test_null_and_misaligned_arguments(name):
    args = GOOD[name]
    assert call(name, shape(), marshalled(args), ctx=None) == B.EVOMOE_EINVAL
    assert call(name, None, marshalled(args)) == B.EVOMOE_EINVAL
    work = name in ("evomoe_gate_logits_bwd", "evomoe_add_rmsnorm_bwd", "evomoe_expert_ffn_mx8")
    for i, a in enumerate(args):
        if isinstance(a, float) or a == BIG:
            continue
        expect = B.EVOMOE_EWORKSPACE if work and i == len(args) - 2 else B.EVOMOE_EINVAL
        if not isinstance(a, B.TopK):
            odd = list(args)
            odd[i] = A + 2
            assert call(name, shape(), marshalled(odd)) == expect, (name, i)
        if i in NULLABLE[name]:
            continue
        gone = list(args)
        gone[i] = None
        assert call(name, shape(), marshalled(gone)) == expect, (name, i)
    if work:
        short = list(args)
        short[-1] = 16
        assert call(name, shape(), marshalled(short)) == B.EVOMOE_EWORKSPACE


@pytest.mark.parametrize("name", sorted(GOOD))
@pytest.mark.parametrize("bad,status", [(dict(T=0), B.EVOMOE_EINVAL), (dict(d=-64), B.EVOMOE_EINVAL), (dict(E=0), B.EVOMOE_EINVAL),
                                        (dict(P=0), B.EVOMOE_EINVAL), (dict(E=65), B.EVOMOE_EUNSUPPORTED),
                                        (dict(d=68), B.EVOMOE_EUNSUPPORTED), (dict(T=1 << 29), B.EVOMOE_EUNSUPPORTED),
                                        (dict(T=(1 << 29) + 1, E=1), B.EVOMOE_EUNSUPPORTED),
                                        (dict(T=1, d=(1 << 30) + 64), B.EVOMOE_EUNSUPPORTED)])
def test_shapes(name, bad, status):
    assert call(name, shape(**bad), marshalled(GOOD[name])) == status


@pytest.mark.parametrize("bad", [dict(k=0), dict(k=5), dict(k=-1), dict(groups=0), dict(groups=3), dict(groups=-4), dict(top_groups=0),
                                 dict(top_groups=5), dict(group_keys=0), dict(group_keys=3), dict(score_id=2), dict(score_id=-1),
                                 dict(renormalise_id=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
                                 dict(scale=float("nan"))])
@pytest.mark.parametrize("name", ["evomoe_topk_gate", "evomoe_topk_gate_bwd"])
def test_topk_options(name, bad):
    assert call(name, shape(), marshalled([topk(**bad)] + GOOD[name][1:])) == B.EVOMOE_EINVAL


def test_norm_arguments():
    args = GOOD["evomoe_add_rmsnorm"]
    for eps in (0.0, -1e-5, float("nan"), float("inf")):
        assert call("evomoe_add_rmsnorm", shape(), args[:3] + [eps] + args[4:]) == B.EVOMOE_EINVAL
    one = lambda **kw: [kw.get(n, None) if n in ("h", "y", "rstd", "q", "qs") else v
                        for n, v in zip(("x", "res", "gamma", "eps", "h", "y", "rstd", "q", "qs"), args)]
    assert call("evomoe_add_rmsnorm", shape(), one(rstd=A)) == B.EVOMOE_EINVAL               # nothing to write
    assert call("evomoe_add_rmsnorm", shape(), one(y=A, q=A)) == B.EVOMOE_EINVAL             # 8 bits without scales
    assert call("evomoe_add_rmsnorm", shape(), one(y=A, qs=A)) == B.EVOMOE_EINVAL
    assert call("evomoe_add_rmsnorm", shape(), one(h=A, y=A)) == B.EVOMOE_EINVAL             # one place for two outputs
    assert call("evomoe_add_rmsnorm", shape(), one(y=A, q=A, qs=2 * A)) == B.EVOMOE_EINVAL
    assert call("evomoe_add_rmsnorm", shape(), one(h=A, q=2 * A, qs=A)) == B.EVOMOE_EINVAL
    assert call("evomoe_add_rmsnorm", shape(), one(y=A, rstd=A)) == B.EVOMOE_EINVAL
    assert call("evomoe_add_rmsnorm", shape(d=72), one(q=A, qs=2 * A)) == B.EVOMOE_EUNSUPPORTED


def test_quantize_arguments():
    q = lambda rows, cols, dtype, src=A, dst=A, s=A, ctx=CTX: B.lib().evomoe_quantize_mx8(ctx, rows, cols, dtype, src, dst, s)
    assert q(4, 64, 0, ctx=None) == B.EVOMOE_EINVAL
    for rows, cols, dtype in ((0, 64, 0), (4, 0, 0), (-1, 64, 0), (4, -64, 0), (4, 64, 2), (4, 64, -1)):
        assert q(rows, cols, dtype) == B.EVOMOE_EINVAL
    assert q(4, 48, 0) == B.EVOMOE_EUNSUPPORTED and q(1 << 40, 1 << 20, 0) == B.EVOMOE_EUNSUPPORTED
    for bad in (dict(src=None), dict(dst=None), dict(s=None), dict(src=A + 4), dict(dst=A + 8), dict(s=A + 1)):
        assert q(4, 64, 1, **bad) == B.EVOMOE_EINVAL


def test_limits_of_the_8_bit_experts():
    args = GOOD["evomoe_expert_ffn_mx8"]
    for bad in (dict(dtype=F32), dict(d=72), dict(F=104), dict(d=65536, F=65536), dict(T=1 << 22, d=1024),
                dict(T=2, d=(1 << 24) + 128, F=128), dict(T=2, d=128, F=(1 << 24) + 128)):
        assert call("evomoe_expert_ffn_mx8", shape(**bad), args) == B.EVOMOE_EUNSUPPORTED
        assert B.evomoe_workspace_bytes_mx8(shape(**bad)) == 0
    for P in (1, 100, 59000):
        s = shape(T=8192, d=64, F=96, P=P)
        assert P * 99 <= B.evomoe_workspace_bytes_mx8(s) <= B.evomoe_workspace_bytes(s)
