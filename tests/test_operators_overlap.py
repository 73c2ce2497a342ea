"""What a call of the operators writes overlaps nothing else that it is given, but a gradient in its logits' place; rows that lie
beside each other in one buffer do not overlap.  No GPU: no such device is there, so that nothing is ever enqueued."""
import pytest
import torch

from paper_1805_08768_amd import binding as sbc

P, NO_DEVICE = 0x10000000, 1 << 20
MIB = 1 << 20
none_here = torch.cuda.device_count() == 0


def refused(name, args, **kw):
    """Whether the overlap is refused; a call without any gets as far as looking for its device."""
    values = [kw.get(n, v) for n, v in args]
    rc = getattr(sbc.load(), name)(*values)
    assert rc in (sbc.SBC_EINVAL, sbc.SBC_EHIP), rc
    return rc == sbc.SBC_EINVAL


def check(name, args, sizes, written, beside=()):
    """sizes: bytes of each pointer; written: the ones that the call writes.  Each pair with one of those in it, the second
    starting at the first's first byte or its last 16."""
    assert not none_here or not refused(name, args)
    for w in written:
        for other in sizes:
            if other == w or (w, other) in beside:
                continue
            for moved, fixed in ((w, other), (other, w)):
                base = dict(args)[fixed]
                for at in (base, base + sizes[fixed] - 16):
                    assert refused(name, args, **{moved: at}), (name, moved, fixed, at - base)
                # ... and next to it is fine
                assert not none_here or not refused(name, args, **{moved: base + (sizes[fixed] + 15) // 16 * 16 + 5 * MIB}), (moved, fixed)


def held(rows, cols):
    return sbc.sbc_mxfp_bytes(rows, cols)


def test_quantize_and_dequantize():
    args = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 0), ("rows", 100), ("cols", 200), ("ld", 200), ("by_rows", P + 8 * MIB), ("by_cols", P + 16 * MIB)]
    check("sbc_mxfp_quantize", args, dict(x=80000, by_rows=held(100, 200), by_cols=held(200, 100)), ["by_rows", "by_cols"])
    args = [("device", NO_DEVICE), ("stream", None), ("q", P), ("rows", 100), ("cols", 200), ("y", P + 8 * MIB), ("type", 1), ("ld", 200)]
    check("sbc_mxfp_dequantize", args, dict(q=held(100, 200), y=40000), ["y"])


def test_products():
    args = [("device", NO_DEVICE), ("stream", None), ("a", P), ("b", P + 8 * MIB), ("m", 100), ("n", 300), ("k", 200), ("c", P + 16 * MIB), ("type", 0), ("ldc", 300)]
    check("sbc_mxfp_matmul", args, dict(a=held(100, 200), b=held(300, 200), c=120000), ["c"])
    assert not none_here or not refused("sbc_mxfp_matmul", args, n=100, b=P)        # (operands are only read: a matrix times itself)
    for m in (4, 100):
        room = max(16, sbc.sbc_mxfp_linear_workspace(m, 200))
        args = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 0), ("ldx", 200), ("m", m), ("w", P + 8 * MIB), ("n", 200), ("k", 200), ("y", P + 16 * MIB), ("ldy", 200),
                ("ws", P + 24 * MIB), ("bytes", room)]
        sizes = dict(x=m * 800, w=held(200, 200), y=m * 800)
        check("sbc_mxfp_linear", args, dict(sizes, ws=room) if m == 100 else sizes, ["y", "ws"] if m == 100 else ["y"])


def test_top_logits():
    room = sbc.sbc_top_logits_workspace(3, 200000, 8)
    args = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 0), ("ld", 200000), ("rows", 3), ("vocab", 200000), ("k", 8), ("t", 1.0), ("index", P + 8 * MIB),
            ("top", P + 16 * MIB), ("lse", P + 24 * MIB), ("ws", P + 32 * MIB), ("bytes", room)]
    sizes = dict(x=2400000, index=96, top=96, ws=room)
    check("sbc_top_logits", args, sizes, ["index", "top", "ws"])
    for other in sizes:
        assert refused("sbc_top_logits", args, lse=dict(args)[other] + 4)


def test_distillation():
    V = 200000
    room = sbc.sbc_distill_workspace(3, V)
    first = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 0), ("ld", V), ("rows", 3), ("vocab", V), ("index", P + 8 * MIB), ("top", P + 16 * MIB), ("k", 8),
             ("lse", P + 24 * MIB), ("t", 1.0)]
    loss = first + [("weight", P + 32 * MIB), ("loss", P + 40 * MIB), ("stats", P + 48 * MIB), ("grad", P + 56 * MIB), ("ldg", V), ("ws", P + 72 * MIB), ("bytes", room)]
    grad = first + [("stats", P + 48 * MIB), ("dloss", P + 32 * MIB), ("grad", P + 56 * MIB), ("ldg", V)]
    sizes = dict(x=12 * V, index=96, top=96, stats=48, grad=12 * V)
    assert room > 0
    for name, args, more, written in (("sbc_distill_loss", loss, dict(ws=room), ["stats", "ws"]), ("sbc_distill_grad", grad, {}, [])):
        check(name, args, dict(sizes, **more), written)
        for other in list(sizes) + list(more):
            if other not in ("x", "grad"):
                assert refused(name, args, grad=dict(args)[other])
        for other in ("lse", "weight", "dloss", "loss"):
            if other in dict(args):
                assert refused(name, args, grad=dict(args)[other])
                if name == "sbc_distill_loss" and other != "loss":
                    assert refused(name, args, loss=dict(args)[other]) and refused(name, args, stats=dict(args)[other])
        assert refused(name, args, grad=P + 16) and refused(name, args, grad=P - 16)
        assert not none_here or not refused(name, args, grad=P)                     # (in place)
        assert refused(name, args, grad=P, ldg=V + 4)


@pytest.mark.skipif(not none_here, reason="only where no device answers can it be told that a call was not refused")
def test_rows_beside_each_other():
    V = 100
    args = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 0), ("ld", 2 * V), ("rows", 3), ("vocab", V), ("index", P + 8 * MIB), ("top", P + 16 * MIB), ("k", 8), ("lse", None),
            ("t", 1.0), ("stats", P + 48 * MIB), ("dloss", None), ("grad", P + 4 * V), ("ldg", 2 * V)]
    name = "sbc_distill_grad"
    assert not refused(name, args) and not refused(name, args, x=P + 4 * V, grad=P)
    assert not refused(name, args, grad=P + 4 * V + 800 * 5) and not refused(name, args, x=P + 8000, grad=P + 4 * V)
    for at in (P + 4 * V - 4, P + 4 * V + 4, P + 4, P + 8 * V - 4 * V + 4, P + 8 * V - 4):
        assert refused(name, args, grad=at), at - P
    assert refused(name, args, ldg=2 * V + 1) and refused(name, args, ldg=4 * V)     # (rows that meet somewhere, or might)
    args = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 1), ("ldx", 300), ("m", 5), ("w", P + 8 * MIB), ("n", 200), ("k", 100), ("y", P + 200), ("ldy", 300), ("ws", None),
            ("bytes", 0)]
    assert not refused("sbc_mxfp_linear", args)
    assert refused("sbc_mxfp_linear", args, y=P + 198) and refused("sbc_mxfp_linear", args, y=P + 202)
    # a vector in the gap between a matrix's rows
    args = [("device", NO_DEVICE), ("stream", None), ("x", P), ("type", 0), ("ld", 300), ("rows", 3), ("vocab", 100), ("k", 8), ("t", 1.0), ("index", P + 8 * MIB),
            ("top", P + 16 * MIB), ("lse", P + 400), ("ws", None), ("bytes", 0)]
    assert not refused("sbc_top_logits", args) and refused("sbc_top_logits", args, lse=P + 396) and refused("sbc_top_logits", args, lse=P + 1196)
    # sizes whose product passes 64 bits
    assert refused("sbc_top_logits", args, ld=(1 << 40) - 1, rows=(1 << 31) - 1)
