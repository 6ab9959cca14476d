"""The limits of pitches and strides, on the host before any device call: products of them and of sizes that pass 64 bits
are refused, not wrapped (pointers are never followed)."""
import pytest

from test_layers_refusals import BIG, CALLS, H, P, SHAPE, mx

LONG = 1 << 28      # the longest side
FAR = 1 << 36       # LONG times it is 2^64: zero in 64 bits


@pytest.fixture(scope="module")
def gl():
    import paper_2504_20437_amd
    return paper_2504_20437_amd


def wide(codes=P, ldq=512, stride_q=0, scales=P, lds=16, stride_s=0):
    from paper_2504_20437_amd.training import MxMatrix
    return MxMatrix(codes, ldq, stride_q, scales, lds, stride_s)


def rows(names, tokens="tokens"):
    """for each matrix of a call: a batch of two at a stride that its rows pass only modulo 2^64, a stride past the limit,
    and rows further apart than memory reaches"""
    fine = {"stride_" + n.lower(): BIG for n in names}
    for n in names:
        low = n.lower()
        yield {tokens: LONG, "batch": 2, **fine, "ld" + low: FAR, "stride_" + low: 0}
        yield {"batch": 2, "stride_" + low: BIG + 1}
        yield {tokens: LONG, "ld" + low: 1 << 30}


PACKED = dict(Q=None, K=None, q8=mx(), k8=mx())
LIMITS = {
    "galore_embedding": [dict(vocab=LONG, ldw=1 << 30), dict(tokens=LONG, ldo=1 << 30)],
    "galore_embedding_grad": [dict(tokens=LONG, lddy=1 << 30), dict(vocab=LONG, ldg=1 << 30)],
    "galore_dropout": list(rows(["X", "R", "Y"])) + [
        dict(tokens=LONG, batch=2, stride_x=BIG, stride_r=BIG, stride_y=BIG, y8=wide(ldq=FAR, stride_q=0, lds=16, stride_s=BIG)),
        dict(tokens=LONG, batch=2, stride_x=BIG, stride_r=BIG, stride_y=BIG, y8=wide(ldq=64, stride_q=BIG, lds=FAR, stride_s=0)),
        dict(batch=2, y8=wide(stride_q=BIG + 16, stride_s=BIG)), dict(batch=2, y8=wide(stride_q=BIG, stride_s=BIG + 4)),
        dict(y8=wide(ldq=BIG + 16)), dict(y8=wide(lds=BIG + 4)), dict(tokens=LONG, y8=wide(ldq=1 << 30)),
        dict(tokens=LONG, y8=wide(lds=1 << 30))],
    "galore_head_norm": [dict(tokens=LONG, **{n: H(token=t, head=h)}) for n in ("Q", "K", "Q_out", "K_out")
                         for t, h in ((FAR, 64), (FAR, FAR + 64 if n[0] == "Q" else 1 << 39), (1 << 30, 64))] + [
        dict(table_rows=LONG, ld_table=1 << 30)],
    "galore_head_norm_backward": [dict(tokens=LONG, **{n: H(token=FAR, head=64)}) for n in ("dQ", "dK", "Q", "K", "dQ_in", "dK_in")] + [
        dict(PACKED, q8=wide(ldq=BIG + 16)), dict(PACKED, k8=wide(lds=BIG + 4)),
        dict(PACKED, tokens=LONG, q8=wide(ldq=1 << 30)), dict(PACKED, tokens=LONG, k8=wide(lds=1 << 30))],
    "galore_recurrence": list(rows(["X", "F", "H"])),
    "galore_recurrence_backward": list(rows(["dH", "X", "F", "dX", "dF"])),
}


@pytest.mark.parametrize("name,change", [(n, c) for n, cases in LIMITS.items() for c in cases])
def test_no_product_passes_64_bits(gl, name, change):
    a = dict(CALLS[name])
    a.update(change)
    assert getattr(gl.lib, name)(*a.values()) == SHAPE


def test_training_operators_batch_strides(gl):
    """the check that the training operators share"""
    assert gl.lib.galore_checkpoint_pack(P, 0, LONG, 64, FAR, 0, wide(stride_q=BIG, ldq=64, stride_s=BIG, lds=4), 2, None) == SHAPE
    assert gl.lib.galore_checkpoint_pack(P, 0, LONG, 64, 64, BIG, wide(ldq=FAR, stride_q=0, lds=4, stride_s=BIG), 2, None) == SHAPE
    assert gl.lib.galore_checkpoint_pack(P, 0, 5, 64, 64, -64, wide(stride_q=BIG, stride_s=BIG), 2, None) == SHAPE


def test_what_memory_holds_is_taken(gl):
    """at the limits themselves; no tokens, so that nothing is launched"""
    none = dict(tokens=0, stream=None)
    assert gl.lib.galore_dropout(*dict(CALLS["galore_dropout"], **none, batch=2, ldx=BIG, stride_x=BIG, stride_y=0).values()) == 0
    assert gl.lib.galore_head_norm(*dict(CALLS["galore_head_norm"], **none, Q=H(token=BIG, head=BIG)).values()) == 0
