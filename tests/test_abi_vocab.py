"""Refusals of the vocabulary losses: before any HIP call, with their status (no GPU)."""
import os

import pytest

from paper_2104_00237_amd import _lib as L

FAKE = 0x10000  # never dereferenced: validation fails before any HIP call


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libopfuse.so not built")
    return L.load()


def desc(**kw):
    a = dict(M=8, V=100, K=64, dtype=L.OF_BF16, grad_dtype=L.OF_BF16)
    a.update(kw)
    return L.OfVocabDesc(**a)


def param(d, **kw):
    a = dict(w=3 * FAKE, m=4 * FAKE, v=5 * FAKE, w_bf16=6 * FAKE, numel=d.V * d.K)
    a.update(kw)
    return L.OfParam(**a)


OPT = dict(kind="adam", lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8)
KINDS = ["xent_fwd", "xent_bwd", "xent_bwd_fused", "distill_fwd", "distill_bwd", "distill_bwd_fused"]


def refused(kind, d=None, W=None, opt=OPT, given=True, **kw):
    """Status of a call all of whose other arguments are right; given=False: without its descriptor."""
    d = d if d is not None else desc(**({"topk": 4} if kind.startswith("distill") else {}))
    a = dict(x=FAKE, ids=2 * FAKE, teacher=7 * FAKE, loss=8 * FAKE, lse=9 * FAKE, zt=10 * FAKE, mean=11 * FAKE, dloss=12 * FAKE,
             dx=13 * FAKE, dw=14 * FAKE, accumulate=0, gW=15 * FAKE, ws=16 * FAKE, size=1 << 50)
    a.update(kw)
    W = W if W is not None else param(d)
    t = [a["ids"]] + ([a["teacher"]] if kind.startswith("distill") else [])
    if kind.endswith("fwd"):
        rest = [a["loss"], a["lse"], a["zt"], a["mean"]]
    elif kind.endswith("fused"):
        rest = [a["lse"], a["zt"], a["dloss"], a["gW"], L.make_opt(opt, 1) if opt else None, a["dx"]]
    else:
        rest = [a["lse"], a["zt"], a["dloss"], a["dx"], a["dw"], a["accumulate"]]
    with pytest.raises(L.OpfuseError) as e:
        getattr(L, "of_vocab_" + kind)(d if given else None, a["x"], W, *t, *rest, a["ws"], a["size"], None)
    return e.value.status


BAD = [(L.OF_EINVAL, dict(M=0)), (L.OF_EINVAL, dict(V=0)), (L.OF_EINVAL, dict(K=-1)), (L.OF_EINVAL, dict(ldx=63)),
       (L.OF_EINVAL, dict(dtype=2)), (L.OF_EINVAL, dict(grad_dtype=-1)), (L.OF_EINVAL, dict(teacher_dtype=5)),
       (L.OF_EINVAL, dict(topk=-1)), (L.OF_EUNSUPPORTED, dict(topk=1025)), (L.OF_EINVAL, dict(softcap=-1.0)),
       (L.OF_EINVAL, dict(softcap=float("nan"))), (L.OF_EUNSUPPORTED, dict(softcap=2.0 ** 41)),
       (L.OF_EINVAL, dict(z_loss=-1e-4)), (L.OF_EINVAL, dict(z_loss=float("inf"))), (L.OF_EINVAL, dict(temperature=-1.0)),
       (L.OF_EUNSUPPORTED, dict(temperature=2.0 ** -41)), (L.OF_EUNSUPPORTED, dict(M=(1 << 22) + 1)),
       (L.OF_EUNSUPPORTED, dict(V=(1 << 20) + 1)), (L.OF_EUNSUPPORTED, dict(K=(1 << 20) + 1)),
       (L.OF_EUNSUPPORTED, dict(M=1 << 20, V=1 << 17)), (L.OF_EUNSUPPORTED, dict(V=1 << 20, K=(1 << 16) + 1)),
       (L.OF_EUNSUPPORTED, dict(ldx=(1 << 21) + 1)), (L.OF_EUNSUPPORTED, dict(M=1 << 20, ldx=1 << 10)),
       (L.OF_EUNSUPPORTED, dict(M=1 << 21, topk=1024))]


@pytest.mark.parametrize("want,kw", BAD)
def test_descriptors(want, kw):
    for op in (L.OF_VOCAB_FWD, L.OF_VOCAB_BWD):
        assert L.of_vocab_workspace_size(desc(**kw), op) == 0
        assert L.of_last_error()
    kind = "distill_bwd" if "topk" in kw else "xent_bwd"
    assert refused(kind, desc(**kw)) == want, L.of_last_error()


@pytest.mark.parametrize("kw", [dict(M=1 << 22, V=1000, K=100), dict(M=1, V=1 << 20, K=1 << 16), dict(M=1 << 16, V=1 << 20, K=64),
                                dict(M=(1 << 20) - 1, V=4096, K=512), dict(M=1, V=1, K=1), dict(M=1 << 21, V=32, K=32, topk=1023),
                                dict(M=500, V=1 << 20, K=1 << 15)])
@pytest.mark.parametrize("dtype", [L.OF_F32, L.OF_BF16])
def test_workspace_of_the_largest(kw, dtype):
    """Grows with what it holds: X, the entries, a gradient of at most 512 MB and partial sums beside it."""
    d = desc(dtype=dtype, grad_dtype=dtype, **kw)
    wide = d.M * d.K * 4
    for op in (L.OF_VOCAB_FWD, L.OF_VOCAB_BWD):
        size = L.of_vocab_workspace_size(d, op)
        assert 0 < size < (1 << 31) + 70 * wide + 24 * d.M * max(d.topk, 1) + 64 * d.V * d.K + d.M * d.V // 8 + (1 << 22), (size, L.of_last_error())


def test_workspace_query():
    assert L.of_vocab_workspace_size(desc(), L.OF_VOCAB_FWD) > 0
    assert L.of_vocab_workspace_size(desc(), L.OF_VOCAB_BWD) > 0
    assert L.of_vocab_workspace_size(desc(), 2) == 0
    # (bf16 gradients of fp32 operands: the forward has no gradients)
    mixed = desc(dtype=L.OF_F32)
    assert L.of_vocab_workspace_size(mixed, L.OF_VOCAB_FWD) > 0
    assert L.of_vocab_workspace_size(mixed, L.OF_VOCAB_BWD) == 0
    assert refused("xent_bwd", mixed) == L.OF_EUNSUPPORTED


@pytest.mark.parametrize("kind", KINDS)
def test_calls(kind):
    distill = kind.startswith("distill")
    more = {"topk": 4} if distill else {}
    assert refused(kind, desc(**more), given=False) == L.OF_EINVAL
    for name in ["x", "ids", "lse", "zt"] + (["teacher"] if distill else []) + (["loss"] if kind.endswith("fwd") else []):
        assert refused(kind, **{name: None}) == L.OF_EINVAL, name
    assert refused(kind, size=L.of_vocab_workspace_size(
        desc(**more), L.OF_VOCAB_FWD if kind.endswith("fwd") else L.OF_VOCAB_BWD) - 1) == L.OF_EWORKSPACE
    assert refused(kind, ws=None) == L.OF_EWORKSPACE
    assert refused(kind, ws=FAKE + 8) == L.OF_EALIGN
    d = desc(**more)
    assert refused(kind, d, param(d, numel=6399)) == L.OF_EINVAL
    assert refused(kind, d, param(d, w_bf16=None)) == L.OF_EINVAL
    assert refused(kind, d, param(d, w_bf16=FAKE + 1)) == L.OF_EALIGN
    f = desc(dtype=L.OF_F32, grad_dtype=L.OF_F32, **more)
    assert refused(kind, f, param(f, w=None, w_bf16=None)) == L.OF_EINVAL
    assert refused(kind, f, param(f, w_bf16=None), x=FAKE + 2) == L.OF_EALIGN
    assert refused(kind, x=FAKE + 1) == L.OF_EALIGN
    assert refused(kind, ids=FAKE + 4) == L.OF_EALIGN
    assert refused(kind, lse=FAKE + 2) == L.OF_EALIGN
    if distill:
        assert refused(kind, teacher=FAKE + 2) == L.OF_EALIGN
        assert refused(kind, desc()) == L.OF_EINVAL                       # no entries
        assert refused(kind, desc(topk=4, z_loss=1e-4)) == L.OF_EINVAL
    else:
        assert refused(kind, desc(topk=2)) == L.OF_EINVAL
        assert refused(kind, desc(temperature=2.0)) == L.OF_EINVAL
    if kind.endswith("fwd"):
        assert refused(kind, loss=9 * FAKE) == L.OF_EINVAL
        assert refused(kind, mean=10 * FAKE) == L.OF_EINVAL
        assert refused(kind, mean=FAKE + 2) == L.OF_EALIGN
        return
    assert refused(kind, dx=FAKE) == L.OF_EINVAL
    assert refused(kind, dx=6 * FAKE) == L.OF_EINVAL
    assert refused(kind, dloss=FAKE + 2) == L.OF_EALIGN
    if kind.endswith("fused"):
        assert refused(kind, opt=None) == L.OF_EINVAL
        assert refused(kind, opt=dict(OPT, lr=float("nan"))) == L.OF_EINVAL
        assert refused(kind, d, param(d, v=None)) == L.OF_EINVAL
        assert refused(kind, gW=FAKE + 2) == L.OF_EALIGN
        assert refused(kind, f, param(f)) == L.OF_EINVAL                  # a shadow beside fp32 operands
    else:
        assert refused(kind, dx=None, dw=None) == L.OF_EINVAL
        assert refused(kind, dx=14 * FAKE) == L.OF_EINVAL
        assert refused(kind, dw=FAKE) == L.OF_EINVAL
        assert refused(kind, dw=6 * FAKE) == L.OF_EINVAL
        assert refused(kind, accumulate=2) == L.OF_EINVAL
        assert refused(kind, dw=FAKE + 1) == L.OF_EALIGN


def size(op, **kw):
    return L.of_vocab_workspace_size(desc(**kw), op)


def test_workspace_of_aligned_operands():
    """bf16 operands of 16-byte pieces that are promised to be aligned: no room for copies of W, nor of a forward's X, and
    none for entries where there are none."""
    M, V, K = 4, 32768, 1024
    kw = dict(M=M, V=V, K=K)
    copy_w, copy_x = V * K * 2, M * K * 2
    for op in (L.OF_VOCAB_FWD, L.OF_VOCAB_BWD):
        assert size(op, **kw) - size(op, aligned=1, **kw) == copy_w + (copy_x if op == L.OF_VOCAB_FWD else 0)
        # not for rows that are no whole pieces, or fp32 (whose planes are made)
        for more in (dict(K=1023), dict(dtype=L.OF_F32, grad_dtype=L.OF_F32)):
            assert size(op, **{**kw, **more}) == size(op, aligned=1, **{**kw, **more})
    odd = dict(kw, ldx=1028, aligned=1)
    assert size(L.OF_VOCAB_FWD, **odd) - size(L.OF_VOCAB_FWD, **kw, aligned=1) == copy_x
    # a few statistics a row and tile
    assert size(L.OF_VOCAB_FWD, aligned=1, **kw) <= 8 * M * V // 128 + (1 << 13)
    # logits in bf16 would be 2 MB, 256 MB, 1 GB (a backward keeps 512 MB of their gradient: half of W at a time)
    assert size(L.OF_VOCAB_FWD, M=32, V=32768, K=1024, aligned=1) < 1 << 17
    assert size(L.OF_VOCAB_FWD, M=4096, V=32768, K=1024, topk=0, aligned=1) < 8 << 20
    big = dict(M=8192, V=65536, K=4096)
    assert size(L.OF_VOCAB_BWD, **big) - size(L.OF_VOCAB_BWD, aligned=1, **big) == 65536 // 2 * 4096 * 2
    assert size(L.OF_VOCAB_FWD, topk=64, **big) > size(L.OF_VOCAB_FWD, **big)


@pytest.mark.parametrize("kind", KINDS)
def test_aligned_operands_are_checked(kind):
    more = {"topk": 4} if kind.startswith("distill") else {}
    assert refused(kind, desc(aligned=2, **more)) == L.OF_EINVAL
    assert refused(kind, desc(aligned=-1, **more)) == L.OF_EINVAL
    d = desc(aligned=1, **more)
    assert refused(kind, d, x=FAKE + 2) == L.OF_EALIGN
    assert refused(kind, d, x=FAKE + 8) == L.OF_EALIGN
    assert refused(kind, d, param(d, w_bf16=FAKE + 8)) == L.OF_EALIGN
    f = desc(aligned=1, dtype=L.OF_F32, grad_dtype=L.OF_F32, **more)
    assert refused(kind, f, param(f, w=FAKE + 4, w_bf16=None)) == L.OF_EALIGN
