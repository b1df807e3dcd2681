"""Refusals of the rotary and attention entry points: before any HIP call, with their status (no GPU)."""
import os

import pytest

from paper_2104_00237_amd import _lib as L

FAKE = 0x10000  # never dereferenced: validation fails before any HIP call


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(L.LIB_PATH):
        pytest.skip("libopfuse.so not built")
    return L.load()


def status(fn, *args):
    with pytest.raises(L.OpfuseError) as e:
        fn(*args)
    return e.value.status


def rotary(**kw):
    a = dict(T=8, H=2, D=64, rot=64, dtype=L.OF_F32, base=10000.0)
    a.update(kw)
    return L.OfRotaryDesc(**a)


@pytest.mark.parametrize("fn", ["of_rotary_fwd", "of_rotary_bwd"])
def test_rotary(fn):
    f = getattr(L, fn)
    bad = lambda want, x=FAKE, pos=None, y=2 * FAKE, **kw: \
        _same(status(f, rotary(**kw), x, pos, y, None), want, kw)  # noqa: E731
    assert status(f, None, FAKE, None, FAKE, None) == L.OF_EINVAL
    bad(L.OF_EINVAL, x=None)
    bad(L.OF_EINVAL, y=None)
    for kw in (dict(T=0), dict(H=0), dict(D=0), dict(rot=0), dict(rot=3), dict(rot=66), dict(rot=-2), dict(interleaved=2),
               dict(dtype=7), dict(seq_len=-1), dict(pos0=-1), dict(pos0=1 << 60), dict(base=1.0), dict(base=float("nan")), dict(scaling=4),
               dict(scaling=-1), dict(scaling=L.OF_ROPE_LINEAR), dict(scaling=L.OF_ROPE_BASE, factor=float("inf")),
               dict(scaling=L.OF_ROPE_BANDS, factor=2.0), dict(mscale=-1.0), dict(mscale=float("nan")),
               dict(scaling=L.OF_ROPE_BANDS, factor=2.0, orig_len=10.0, low_turns=4.0, high_turns=4.0),
               dict(ldx=63), dict(hsx=63), dict(ldx=100), dict(ldy=100), dict(ldx=64, hsx=100)):
        bad(L.OF_EINVAL, **kw)
    bad(L.OF_EUNSUPPORTED, D=600, rot=600)
    bad(L.OF_EUNSUPPORTED, T=1 << 31)
    bad(L.OF_EUNSUPPORTED, H=1 << 20)
    bad(L.OF_EUNSUPPORTED, T=1 << 24, H=256)    # one row a workgroup: 2^32 threads
    bad(L.OF_EUNSUPPORTED, ldx=1 << 23)
    bad(L.OF_EALIGN, x=FAKE + 2)
    bad(L.OF_EALIGN, y=FAKE + 1, dtype=L.OF_BF16)
    bad(L.OF_EALIGN, pos=FAKE + 4)
    bad(L.OF_EINVAL, y=FAKE, ldx=256)     # in place in two layouts


def _same(got, want, kw):
    assert got == want, (kw, L.of_last_error())


def attn(**kw):
    a = dict(Tq=64, Tk=64, nseq=2, Hq=4, Hkv=2, D=64, dtype=L.OF_BF16, grad_dtype=L.OF_BF16)
    a.update(kw)
    return L.OfAttnDesc(**a)


BAD = [(L.OF_EINVAL, dict(Tq=0)), (L.OF_EINVAL, dict(Tk=0)), (L.OF_EINVAL, dict(nseq=0)), (L.OF_EINVAL, dict(Hq=0)),
       (L.OF_EINVAL, dict(Hkv=0)), (L.OF_EINVAL, dict(Hq=3)), (L.OF_EINVAL, dict(D=0)), (L.OF_EUNSUPPORTED, dict(D=257)),
       (L.OF_EINVAL, dict(dtype=3)), (L.OF_EINVAL, dict(grad_dtype=3)), (L.OF_EINVAL, dict(causal=2)),
       (L.OF_EINVAL, dict(window=-1)), (L.OF_EINVAL, dict(scale=-1.0)), (L.OF_EINVAL, dict(scale=float("nan"))),
       (L.OF_EUNSUPPORTED, dict(Tq=1 << 30)), (L.OF_EUNSUPPORTED, dict(Tk=1 << 31)), (L.OF_EUNSUPPORTED, dict(Tk=1 << 30)),
       (L.OF_EUNSUPPORTED, dict(Hq=1 << 29, Hkv=1 << 29, hsq=1 << 40)),
       (L.OF_EUNSUPPORTED, dict(nseq=1 << 26, Tq=1 << 26, Tk=1 << 26)), (L.OF_EINVAL, dict(Tq=65)),
       (L.OF_EINVAL, dict(Tk=65)), (L.OF_EALIGN, dict(q_off=FAKE + 2)), (L.OF_EALIGN, dict(k_len=FAKE + 1)),
       (L.OF_EINVAL, dict(ldq=63)), (L.OF_EINVAL, dict(hsk=63)), (L.OF_EINVAL, dict(ldv=100)),
       (L.OF_EINVAL, dict(ldo=64, hso=64 * 63)), (L.OF_EUNSUPPORTED, dict(ldo=(1 << 22) + 8)),
       (L.OF_EUNSUPPORTED, dict(scale=2.0 ** -101)), (L.OF_EUNSUPPORTED, dict(scale=2.0 ** 101)),
       # a launch has fewer than 2^32 threads; the last tile's row numbers are ints
       (L.OF_EUNSUPPORTED, dict(nseq=1 << 23, Tq=1 << 23, Tk=1 << 23)),
       (L.OF_EUNSUPPORTED, dict(nseq=1, Hq=1, Hkv=1, Tk=(1 << 31) - 512))]


def test_attention_backward_workgroups():
    d = attn(nseq=1, Hq=1, Hkv=1, Tk=1 << 30)      # two column parts of 2^23 tiles of keys
    assert L.of_attn_workspace_size(d, L.OF_ATTN_FWD) > 0
    assert L.of_attn_workspace_size(d, L.OF_ATTN_BWD) == 0
    assert "workgroups" in L.of_last_error()


@pytest.mark.parametrize("want,kw", BAD, ids=str)
def test_attention_descriptors(want, kw):
    d = attn(**kw)
    big = 1 << 40
    _same(status(L.of_attn_fwd, d, FAKE, FAKE, FAKE, 2 * FAKE, None, FAKE, big, None), want, kw)
    _same(status(L.of_attn_bwd, d, *[FAKE * i for i in range(1, 10)], FAKE, big, None), want, kw)
    for op in (L.OF_ATTN_FWD, L.OF_ATTN_BWD):
        assert L.of_attn_workspace_size(d, op) == 0


def test_attention_arguments():
    big = 1 << 40
    fwd = [FAKE, 2 * FAKE, 3 * FAKE, 4 * FAKE]
    bwd = [FAKE * i for i in range(1, 10)]
    assert status(L.of_attn_fwd, None, *fwd, None, FAKE, big, None) == L.OF_EINVAL
    for i in range(4):
        a = list(fwd)
        a[i] = None
        assert status(L.of_attn_fwd, attn(), *a, None, FAKE, big, None) == L.OF_EINVAL
        a[i] = FAKE * (i + 1) + 1
        assert status(L.of_attn_fwd, attn(), *a, None, FAKE, big, None) == L.OF_EALIGN
    assert status(L.of_attn_fwd, attn(), *fwd, FAKE + 2, FAKE, big, None) == L.OF_EALIGN
    assert status(L.of_attn_fwd, attn(), FAKE, FAKE, FAKE, FAKE, None, FAKE, big, None) == L.OF_EINVAL
    for i in range(9):
        a = list(bwd)
        a[i] = None
        assert status(L.of_attn_bwd, attn(), *a, FAKE, big, None) == L.OF_EINVAL
        a[i] = FAKE * (i + 1) + 1
        assert status(L.of_attn_bwd, attn(), *a, FAKE, big, None) == L.OF_EALIGN
        if i >= 6:
            a[i] = FAKE
            assert status(L.of_attn_bwd, attn(), *a, FAKE, big, None) == L.OF_EINVAL
    a = list(bwd)
    a[7] = a[6]
    assert status(L.of_attn_bwd, attn(), *a, FAKE, big, None) == L.OF_EINVAL
    # fp32 operands have fp32 gradients
    assert status(L.of_attn_bwd, attn(dtype=L.OF_F32), *bwd, FAKE, big, None) == L.OF_EUNSUPPORTED
    need = L.of_attn_workspace_size(attn(), L.OF_ATTN_BWD)
    assert need > 0
    assert status(L.of_attn_bwd, attn(), *bwd, FAKE, need - 1, None) == L.OF_EWORKSPACE
    assert status(L.of_attn_bwd, attn(), *bwd, None, need, None) == L.OF_EWORKSPACE
    assert status(L.of_attn_bwd, attn(), *bwd, FAKE + 8, need, None) == L.OF_EALIGN
    # one token over a long cache is split, and needs room for the parts
    d = attn(Tq=2, Tk=20000)
    need = L.of_attn_workspace_size(d, L.OF_ATTN_FWD)
    assert need > 0
    assert status(L.of_attn_fwd, d, *fwd, None, FAKE, need - 1, None) == L.OF_EWORKSPACE
    assert L.of_attn_workspace_size(attn(), 2) == 0
    assert "of_attn_op" in L.of_last_error()
    assert L.of_attn_workspace_size(attn(Tk=0), L.OF_ATTN_FWD) == 0
