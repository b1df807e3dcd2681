"""of_attn_fwd and of_attn_bwd against float64, element by element within the rounding bounds of
tests/attn_reference.py: types, head widths and layouts, ragged and empty sequences, masks that leave
rows empty, rows of no sequence, one token over a long cache, streams and graphs."""
import math

import pytest
import torch

from attn_reference import backward, forward, sees
from paper_2104_00237_amd import _lib as L

pytestmark = pytest.mark.gpu
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
KINDS = {"f32": L.OF_F32, "bf16": L.OF_BF16}
PAD = float("nan")   # in every row of no sequence


class Call:
    """A set of sequences, their buffers on the device, and the descriptor."""

    def __init__(self, ql, kl, Hq=2, Hkv=1, D=64, dtype="bf16", grad=None, causal=0, window=0, slots=False,
                 layout="rows", scale=0.0, tail=0, shift=0, seed=0, gpu="cuda:0"):
        self.ql, self.kl, self.Hq, self.Hkv, self.D = ql, kl, Hq, Hkv, D
        self.dtype, self.grad, self.causal, self.window, self.scale = dtype, grad or dtype, causal, window, scale
        g = torch.Generator().manual_seed(seed)
        self.gpu = gpu
        slot_q, slot_k = (max(ql) + 2, max(kl) + 3) if slots else (0, 0)

        def offsets(lens, slot):
            off = [0 if slot else tail]      # packed: also rows before the first sequence
            for n in lens:
                off.append(off[-1] + (slot or n))
            return off
        self.qo, self.ko = offsets(ql, slot_q), offsets(kl, slot_k)
        self.Tq = max(1, self.qo[-1] + (0 if slots else tail))
        self.Tk = max(1, self.ko[-1] + (0 if slots else tail))

        def tensor(T, H, t, lens, off, scale=1.0):
            """[T, H, D] view in the layout asked for, NaN in rows of no sequence."""
            x = torch.full((T, H, D), PAD, dtype=torch.float32)
            for n, o in zip(lens, off):
                x[o:o + n] = torch.randn(n, H, D, generator=g) * scale
            return self.place(x.to(TYPES[t]), layout, shift)
        self.q = tensor(self.Tq, Hq, dtype, ql, self.qo)
        self.k = tensor(self.Tk, Hkv, dtype, kl, self.ko)
        self.v = tensor(self.Tk, Hkv, dtype, kl, self.ko)
        self.do = tensor(self.Tq, Hq, self.grad, ql, self.qo)
        same = lambda x, t: self.place(torch.full(x.shape, 7.0, dtype=TYPES[t]), layout, shift)  # noqa: E731
        self.o = same(self.q, dtype)
        self.dq, self.dk, self.dv = same(self.q, self.grad), same(self.k, self.grad), same(self.v, self.grad)
        self.lse = torch.full((Hq, self.Tq), 7.0, device=gpu)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=gpu)  # noqa: E731
        self.keep = [i32(self.qo), i32(self.ko), i32(ql), i32(kl)]
        d = L.OfAttnDesc(Tq=self.Tq, Tk=self.Tk, nseq=len(ql), Hq=Hq, Hkv=Hkv, D=D, dtype=KINDS[dtype],
                         grad_dtype=KINDS[self.grad], causal=causal, window=window, scale=scale,
                         ldq=self.q.stride(0), hsq=self.q.stride(1), ldk=self.k.stride(0), hsk=self.k.stride(1),
                         ldv=self.v.stride(0), hsv=self.v.stride(1), ldo=self.o.stride(0), hso=self.o.stride(1))
        if slots:
            d.q_len, d.k_len = self.keep[2].data_ptr(), self.keep[3].data_ptr()
        else:
            d.q_off, d.k_off = self.keep[0].data_ptr(), self.keep[1].data_ptr()
        self.d = d
        self.ws = {}
        for op in (L.OF_ATTN_FWD, L.OF_ATTN_BWD):
            n = L.of_attn_workspace_size(d, op)
            self.ws[op] = (torch.full((max(n, 16) // 4,), PAD, device=gpu), n)

    def place(self, x, layout, shift):
        """x on the device: rows of heads, heads behind each other, rows with a gap, rows or heads so far
        apart that offsets pass 32 bits; `shift` elements off the allocation's alignment."""
        T, H, D = x.shape
        ld, hs = {"rows": (H * D, D), "heads": (D, T * D), "gap": (H * D + 8, D), "odd": (H * D + 3, D),
                  "wide": (1 << 21, D), "far": (D, (1 << 31) + 64)}[layout]
        size = (T - 1) * ld + (H - 1) * hs + D + shift
        flat = torch.zeros(size, dtype=x.dtype, device=self.gpu)
        y = flat[shift:].as_strided((T, H, D), (ld, hs, 1))
        y.copy_(x)
        return y

    def fwd(self, stream=None, lse=True):
        ws, n = self.ws[L.OF_ATTN_FWD]
        s = stream if stream is not None else torch.cuda.current_stream().cuda_stream
        L.of_attn_fwd(self.d, self.q.data_ptr(), self.k.data_ptr(), self.v.data_ptr(), self.o.data_ptr(),
                      self.lse.data_ptr() if lse else None, ws.data_ptr(), n, s)
        return self

    def bwd(self, stream=None):
        ws, n = self.ws[L.OF_ATTN_BWD]
        s = stream if stream is not None else torch.cuda.current_stream().cuda_stream
        L.of_attn_bwd(self.d, *[x.data_ptr() for x in (self.q, self.k, self.v, self.o, self.lse, self.do, self.dq,
                                                       self.dk, self.dv)], ws.data_ptr(), n, s)
        return self

    def check(self, back=True):
        G, scale = self.Hq // self.Hkv, self.scale or 1.0 / math.sqrt(self.D)
        c = {n: getattr(self, n).detach().cpu() for n in ("q", "k", "v", "do", "o", "lse", "dq", "dk", "dv")}
        rows_q = torch.zeros(self.Tq, dtype=torch.bool)
        rows_k = torch.zeros(self.Tk, dtype=torch.bool)
        for s, (nq, nk) in enumerate(zip(self.ql, self.kl)):
            rq, rk = slice(self.qo[s], self.qo[s] + nq), slice(self.ko[s], self.ko[s] + nk)
            rows_q[rq], rows_k[rk] = True, True
            ok = sees(nq, nk, self.causal, self.window)
            for hk in range(self.Hkv):
                k, v = c["k"][rk, hk], c["v"][rk, hk]
                sums = [torch.zeros(nk, self.D, dtype=torch.float64) for _ in range(4)]
                for h in range(hk * G, hk * G + G):
                    q = c["q"][rq, h]
                    what = f"sequence {s} head {h}"
                    o, lse, bo, bl, _ = forward(q, k, v, ok, scale, self.dtype)
                    self.near(c["o"][rq, h], o, bo, what + " o")
                    empty = torch.isinf(lse)
                    got = c["lse"][h, rq].double()
                    assert torch.equal(got[empty], lse[empty]), what + " lse of empty rows"
                    self.near(got[~empty], lse[~empty], bl[~empty], what + " lse")
                    if not back:
                        continue
                    do = c["do"][rq, h].to(TYPES[self.dtype])   # as an operand
                    (dq, dk, dv), (bq, bk, bv) = backward(q, k, v, do, ok, scale, self.dtype, self.grad)
                    self.near(c["dq"][rq, h], dq, bq, what + " dq")
                    for i, x in enumerate((dk, dv, bk, bv)):
                        sums[i] += x
                if back:
                    self.near(c["dk"][rk, hk], sums[0], sums[2], f"sequence {s} key head {hk} dk")
                    self.near(c["dv"][rk, hk], sums[1], sums[3], f"sequence {s} key head {hk} dv")
        for n, rows in (("o", rows_q), ("dq", rows_q), ("dk", rows_k), ("dv", rows_k)):
            if n == "o" or back:
                assert (c[n][~rows] == 7).all(), f"{n}: a row of no sequence was written"
        assert (c["lse"][:, ~rows_q] == 7).all()

    @staticmethod
    def near(got, want, bound, what):
        err = (got.double() - want).abs()
        bad = ~(err <= bound + 1e-30)
        assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / (bound + 1e-30)).max()):.3g} bounds"


MASKS = {"whole": (0, 0), "causal": (1, 0), "causal_window": (1, 37), "window": (0, 21)}
SEQS = {"one": ([1], [1]), "ragged": ([5, 0, 130, 64, 1, 97], [5, 0, 130, 64, 1, 97]),
        "cross": ([3, 70, 0, 9, 33], [200, 31, 12, 0, 33]), "empty_rows": ([150, 40], [20, 1])}


@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("seqs", SEQS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_masks_and_sequences(gpu, dtype, seqs, mask):
    ql, kl = SEQS[seqs]
    causal, window = MASKS[mask]
    Call(ql, kl, Hq=4, Hkv=2, D=64, dtype=dtype, causal=causal, window=window, tail=3).fwd().bwd().check()


@pytest.mark.parametrize("D", [1, 16, 33, 40, 64, 72, 96, 128, 160, 200, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_head_widths(gpu, dtype, D):
    Call([100, 37], [100, 37], Hq=3, Hkv=1, D=D, dtype=dtype, causal=1).fwd().bwd().check()


@pytest.mark.parametrize("layout,shift", [("rows", 0), ("heads", 0), ("gap", 0), ("odd", 0), ("rows", 1), ("gap", 8)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layouts(gpu, dtype, layout, shift):
    for D in (64, 36):
        Call([66, 80], [66, 80], Hq=4, Hkv=2, D=D, dtype=dtype, causal=1, layout=layout, shift=shift).fwd().bwd().check()


@pytest.mark.parametrize("dtype,layout,shift", [("bf16", "wide", 0), ("bf16", "wide", 1), ("bf16", "far", 0), ("f32", "far", 0)])
def test_offsets_past_32_bits(gpu, dtype, layout, shift):
    """Row 1024 of rows 2^21 elements apart is 2^31 elements on; head 1 of heads 2^31 apart."""
    c = Call([3, 1090], [3, 1090], Hq=2, Hkv=2, D=64, dtype=dtype, causal=1, window=200, layout=layout, shift=shift)
    c.fwd().bwd().check()
    del c
    torch.cuda.empty_cache()


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (6, 2), (7, 1), (8, 8), (16, 2), (130, 1)])
def test_head_groups(gpu, Hq, Hkv):
    Call([70, 33], [90, 33], Hq=Hq, Hkv=Hkv, D=32, causal=1).fwd().bwd().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_slots_with_lengths(gpu, dtype):
    """A padded batch: rows behind a length hold NaN and stay as they were."""
    Call([5, 70, 0, 31], [5, 70, 9, 64], Hq=4, Hkv=4, D=64, dtype=dtype, causal=1, slots=True).fwd().bwd().check()


@pytest.mark.parametrize("D", [40, 64, 128, 256])
def test_fp32_gradients_of_bf16_operands(gpu, D):
    """dout is rounded to bf16 as an operand; dq, dk, dv come in fp32."""
    Call([140, 9], [140, 9], Hq=4, Hkv=2, D=D, grad="f32", causal=1).fwd().bwd().check()
    Call([60, 9], [60, 9], Hq=2, Hkv=2, D=D, grad="f32", causal=1, shift=1, layout="odd").fwd().bwd().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_one_token_over_long_caches(gpu, dtype, D):
    """Split over the keys and joined; lengths from nothing to several splits."""
    c = Call([1, 1, 1, 1, 2], [5000, 1, 0, 1025, 700], Hq=8, Hkv=2, D=D, dtype=dtype, causal=1, slots=True)
    assert c.ws[L.OF_ATTN_FWD][1] > 0      # a split call
    c.fwd().check(back=False)
    c = Call([1], [3000], Hq=2, Hkv=1, D=D, dtype=dtype, window=100, causal=1).fwd()
    c.check(back=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_longer_sequences(gpu, dtype):
    """Many tiles, large logits (scale 1), a window that skips whole tiles."""
    Call([700], [700], Hq=2, Hkv=1, D=64, dtype=dtype, causal=1, scale=0.5).fwd().bwd().check()
    Call([900, 300], [1100, 300], Hq=2, Hkv=1, D=64, dtype=dtype, causal=1, window=150).fwd().bwd().check()
    Call([500], [800], Hq=1, Hkv=1, D=128, dtype=dtype).fwd().bwd().check()


@pytest.mark.parametrize("D", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_split_backward(gpu, dtype, D):
    """Few key tiles, many queries: dK and dV in parts over the queries of several heads, and their sum."""
    c = Call([1200, 40], [300, 40], Hq=4, Hkv=1, D=D, dtype=dtype, causal=1, tail=2)
    stats = 4 * (4 * c.Tq + 3)
    assert c.ws[L.OF_ATTN_BWD][1] > stats
    c.fwd().bwd().check()
    Call([700], [700], Hq=4, Hkv=2, D=D, dtype=dtype, causal=1, window=90, slots=True, grad="f32").fwd().bwd().check()


def test_offsets_with_lengths(gpu):
    """Slots of different sizes, given by offsets, filled in part: keys in a cache, packed queries."""
    c = Call([3, 40, 1, 17], [100, 40, 9, 64], Hq=4, Hkv=2, D=64, causal=1, slots=True)
    c.d.q_off, c.d.k_off = c.keep[0].data_ptr(), c.keep[1].data_ptr()
    c.fwd().bwd().check()


@pytest.mark.parametrize("name", ["q", "k", "v", "o", "do", "dq", "dk", "dv"])
def test_one_tensor_off_alignment(gpu, name):
    """Each tensor alone two bytes off a 16-byte address, the others on one."""
    c = Call([70, 9], [70, 9], Hq=4, Hkv=2, D=64, causal=1)
    setattr(c, name, c.place(getattr(c, name).cpu(), "rows", 1))
    c.fwd().bwd().check()


def test_more_queries_than_keys_in_a_window(gpu):
    for causal in (0, 1):
        Call([300], [70], Hq=2, Hkv=1, D=64, causal=causal, window=20).fwd().bwd().check()
        Call([70], [300], Hq=2, Hkv=1, D=64, causal=causal, window=20).fwd().bwd().check()


def test_large_logits(gpu):
    """Maxima that grow from tile to tile by more and by less than the kernel's step of its running
    maximum, in both orders; rows of one huge logit.  (fp32: the logits' own error grows with them, and
    the bound with it.)"""
    for dtype in ("bf16", "f32"):
        c = Call([260], [260], Hq=1, Hkv=1, D=64, dtype=dtype)
        f = torch.linspace(0.1, 6.0, 260, device=gpu)[:, None, None]
        c.k.copy_(c.k.float() * f)
        c.fwd().bwd().check()
        c.k.copy_(c.k.flip(0))
        c.fwd().bwd().check()


def test_many_sequences(gpu):
    lens = [(i * 7) % 13 for i in range(300)]
    Call(lens, lens, Hq=2, Hkv=1, D=16, causal=1).fwd().bwd().check()


def test_offsets_out_of_range_are_cut(gpu):
    """Offsets and lengths that would leave the tensors: rows that can be found are computed, nothing
    else is touched (the cutting itself is tested on the CPU)."""
    c = Call([30, 50], [30, 50], Hq=2, Hkv=1, D=64, causal=1)
    want = c.fwd().o.clone()
    c.keep[0].copy_(torch.tensor([0, 30, 1 << 30], dtype=torch.int32))
    c.keep[1].copy_(torch.tensor([-5, 30, 1 << 30], dtype=torch.int32))
    c.o.fill_(7)
    c.fwd().bwd()
    torch.cuda.synchronize()
    assert torch.equal(c.o, want)


def test_no_lse(gpu):
    c = Call([65], [65], causal=1)
    c.fwd(lse=False)
    assert (c.lse == 7).all()
    a = c.o.clone()
    c.fwd()
    assert torch.equal(a, c.o)


def test_deterministic_streams_and_graphs(gpu):
    """The same bits on another stream, and in every replay of a captured pair of calls with other work
    and other inputs between; two graphs with workspaces of their own do not disturb each other."""
    cs = [Call([200, 64], [200, 64], Hq=4, Hkv=2, D=64, causal=1, seed=s) for s in (1, 2)]
    # (a split call, its partial sums in the workspace)
    cs.append(Call([1, 1], [2000, 300], Hq=4, Hkv=2, D=64, causal=1, seed=3))
    want = []
    for c in cs:
        c.fwd().bwd()
        torch.cuda.synchronize()
        want.append([x.clone() for x in (c.o, c.lse, c.dq, c.dk, c.dv)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for c in cs:
        for x in (c.o, c.dq, c.dk, c.dv):
            x.fill_(3)
    torch.cuda.synchronize()
    for c, w in zip(cs, want):
        c.fwd(side.cuda_stream).bwd(side.cuda_stream)
        side.synchronize()
        for x, y in zip((c.o, c.lse, c.dq, c.dk, c.dv), w):
            assert torch.equal(x, y)
    graphs = []
    for c in cs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            c.fwd(side.cuda_stream).bwd(side.cuda_stream)
        graphs.append(g)
    for k in range(3):
        for c in cs:
            for x in (c.o, c.lse, c.dq, c.dk, c.dv):
                x.fill_(float(k))
        torch.randn(1000, device=gpu).sum()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, w in zip(cs, want):
            for x, y in zip((c.o, c.lse, c.dq, c.dk, c.dv), w):
                assert torch.equal(x, y)
    # new inputs in the captured buffers
    c = cs[0]
    c.q.copy_(c.q.flip(0))
    graphs[0].replay()
    torch.cuda.synchronize()
    c.check()


def test_gradient_against_differences(gpu):
    """fp32, central differences of sum(o * do) in one random direction each for q, k and v: the
    difference quotient of a loss L ~ 1 with step h has an error of h^2 L''' / 6 + 2 e |L| / h; with
    h = 2^-7 and O(1) derivatives both stay below 1e-3 of the directional derivative's scale."""
    c = Call([40, 25], [50, 25], Hq=4, Hkv=2, D=32, dtype="f32", causal=1)
    c.fwd().bwd()
    g = torch.Generator(device=gpu).manual_seed(5)
    ok = [torch.isfinite(c.q), torch.isfinite(c.k)]

    def loss():
        c.fwd()
        torch.cuda.synchronize()
        return float((c.o.double() * c.do.double())[ok[0]].sum())
    for name, grad in (("q", c.dq.clone()), ("k", c.dk.clone()), ("v", c.dv.clone())):
        x = getattr(c, name)
        e = torch.randn(x.shape, generator=g, device=gpu)
        h = 2.0 ** -7
        x0 = x.clone()
        x.copy_(x0 + h * e)
        up = loss()
        x.copy_(x0 - h * e)
        down = loss()
        x.copy_(x0)
        slope = float((grad.double() * e.double()).sum())
        size = float((grad.double() ** 2).sum().sqrt())
        assert abs((up - down) / (2 * h) - slope) <= 1e-2 * max(size, 1.0), name
