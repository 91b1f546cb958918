"""Calls over packed caches that test_gpu_packed.py does not make, against the same reference, with the kernels that a call
launched read from a captured copy of it."""
import ctypes
import re

import numpy as np
import pytest
import torch

import paper_2609_17983_amd as kvr
from tests import packed_ref as ref
from tests.gpu_util import TOL, say
from tests.test_gpu_packed import BF16, F32, TDT, Ctx, fill, rows_like, stream

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------- what a call launched


class _Dim3(ctypes.Structure):
    _fields_ = [("x", ctypes.c_uint), ("y", ctypes.c_uint), ("z", ctypes.c_uint)]


class _KernelNode(ctypes.Structure):
    _fields_ = [("block", _Dim3), ("extra", ctypes.c_void_p), ("func", ctypes.c_void_p), ("grid", _Dim3),
                ("params", ctypes.c_void_p), ("lds", ctypes.c_uint)]


def launched(call):
    """The packed-attention kernels of a call (captured, not run): (name, template arguments, threads of a block)."""
    hip = ctypes.CDLL("libamdhip64.so")
    hip.hipKernelNameRefByPtr.restype = ctypes.c_char_p
    g = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(g):
        call()
    raw, n = ctypes.c_void_p(g.raw_cuda_graph()), ctypes.c_size_t(0)
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(n)) == 0
    nodes = (ctypes.c_void_p * n.value)()
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(n)) == 0
    out = []
    for node in nodes:
        p = _KernelNode()
        if hip.hipGraphKernelNodeGetParams(ctypes.c_void_p(node), ctypes.byref(p)) != 0:
            continue  # no kernel
        name = hip.hipKernelNameRefByPtr(ctypes.c_void_p(p.func), None).decode()
        m = re.search(r"(attention_packed\w*?_kernel)I([tf]?)((?:Li\d+E)+)E", name)
        if m and "combine" not in m[1]:
            out.append((m[1], m[2], tuple(int(x) for x in re.findall(r"Li(\d+)E", m[3])), p.block.x))
    return out


# ---------------------------------------------------------------------------- attention


class Case:
    """Query rows over packed caches, and what they should give."""

    def __init__(self, c, bits, docs, packs, decs, seed=0, spoil=False):
        """docs: (index into packs, positions).  spoil: rows at -1 hold NaN."""
        self.bits, self.docs, self.dtype = bits, docs, c.dtype
        R = sum(len(p) for _, p in docs)
        self.x, t = rows_like((R, c.Hq * c.hd), c.dtype, seed + 77)
        if spoil:
            t[[p < 0 for _, d in docs for p in d]] = float("nan")
        self.q, self.packs = t.cuda(), [p.cuda() for p in packs]
        self.want, self.bound = np.zeros((2, R, c.Hq, c.hd)), np.zeros((2, R, c.Hq))
        self.want = self.want[0]
        half = torch.finfo(TDT[c.dtype]).eps / 2
        at = 0
        for i, pos in docs:
            q = self.x[at:at + len(pos)].reshape(-1, c.Hq, c.hd)
            self.want[at:at + len(pos)] = ref.attend(q, pos, ref.values(*decs[i][0]), ref.values(*decs[i][1]))
            for pairs in (0, 1):
                self.bound[pairs, at:at + len(pos)] = ref.attend_bound(q, pos, *decs[i], bits, c.dtype == F32, pairs == 1)
            at += len(pos)
        self.tol = self.bound[..., None] * (1 + half) + half * np.abs(self.want) + 1e-30

    def call(self, c, out):
        lst = kvr.make_packed_rows([(self.packs[i].data_ptr(), self.packs[i].shape[3] * 32, p) for i, p in self.docs])
        n = c.Hq * c.hd
        return lambda: kvr.kvr_attention_packed(c.ctx, c.layers - 1, self.bits, lst, self.q.data_ptr(), n, out.data_ptr(), n,
                                                stream())

    def check(self, c, kernel=None, tag=""):
        """Runs the call and holds it to the bound of the kernel that it launched; kernel: the name and block that it has to
        be.  Returns the output."""
        out = torch.full((self.q.shape[0], c.Hq * c.hd), 3.0, dtype=TDT[c.dtype], device="cuda")
        call = self.call(c, out)
        call()
        torch.cuda.synchronize()
        ran = launched(call)
        if kernel:
            assert {(k[0], k[3]) for k in ran} == {kernel}, ran
        y = out.cpu().float().numpy().reshape(self.want.shape).astype(np.float64)
        off = np.abs(y - self.want) / self.tol[int(any("rows" in k[0] for k in ran))]
        say(f"attention {tag} {sorted(set(ran))}: worst error over bound {np.nanmax(off):.3f}")
        assert np.array_equal(np.isnan(y), np.isnan(self.want)) and np.nanmax(off) <= 1.0
        # and over all of them: the output's rounding alone in bf16, the repository's tolerance in fp32
        ok = np.isfinite(self.want)
        rel = np.linalg.norm(y[ok] - self.want[ok]) / np.linalg.norm(self.want[ok])
        assert rel <= (TOL[F32] if c.dtype == F32 else torch.finfo(TDT[c.dtype]).eps / 2)
        return out


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,bits", [(BF16, 8, 2, 64, 4), (BF16, 32, 8, 128, 8), (F32, 4, 4, 64, 8)])
def test_consecutive_rows_with_others(dtype, Hq, Hkv, hd, bits):
    """Runs and short pieces of a list that no table holds whole: every row lands where it belongs."""
    with Ctx(dtype, Hq, Hkv, hd, max_ctx=1152) as c:
        packs, decs = zip(*[fill(c, n, bits, n) for n in (1100, 60)])
        docs = [(1, [59, 3]), (0, [7, -1] + list(range(30, 700)) + [5] + list(range(0, 600, 5)) + list(range(800, 1100))),
                (1, list(range(60)))]
        case = Case(c, bits, docs, packs, decs)
        case.check(c, tag="runs")


SHAPES = {114: "attention_packed_kernel", 118: "attention_packed_kernel", 124: "attention_packed_kernel",
          128: "attention_packed_kernel", 144: "attention_packed_kernel", 148: "attention_packed_kernel",
          218: "attention_packed_kernel", 418: "attention_packed_kernel", 818: "attention_packed_rows_kernel"}


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,bits", [
    (BF16, 8, 2, 128, 4), (BF16, 14, 2, 96, 8), (BF16, 12, 3, 64, 4), (BF16, 8, 2, 40, 8), (F32, 8, 2, 128, 4), (F32, 4, 2, 64, 8)])
def test_attention_in_every_shape(dtype, Hq, Hkv, hd, bits, monkeypatch):
    """Blocks of four and of eight wavefronts, copies of the columns, column tiles and the kernel for many rows, each made to
    take single rows, several rows, split and unsplit keys, repeated and idle rows."""
    with Ctx(dtype, Hq, Hkv, hd, layers=2, max_ctx=1184) as c:
        packs, decs = zip(*[fill(c, n, bits, n, slots) for n, slots in ((1100, 1180), (33, 64), (300, 300))])
        docs = [(0, [1099]), (1, [32]), (2, [299, -1, 16, 299]), (0, list(range(900, 948))), (1, [-1]), (2, [0])]
        case = Case(c, bits, docs, packs, decs, spoil=True)
    for shape, name in SHAPES.items():
        if shape == 818 and dtype == F32:
            continue
        monkeypatch.setenv("KVR_PACKED_SHAPE", str(shape))
        with Ctx(dtype, Hq, Hkv, hd, layers=2, max_ctx=1184) as c:
            case.check(c, (name, 64 * (shape % 10)), str(shape))


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,bits,rows", [
    (BF16, 32, 8, 128, 4, 120), (BF16, 28, 4, 128, 8, 120), (BF16, 32, 2, 64, 4, 240), (F32, 8, 8, 64, 8, 120)])
def test_attention_of_a_large_batch_of_single_rows(dtype, Hq, Hkv, hd, bits, rows):
    """Enough work for blocks of four wavefronts, and more documents than a table holds (they share a cache)."""
    with Ctx(dtype, Hq, Hkv, hd, max_ctx=1536) as c:
        pack, dec = fill(c, 1500, bits, 3)
        docs = [(0, [-1 if i % 17 == 5 else 1499 - i % 40]) for i in range(rows)]
        Case(c, bits, docs, [pack], [dec]).check(c, ("attention_packed_kernel", 256), "batch")


def cancelling(p, n, hd, bits, monkeypatch):
    """Fills the planes p [2][heads][blocks][bytes] of one layer: positions 2 i and 2 i + 1 have equal keys, and values
    m + s c and -(m + s c); the last 16 add small ones.  Returns what ref.read gives."""
    rng = np.random.default_rng(bits)
    top, heads = (1 << bits) - 1, p.shape[1]
    keys = np.repeat(0.3 * rng.standard_normal((heads, n // 2, hd)).astype(np.float32), 2, 1)
    ref.write(p[0], keys, range(n), bits, False)
    codes = rng.integers(0, top + 1, (heads, n // 2, hd))
    codes = np.stack([codes, top - codes], 2).reshape(heads, n, hd)
    scale = np.full((heads, n, hd // 64), 2.0 ** -bits, np.float32)
    offset = np.tile(np.repeat(np.float32([-(top + 1) / 2, -(top - 1) / 2])[:, None], hd // 64, 1), (heads, n // 2, 1)) * scale
    scale[:, -16:] *= 2.0 ** -9
    offset[:, -16:] = 2.0 ** -9
    with monkeypatch.context() as m:  # these codes, not what the format would make of some values
        m.setattr(ref, "quantise", lambda *_: (codes, scale, offset.astype(np.float32)))
        ref.write(p[1], np.zeros((heads, n, hd), np.float32), range(n), bits, True)
    dec = [ref.read(p[kv], n, hd, bits, kv == 1) for kv in range(2)]
    assert np.array_equal(dec[1][0], codes) and np.array_equal(dec[1][1], scale) and np.array_equal(dec[1][2], offset)
    v = ref.values(*dec[1])[:, :-16].reshape(heads, -1, 2, hd)
    assert (v[:, :, 0] == -v[:, :, 1]).all() and np.abs(v).max() > 0.4
    return dec


@pytest.mark.parametrize("shape", [148, 144, 418, 818])
@pytest.mark.parametrize("bits", [4, 8])
def test_attention_of_values_that_cancel(bits, shape, monkeypatch):
    """Outputs below 2^-11 of their terms: each value has its opposite under an equal key.  The pieces' rounding is part of
    the largest value, as the bound states it, not of the output."""
    monkeypatch.setenv("KVR_PACKED_SHAPE", str(shape))
    n, hd = 512, 128
    with Ctx(BF16, 8, 2, hd, max_ctx=n) as c:
        p = c.packed(n, bits).numpy()
        dec = cancelling(p[0], n, hd, bits, monkeypatch)
        case = Case(c, bits, [(0, [n - 1] * 40)], [torch.tensor(p)], [dec])
        terms = np.abs(ref.values(*dec[1])).max()
        assert 0 < np.abs(case.want).max() < 2.0 ** -11 * terms
        out = torch.zeros((40, 8 * hd), dtype=torch.bfloat16, device="cuda")
        call = case.call(c, out)
        call()
        torch.cuda.synchronize()
        assert {(k[0], k[3]) for k in launched(call)} == {(SHAPES[shape], 64 * (shape % 10))}
        err = np.abs(out.cpu().double().numpy().reshape(case.want.shape) - case.want)
        say(f"cancelling values, {bits} bits, {shape}: error {err.max() / terms:.1e} of the terms, "
            f"{np.linalg.norm(err) / np.linalg.norm(case.want):.1e} of the outputs")
        assert (err <= case.tol[int(shape == 818)]).all()


@pytest.mark.parametrize("shape", [0, 418, 818])
def test_attention_beyond_32_bit_offsets(shape, monkeypatch):
    """The last plane of a packed cache of more than 4 GiB: queries that find the first and the very last position among
    200000, whose keys are zero elsewhere."""
    monkeypatch.setenv("KVR_PACKED_SHAPE", str(shape))
    layers, n, Hkv, hd = 17, 200000, 8, 128
    with Ctx(BF16, Hkv, Hkv, hd, layers=layers, max_ctx=n) as c:
        size = kvr.kvr_packed_bytes(c.dims, n, 8)
        assert size > 1 << 32
        dev = torch.zeros(size, dtype=torch.uint8, device="cuda")
        pos = [0, 5, n - 1]
        rng = np.random.default_rng(4)
        t = torch.tensor(rng.standard_normal((2, 3, Hkv * hd)), dtype=torch.float32).bfloat16()
        kv, x = t.cuda(), t.float().numpy()
        docs = kvr.make_packed_rows([(dev.data_ptr(), n, pos)])
        kvr.kvr_append_packed(c.ctx, layers - 1, 8, docs, kv.data_ptr(), kv.data_ptr() + 3 * Hkv * hd * 2, Hkv * hd, stream())
        dec = []
        for v in range(2):  # the written rows as slots 0, 5 and 63 of two blocks
            p = np.zeros((Hkv, 2, ref.block_bytes(hd, 8)), np.uint8)
            ref.write(p, x[v].reshape(3, Hkv, hd).transpose(1, 0, 2), [0, 5, 63], 8, v == 1)
            dec.append(ref.read(p, 64, hd, 8, v == 1))
        k, v = (ref.values(*d)[:, [0, 5, 63]] for d in dec)
        # rows that look for the three positions, and one that looks for the last one and does not see it
        seen = [n - 1, n - 1, n - 1, n - 2]
        q = torch.tensor(4.0 * x[0][[0, 1, 2, 2]]).bfloat16()
        qn = q.float().numpy().reshape(4, Hkv, hd)

        def expect(visible):
            """By the softmax over the written rows that are visible and the zero rows, whose scores and values are zero."""
            want = np.zeros((4, Hkv, hd))
            for r in range(4):
                for h in range(Hkv):
                    s = np.where(visible[r], qn[r, h].astype(np.float64) @ k[h].T / np.sqrt(hd), -np.inf)
                    w = np.exp(s - s.max())
                    want[r, h] = w @ v[h] / (w.sum() + (seen[r] + 1 - np.isfinite(s).sum()) * np.exp(-s.max()))
            return want

        see = np.array([[True, True, p == n - 1] for p in seen])
        want = expect(see)
        V = float((256 * dec[1][1].astype(np.float64) + np.abs(dec[1][2])).max())
        # the bound over the written rows, and the sums over all slots
        tol = ref.attend_bound(qn, [63] * 4, dec[0], dec[1], 8, False, shape == 818)[..., None] + \
            2 * (n / 32) * 2.0 ** -24 * V + 2.0 ** -8 * np.abs(want)
        without = see.copy()
        without[:, 2] = False
        for wrong in (expect(without), 0 * want, 2 * want):  # the bound sees what it is for
            assert (np.abs(wrong - want)[2] > tol[2]).mean() > 0.9
        dq, out = q.cuda(), torch.full((4, Hkv * hd), 3.0, dtype=torch.bfloat16, device="cuda")
        rows = kvr.make_packed_rows([(dev.data_ptr(), n, seen)])
        kvr.kvr_attention_packed(c.ctx, layers - 1, 8, rows, dq.data_ptr(), Hkv * hd, out.data_ptr(), Hkv * hd, stream())
        torch.cuda.synchronize()
        off = np.abs(out.cpu().double().numpy().reshape(want.shape) - want) / tol
        say(f"beyond 32 bits, shape {shape}: worst error over bound {off.max():.3f}")
        assert off.max() <= 1.0
