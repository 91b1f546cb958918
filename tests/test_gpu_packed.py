"""Packed caches on the GPU: quantising, reading back and attending, each against
tests/packed_ref.py (codes and stored values bit for bit; attention within the bound
derived there), and the calls that are refused."""
import numpy as np
import pytest
import torch

import paper_2609_17983_amd as kvr
from tests import packed_ref as ref
from tests.gpu_util import TOL, say

pytestmark = pytest.mark.gpu

BF16, F32 = kvr.KVR_BF16, kvr.KVR_F32
TDT = {BF16: torch.bfloat16, F32: torch.float32}


class Ctx:
    """A context that carries a cache layout; its weights are never read."""

    def __init__(self, dtype, Hq, Hkv, hd, layers=1, max_ctx=4096):
        self.dtype, self.Hq, self.Hkv, self.hd, self.layers = dtype, Hq, Hkv, hd, layers
        self.dims = kvr.kvr_dims(layers, 4, Hq, Hkv, hd, 4, 4, 0, 1e-5, 1e4, max_ctx, 1, dtype)
        self.t = torch.zeros(4096, dtype=TDT[dtype], device="cuda")
        lw = {k: self.t for k in ("attn_norm", "wq", "wk", "wv", "wo", "mlp_norm", "w_gate", "w_up", "w_down")}
        self.ws = kvr.weights_struct({"embed": self.t, "final_norm": self.t, "layers": [lw] * layers})
        self.ctx = kvr.kvr_create(self.dims, self.ws)

    def __enter__(self):
        return self

    def __exit__(self, *_):
        torch.cuda.synchronize()
        kvr.kvr_destroy(self.ctx)

    def packed(self, n_cap, bits, seed=0):
        """A packed cache of arbitrary bytes [L][2][Hkv][blocks][bytes]."""
        g = torch.Generator().manual_seed(seed)
        shape = (self.layers, 2, self.Hkv, ref.blocks(n_cap), ref.block_bytes(self.hd, bits))
        t = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)
        assert t.numel() == kvr.kvr_packed_bytes(self.dims, n_cap, bits)
        return t


def stream():
    return torch.cuda.current_stream().cuda_stream


def rows_like(shape, dtype, seed):
    """Values with channels of different size, rounded to the dtype; fp32 numpy and the tensor."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-1.5, 1.5, (1,) * (len(shape) - 1) + (shape[-1],)))
    t = torch.tensor(x, dtype=torch.float32).to(TDT[dtype])
    return t.float().numpy(), t


def edge_rows(x, t):
    """Rows of zeros, of one value, of tiny and huge ones, and of values that are not finite."""
    flat = t.view(-1, t.shape[-1])
    flat[0] = 0.0
    flat[1] = -2.5
    flat[2] = 1e-40
    flat[2, 0] = -1e-39
    flat[3, 0], flat[3, 1] = 3e38, -3e38
    flat[4, -1] = float("inf")
    flat[5, 0] = float("nan")
    flat[6] = flat[6] * 1e30
    flat[7, 0] = float("-inf")
    return t.float().numpy()


# ---------------------------------------------------------------------------- pack, unpack


def check_packed(got, before, cache, positions, bits):
    """got, before: packed bytes; cache fp32 [L, 2, Hkv, n, hd]: the listed positions hold its codes, the rest is as before."""
    want = before.copy()
    for l in range(want.shape[0]):
        for kv in range(2):
            ref.write(want[l, kv], cache[l, kv][:, positions], positions, bits, kv == 1)
    assert np.array_equal(got, want)
    return want


def stored(packed, n, hd, bits, tdt):
    """What packed bytes stand for, rounded to the dtype, [L, 2, Hkv, n, hd]."""
    v = np.stack([np.stack([ref.values(*ref.read(packed[l, kv], n, hd, bits, kv == 1)) for kv in range(2)])
                  for l in range(packed.shape[0])])
    with np.errstate(all="ignore"):
        return torch.tensor(v.astype(np.float32)).to(tdt)


LISTS = {
    "all": lambda n: None,
    "one": lambda n: [n - 1],
    "run": lambda n: list(range(n // 3, n)),
    "spread": lambda n: list(range(1, n, 3)),
    "mixed": lambda n: [0] + list(range(5, min(n, 40))) + list(range(41, n, 2)),
}


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,Hkv,hd,n_cap,extra,which", [
    (BF16, 2, 128, 70, 5, "all"), (BF16, 3, 64, 33, 0, "spread"), (F32, 2, 128, 64, 40, "mixed"),
    (F32, 1, 64, 45, 0, "all"), (BF16, 2, 96, 50, 1, "run"), (F32, 2, 40, 64, 0, "mixed"), (BF16, 1, 2, 32, 0, "all"),
    (BF16, 2, 66, 31, 3, "mixed"), (BF16, 1, 128, 41, 0, "one"), (F32, 2, 80, 100, 0, "spread"), (F32, 1, 6, 65, 0, "run"),
])
def test_pack_and_unpack_match_the_format(bits, dtype, Hkv, hd, n_cap, extra, which):
    with Ctx(dtype, 2 * Hkv, Hkv, hd, layers=2) as c:
        _, t = rows_like((2, 2, Hkv, n_cap, hd), dtype, hd + bits)
        x = edge_rows(None, t)
        positions = LISTS[which](n_cap)
        plist = list(range(n_cap)) if positions is None else positions
        before = c.packed(n_cap + extra, bits)
        packed, cache = before.cuda(), t.cuda()
        arg = n_cap if positions is None else positions
        say(f"pack {bits} bits hd={hd} {which}")
        kvr.kvr_pack(c.ctx, kvr.make_pack_docs([(cache.data_ptr(), n_cap, packed.data_ptr(), n_cap + extra, arg)]), bits, stream())
        torch.cuda.synchronize()
        want = check_packed(packed.cpu().numpy(), before.numpy(), x, plist, bits)
        assert torch.equal(cache.cpu().view(torch.uint8), t.view(torch.uint8))
        # back into a cache of another capacity; other slots keep what they held
        sentinel = torch.full((2, 2, Hkv, n_cap + 7, hd), 7.0, dtype=TDT[dtype])
        out = sentinel.cuda()
        kvr.kvr_unpack(c.ctx, kvr.make_pack_docs([(out.data_ptr(), n_cap + 7, packed.data_ptr(), n_cap + extra, arg)]), bits,
                       stream())
        torch.cuda.synchronize()
        got = out.cpu()
        sentinel[:, :, :, plist] = stored(want, n_cap, hd, bits, TDT[dtype])[:, :, :, plist]
        assert torch.equal(torch.isnan(got), torch.isnan(sentinel))
        assert torch.equal(torch.nan_to_num(got.float()), torch.nan_to_num(sentinel.float()))


@pytest.mark.parametrize("bits", [4, 8])
def test_pack_of_many_documents_and_long_lists(bits):
    """More documents than one launch's table holds, a scattered list longer than one, empty lists between them."""
    with Ctx(BF16, 1, 1, 64) as c:
        ns = [2500] + [20 + i % 23 for i in range(90)]
        lists = [list(range(0, 2500, 2)) + [2499]] + [[] if i % 7 == 3 else list(range(i % 5, n, 2 if i % 2 else 1))
                                                      for i, n in enumerate(ns[1:])]
        xs = [rows_like((1, 2, 1, n, 64), BF16, n + i) for i, n in enumerate(ns)]
        befores = [c.packed(n, bits, seed=i) for i, n in enumerate(ns)]
        packs, caches = [b.cuda() for b in befores], [t.cuda() for _, t in xs]
        docs = kvr.make_pack_docs([(t.data_ptr(), n, p.data_ptr(), n, l) for t, n, p, l in zip(caches, ns, packs, lists)])
        kvr.kvr_pack(c.ctx, docs, bits, stream())
        torch.cuda.synchronize()
        wants = [check_packed(p.cpu().numpy(), b.numpy(), x, l, bits) for p, b, (x, _), l in zip(packs, befores, xs, lists)]
        outs = [torch.zeros_like(t) for t in caches]
        kvr.kvr_unpack(c.ctx, kvr.make_pack_docs([(o.data_ptr(), n, p.data_ptr(), n, l)
                                                  for o, n, p, l in zip(outs, ns, packs, lists)]), bits, stream())
        torch.cuda.synchronize()
        for o, n, w, l in zip(outs, ns, wants, lists):
            v = torch.zeros((1, 2, 1, n, 64), dtype=torch.bfloat16)
            v[:, :, :, l] = stored(w, n, 64, bits, torch.bfloat16)[:, :, :, l]
            assert torch.equal(o.cpu(), v)


# ---------------------------------------------------------------------------- append


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,Hkv,hd,stride_extra,offset", [
    (BF16, 2, 128, 0, 0), (F32, 3, 64, 64, 0), (BF16, 1, 96, 1, 3), (F32, 2, 40, 7, 1), (BF16, 5, 64, 640, 0)])
def test_append_writes_rows_of_one_layer(bits, dtype, Hkv, hd, stride_extra, offset):
    with Ctx(dtype, Hkv, Hkv, hd, layers=2) as c:
        lists = [[5], list(range(30, 70)), [], [0, 1, 2, 31, 32, 33, 64, 90], list(range(3, 1200, 2))]
        caps = [6, 70, 1, 91, 1200]
        R = sum(map(len, lists))
        stride = Hkv * hd + stride_extra
        x, t = rows_like((2, R, stride), dtype, bits)
        # keys and values anywhere in memory, aligned to their type
        buf = torch.zeros(2 * R * stride + offset, dtype=TDT[dtype], device="cuda")
        buf[offset:] = t.view(-1).cuda()
        befores = [c.packed(n, bits, seed=n) for n in caps]
        packs = [b.cuda() for b in befores]
        docs = kvr.make_packed_rows([(p.data_ptr(), n, l) for p, n, l in zip(packs, caps, lists)])
        es = buf.element_size()
        kvr.kvr_append_packed(c.ctx, 1, bits, docs, buf.data_ptr() + offset * es, buf.data_ptr() + (offset + R * stride) * es,
                              stride, stream())
        torch.cuda.synchronize()
        at = 0
        for p, b, l in zip(packs, befores, lists):
            want = b.numpy().copy()
            for kv in range(2):
                rows = x[kv, at:at + len(l), :Hkv * hd].reshape(len(l), Hkv, hd).transpose(1, 0, 2)
                if l:
                    ref.write(want[1, kv], rows, l, bits, kv == 1)
            at += len(l)
            assert np.array_equal(p.cpu().numpy(), want)


def test_append_to_more_documents_than_a_table_holds():
    with Ctx(BF16, 2, 1, 64) as c:
        n, cap = 150, 64
        x, t = rows_like((2, n, 64), BF16, 3)
        befores = [c.packed(cap, 4, seed=i) for i in range(n)]
        packs = [b.cuda() for b in befores]
        kv = t.cuda()
        docs = kvr.make_packed_rows([(p.data_ptr(), cap, [i % cap]) for i, p in enumerate(packs)])
        kvr.kvr_append_packed(c.ctx, 0, 4, docs, kv.data_ptr(), kv.data_ptr() + n * 64 * 2, 64, stream())
        torch.cuda.synchronize()
        for i, (p, b) in enumerate(zip(packs, befores)):
            want = b.numpy().copy()
            for v in range(2):
                ref.write(want[0, v], x[v, i].reshape(1, 1, 64), [i % cap], 4, v == 1)
            assert np.array_equal(p.cpu().numpy(), want)


# ---------------------------------------------------------------------------- attention


def fill(c, n, bits, seed, slots=None):
    """A packed cache with its positions [0, n) written by the reference, arbitrary bytes behind them; the cache's
    (codes, scale, offset) of layer `layers - 1`."""
    p = c.packed(n if slots is None else slots, bits, seed=seed).numpy()
    dec = []
    x, _ = rows_like((2, c.Hkv, n, c.hd), c.dtype, seed + 1)
    for kv in range(2):
        if n:
            ref.write(p[-1, kv], x[kv], list(range(n)), bits, kv == 1)
        dec.append(ref.read(p[-1, kv], n, c.hd, bits, kv == 1))
    return torch.tensor(p), dec


def check_attention(c, bits, docs, packs, decs, q_extra=0, o_extra=0, q_off=0, o_off=0, seed=0, call=None):
    """docs: (index into packs, positions)."""
    Hq, hd = c.Hq, c.hd
    R = sum(len(p) for _, p in docs)
    qs, os_ = Hq * hd + q_extra, Hq * hd + o_extra
    x, t = rows_like((R, qs), c.dtype, seed + 77)
    q = torch.zeros(R * qs + q_off, dtype=TDT[c.dtype], device="cuda")
    q[q_off:] = t.view(-1).cuda()
    out = torch.full((R * os_ + o_off + 5,), 3.0, dtype=TDT[c.dtype], device="cuda")
    dev = [p.cuda() for p in packs]
    lst = kvr.make_packed_rows([(dev[i].data_ptr(), dev[i].shape[3] * 32, p) for i, p in docs])
    es = q.element_size()
    args = (c.ctx, c.layers - 1, bits, lst, q.data_ptr() + q_off * es, qs, out.data_ptr() + o_off * es, os_)
    (call or (lambda: kvr.kvr_attention_packed(*args, stream())))() if call is None else call(args, out)
    torch.cuda.synchronize()
    got = out.cpu()
    assert (got[:o_off] == 3.0).all() and (got[R * os_ + o_off:] == 3.0).all()
    body = got[o_off:R * os_ + o_off].view(R, os_)
    assert (body[:, Hq * hd:] == 3.0).all()
    y = body[:, :Hq * hd].float().numpy().reshape(R, Hq, hd).astype(np.float64)
    qn = x[:, :Hq * hd].reshape(R, Hq, hd)
    at, worst, full = 0, 0.0, np.zeros_like(y)
    half = torch.finfo(TDT[c.dtype]).eps / 2
    # (more than 64 columns of a document in bf16: the kernel for many rows)
    pairs = c.dtype == BF16 and max(len(p) for _, p in docs) * Hq // c.Hkv > 64
    for i, pos in docs:
        kc, vc = decs[i]
        qq = qn[at:at + len(pos)]
        want = ref.attend(qq, pos, ref.values(*kc), ref.values(*vc))
        tol = ref.attend_bound(qq, pos, kc, vc, bits, c.dtype == F32, pairs)[..., None] * (1 + half) + half * np.abs(want) + 1e-30
        diff = np.abs(y[at:at + len(pos)] - want)
        full[at:at + len(pos)] = want
        assert np.array_equal(np.isnan(diff), np.isnan(want))
        worst = max(worst, float(np.nan_to_num(diff / tol).max(initial=0.0)))
        at += len(pos)
    # and over all of them: the output's rounding alone in bf16, the repository's tolerance in fp32
    ok = np.isfinite(full)
    rel = float(np.linalg.norm(y[ok] - full[ok]) / max(np.linalg.norm(full[ok]), 1e-300))
    say(f"attention {bits} bits hd={hd} Hq={Hq}/{c.Hkv} rows={R}: worst error over bound {worst:.3f}, of all {rel:.2e}")
    assert worst <= 1.0 and rel <= (TOL[F32] if c.dtype == F32 else half)
    return body


HEADS = [(BF16, 32, 8, 128), (BF16, 28, 4, 128), (BF16, 4, 4, 64), (F32, 4, 4, 64), (F32, 4, 2, 128), (BF16, 32, 8, 64),
         (BF16, 12, 4, 96), (F32, 6, 2, 40), (BF16, 3, 1, 80), (BF16, 40, 1, 64), (BF16, 2, 2, 2), (F32, 20, 1, 128)]


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", HEADS)
def test_attention_single_tokens(bits, dtype, Hq, Hkv, hd):
    """One row a document; lengths from one slot over the 16- and 32-position edges to long ones, an idle row, an empty list."""
    with Ctx(dtype, Hq, Hkv, hd, layers=2) as c:
        ns = [1, 2, 16, 17, 31, 32, 33, 64, 65, 129, 500, 1537]
        packs, decs = zip(*[fill(c, n, bits, n) for n in ns])
        docs = [(i, [n - 1]) for i, n in enumerate(ns)] + [(3, [-1]), (4, []), (9, [40])]
        check_attention(c, bits, docs, packs, decs)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,Hq,Hkv,hd", HEADS)
def test_attention_rows(bits, dtype, Hq, Hkv, hd):
    """Several rows: consecutive, scattered, repeated, out of order, idle between them; slots behind the rows hold
    arbitrary bytes (scales that are not finite among them)."""
    with Ctx(dtype, Hq, Hkv, hd) as c:
        packs, decs = zip(*[fill(c, n, bits, n, slots) for n, slots in ((200, 320), (33, 64), (700, 700))])
        docs = [(0, list(range(150, 200))), (1, [32, 3, -1, 3, 0, 31]), (2, list(range(0, 700, 9))), (0, [7])]
        check_attention(c, bits, docs, packs, decs)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,q_extra,o_extra,q_off,o_off", [
    (BF16, 8, 2, 128, 512, 0, 0, 0), (BF16, 8, 2, 128, 1, 3, 1, 3), (F32, 4, 4, 64, 5, 1, 3, 1), (BF16, 6, 2, 96, 8, 4, 8, 4),
    (BF16, 6, 3, 40, 2, 2, 2, 2), (F32, 4, 2, 6, 0, 0, 1, 1)])
def test_attention_strides(bits, dtype, Hq, Hkv, hd, q_extra, o_extra, q_off, o_off):
    with Ctx(dtype, Hq, Hkv, hd) as c:
        pack, dec = fill(c, 90, bits, 5)
        check_attention(c, bits, [(0, [89]), (0, list(range(20, 60)))], [pack], [dec], q_extra, o_extra, q_off, o_off)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("dtype,Hq,Hkv,hd,n", [(BF16, 8, 2, 128, 700), (F32, 4, 4, 64, 300), (BF16, 8, 2, 64, 300)])
def test_attention_of_a_whole_prompt(bits, dtype, Hq, Hkv, hd, n):
    with Ctx(dtype, Hq, Hkv, hd) as c:
        pack, dec = fill(c, n, bits, 5)
        check_attention(c, bits, [(0, list(range(n)))], [pack], [dec])


@pytest.mark.parametrize("Hq,Hkv,hd,bits", [(256, 16, 128, 4), (256, 16, 128, 8), (240, 16, 96, 4), (256, 16, 64, 4),
                                            (256, 16, 64, 8), (256, 16, 40, 8), (256, 16, 66, 4)])
def test_attention_of_a_prompt_with_many_heads(Hq, Hkv, hd, bits):
    """Enough columns for the kernel that goes through the keys once for many rows; slots behind the rows hold arbitrary
    bytes."""
    with Ctx(BF16, Hq, Hkv, hd) as c:
        pack, dec = fill(c, 420, bits, 5, 500)
        check_attention(c, bits, [(0, list(range(420)))], [pack], [dec])


def test_attention_of_many_rows_over_split_keys():
    """The same kernel with its keys cut into ranges."""
    with Ctx(BF16, 256, 4, 128) as c:
        pack, dec = fill(c, 2990, 4, 5)
        check_attention(c, 4, [(0, list(range(2890, 2990)))], [pack], [dec])


@pytest.mark.parametrize("dtype,Hq,Hkv,hd,bits", [(BF16, 32, 8, 128, 4), (F32, 8, 8, 64, 8)])
def test_attention_of_documents_with_one_row_beside_one_with_many(dtype, Hq, Hkv, hd, bits):
    """A batch that decodes while a prompt runs: the two kinds are launched apart, and every row lands where it belongs."""
    with Ctx(dtype, Hq, Hkv, hd) as c:
        ns = [700 + 20 * i for i in range(40)]
        packs, decs = zip(*[fill(c, n, bits, n) for n in ns])
        docs = [(i, [n - 1]) for i, n in enumerate(ns)]
        docs[17] = (17, list(range(ns[17] - 300, ns[17])))
        docs[30] = (30, [-1])
        check_attention(c, bits, docs, packs, decs)


def test_attention_of_more_documents_and_positions_than_a_table_holds():
    with Ctx(BF16, 4, 2, 64) as c:
        ns = [1 + (37 * i) % 211 for i in range(160)]
        made = [fill(c, n, 4, i) for i, n in enumerate(ns)] + [fill(c, 2100, 4, 999)]
        packs, decs = zip(*made)
        docs = [(i, [n - 1]) for i, n in enumerate(ns)] + [(160, list(range(0, 2100, 2)))]
        check_attention(c, 4, docs, packs, decs)


def test_attention_of_a_long_document():
    """Many key ranges, one row; and the same row beside others."""
    with Ctx(BF16, 8, 2, 128, max_ctx=20000) as c:
        pack, dec = fill(c, 20000, 4, 1)
        alone = check_attention(c, 4, [(0, [19999])], [pack], [dec])
        again = check_attention(c, 4, [(0, [19999])], [pack], [dec])
        assert torch.equal(alone, again)  # no order of additions is left to chance


@pytest.mark.parametrize("bits", [4, 8])
def test_attention_sees_values_that_are_not_finite_only_where_it_should(bits):
    """A NaN group of keys makes every row that sees it NaN; of values, that group's dimensions; rows before it are exact."""
    with Ctx(BF16, 4, 2, 128) as c:
        pack, _ = fill(c, 100, bits, 8)
        p = pack.numpy()
        bad = np.ones((2, 1, 128), np.float32)
        bad[:, :, 70] = np.nan
        ref.write(p[0, 1], bad, [60], bits, True)  # values: the second group
        ref.write(p[0, 0], bad, [80], bits, False)
        decs = [[ref.read(p[0, kv], 100, 128, bits, kv == 1) for kv in range(2)]]
        body = check_attention(c, bits, [(0, [99, 80, 79, 60, 59, 10])], [torch.tensor(p)], decs)
        y = body.view(6, 4, 128).float()
        assert torch.isnan(y[:2]).all() and torch.isnan(y[2:4, :, 64:]).all()
        assert torch.isfinite(y[2:4, :, :64]).all() and torch.isfinite(y[4:]).all()


@pytest.mark.parametrize("hd,bits", [(64, 8), (128, 4)])
def test_many_heads_see_values_that_are_not_finite_only_where_they_should(hd, bits):
    """A NaN value is seen by the rows behind it only, in its group's dimensions only, also when the next blocks are staged
    over it."""
    n = 420
    with Ctx(BF16, 256, 16, hd) as c:
        pack, _ = fill(c, n, bits, 8, n + 44)
        p = pack.numpy()
        bad = np.ones((16, 1, hd), np.float32)
        bad[:, :, hd - 1] = np.nan  # the last group
        ref.write(p[0, 1], bad, [137], bits, True)
        ref.write(p[0, 1], bad, [301], bits, True)
        ref.write(p[0, 0], bad, [370], bits, False)
        decs = [[ref.read(p[0, kv], n, hd, bits, kv == 1) for kv in range(2)]]
        rows = list(range(n))
        body = check_attention(c, bits, [(0, rows)], [torch.tensor(p)], decs)
        y = body.view(n, 256, hd).float()
        for r in rows:
            assert torch.isnan(y[r, :, hd - 64:]).all() == (r >= 137)
            if hd > 64:  # the other group's dimensions
                assert torch.isfinite(y[r, :, :hd - 64]).all() == (r < 370)


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hd", [64, 128])
def test_many_rows_see_values_that_are_not_finite_only_where_they_should(bits, hd):
    """The same for rows of few heads."""
    with Ctx(BF16, 8, 2, hd) as c:
        pack, _ = fill(c, 300, bits, 8, 320)
        p = pack.numpy()
        bad = np.ones((2, 1, hd), np.float32)
        bad[:, :, hd - 1] = np.nan  # the last group
        ref.write(p[0, 1], bad, [37], bits, True)
        ref.write(p[0, 1], bad, [201], bits, True)
        ref.write(p[0, 0], bad, [250], bits, False)
        decs = [[ref.read(p[0, kv], 300, hd, bits, kv == 1) for kv in range(2)]]
        rows = list(range(20, 60)) + list(range(190, 210)) + list(range(240, 300, 7))
        body = check_attention(c, bits, [(0, rows)], [torch.tensor(p)], decs)
        y = body.view(len(rows), 8, hd).float()
        for i, r in enumerate(rows):
            assert torch.isnan(y[i, :, hd - 64:]).all() == (r >= 37)
            if hd > 64:  # the other group's dimensions
                assert torch.isfinite(y[i, :, :hd - 64]).all() == (r < 250)


def test_attention_of_large_scores():
    """Scores far apart and far from zero: one key takes the softmax, and the running maximum rises again and again."""
    with Ctx(BF16, 4, 2, 64) as c:
        p = c.packed(400, 8).numpy()
        rng = np.random.default_rng(0)
        x = rng.standard_normal((2, 2, 400, 64)).astype(np.float32)
        x[0] *= np.linspace(0.01, 30.0, 400, dtype=np.float32)[None, :, None]  # keys grow with their position
        x = torch.tensor(x).bfloat16().float().numpy()
        for kv in range(2):
            ref.write(p[0, kv], x[kv], list(range(400)), 8, kv == 1)
        dec = [ref.read(p[0, kv], 400, 64, 8, kv == 1) for kv in range(2)]
        check_attention(c, 8, [(0, list(range(390, 400))), (0, [5])], [torch.tensor(p)], [dec])
        check_attention(c, 8, [(0, list(range(300, 400))), (0, [5])], [torch.tensor(p)], [dec])


# ---------------------------------------------------------------------------- streams, graphs, offsets


def test_attention_captured_and_replayed():
    """A captured call keeps its own documents and positions: replays give its result, whatever ran in between."""
    with Ctx(BF16, 8, 2, 128) as c:
        packs, decs = zip(*[fill(c, n, 4, n) for n in (300, 1000)])

        def call(args, out):
            kvr.kvr_attention_packed(*args, stream())  # an eager call first
            torch.cuda.synchronize()
            eager = out.clone()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                kvr.kvr_attention_packed(*args, stream())
            # other work of the same context between the replays
            other = torch.zeros_like(out)
            dev = packs[1].cuda()
            lst = kvr.make_packed_rows([(dev.data_ptr(), 1024, [999, 5])])
            for _ in range(3):
                out.fill_(3.0)
                kvr.kvr_attention_packed(c.ctx, 0, 4, lst, args[4], args[5], other.data_ptr(), 1024, stream())
                g.replay()
                torch.cuda.synchronize()
                assert torch.equal(out, eager)

        check_attention(c, 4, [(0, [299]), (1, [999]), (1, list(range(400, 440)))], packs, decs, call=call)


def test_append_and_attention_on_another_stream():
    """Append, attention and unpack in order on a stream that is not the current one; another context on its own stream
    beside them."""
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    results = []
    with Ctx(BF16, 8, 2, 64) as a, Ctx(BF16, 8, 2, 64) as b:
        pack, _ = fill(a, 64, 4, 4, 96)
        x, t = rows_like((10, 12 * 64), BF16, 9)
        fused = t.cuda()
        torch.cuda.synchronize()
        for c, s in ((a, s1), (b, s2)):
            dev = pack.cuda()
            out = torch.zeros((10, 512), dtype=torch.bfloat16, device="cuda")
            back = torch.zeros((1, 2, 2, 96, 64), dtype=torch.bfloat16, device="cuda")
            torch.cuda.synchronize()
            docs = kvr.make_packed_rows([(dev.data_ptr(), 96, list(range(64, 74)))])
            es = 2
            kvr.kvr_append_packed(c.ctx, 0, 4, docs, fused.data_ptr() + 512 * es, fused.data_ptr() + 640 * es, 768, s.cuda_stream)
            kvr.kvr_attention_packed(c.ctx, 0, 4, docs, fused.data_ptr(), 768, out.data_ptr(), 512, s.cuda_stream)
            kvr.kvr_unpack(c.ctx, kvr.make_pack_docs([(back.data_ptr(), 96, dev.data_ptr(), 96, 74)]), 4, s.cuda_stream)
            results.append((dev, out, back))
        torch.cuda.synchronize()
        p = pack.numpy().copy()
        for kv in range(2):
            rows = x[:, 512 + 128 * kv:640 + 128 * kv].reshape(10, 2, 64).transpose(1, 0, 2)
            ref.write(p[0, kv], rows, list(range(64, 74)), 4, kv == 1)
        dec = [ref.read(p[0, kv], 74, 64, 4, kv == 1) for kv in range(2)]
        want = ref.attend(x[:, :512].reshape(10, 8, 64), range(64, 74), ref.values(*dec[0]), ref.values(*dec[1]))
        tol = ref.attend_bound(x[:, :512].reshape(10, 8, 64), range(64, 74), dec[0], dec[1], 4, False)[..., None] * 1.01 + \
            2.0 ** -8 * np.abs(want)
        for dev, out, back in results:
            assert np.array_equal(dev.cpu().numpy(), p)
            assert (np.abs(out.cpu().float().numpy().reshape(10, 8, 64) - want) <= tol).all()
            assert torch.equal(back[:, :, :, :74].cpu(), stored(p, 74, 64, 4, torch.bfloat16))
            assert (back[:, :, :, 74:] == 0).all()


def test_planes_beyond_32_bit_offsets():
    """The last plane of a packed cache of more than 4 GiB."""
    layers, n_cap = 17, 200000
    with Ctx(BF16, 8, 8, 128, layers=layers, max_ctx=n_cap) as c:
        size = kvr.kvr_packed_bytes(c.dims, n_cap, 8)
        assert size > 1 << 32
        dev = torch.zeros(size, dtype=torch.uint8, device="cuda")
        pos = [0, 5, n_cap - 1]
        x, t = rows_like((2, 3, 8 * 128), BF16, 2)
        kv = t.cuda()
        docs = kvr.make_packed_rows([(dev.data_ptr(), n_cap, pos)])
        kvr.kvr_append_packed(c.ctx, layers - 1, 8, docs, kv.data_ptr(), kv.data_ptr() + 3 * 1024 * 2, 1024, stream())
        planes = dev.view(layers, 2, 8, ref.blocks(n_cap), ref.block_bytes(128, 8))
        want = np.zeros((2, 8, 2, ref.block_bytes(128, 8)), np.uint8)  # the first and the last block
        last = (n_cap - 1) % 32 + 32
        for v in range(2):
            ref.write(want[v], x[v].reshape(3, 8, 128).transpose(1, 0, 2), [0, 5, last], 8, v == 1)
        got = planes[layers - 1][:, :, [0, -1]].cpu().numpy()
        assert np.array_equal(got, want)
        assert int(planes[0, 0, 0].max()) == 0
        # one row attends over all of it: 199997 slots hold zero rows, whose scores are zero
        q = torch.zeros((1, 1024), dtype=torch.bfloat16, device="cuda")
        out = torch.full((1, 1024), 3.0, dtype=torch.bfloat16, device="cuda")
        row = kvr.make_packed_rows([(dev.data_ptr(), n_cap, [n_cap - 1])])
        kvr.kvr_attention_packed(c.ctx, layers - 1, 8, row, q.data_ptr(), 1024, out.data_ptr(), 1024, stream())
        torch.cuda.synchronize()
        v = ref.values(*ref.read(want[1], 64, 128, 8, True))[:, [0, 5, last]].sum(1) / n_cap
        y = out.cpu().float().numpy().reshape(8, 128)
        big = np.abs(x[1]).max() * 3  # of all terms; the sums run over n / 32 steps at most, see attend_bound
        assert (np.abs(y - v) <= 2.0 ** -8 * np.abs(v) + big * (2 * (n_cap / 32 + 64) * 2.0 ** -24 + 2.0 ** -16) / n_cap * 400).all()


# ---------------------------------------------------------------------------- refusals


def refused(status, fn, *args):
    with pytest.raises(kvr.KvrError) as e:
        fn(*args)
    assert e.value.status == status, str(e.value)


def test_refusals():
    with Ctx(BF16, 4, 2, 64, layers=2, max_ctx=128) as c:
        p = c.packed(128, 8).cuda()
        keep = p.clone()
        cache = torch.zeros((2, 2, 2, 128, 64), dtype=torch.bfloat16, device="cuda")
        q = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
        s, P, C, Q = stream(), p.data_ptr(), cache.data_ptr(), q.data_ptr()
        A, R, U = kvr.KVR_E_ARG, kvr.KVR_E_RANGE, kvr.KVR_E_UNSUPPORTED
        for fn in (kvr.kvr_pack, kvr.kvr_unpack):
            d = lambda *a: kvr.make_pack_docs([a])  # noqa: E731
            refused(U, fn, c.ctx, d(C, 128, P, 128, 10), 5, s)
            refused(A, fn, c.ctx, d(None, 128, P, 128, 10), 4, s)
            refused(A, fn, c.ctx, d(C, 128, P + 8, 128, 10), 4, s)
            refused(A, fn, c.ctx, d(C, 128, P, 128, -1), 4, s)
            refused(R, fn, c.ctx, d(C, 128, P, 64, 65), 4, s)
            refused(R, fn, c.ctx, d(C, 128, P, 64, [64]), 4, s)
            refused(R, fn, c.ctx, d(C, 128, P, 128, [-1]), 4, s)
            refused(R, fn, c.ctx, d(C, 128, P, 2 ** 30 + 1, [1]), 4, s)
            refused(A, fn, c.ctx, d(C, 128, P, 128, [3, 3]), 4, s)
            refused(A, fn, c.ctx, d(C, 128, P, 128, [3, 2]), 4, s)
            two = kvr.make_pack_docs([(C, 64, P, 64, 10), (C, 64, P, 64, 10)])
            refused(A, fn, c.ctx, two, 4, s)
            refused(A, fn, c.ctx, d(P, 64, P, 64, 10), 4, s)
            fn(c.ctx, d(None, 0, None, 0, []), 4, s)  # nothing to do
        d = lambda *a: kvr.make_packed_rows([a])  # noqa: E731
        att = lambda docs, layer=0, bits=4, qq=Q, qs=256, o=Q + 4096, os_=256: (  # noqa: E731
            c.ctx, layer, bits, docs, qq, qs, o, os_, s)
        app = lambda docs, layer=0, bits=4, k=Q, v=Q + 4096, st=128: (c.ctx, layer, bits, docs, k, v, st, s)  # noqa: E731
        for fn, a in ((kvr.kvr_attention_packed, att), (kvr.kvr_append_packed, app)):
            refused(U, fn, *a(d(P, 128, [1]), bits=16))
            refused(R, fn, *a(d(P, 128, [1]), layer=2))
            refused(R, fn, *a(d(P, 128, [1]), layer=-1))
            refused(A, fn, *a(d(None, 128, [1])))
            refused(A, fn, *a(d(P + 4, 128, [1])))
            refused(R, fn, *a(d(P, 129, [1])))
            refused(R, fn, *a(d(P, 0, [0])))
            refused(R, fn, *a(d(P, 128, [128])))
            fn(*a(kvr.make_packed_rows([])))
            fn(*a(d(P, 128, [])))
        refused(R, kvr.kvr_attention_packed, *att(d(P, 128, [-2])))
        refused(R, kvr.kvr_attention_packed, *att(d(P, 128, [1]), qs=255))
        refused(R, kvr.kvr_attention_packed, *att(d(P, 128, [1]), os_=255))
        refused(A, kvr.kvr_attention_packed, *att(d(P, 128, [1]), qq=None))
        refused(A, kvr.kvr_attention_packed, *att(d(P, 128, [1]), o=Q + 1))
        refused(R, kvr.kvr_append_packed, *app(d(P, 128, [-1])))
        refused(A, kvr.kvr_append_packed, *app(d(P, 128, [4, 4])))
        refused(R, kvr.kvr_append_packed, *app(d(P, 128, [4]), st=127))
        refused(A, kvr.kvr_append_packed, *app(d(P, 128, [4]), k=None))
        refused(A, kvr.kvr_append_packed, *app(kvr.make_packed_rows([(P, 64, [4]), (P, 64, [5])])))
        tok = torch.zeros(128, dtype=torch.int32, device="cuda").data_ptr()
        refused(U, kvr.kvr_prefill_packed, c.ctx, tok, 10, 128, P, 3, None, s)
        refused(R, kvr.kvr_prefill_packed, c.ctx, tok, 10, 129, P, 4, None, s)
        refused(U, kvr.kvr_repair_packed, c.ctx, [], 0, s)
        refused(A, kvr.kvr_score_packed, c.ctx, P + 2, 4, 5, 128, tok, 1, None, None, s)
        refused(R, kvr.kvr_generate_packed, c.ctx, P, 4, 120, 128, tok, 5, 10, s)
        torch.cuda.synchronize()
        assert torch.equal(p, keep)
