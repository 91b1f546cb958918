"""The decoder over packed caches against a 64-bit decoder: kvr_prefill_packed, kvr_repair_packed, kvr_score_packed
and kvr_generate_packed, and the operators run together as a server would use them.

A code is a rounding, and the library's keys and values differ from the reference's by the rounding of its arithmetic,
so a value next to the middle of two codes may take the other one.  The reference therefore runs with the library's
own stored rows: at each layer its keys and values have to be within half a step of what the library stored (plus the
tolerance of the compared precision), and it then attends over the stored ones.
"""
import numpy as np
import pytest
import torch

import paper_2609_17983_amd as kvr
import synth
from oracle import decoder as od
from tests import packed_ref as ref
from tests.gpu_util import TOL, Engine, OracleWeights, relmax, say, to_device_weights

pytestmark = pytest.mark.gpu

MID = synth.ModelShape("mid-bf16", 2, 512, 8, 2, 128, 1024, 2048, 1e-5, 500000.0)
QBIAS = synth.ModelShape("bias-heads64", 2, 448, 7, 1, 64, 576, 512, 1e-6, 1e6, qkv_bias=True)
ODD = synth.ModelShape("odd-heads40", 2, 200, 5, 1, 40, 300, 404, 1e-5, 1e4)


def stream():
    return torch.cuda.current_stream().cuda_stream


class Packed:
    """An engine and a packed cache of arbitrary bytes."""

    def __init__(self, shape, dtype, n_cap, rows, bits, seed=0):
        tdt = torch.bfloat16 if dtype == kvr.KVR_BF16 else torch.float32
        w = synth.make_weights(shape, dtype=tdt, seed=seed)
        w["lm_head"] = synth.make_lm_head(shape, dtype=tdt, seed=seed)
        self.lm = w["lm_head"].double().numpy()
        self.shape, self.dtype, self.bits, self.n_cap = shape, dtype, bits, n_cap
        self.ow = OracleWeights(w, cache=True)
        self.eng = Engine(shape, to_device_weights(w) | {"lm_head": w["lm_head"].cuda()}, dtype, n_cap, rows)
        g = torch.Generator().manual_seed(seed)
        self.cache = torch.randint(0, 256, (shape.n_layers, 2, shape.n_kv_heads, ref.blocks(n_cap),
                                            ref.block_bytes(shape.head_dim, bits)), generator=g, dtype=torch.uint8).cuda()

    def __enter__(self):
        return self

    def __exit__(self, *_):
        torch.cuda.synchronize()
        self.eng.close()

    @property
    def ctx(self):
        return self.eng.ctx

    def pack(self, plain, n):
        kvr.kvr_pack(self.ctx, kvr.make_pack_docs([(plain.data_ptr(), plain.shape[3], self.cache.data_ptr(), self.n_cap, n)]),
                     self.bits, stream())

    def bytes(self):
        torch.cuda.synchronize()
        return self.cache.cpu().numpy()

    def decode(self, packed, n):
        """(values, scales) [L][2][Hkv][n][hd] of a packed cache's positions [0, n)."""
        v, s = [], []
        for l in range(self.shape.n_layers):
            for kv in range(2):
                c, sc, m = ref.read(packed[l, kv], n, self.shape.head_dim, self.bits, kv == 1)
                v.append(ref.values(c, sc, m))
                s.append(sc[..., np.arange(self.shape.head_dim) // 64].astype(np.float64))
        full = (self.shape.n_layers, 2, *v[0].shape)
        return np.stack(v).reshape(full), np.stack(s).reshape(full)


def check_pass(p, before, after, tokens, P, n, tag):
    """The rows P of one pass: `after` holds stored rows within half a step of the reference's, every other row's bytes are
    `before`'s.  Returns the reference's final-norm rows."""
    shape, tol = p.shape, TOL[p.dtype]
    P = np.asarray(P, np.int64)
    cache, scale = p.decode(after, n)
    old, _ = p.decode(before, n)
    keep = np.setdiff1d(np.arange(n), P)
    assert np.array_equal(cache[:, :, :, keep], old[:, :, :, keep], equal_nan=True), tag
    h = p.ow.embed_rows(np.asarray(tokens, np.int64)[P])
    for l in range(shape.n_layers):
        w = p.ow.layer(l)
        x = od.rms_norm(h, w["attn_norm"], shape.rms_eps)
        q, k, v = x @ w["wq"].T, x @ w["wk"].T, x @ w["wv"].T
        if w.get("bq") is not None:
            q, k, v = q + w["bq"], k + w["bk"], v + w["bv"]
        R, hd = len(P), shape.head_dim
        q = od.rope(q.reshape(R, shape.n_heads, hd), P, shape.rope_theta)
        k = od.rope(k.reshape(R, shape.n_kv_heads, hd), P, shape.rope_theta)
        for kv, fresh in ((0, k), (1, v.reshape(R, shape.n_kv_heads, hd))):
            fresh = fresh.transpose(1, 0, 2)
            off = np.abs(cache[l, kv][:, P] - fresh)
            # half a step (and its fp32 roundings), and the pass's own error; the offset and the scale move with it
            room = 0.5001 * scale[l, kv][:, P] + 2 * tol * np.abs(fresh).max()
            assert (off <= room).all(), (tag, l, kv, float((off / room).max()))
        o = od.attend(q, P, cache[l, 0], cache[l, 1]).reshape(R, -1)
        h = h + o @ w["wo"].T
        x = od.rms_norm(h, w["mlp_norm"], shape.rms_eps)
        h = h + (od.silu(x @ w["w_gate"].T) * (x @ w["w_up"].T)) @ w["w_down"].T
    return od.rms_norm(h, p.ow.final_norm, shape.rms_eps)


CASES = [(MID, kvr.KVR_BF16, 4), (MID, kvr.KVR_BF16, 8), (synth.TINY, kvr.KVR_F32, 4), (QBIAS, kvr.KVR_BF16, 4),
         (ODD, kvr.KVR_F32, 8), (ODD, kvr.KVR_BF16, 4)]


@pytest.mark.parametrize("shape,dtype,bits", CASES)
def test_prefill_packed(shape, dtype, bits):
    n = 150
    with Packed(shape, dtype, n + 9, 64, bits) as p:
        toks = synth.make_tokens(n, shape.vocab)
        before = p.bytes().copy()
        hidden = torch.zeros((n, shape.d_model), device="cuda")
        dev = toks.cuda()
        kvr.kvr_prefill_packed(p.ctx, dev.data_ptr(), n, n + 9, p.cache.data_ptr(), bits, hidden.data_ptr(), stream())
        after = p.bytes()
        y = check_pass(p, before, after, toks.numpy(), range(n), n + 9, "prefill")
        e = relmax(hidden.cpu().numpy(), y)
        say(f"prefill {shape.name} {bits} bits: hidden {e:.2e}")
        assert e <= TOL[dtype]


def test_prefill_packed_with_many_heads():
    """Enough columns for the attention kernel for many rows, with the decoder's compensated queries."""
    n, shape = 300, synth.ModelShape("many-heads", 1, 256, 256, 16, 128, 320, 512, 1e-5, 1e5)
    with Packed(shape, kvr.KVR_BF16, n + 9, n, 4) as p:
        toks = synth.make_tokens(n, shape.vocab)
        before = p.bytes().copy()
        hidden = torch.zeros((n, shape.d_model), device="cuda")
        dev = toks.cuda()
        kvr.kvr_prefill_packed(p.ctx, dev.data_ptr(), n, n + 9, p.cache.data_ptr(), 4, hidden.data_ptr(), stream())
        y = check_pass(p, before, p.bytes(), toks.numpy(), range(n), n + 9, "prefill")
        e = relmax(hidden.cpu().numpy(), y)
        say(f"prefill {shape.name}: hidden {e:.2e}")
        assert e <= TOL[kvr.KVR_BF16]


@pytest.mark.parametrize("shape,dtype,bits", CASES)
@pytest.mark.parametrize("span,K", [(8, 24), (3, 0), (16, 130)])
def test_repair_packed(shape, dtype, bits, span, K):
    """A cache goes to rest, is edited, and its packed rows are repaired in place; scattered and consecutive rows."""
    n, s0 = 260, 70
    with Packed(shape, dtype, n, 200, bits) as p:
        tdt = p.eng.tdtype
        plain = synth.make_stale_cache(shape, n, dtype=tdt).cuda()
        p.pack(plain, n)
        before = p.bytes().copy()
        toks = synth.apply_edit(synth.make_tokens(n, shape.vocab), s0, span, shape.vocab)
        A = kvr.kvr_select(kvr.KVR_RANDOM, n, s0, s0 + span, K, 3)
        P = sorted(set(range(s0, s0 + span)) | set(A))
        hidden = torch.zeros((len(P), shape.d_model), device="cuda")
        dev = toks.cuda()
        doc = kvr.make_doc(p.cache.data_ptr(), n, n, dev.data_ptr(), s0, s0 + span, A, hidden.data_ptr())
        kvr.kvr_repair_packed(p.ctx, [doc], bits, stream())
        y = check_pass(p, before, p.bytes(), toks.numpy(), P, n, "repair")
        e = relmax(hidden.cpu().numpy(), y)
        say(f"repair {shape.name} {bits} bits: hidden {e:.2e}")
        assert e <= TOL[dtype]


def test_repair_packed_of_several_documents():
    """One call over documents equals a call for each, bit for bit in what is stored."""
    shape, bits = MID, 4
    ns = [100, 33, 260]
    caches, hid = [], []
    with Packed(shape, kvr.KVR_BF16, 260, 200, bits) as p:
        plain = [synth.make_stale_cache(shape, n, label=n).cuda() for n in ns]
        toks = [synth.make_tokens(n, shape.vocab, seed=n).cuda() for n in ns]
        size = [kvr.kvr_packed_bytes(p.eng.dims, n, bits) for n in ns]
        for together in (True, False):
            packed = [torch.zeros(z, dtype=torch.uint8, device="cuda") for z in size]
            kvr.kvr_pack(p.ctx, kvr.make_pack_docs([(a.data_ptr(), n, b.data_ptr(), n, n) for a, b, n in zip(plain, packed, ns)]),
                         bits, stream())
            hidden = [torch.zeros((12, shape.d_model), device="cuda") for _ in ns]
            docs = [kvr.make_doc(b.data_ptr(), n, n, t.data_ptr(), n // 2, n // 2 + 4, list(range(n - 9, n - 1)), h.data_ptr())
                    for b, n, t, h in zip(packed, ns, toks, hidden)]
            if together:
                kvr.kvr_repair_packed(p.ctx, docs, bits, stream())
            else:
                for d in docs:
                    kvr.kvr_repair_packed(p.ctx, [d], bits, stream())
            torch.cuda.synchronize()
            caches.append([b.cpu() for b in packed])
            hid.append([h.cpu() for h in hidden])
        for i, n in enumerate(ns):
            assert relmax(hid[0][i].numpy(), hid[1][i].numpy()) <= TOL[kvr.KVR_BF16]
        with pytest.raises(kvr.KvrError) as e:
            kvr.kvr_repair_packed(p.ctx, [docs[0], docs[0]], bits, stream())
        assert e.value.status == kvr.KVR_E_ARG


@pytest.mark.parametrize("shape,dtype,bits", CASES)
def test_score_and_generate_packed(shape, dtype, bits):
    n, m, new = 200, 20, 6
    n_cap = n + m + new
    with Packed(shape, dtype, n_cap, 64, bits) as p:
        plain = synth.make_stale_cache(shape, n, dtype=p.eng.tdtype).cuda()
        p.pack(plain, n)
        toks = torch.zeros(n_cap, dtype=torch.int32)
        toks[:n + m] = synth.make_tokens(n + m, shape.vocab)
        dev = toks.cuda()
        before = p.bytes().copy()
        lp = torch.zeros(m, device="cuda")
        best = torch.zeros(m, dtype=torch.int32, device="cuda")
        kvr.kvr_score_packed(p.ctx, p.cache.data_ptr(), bits, n, n_cap, dev.data_ptr(), m, lp.data_ptr(), best.data_ptr(), stream())
        after = p.bytes().copy()
        y = check_pass(p, before, after, toks.numpy(), range(n, n + m), n_cap, "score")
        logits = y @ p.lm.T
        logits -= logits.max(-1, keepdims=True)
        want = logits - np.log(np.exp(logits).sum(-1, keepdims=True))
        want = want[np.arange(m - 1), toks.numpy()[n + 1:n + m]]
        e = relmax(lp[:m - 1].cpu().numpy(), want)
        say(f"score {shape.name} {bits} bits: {e:.2e}")
        assert e <= TOL[dtype]
        # the continuation: each step's pass is the reference's, with the tokens that the library chose
        kvr.kvr_generate_packed(p.ctx, p.cache.data_ptr(), bits, n, n_cap, dev.data_ptr(), m, new, stream())
        end = p.bytes()
        got = dev.cpu().numpy()
        assert np.array_equal(got[:n + m], toks.numpy()[:n + m])
        check_pass(p, after, end, got, range(n, n + m + new - 1), n_cap, "generate")
        top2 = np.sort(logits[-1])[-2:]
        if top2[1] - top2[0] > 2 * TOL[dtype] * np.abs(logits).max():
            assert got[n + m] == int(np.argmax(logits[-1]))


def test_generate_packed_captured():
    """A captured generation, replayed with other calls of the context in between, writes what an eager one does."""
    shape, bits, n, q, new = MID, 4, 120, 5, 8
    n_cap = n + q + new
    with Packed(shape, kvr.KVR_BF16, n_cap, 64, bits) as p:
        plain = synth.make_stale_cache(shape, n).cuda()
        p.pack(plain, n)
        torch.cuda.synchronize()
        start = p.cache.clone()
        toks = torch.zeros(n_cap, dtype=torch.int32, device="cuda")
        toks[:n + q] = synth.make_tokens(n + q, shape.vocab).cuda()
        first = toks.clone()
        run = lambda: kvr.kvr_generate_packed(p.ctx, p.cache.data_ptr(), bits, n, n_cap, toks.data_ptr(), q, new,  # noqa: E731
                                              torch.cuda.current_stream().cuda_stream)
        run()
        torch.cuda.synchronize()
        want, kept = toks.clone(), p.cache.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        other = start.clone()
        for _ in range(3):
            toks.copy_(first)
            p.cache.copy_(start)
            doc = kvr.make_doc(other.data_ptr(), n, n_cap, first.data_ptr(), 4, 9, [30, 31], None)
            kvr.kvr_repair_packed(p.ctx, [doc], bits, stream())
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(toks, want) and torch.equal(p.cache, kept)


def test_operators_together():
    """A server's round: prefill, rest, a token's rows appended and attended layer by layer, an edit repaired in the
    unpacked cache, the repaired positions packed again."""
    shape, bits, n = MID, 4, 180
    with Packed(shape, kvr.KVR_BF16, n + 8, 64, bits) as p:
        toks = synth.make_tokens(n, shape.vocab)
        dev = toks.cuda()
        plain = p.eng.new_cache(n)
        kvr.kvr_prefill(p.ctx, dev.data_ptr(), n, n, plain.data_ptr(), None, stream())
        p.pack(plain, n)
        before = p.bytes().copy()
        # one token's projections for both layers (as a program with layers of its own would have them)
        Hq, Hkv, hd = shape.n_heads, shape.n_kv_heads, shape.head_dim
        g = torch.Generator().manual_seed(5)
        fused = torch.randn((2, (Hq + 2 * Hkv) * hd), generator=g).bfloat16()
        f = fused.cuda()
        out = torch.zeros((2, Hq * hd), dtype=torch.bfloat16, device="cuda")
        row = kvr.make_packed_rows([(p.cache.data_ptr(), n + 8, [n])])
        for l in range(2):
            at = f.data_ptr() + l * f.shape[1] * 2
            kvr.kvr_append_packed(p.ctx, l, bits, row, at + Hq * hd * 2, at + (Hq + Hkv) * hd * 2, f.shape[1], stream())
            kvr.kvr_attention_packed(p.ctx, l, bits, row, at, f.shape[1], out.data_ptr() + l * Hq * hd * 2, Hq * hd, stream())
        after = p.bytes().copy()
        want = before.copy()
        x = fused.float().numpy()
        half = torch.finfo(torch.bfloat16).eps / 2
        for l in range(2):
            dec = []
            for kv in range(2):
                rows = x[l, (Hq + kv * Hkv) * hd:(Hq + (kv + 1) * Hkv) * hd].reshape(Hkv, 1, hd)
                ref.write(want[l, kv], rows, [n], bits, kv == 1)
                dec.append(ref.read(want[l, kv], n + 1, hd, bits, kv == 1))
            q = x[l:l + 1, :Hq * hd].reshape(1, Hq, hd)
            y = ref.attend(q, [n], ref.values(*dec[0]), ref.values(*dec[1]))
            tol = ref.attend_bound(q, [n], dec[0], dec[1], bits, False)[..., None] * (1 + half) + half * np.abs(y)
            assert (np.abs(out[l].cpu().float().numpy().reshape(1, Hq, hd) - y) <= tol).all()
        assert np.array_equal(after, want)
        # an edit: the cache is read back, repaired, and the repaired positions return to the packed cache
        new = synth.apply_edit(toks, 50, 4, shape.vocab)
        nd = new.cuda()
        doc = lambda pos: kvr.make_pack_docs([(plain.data_ptr(), n, p.cache.data_ptr(), n + 8, pos)])  # noqa: E731
        kvr.kvr_unpack(p.ctx, doc(n), bits, stream())
        A = kvr.kvr_select(kvr.KVR_EDIT_LOCAL, n, 50, 54, 20)
        kvr.kvr_repair(p.ctx, [kvr.make_doc(plain.data_ptr(), n, n, nd.data_ptr(), 50, 54, A, None)], stream())
        P = sorted(set(range(50, 54)) | set(A))
        kvr.kvr_pack(p.ctx, doc(P), bits, stream())
        end = p.bytes()
        host = plain.float().cpu().numpy()
        for l in range(2):
            for kv in range(2):
                ref.write(want[l, kv], host[l, kv][:, P], P, bits, kv == 1)
        assert np.array_equal(end, want)
