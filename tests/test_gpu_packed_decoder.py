"""The decoder over packed caches in the kernels and passes that test_gpu_packed_paths.py does not reach: every form of
attention with its compensated queries, prompts of more than one pass, more documents than a launch's table holds."""
import numpy as np
import pytest
import torch

import paper_2609_17983_amd as kvr
import synth
from tests import packed_ref as ref
from tests.gpu_util import TOL, relmax, say
from tests.test_gpu_packed_calls import SHAPES, launched
from tests.test_gpu_packed_paths import MID, QBIAS, Packed, check_pass, stream

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("model,bits", [(MID, 4), (MID, 8), (QBIAS, 4), (QBIAS, 8)])
@pytest.mark.parametrize("shape", [818, 418, 124, 144])
def test_prefill_packed_in_every_shape(model, bits, shape, monkeypatch):
    monkeypatch.setenv("KVR_PACKED_SHAPE", str(shape))
    n = 100
    with Packed(model, kvr.KVR_BF16, n + 9, 64, bits) as p:
        toks = synth.make_tokens(n, model.vocab)
        before = p.bytes().copy()
        hidden = torch.zeros((n, model.d_model), device="cuda")
        dev = toks.cuda()
        call = lambda: kvr.kvr_prefill_packed(p.ctx, dev.data_ptr(), n, n + 9, p.cache.data_ptr(), bits,  # noqa: E731
                                              hidden.data_ptr(), stream())
        call()
        y = check_pass(p, before, p.bytes(), toks.numpy(), range(n), n + 9, f"prefill {shape}")
        e = relmax(hidden.cpu().numpy(), y)
        ran = launched(call)
        say(f"prefill {model.name} {bits} bits {sorted(set(ran))}: hidden {e:.2e}")
        assert e <= TOL[kvr.KVR_BF16]
        # two pieces a query: the third template argument of both kernels
        assert {(k[0], k[2][:3], k[3]) for k in ran} == {(SHAPES[shape], (ref.width(model.head_dim), bits, 2), 64 * (shape % 10))}


@pytest.mark.parametrize("model,dtype,bits", [(synth.TINY, kvr.KVR_F32, 4), (MID, kvr.KVR_BF16, 8)])
def test_prefill_packed_of_more_than_one_pass(model, dtype, bits):
    """The rows of a second pass attend over what the first one stored."""
    n = 8192 + 70
    with Packed(model, dtype, n, 64, bits) as p:
        toks = synth.make_tokens(n, model.vocab)
        hidden = torch.zeros((n, model.d_model), device="cuda")
        dev = toks.cuda()
        kvr.kvr_prefill_packed(p.ctx, dev.data_ptr(), n, n, p.cache.data_ptr(), bits, hidden.data_ptr(), stream())
        after = p.bytes()
        rows = [0, 5, 4000, 8190, 8191, 8192, 8193, 8230, n - 1]
        y = check_pass(p, after, after, toks.numpy(), rows, n, "prefill")
        e = relmax(hidden.cpu().numpy()[rows], y)
        say(f"prefill of {n} tokens, {model.name} {bits} bits: hidden {e:.2e}")
        assert e <= TOL[dtype]


def test_repair_packed_of_more_documents_than_a_table_holds():
    """A row or three of each of 100 documents in one call."""
    bits, docs = 4, 100
    ns = [20 + i % 37 for i in range(docs)]
    with Packed(MID, kvr.KVR_BF16, 64, 200, bits) as p:
        plain = [synth.make_stale_cache(MID, n, label=n).cuda() for n in ns]
        toks = [synth.make_tokens(n, MID.vocab, seed=n).cuda() for n in ns]
        packed = [torch.zeros((MID.n_layers, 2, MID.n_kv_heads, ref.blocks(n), ref.block_bytes(MID.head_dim, bits)),
                              dtype=torch.uint8, device="cuda") for n in ns]
        kvr.kvr_pack(p.ctx, kvr.make_pack_docs([(a.data_ptr(), n, b.data_ptr(), n, n) for a, b, n in zip(plain, packed, ns)]),
                     bits, stream())
        torch.cuda.synchronize()
        before = [b.cpu().numpy().copy() for b in packed]
        lists = [[3, n - 2] if i % 2 else [] for i, n in enumerate(ns)]
        hidden = [torch.full((1 + len(l), MID.d_model), 9.0, device="cuda") for l in lists]
        call = lambda: kvr.kvr_repair_packed(  # noqa: E731
            p.ctx, [kvr.make_doc(b.data_ptr(), n, n, t.data_ptr(), n // 2, n // 2 + 1, l, h.data_ptr())
                    for b, n, t, l, h in zip(packed, ns, toks, lists, hidden)], bits, stream())
        call()
        torch.cuda.synchronize()
        for i, n in enumerate(ns):
            P = sorted([n // 2] + lists[i])
            y = check_pass(p, before[i], packed[i].cpu().numpy(), toks[i].cpu().numpy(), P, n, f"document {i}")
            assert relmax(hidden[i].cpu().numpy(), y) <= TOL[kvr.KVR_BF16], i
        assert len(launched(call)) > MID.n_layers  # more than one launch a layer


@pytest.mark.parametrize("model,dtype,bits", [(MID, kvr.KVR_BF16, 4), (synth.TINY, kvr.KVR_F32, 8)])
def test_score_and_generate_packed_from_nothing(model, dtype, bits):
    """A cache without a context, more rows than the LM head takes at once, and a continuation by one token."""
    m = 150
    with Packed(model, dtype, m + 2, 64, bits) as p:
        toks = torch.zeros(m + 2, dtype=torch.int32)
        toks[:m] = synth.make_tokens(m, model.vocab)
        dev, lp = toks.cuda(), torch.zeros(m, device="cuda")
        before = p.bytes().copy()
        kvr.kvr_score_packed(p.ctx, p.cache.data_ptr(), bits, 0, m + 2, dev.data_ptr(), m, lp.data_ptr(), None, stream())
        after = p.bytes().copy()
        logits = check_pass(p, before, after, toks.numpy(), range(m), m + 2, "score") @ p.lm.T
        want = logits - logits.max(-1, keepdims=True)
        want -= np.log(np.exp(want).sum(-1, keepdims=True))
        assert relmax(lp[:m - 1].cpu().numpy(), want[np.arange(m - 1), toks.numpy()[1:m]]) <= TOL[dtype]
        kvr.kvr_generate_packed(p.ctx, p.cache.data_ptr(), bits, 0, m + 2, dev.data_ptr(), 1, 2, stream())
        end, got = p.bytes(), dev.cpu().numpy()
        check_pass(p, after, end, got, range(2), m + 2, "generate")
