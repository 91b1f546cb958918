"""The reference of packed caches holds to the format's statements, and the library's
sizes and refusals that need no GPU."""
import ctypes

import numpy as np
import pytest

import paper_2609_17983_amd as kvr
from tests import packed_ref as ref


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("hd", [2, 40, 64, 96, 128])
@pytest.mark.parametrize("value", [False, True])
def test_layout_is_a_bijection(bits, hd, value):
    seen = set()
    for r in range(32):
        for d in range(hd):
            byte, bit = ref.code_place(hd, bits, value, r, d)
            assert 0 <= byte < 4 * ref.width(hd) * bits and bit + bits <= 8
            seen.add((byte, bit))
    assert len(seen) == 32 * hd


@pytest.mark.parametrize("bits", [4, 8])
def test_quantise_is_off_by_half_a_step(bits):
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((500, 96)) * np.exp(rng.uniform(-8, 8, (500, 1)))).astype(np.float32)
    c, s, m = ref.quantise(x, bits)
    g = np.arange(96) // 64
    # half a step, and the fp32 roundings of the difference, the reciprocal and the product (2^-24 each of at most 2^bits)
    err = np.abs(ref.values(c, s, m) - x)
    assert (err <= s[..., g].astype(np.float64) * (0.5 + 3 * 2.0 ** (bits - 24))).all()
    assert (m <= np.stack([x[:, :64].min(1), x[:, 64:].min(1)], 1)).all()
    assert c.max() == (1 << bits) - 1 and c.min() == 0


@pytest.mark.parametrize("bits", [4, 8])
def test_quantise_edges(bits):
    x = np.zeros((7, 64), np.float32)
    x[1] = 3.25                      # one value: held exactly, as bf16 holds it
    x[2, 5] = np.inf
    x[3, 0] = np.nan
    x[4, 0], x[4, 1] = 3e38, -3e38   # the range overflows
    x[5, 3] = 1e-40                  # a scale below the normal numbers
    x[6] = np.linspace(-1, 1, 64)
    c, s, m = ref.quantise(x, bits)
    v = ref.values(c, s, m)
    assert (v[0] == 0).all() and (v[1] == 3.25).all()
    assert np.isnan(v[2]).all() and np.isnan(v[3]).all() and np.isnan(v[4]).all()
    assert s[5, 0] == np.float32(2.0 ** -126) and (v[5] == 0).all()
    assert np.isfinite(v[6]).all()


def test_write_read_round_trip():
    rng = np.random.default_rng(1)
    for bits in (4, 8):
        for hd in (40, 128):
            packed = rng.integers(0, 256, (2, 2, ref.block_bytes(hd, bits)), dtype=np.uint8)
            before = packed.copy()
            rows = rng.standard_normal((2, 3, hd)).astype(np.float32)
            for value in (False, True):
                ref.write(packed, rows, [1, 31, 40], bits, value)
                got = ref.read(packed, 64, hd, bits, value)
                want = ref.quantise(rows, bits)
                for a, b in zip(got, want):
                    assert np.array_equal(a[:, [1, 31, 40]], b)
                old = ref.read(before, 64, hd, bits, value)
                keep = [p for p in range(64) if p not in (1, 31, 40)]
                assert np.array_equal(got[0][:, keep], old[0][:, keep])
                packed = before.copy()


def _dims(**kw):
    base = dict(n_layers=3, d_model=256, n_heads=4, n_kv_heads=2, head_dim=128, d_ffn=64, vocab=64, qkv_bias=0,
                rms_eps=1e-5, rope_theta=10000.0, max_ctx=512, max_rows=64, dtype=kvr.KVR_BF16)
    base.update(kw)
    return kvr.kvr_dims(**base)


@pytest.mark.parametrize("hd", [2, 40, 64, 66, 96, 128])
@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("n_cap", [0, 1, 32, 33, 8192])
def test_packed_bytes(hd, bits, n_cap):
    assert kvr.kvr_packed_bytes(_dims(head_dim=hd), n_cap, bits) == 3 * 2 * 2 * ref.blocks(n_cap) * ref.block_bytes(hd, bits)


def test_packed_bytes_refusals():
    assert kvr.kvr_packed_bytes(_dims(), 32, 5) == 0
    assert kvr.kvr_packed_bytes(_dims(), -1, 4) == 0
    assert kvr.kvr_packed_bytes(_dims(), 2 ** 30, 4) > 2 ** 30
    assert kvr.kvr_packed_bytes(_dims(), 2 ** 30 + 1, 4) == 0
    assert kvr.kvr_packed_bytes(_dims(), 2 ** 31 - 1, 4) == 0
    assert kvr.kvr_packed_bytes(_dims(head_dim=256), 32, 4) == 0
    assert kvr.load().kvr_packed_bytes(None, 32, 4) == 0


def test_null_context_is_refused():
    lib = kvr.load()
    assert lib.kvr_pack(None, None, 0, 4, None) == kvr.KVR_E_ARG
    assert lib.kvr_unpack(None, None, 0, 4, None) == kvr.KVR_E_ARG
    assert lib.kvr_append_packed(None, 0, 4, None, 0, None, None, 0, None) == kvr.KVR_E_ARG
    assert lib.kvr_attention_packed(None, 0, 4, None, 0, None, 0, None, 0, None) == kvr.KVR_E_ARG
    assert lib.kvr_prefill_packed(None, None, 1, 1, None, 4, None, None) == kvr.KVR_E_ARG
    assert lib.kvr_repair_packed(None, None, 0, 4, None) == kvr.KVR_E_ARG
    assert lib.kvr_score_packed(None, None, 4, 1, 1, None, 1, None, None, None) == kvr.KVR_E_ARG
    assert lib.kvr_generate_packed(None, None, 4, 1, 1, None, 1, 1, None) == kvr.KVR_E_ARG
    assert "kvr_generate_packed" in kvr.kvr_last_error(None)


def test_document_lists():
    docs = kvr.make_pack_docs([(4096, 10, 8192, 12, 7), (4096, 10, 8192, 12, [1, 5])])
    assert docs._count == 2 and docs[0].n_positions == 7 and not docs[0].h_positions
    assert docs[1].n_positions == 2 and list(docs[1].h_positions[:2]) == [1, 5]
    rows = kvr.make_packed_rows([(4096, 10, [3]), (8192, 20, [])])
    assert rows._count == 2 and rows[0].h_positions[0] == 3 and rows[1].n_rows == 0
    assert ctypes.sizeof(kvr.kvr_packed_rows) == 32 and ctypes.sizeof(kvr.kvr_pack_doc) == 48
