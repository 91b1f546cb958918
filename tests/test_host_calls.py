"""Host code of the packed calls, on the CPU: the library runs on a HIP runtime that records launches (host_runtime.py)."""
import pytest

import paper_2609_17983_amd as kvr
from tests.host_runtime import run

SHORT_OF_MEMORY = """
def outcomes(call):
    # [status, launches] with the library's k-th allocation failing, for every k until none does
    out = []
    for k in range(60):
        c = context(dims(2, 4, 2, 64, max_ctx=9000, max_rows=80))
        host.host_clear()
        host.host_fail_after(k)
        try:
            call(c)
            status = 0
        except kvr.KvrError as e:
            status = e.status
        failed = host.host_failed()
        host.host_fail_after(-1)
        out.append([status, len(launched())])
        kvr.kvr_destroy(c)
        if not failed:
            return out
"""


@pytest.mark.parametrize("call", [
    "kvr.kvr_generate_packed(c, P, 4, 10, 100, P, 3, 5)",  # five passes
    "kvr.kvr_prefill_packed(c, P, 9000, 9000, P, 4)",  # two
    "kvr.kvr_score_packed(c, P, 8, 10, 100, P, 70, P)",
    "kvr.kvr_repair_packed(c, [kvr.make_doc(P, 50, 60, P, 4, 9, [20, 22], None)], 4)",
    "kvr.kvr_attention_packed(c, 1, 4, kvr.make_packed_rows([(P, 9000, [5]), (P, 9000, list(range(0, 2000, 2)))]), P, 256, P, 256)",
    "kvr.kvr_append_packed(c, 1, 4, kvr.make_packed_rows([(P, 9000, list(range(0, 2000, 2)))]), P, P, 128)",
    "kvr.kvr_pack(c, kvr.make_pack_docs([(P, 9000, P + (1 << 30), 9000, list(range(0, 9000, 40)))]), 4)"], ids=["generate", "prefill", "score", "repair", "attention", "append", "pack"])
def test_out_of_host_memory_before_anything_is_enqueued_or_said_to_be_later(call):
    """KVR_E_NOMEM means that nothing was enqueued, whichever allocation fails."""
    *failures, last = run(SHORT_OF_MEMORY + f"result = outcomes(lambda c: {call})")
    assert last[0] == kvr.KVR_OK and last[1] > 0
    assert failures
    for status, launches in failures:
        assert (status == kvr.KVR_E_NOMEM and launches == 0) or (status == kvr.KVR_E_HIP and launches > 0)


def test_planning_again_allocates_nothing():
    """A generation's later passes plan in the memory of its first ones."""
    *failures, last = run(SHORT_OF_MEMORY + "result = outcomes(lambda c: kvr.kvr_generate_packed(c, P, 4, 10, 100, P, 3, 5))")
    assert last[0] == kvr.KVR_OK and all(launches == 0 for _, launches in failures)


def test_key_ranges_are_for_the_contexts_device():
    """Which device a process asked first has no say in another device's plans."""
    body = """
    host.host_units(1, 32)
    result = []
    for device in %s:
        host.hipSetDevice(device)
        c = context(dims(max_ctx=8000))
        host.hipSetDevice(0)  # (a call works on its context's device)
        result.append([attend(c, 4, [(8000, list(range(8000 - rows, 8000)))])[0]["grid"] for rows in (1, 48)])
    """
    both, one, other = (run(body % devices) for devices in ("(0, 1)", "(0,)", "(1,)"))
    assert both == one + other
    assert all(a != b for a, b in zip(*both))


def test_consecutive_rows_with_others_are_one_launch():
    """A prompt beside idle, repeated or further rows takes as few launches as alone."""
    alone, *rest = run("""
    c = context(dims(max_ctx=8000, max_rows=1))
    prompt = list(range(5000))
    result = [attend(c, 4, [(8000, prompt)])]
    for extra in ([7], [-1, -1], [3, 900, 40], list(range(100, 140))):
        result += [attend(c, 4, [(8000, extra + prompt)]), attend(c, 4, [(8000, prompt + extra)])]
    """)
    for launches in rest:
        assert len(launches) == len(alone) == 1 and launches[0]["name"] == alone[0]["name"]
        # (32 heads of 8, columns by 256: at most a group more for each piece)
        assert alone[0]["grid"][1] <= launches[0]["grid"][1] <= alone[0]["grid"][1] + 3


def test_scattered_rows_are_one_entry():
    """Rows that a table holds are not cut at their runs, whose last column groups would be part empty."""
    launches = run("""
    c = context(dims(max_ctx=8000, max_rows=1))
    result = attend(c, 4, [(8000, [40 * i + j for i in range(40) for j in range(13)])])
    """)
    assert len(launches) <= 2  # (a combine, if the keys are split)
    # 520 rows of four heads in groups of 32, 64 or 256 columns; by runs they were 80 or 40 groups
    assert any(launches[0]["grid"][1] % -(-520 * 4 // cols) == 0 for cols in (32, 64, 256))


def test_shapes_can_be_chosen():
    """KVR_PACKED_SHAPE, read when a context is made: each form of the kernels; other numbers have no effect."""
    got = run("""
    import os
    result = {}
    for shape in (0, 114, 118, 124, 128, 144, 148, 218, 418, 818, 814, 999, 7):
        os.environ["KVR_PACKED_SHAPE"] = str(shape)
        c = context(dims(max_ctx=4096))
        del os.environ["KVR_PACKED_SHAPE"]
        result[shape] = [attend(c, 4, [(4096, [4000])])[0], attend(c, 8, [(4096, list(range(48)))])[0]]
    """)
    for shape, launches in got.items():
        if shape in ("0", "814", "999", "7"):
            assert launches == got["0"]
            continue
        for l, bits in zip(launches, (4, 8)):
            assert l["threads"] == 64 * int(shape[2])
            kernel = "attention_packed_rows_kernel<128, %d, 1>" if shape == "818" else \
                "attention_packed_kernel<unsigned short, 128, %d, 1, " + shape[1] + ", 64>"
            assert l["name"] == kernel % bits


def test_a_repairs_rows_are_one_entry():
    """A pass has its positions in memory: its lists need no room in the launch's table, however long."""
    launches = run("""
    c = context(dims(max_ctx=4000, max_rows=1200))
    host.host_clear()
    kvr.kvr_repair_packed(c, [kvr.make_doc(P, 4000, 4000, P, 10, 605, list(range(700, 1510, 2)), None)], 4)
    result = [l for l in launched() if l["name"].startswith("attention_packed_") and "combine" not in l["name"]]
    """)
    # 1000 rows of four heads; 595 and 405 apart were 10 + 7 groups of 256 columns, 38 + 26 of 64, 75 + 51 of 32
    groups = (16,) if "rows" in launches[0]["name"] else (63, 125)
    assert len(launches) == 1 and any(launches[0]["grid"][1] % g == 0 for g in groups)


def test_profile_counts_the_launches_of_packed_passes():
    steps, launches = run("""
    c = context(dims(3, 4, 2, 64, max_ctx=4000))
    kvr.kvr_profile_enable(c, True)
    host.host_clear()
    kvr.kvr_generate_packed(c, P, 4, 3000, 4000, P, 3, 2)
    counted = kvr.kvr_profile_read(c)
    made = launched()
    kvr.kvr_attention_packed(c, 0, 4, kvr.make_packed_rows([(P, 4000, [9])]), P, 256, P, 256)  # no pass, not counted
    assert kvr.kvr_profile_read(c) == {} or not any(n for _, n in kvr.kvr_profile_read(c).values())
    result = [{k: n for k, (_, n) in counted.items()}, made]
    """)
    names = [l["name"] for l in launches]
    assert steps["attention"] == sum(n.startswith("attention_packed_kernel") for n in names) == 3 * 2
    assert steps["attention_combine"] == sum("combine" in n for n in names)
    assert steps["rope_scatter"] == sum(n.startswith("rope_pack_kernel") for n in names) == 3 * 2
