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


@pytest.mark.parametrize("rows", [1, 48])
def test_key_ranges_are_for_the_contexts_device(rows):
    """Which device a process asked first has no say in another device's plans."""
    body = """
    host.host_units(1, 32)
    grids = []
    for device in %s:
        host.hipSetDevice(device)
        c = context(dims(max_ctx=8000))
        host.hipSetDevice(0)  # (a call works on its context's device)
        grids.append(attend(c, 4, [(8000, list(range(8000 - %d, 8000)))])[0]["grid"])
    result = grids
    """
    both, one, other = (run(body % (devices, rows)) for devices in ((0, 1), (0,), (1,)))
    assert both == one + other and one != other
