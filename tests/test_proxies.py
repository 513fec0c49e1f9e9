"""Shared memory that ordinary stores or cp.async wrote is refilled by a bulk copy
(cp.async.bulk, which writes through the async proxy) only behind a proxy fence,
read in the sources: no run shows a breach reliably."""
import os
import re

from helpers import ROOT

SOURCE = os.path.join(ROOT, "paper_2608_10139_gb300", "csrc", "decode_q8.cu")


def _code():
    return re.sub(r"//[^\n]*", "", open(SOURCE).read())


def _kernels(src):
    return dict(re.findall(r"__global__[^;{]*?\b(k_\w+)\s*\([^{]*\)\s*\{(.*?)\n\}", src, flags=re.S))


def test_rows_slots_are_fenced_before_a_bulk_copy_refills_them():
    src = _code()
    m = re.search(r"void rows_used\(\) \{(.*?)\n  \}", src, flags=re.S)
    assert m and re.fullmatch(r"\s*fence_proxy_async_smem\(\);\s*__syncwarp\(\);", m.group(1))
    bodies = {k: b for k, b in _kernels(src).items() if "open_block<" in b}
    assert set(bodies) == {"k_decode_q8_stream", "k_decode_q8_split"}
    # whoever goes on to refill slots after the open block (its rows stood in two of them) fences first
    for body in bodies.values():
        after = body[body.rindex("open_block<"):]
        refill = re.search(r"\bproduce\(\)|\bissue_tile\(|\bbulk_copy_g2s\(", after)
        if refill:
            assert "rows_used()" in after[:refill.start()]
    assert "produce()" in bodies["k_decode_q8_stream"][bodies["k_decode_q8_stream"].rindex("open_block<"):]
