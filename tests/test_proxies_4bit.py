"""A slot of shared memory that the step's token was stored into is refilled by a bulk copy
(cp.async.bulk, which writes through the async proxy) only behind a proxy fence of every lane,
read in the source: no run shows a breach reliably."""
import os
import re

from helpers import ROOT

SOURCE = os.path.join(ROOT, "paper_2608_10139_gb300", "csrc", "decode_q4.cu")


def _kernels():
    src = re.sub(r"//[^\n]*", "", open(SOURCE).read())
    return dict(re.findall(r"__global__[^;{]*?\b(k_\w+)\s*\([^{]*\)\s*\{(.*?)\n\}", src, flags=re.S))


def test_slots_are_fenced_before_a_bulk_copy_refills_them():
    bodies = {k: b for k, b in _kernels().items() if "append<" in b}
    assert set(bodies) == {"k_decode_q4_stream", "k_decode_q4_split"}
    for body in bodies.values():
        assert body.count("append<") == 1
        after = body[body.index("append<"):]
        refill = after[:after.index("produce()")]
        # the fence of whoever stored, then all lanes, and nothing that stores into a slot between
        assert re.search(r"if \((?:x\.)?info & kAppend\) fence_proxy_async_smem\(\);\s*__syncwarp\(\);\s*$", refill)
        assert not re.search(r"\bissue\(|\bbulk_copy", refill)


def test_a_slot_is_refilled_only_once_it_is_used_up():
    for body in _kernels().values():
        if "ring.wait()" not in body:
            continue
        loop = body[body.index("ring.wait()"):]
        assert loop.index("at.tile(") < loop.index("++ring.got;") < loop.index("produce()")


def test_heads_that_no_wait_orders_are_read_behind_a_barrier():
    """Lane 0 stores an entry's head; the others read it behind their wait for that entry's copies, or, where
    they have not waited for it (the first, the one ahead), behind a barrier of the warp."""
    body = _kernels()["k_decode_q4_stream"]
    reads = [m.start() for m in re.finditer(r"ring\.head\(", body)]
    assert len(reads) == 3
    first, waited, ahead = (body[:at] for at in reads)
    assert re.search(r"__syncwarp\(\);\s*if \(ring\.more\(\)\) fetch\($", first)
    assert re.search(r"if \(!ring\.wait\(\)\) return;\s*const Head4 x = $", waited)
    assert re.search(r"\{\s*__syncwarp\(\);\s*fetch\($", ahead) and body[reads[2]:].startswith("ring.head(1)")
    split = _kernels()["k_decode_q4_split"]
    assert len(re.findall(r"ring\.head\(", split)) == 1
    assert re.search(r"if \(!ring\.wait\(\)\) break;\s*const int info = ring\.head\(\)", split)
