"""The waits of the feed-forward products' epilogue that goes by blocks (large tile, 16-bit matrices),
when they give up: what the source does there, and a model of the barriers of the saved projections'
slots."""
import os
import re

import paper_2608_27735_gb300 as ab


def block_epilogue():
    src = open(os.path.join(os.path.dirname(ab.__file__), "csrc", "ffproduct.cuh")).read()
    start = src.index("} else if constexpr (P::kBlocks) {")
    return src[start:src.index("tma_store_done();", start)]


def test_a_wait_gives_up_for_all_lanes_of_a_warp():
    """Below the waits the lanes meet at warp barriers, some of them only where the wait did not give
    up: so all lanes take one and the same decision.  (The slots' loader is a single lane.)"""
    waits = re.findall(r"(?m)^ *ok = (.*mbar_wait.*);$", block_epilogue())
    assert len(waits) == 2 and all(w.startswith("__all_sync(~0u, ok && mbar_wait(") for w in waits)
