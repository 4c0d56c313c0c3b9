"""The order in which a part of a split tile is published (decode kernel of the paged attention). The
kernel's memory order cannot be observed from a test on the GPU, where a warp that happens to run in
step hides a missing barrier, so the steps are read off the source: every lane's stores, a device fence
by every lane, the warp together, one lane's word; then every lane's look at the other words behind a
fence, and a fence before what they stand for is read."""
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_20538_gb300", "csrc", "cg_paged_attn.cu")


def _body(name):
    text = re.sub(r"//[^\n]*", "", open(SRC).read())
    at = text.index("{", re.search(r"\b%s\([^;{]*\)\s*\{" % name, text).start())
    depth = 0
    for i in range(at, len(text)):
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        if not depth:
            return text[at:i]


def test_a_part_is_published_by_the_whole_warp():
    steps = re.findall(r"__threadfence\(\)|__syncwarp\(\)|\[mine\] = epoch|== epoch|__all_sync|= 0ull", _body("all_written"))
    assert steps == ["__threadfence()", "__syncwarp()", "[mine] = epoch", "__syncwarp()", "__threadfence()", "== epoch",
                     "__threadfence()", "__all_sync", "= 0ull"]
