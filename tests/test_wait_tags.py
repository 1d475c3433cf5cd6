"""A wait that runs out names its kernel: every kernel file but the attention kernel's, which says that it records no location, gives its waits a tag of
its own, and recache_poll_status has a text for each tag.  (Looked for in the sources: no kernel is made to wait for nothing here.)"""
import glob
import os
import re

from test_barrier_init import CSRC

TEXT = {os.path.basename(p): open(p).read() for p in glob.glob(os.path.join(CSRC, "*.cu*"))}
TAGS = dict(re.findall(r"constexpr uint32_t (RC_WHERE_\w+) = (\d+);", TEXT["common.cuh"]))


def test_tags_differ_and_have_texts():
    assert len(TAGS) >= 4 and len(set(TAGS.values())) == len(TAGS) and "0" not in TAGS.values()
    poll = TEXT["api.cu"][TEXT["api.cu"].index("recache_status recache_poll_status"):]
    poll = poll[:poll.index("\n}\n")]
    for tag in TAGS:
        assert re.search(r"\(w >> 28\) == " + tag + r"\)\s+snprintf\(", poll), tag


def test_each_kernel_file_has_a_tag_of_its_own():
    used = {}
    for name, text in TEXT.items():
        if name == "common.cuh":
            continue
        alias = dict(re.findall(r"constexpr uint32_t (\w+) = (RC_WHERE_\w+);", text))
        used[name] = {alias.get(t, t) for t in re.findall(r"rc_mbar_wait<\w+, (\w+)>", text)}
    used = {name: tags for name, tags in used.items() if tags}
    assert used.pop("attn_tc.cu") == {"0"} and len(used) >= 4
    for name, tags in used.items():
        assert len(tags) == 1 and tags <= set(TAGS), (name, tags)
    assert len(set.union(*used.values())) == len(used)
