"""The order between ordinary stores to shared memory and asynchronous copies over the same bytes: read from the sources, since a
violation would be a race on the device."""
import re

from tests.test_launch_rules import _body, _sources


def test_what_a_join_copies_by_hand_is_fenced_before_the_slots_next_row():
    """A slot of the ring is filled by bulk copies, but a row's pieces that reach over its tensor's ends by ordinary stores: the thread
    that made them fences them, on every way out, before it reports the row."""
    text = _sources()["qbp_resnorm.cuh"]
    body = _body(text, text.index("void join_copy_from_before("))
    stores = [m.start() for m in re.finditer(r"\*reinterpret_cast<T \*>\(section", body)]
    assert len(stores) == 2
    after = body[stores[-1]:]
    fence = after.index("fence_proxy_async();")
    assert after.index(";") < fence < after.index("return") and "bulk_load" not in after[:fence]
    assert "return" not in body[:stores[-1]]
    # the row is reported behind the copies of every tensor
    copy = _body(text, text.index("void join_copy("))
    assert copy.rindex("join_copy_from_before") < copy.index("mbar_arrive(full)")
