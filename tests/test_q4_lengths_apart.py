"""kv_append_q4 and kv_commit_q4 write the new lengths while other workgroups still read counts and places: into buffers of their own only."""
import pytest

from host_context import HostContext
from test_q4_refusals import APPEND, COMMIT, INVALID

FAR = 8192  # another address: never read on the host


@pytest.mark.parametrize("name,args,key", [("kv_append_q4", APPEND, "n"), ("kv_commit_q4", COMMIT, "alen"), ("kv_commit_q4", COMMIT, "path"),
                                           ("kv_append_q4", APPEND, "ctx"), ("kv_commit_q4", COMMIT, "ctx")])
def test_new_lengths_over_what_is_still_read_are_refused(name, args, key):
    HostContext().refuses(name, list(dict(args, **{key: FAR, "out": FAR}).values()), INVALID, "ctx_len_out")
