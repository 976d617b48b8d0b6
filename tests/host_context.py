"""A context in host memory, for what the calls refuse before they reach the GPU: the fields that the checks read (the stream, the
device, the limits), the error text, and nothing else."""
import ctypes

import paper_2412_00061_amd as pkg
from paper_2412_00061_amd import binding


class _Head(ctypes.Structure):
    _fields_ = [("stream", ctypes.c_void_p), ("device", ctypes.c_int), ("lim", binding._Limits), ("err", ctypes.c_char * 256),
                ("rest", ctypes.c_char * 4096)]


class HostContext:
    def __init__(self, **limits):
        lim = dict(max_batch=8, max_slots=4, max_topk=1, max_vocab_rows=64, max_nodes=64, max_heads=8, max_head_dim=128)
        lim.update(limits)
        self.lib = pkg.load_library()
        self.head = _Head(lim=binding._Limits(**lim))
        self.handle = ctypes.c_void_p(ctypes.addressof(self.head))

    def refuses(self, name, args, code, text):
        """The call returns `code` and says `text`; nothing is launched."""
        self.head.err = b""
        rc = getattr(self.lib, name)(self.handle, *args)
        said = self.lib.ctcspec_last_error(self.handle).decode()
        assert rc == code and text in said, (name, rc, said)
