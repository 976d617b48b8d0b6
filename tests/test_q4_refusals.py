"""What the calls on a 4-bit cache refuse, before anything reaches the GPU."""
import ctypes

import pytest
import torch

import paper_2412_00061_amd as pkg
from host_context import HostContext
from paper_2412_00061_amd import binding

P = 4096  # an address, 16-byte aligned: never read on the host
INVALID, UNSUPPORTED = -1, -2


def cache(k_codes=P, k_scales=P, v_codes=P, v_scales=P):
    return ctypes.byref(binding._Q4Cache(k_codes, k_scales, v_codes, v_scales))


APPEND = dict(dt=1, k=P, v=P, n=P, max_rows=10, cache=cache(), off=P, ctx=P, cap=100, B=2, H=4, dh=64, out=None)
COMMIT = dict(dt=1, k=P, v=P, alen=P, path=P, T=4, cache=cache(), off=P, ctx=P, cap=100, B=2, H=4, dh=64, N=20, out=None)
READ = dict(cache=cache(), off=P, first=P, n=P, max_rows=10, cap=100, B=2, H=4, dh=64, dt=1, k=P, v=P)
ATTN = dict(dt=1, q=P, cache=cache(), off=P, ctx=P, cap=100, k=P, v=P, n=P, depth=P, mask=P, B=2, H=4, Hkv=2, dh=64, N=20, scale=0.125, window=9, sink=2,
            ws=P, ws_bytes=1 << 40, out_dt=0, out=P, lse=P)
CALLS = {"kv_append_q4": APPEND, "kv_commit_q4": COMMIT, "kv_read_q4": READ}

BAD = [(name, key, None, INVALID, "null pointer") for name, args in CALLS.items() for key in args
       if key in ("k", "v", "n", "alen", "path", "cache", "off", "ctx", "first")]
BAD += [(name, "cache", cache(**{part: None}), INVALID, "null pointer") for name in CALLS for part in ("k_codes", "k_scales", "v_codes", "v_scales")]
BAD += [(name, key, value, INVALID, "positive") for name, args in CALLS.items() for key in ("B", "H", "dh", "cap", "max_rows", "N", "T") if key in args
        for value in (0, -3)]
BAD += [(name, "dt", 2, INVALID, "element type") for name in CALLS]
BAD += [(name, "dh", value, UNSUPPORTED, "multiple of 8") for name in CALLS for value in (12, 136)]
BAD += [(name, key, value, UNSUPPORTED, "limits") for name, args in CALLS.items()
        for key, value in (("B", 9), ("H", 9), ("dh", 128), ("cap", (1 << 30) + 1), ("max_rows", (1 << 30) + 1), ("N", 65)) if key in args]
BAD += [(name, key, P + 8, INVALID, "aligned") for name in CALLS for key in ("k", "v")]
BAD += [(name, "cache", cache(**{part: P + 4}), INVALID, "aligned") for name in CALLS for part in ("k_codes", "v_codes")]
BAD += [(name, "cache", cache(**{part: P + 2}), INVALID, "4-byte") for name in [*CALLS, "q4_verify_attn"] for part in ("k_scales", "v_scales")]
BAD += [(name, "max_rows", (1 << 27) + 1, UNSUPPORTED, "2^27") for name in ("kv_append_q4", "kv_read_q4")]
BAD += [("kv_commit_q4", "T", 9, UNSUPPORTED, "T <= 8"), ("kv_append_q4", "out", P, INVALID, "ctx_len_out"), ("kv_commit_q4", "out", P, INVALID, "ctx_len_out")]


CALLS["q4_verify_attn"] = ATTN
BAD += [("q4_verify_attn", key, None, INVALID, "null pointer") for key in ("q", "cache", "off", "ctx", "k", "v", "n", "mask", "ws", "out")]
BAD += [("q4_verify_attn", "cache", cache(**{part: None}), INVALID, "null pointer") for part in ("k_codes", "k_scales", "v_codes", "v_scales")]
BAD += [("q4_verify_attn", key, value, INVALID, "positive") for key in ("B", "H", "Hkv", "dh", "N") for value in (0, -1)] + [("q4_verify_attn", "cap", -1, INVALID, "positive")]
BAD += [("q4_verify_attn", "Hkv", 3, INVALID, "multiple of H_kv"), ("q4_verify_attn", "dt", 0, UNSUPPORTED, "bf16"), ("q4_verify_attn", "out_dt", 2, INVALID, "element type"),
        ("q4_verify_attn", "window", -1, INVALID, "negative"), ("q4_verify_attn", "sink", -1, INVALID, "negative"), ("q4_verify_attn", "depth", None, INVALID, "node_depth"),
        ("q4_verify_attn", "dh", 60, UNSUPPORTED, "multiple of 8"), ("q4_verify_attn", "dh", 136, UNSUPPORTED, "multiple of 8"), ("q4_verify_attn", "N", 129, UNSUPPORTED, "max_nodes"),
        ("q4_verify_attn", "ws_bytes", 1000, INVALID, "workspace of"), ("q4_verify_attn", "cap", (1 << 30) + 1, UNSUPPORTED, "2^30")]
BAD += [("q4_verify_attn", "scale", value, INVALID, "scale") for value in (0.0, -1.0, float("nan"), float("inf"), 3e38)]
BAD += [("q4_verify_attn", key, value, UNSUPPORTED, "limits") for key, value in (("B", 9), ("H", 10), ("dh", 128), ("N", 65))]
BAD += [("q4_verify_attn", key, P + 8, INVALID, "aligned") for key in ("q", "k", "v", "ws", "out")]
BAD += [("q4_verify_attn", "cache", cache(**{part: P + 4}), INVALID, "aligned") for part in ("k_codes", "v_codes")]


@pytest.mark.parametrize("name,key,value,code,text", BAD)
def test_refusals(name, key, value, code, text):
    args = dict(CALLS[name], **{key: value})
    HostContext(max_head_dim=64 if key == "dh" else 128).refuses(name, list(args.values()), code, text)


def test_prepared_calls_take_the_cache(monkeypatch):
    """(What is refused shows that the struct arrived: its code pointers were looked at.)"""
    ctx = HostContext()
    ctx._check = lambda rc, what: (_ for _ in ()).throw(pkg.CtcspecError(ctx.lib.ctcspec_last_error(ctx.handle).decode()))
    args = {k: v for k, v in READ.items() if k != "cache"}
    with pytest.raises(pkg.CtcspecError, match="null pointer"):
        pkg.prepared(ctx, "kv_read_q4", binding._Q4Cache(P, P, None, P), *args.values())()
    with pytest.raises(pkg.CtcspecError, match="limits"):
        pkg.prepared(ctx, "kv_read_q4", binding._Q4Cache(P, P, P, P), *dict(args, B=9).values())()


def test_no_context():
    lib = pkg.load_library()
    for name, args in CALLS.items():
        assert getattr(lib, name)(None, *args.values()) == INVALID


def test_the_binding_looks_at_shapes(monkeypatch):
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None: None if t is None else ctypes.c_void_p(t.data_ptr()))
    u8 = lambda n: torch.zeros(n, dtype=torch.uint8)  # noqa: E731
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)  # noqa: E731
    with pytest.raises(pkg.CtcspecError, match="16 bytes of codes"):
        pkg.q4_cache(u8(64), u8(4), u8(64), u8(5))
    c, off = pkg.q4_cache(u8(64), u8(4), u8(64), u8(4)), torch.zeros(2, dtype=torch.int64)
    rows = torch.zeros((2, 1, 1, 32))
    with pytest.raises(pkg.CtcspecError, match="n_rows"):
        pkg.kv_append_q4(None, rows, rows, i32(3), c, off, i32(2), 2)
    with pytest.raises(pkg.CtcspecError, match="v_rows"):
        pkg.kv_append_q4(None, rows, rows[:1], i32(2), c, off, i32(2), 2)
    with pytest.raises(pkg.CtcspecError, match="q4_cache"):
        pkg.kv_append_q4(type("C", (), {"lib": type("L", (), {"kv_append_q4": None}), "handle": None}), rows, rows, i32(2), u8(64), off, i32(2), 2)
    with pytest.raises(pkg.CtcspecError, match="accept_len"):
        pkg.kv_commit_q4(None, rows, rows, i32(1), torch.zeros((2, 5), dtype=torch.int32), c, off, i32(2), 2)
    q, mask = torch.zeros((2, 2, 1, 32)), torch.zeros((2, 1, 1), dtype=torch.int64)
    for bad, match in ((dict(k_tree=rows[:1]), "k_tree"), (dict(v_tree=rows[:1]), "v_tree"), (dict(anc_mask=mask[:1]), "anc_mask"), (dict(n_nodes=i32(1)), "n_nodes"),
                       (dict(node_depth=i32(2)), "node_depth")):
        with pytest.raises(pkg.CtcspecError, match=match):
            pkg.q4_verify_attn(None, **dict(dict(q=q, cache=c, kv_off=off, ctx_len=i32(2), kv_cap=2, k_tree=rows, v_tree=rows, n_nodes=i32(2), anc_mask=mask,
                                                 scale=1.0), **bad))
    with pytest.raises(pkg.CtcspecError, match="first"):
        pkg.kv_read_q4(None, c, off, i32(1), i32(2), 1, 2, 1, 32)
