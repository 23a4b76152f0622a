"""The calls of positions and windows marshalled in C hand the library what the ctypes path hands it, or leave the call to it."""
import ctypes as C
import dataclasses
import types

import pytest
import torch

import paper_2605_19218_amd as rk

B, HQ, HKV, N = 2, 8, 2, 6
vp, f32, sz, i32, u32 = C.c_void_p, C.c_float, C.c_size_t, C.c_int, C.c_uint32
PL, PT, PH, PO = C.POINTER(rk.rk_layout), C.POINTER(rk.rk_text), C.POINTER(rk.rk_heads), C.POINTER(rk.rk_rotary)
SIGNATURES = {
    "rk_rope": [vp, PL, PO, i32, vp, PH, PH, PH, PH, u32, vp],
    "rk_rope_append_text": [vp, PL, PO, i32, vp, PH, PH, PH, PH, PT, vp, vp],
    "rk_prefill_attn_window": [vp, PL, PH, i32, vp, PT, i32, i32, f32, PH, vp, sz, vp],
    "rk_decode_attn_window": [vp, PL, vp, vp, vp, vp, vp, PT, i32, i32, f32, vp, vp, sz, vp],
    "rk_decode_attn_window_quant": [vp, PL, vp, vp, vp, vp, vp, PT, i32, i32, f32, vp, vp, sz, vp],
}
DROP = object()


class OtherHeads(rk.Heads):
    pass


def tensor(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def layout(**more):
    return rk.Layout(B, HQ, HKV, 16, rk.RK_BF16, 64, 40, **{"seq_len": tensor(B, dtype=torch.int32), **more})


def text(**more):
    return rk.Text(**{"k": tensor(B, HKV, 48, 128), "v": tensor(B, HKV, 48, 128), "max_len": 33, "len": tensor(B, dtype=torch.int32), **more})


def heads(H=HKV, cls=rk.Heads, **more):
    return cls(**{"data": tensor(B, H, N, 128), **more})


def rope(axis=(0, 1, 2, 2, 0), **more):
    return rk.Rope(**{"pos": tensor(3, B, N, dtype=torch.int32), "inv_freq": tensor(5, dtype=torch.float32), "axis": axis, **more})


def call(name, lay=None, rp=None, h=None, txt=None, n=N, count=None, ints=(4, 2), flags=1, scale=0.5, kv=None, ws=None, out=None, ctx=77):
    """(positional, keywords)"""
    lay, txt, h = lay or layout(), txt or text(), h or heads()
    if name == "rk_rope":
        return [ctx, lay, rp or rope(), n, heads(HQ), heads(HQ), h, heads()], {"flags": flags, "n_tokens_dev": count}
    if name == "rk_rope_append_text":
        return [ctx, lay, rp or rope(), n, None, None, h, heads(), txt, tensor(B, dtype=torch.int32)], {"n_tokens_dev": count}
    ws = torch.empty(100) if ws is None else None if ws is DROP else ws
    if name == "rk_prefill_attn_window":
        return [ctx, lay, h, n, txt, *ints, scale, heads(HQ), ws], {"n_tokens_dev": count}
    return [ctx, lay, tensor(B, HQ, 128), kv, kv, tensor(4), None, txt, *ints, scale, tensor(B, HQ, 128), ws], {}


@pytest.fixture
def paths(monkeypatch):
    """record(name, positional, keywords, fast): the arguments that reached the entry point"""
    rk.lib()
    if rk._bind is None:
        pytest.fail("_rkbind.so is not built")
    seen, keep = [], []

    def plain(v):
        return bytes(v) if isinstance(v, C.Array) else v

    def entry(kinds):
        def f(*a):
            seen.append([[plain(getattr(x.contents, n)) for n, _ in x.contents._fields_] if kind in (PL, PT, PH, PO) and x
                         else None if kind in (PL, PT, PH, PO) else x for x, kind in zip(a, kinds)])
            return 0
        return C.CFUNCTYPE(i32, *kinds)(f)

    stub = types.SimpleNamespace()
    for name, kinds in SIGNATURES.items():
        keep.append(entry(kinds))
        keep[-1].argtypes, keep[-1].restype = kinds, i32
        setattr(stub, name, keep[-1])
    real, bind = rk.lib(), rk._bind
    bind.bind_window(rk.Heads, rk.Rope, *[C.cast(getattr(stub, n), vp).value for n in SIGNATURES])

    def record(name, args, kw, fast, through=None):
        seen.clear()
        monkeypatch.setattr(rk, "_bind", bind if fast else None)
        monkeypatch.setattr(rk, "_lib", None if fast and through is None else stub)
        if fast and through is None:                # the ctypes path must not be needed
            monkeypatch.setattr(rk, "lib", lambda: pytest.fail("the ctypes path was taken"))
        getattr(rk, name)(*args, **kw)
        monkeypatch.undo()
        assert len(seen) == 1
        return list(seen[0])

    yield record
    bind.bind_window(rk.Heads, rk.Rope, *[C.cast(getattr(real, n), vp).value for n in SIGNATURES])


@pytest.mark.parametrize("name", list(SIGNATURES))
def test_same_arguments(paths, name):
    attn = "attn" in name
    forms = [({}, {}), (dict(lay=layout(seq_len=None, head_dim=64), txt=text(len=None), rp=rope(pairing=rk.RK_ROPE_ADJACENT), scale=1), {"stream": 12345}),
             (dict(count=tensor(B, dtype=torch.int32), h=heads(strides=(5, 4, 3)), rp=rope(axis=None), n=1, flags=0), {"stream": None}),
             (dict(h=heads(data=1 << 40, strides=(16, 8, 8)), txt=text(strides=(9, 8, 7), capacity=40), count=1 << 41, kv=1 << 42, ints=(0, 0)),
              {"stream": types.SimpleNamespace(cuda_stream=321)}),
             (dict(rp=rope(pos=tensor(2, B, 9, dtype=torch.int32)[:, :, :N], axis=[1] * 64), ctx=None, ws=DROP), {"workspace_bytes": 0} if attn else {}),
             (dict(rp=rope(strides=(6, 3), n_axes=3)), {}),
             (dict(ws=1 << 40), {"workspace_bytes": 99} if attn else {})]
    for form, kw in forms:
        args, more = call(name, **form)
        assert record_both(paths, name, args, {**more, **kw})


def record_both(record, name, args, kw):
    return record(name, args, kw, True) == record(name, args, kw, False)


@pytest.mark.parametrize("name", list(SIGNATURES))
def test_other_forms_go_to_ctypes(paths, name):
    """What the C marshalling does not take arrives all the same, as by ctypes alone."""
    forms = []
    if "decode" not in name:
        forms += [dict(h=heads(cls=OtherHeads)), dict(h=heads(strides=[1, 2, 3])), dict(n=True)]
    if "rope" in name:
        forms += [dict(rp=rope(strides=[6, 3])), dict(rp=rope(n_axes=True))]
    if "append" in name or "attn" in name:
        forms += [dict(txt=text(strides=[1, 2, 3]))]
    if "attn" in name:
        forms += [dict(scale=True), dict(ints=(True, 2))]
    for form in forms:
        args, kw = call(name, **form)
        assert paths(name, args, kw, True, through="ctypes") == paths(name, args, kw, False)


def test_axes_are_bytes():
    assert rope().axis == bytes([0, 1, 2, 2, 0]) and rope(axis=None).axis == bytes(5) and rope(axis=bytes([2, 1])).axis == bytes([2, 1])
    r = dataclasses.replace(rope(), axis=[2, 1])
    assert list(r.c().axis)[:3] == [2, 1, 0] and r.c().n_pairs == 2
    for axis in ([256], [-1], [0] * 65, bytes(65)):
        with pytest.raises(ValueError):
            rope(axis=axis)


def test_what_is_made_stays():
    """Strides belong to the data they were taken from: both are given once."""
    h, r = heads(), rope()
    assert h.strides == tuple(h.data.stride()[:3]) and r.strides == tuple(r.pos.stride()[:2]) and r.n_axes == 3
    for x, name in ((h, "data"), (h, "strides"), (r, "pos"), (r, "axis")):
        with pytest.raises(dataclasses.FrozenInstanceError):
            setattr(x, name, None)
    other = dataclasses.replace(r, pos=tensor(4, B, 2 * N, dtype=torch.int32), strides=None, n_axes=None)
    assert other.strides == (2 * N * B, 2 * N) and other.n_axes == 4 and other.axis == r.axis


@pytest.mark.parametrize("name", list(SIGNATURES))
def test_an_interrupt_is_not_swallowed(paths, name):
    class Interrupted:
        def __init__(self):
            self.asked = 0

        def data_ptr(self):
            self.asked += 1
            if self.asked == 1:
                raise KeyboardInterrupt
            return 4096

    args, kw = call(name, txt=text(k=Interrupted(), strides=(9, 8, 7), capacity=40), count=Interrupted())
    with pytest.raises(KeyboardInterrupt):
        paths(name, args, kw, True)


def test_statuses():
    """Errors come out as from the ctypes path, with the library's text."""
    ctx = rk.rk_create(rk.RK_DEVICE_NONE)
    try:
        for n, status in ((N, rk.RK_ERR_NO_DEVICE), (-1, rk.RK_ERR_INVALID_ARG)):
            texts = []
            for bind in (rk._bind, None):
                old, rk._bind = rk._bind, bind
                try:
                    with pytest.raises(rk.RotateKError) as e:
                        rk.rk_rope(ctx, layout(), rope(), n, None, None, heads(data=4096, strides=(2048, 1024, 128)), heads(data=4096, strides=(2048, 1024, 128)))
                finally:
                    rk._bind = old
                assert e.value.status == status
                texts.append(str(e.value))
            assert texts[0] == texts[1]
    finally:
        rk.rk_destroy(ctx)
