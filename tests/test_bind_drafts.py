"""The calls over 8-bit caches and of drafted tokens marshalled in C hand the library what the ctypes path hands it, or leave the call to it."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

import paper_2605_19218_amd as rk

B, HQ, HKV, T = 2, 8, 2, 6
vp, f32, sz, i32 = C.c_void_p, C.c_float, C.c_size_t, C.c_int
PL, PT, PD, PR = C.POINTER(rk.rk_layout), C.POINTER(rk.rk_text), C.POINTER(rk.rk_drafts), C.POINTER(rk.rk_rows)
SIGNATURES = {
    "rk_append_quant": [vp, PL, vp, vp, vp, vp, vp, vp, vp],
    "rk_decode_attn_quant": [vp, PL, vp, vp, vp, vp, vp, PT, f32, vp, vp, sz, vp],
    "rk_decode_attn_tree": [vp, PL, vp, vp, vp, vp, vp, PT, PD, f32, vp, vp, sz, vp],
    "rk_decode_attn_tree_quant": [vp, PL, vp, vp, vp, vp, vp, PT, PD, f32, vp, vp, sz, vp],
    "rk_append_text_path": [vp, PL, PT, PD, vp, i32, vp, vp, vp],
    "rk_compress_quant": [vp, PL, PR, vp, vp, PR, vp, vp, vp],
    "rk_unpack_cache_quant": [vp, PL, vp, vp, vp, vp, vp],
}
FAST = {"rk_append_quant": "append_quant", "rk_decode_attn_quant": "decode_quant", "rk_decode_attn_tree": "tree",
        "rk_decode_attn_tree_quant": "tree_quant", "rk_append_text_path": "append_path", "rk_compress_quant": "compress_quant",
        "rk_unpack_cache_quant": "unpack_quant"}


class OtherDrafts(rk.Drafts):
    pass


def tensor(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def layout(**more):
    return rk.Layout(B, HQ, HKV, 16, rk.RK_BF16, 64, 40, **{"seq_len": tensor(B, dtype=torch.int32), **more})


def text(**more):
    return rk.Text(tensor(B, HKV, 48, 128), tensor(B, HKV, 48, 128), 33, **{"len": tensor(B, dtype=torch.int32), **more})


def drafts(cls=rk.Drafts, **more):
    a = {"k": tensor(B, HKV, T, 128), "v": tensor(B, HKV, T, 128), "n_tokens": T, "mask": tensor(B, T, dtype=torch.int64),
         "n_tokens_dev": tensor(B, dtype=torch.int32)}
    return cls(**{**a, **more})


def rows(cls=rk.Rows, **more):
    return cls(**{"data": tensor(B, HKV, 50, 128), "n_tokens": 50, **more})


def call(name, lay=None, txt=None, d=None, ws=None, scale=0.0, kv=None, ctx=77, n=None, rw=None):
    """positional arguments of an entry point; kv: in the place of a tensor"""
    lay = lay or layout()
    t = [tensor(4, 16) for _ in range(6)]
    if kv is not None:
        t[1] = kv
    if name == "rk_append_quant":
        return [ctx, lay, *t]
    if name == "rk_unpack_cache_quant":
        return [ctx, lay, *t[:4]]
    if name == "rk_compress_quant":
        return [ctx, lay, rw or rows(), t[0], t[1], rows(n_tokens=49), *t[2:4]]
    if name == "rk_append_text_path":
        return [ctx, lay, txt, d, kv if kv is not None else tensor(B, 5, dtype=torch.int32), t[2], t[3], n]
    return [ctx, lay, *t[:5], txt, *([d] if "tree" in name else []), scale, tensor(4, 16), ws]


@pytest.fixture
def paths(monkeypatch):
    """record(name, positional, keywords, fast): the arguments that reached the entry point"""
    rk.lib()
    if rk._bind is None:
        pytest.fail("_rkbind.so is not built")
    seen, keep = [], []

    def entry(kinds):
        def f(*a):
            seen.append([[getattr(x.contents, n) for n, _ in x.contents._fields_] if kind in (PL, PT, PD, PR) and x else None if kind in (PL, PT, PD, PR)
                         else x for x, kind in zip(a, kinds)])
            return 0
        return C.CFUNCTYPE(i32, *kinds)(f)

    stub = types.SimpleNamespace()
    for name, kinds in SIGNATURES.items():
        keep.append(entry(kinds))
        keep[-1].argtypes, keep[-1].restype = kinds, i32
        setattr(stub, name, keep[-1])
    real, bind = rk.lib(), rk._bind
    bind.bind_drafts(rk.Drafts, rk.Rows, *[C.cast(getattr(stub, n), vp).value for n in SIGNATURES])

    def record(name, args, kw, fast):
        seen.clear()
        monkeypatch.setattr(rk, "_bind", bind if fast else None)
        monkeypatch.setattr(rk, "_lib", None if fast else stub)
        if fast:                                    # the ctypes path must not be needed
            monkeypatch.setattr(rk, "lib", lambda: pytest.fail("the ctypes path was taken"))
        getattr(rk, name)(*args, **kw)
        monkeypatch.undo()
        assert len(seen) == 1
        return list(seen[0])

    yield record, bind
    bind.bind_drafts(rk.Drafts, rk.Rows, *[C.cast(getattr(real, n), vp).value for n in SIGNATURES])


@pytest.mark.parametrize("name", list(SIGNATURES))
def test_same_arguments(paths, name):
    record, _ = paths
    ws = torch.empty(1000, dtype=torch.float32)
    attn = "attn" in name
    forms = [(dict(txt=text(), d=drafts(), ws=ws), {}),
             (dict(lay=layout(seq_len=None, head_dim=64), txt=text(len=None), d=drafts(mask=None, n_tokens_dev=None), ws=ws, scale=0.25), {"stream": 12345}),
             (dict(lay=layout(seq_len=1 << 47), txt=text(strides=(9, 8, 7), capacity=40), d=drafts(strides=(5, 4, 3), n_tokens=1), scale=1), {"stream": None}),
             (dict(txt=text(), d=drafts(k=1 << 40, v=(1 << 64) - 16, strides=(16, 8, 8)), ws=1 << 40), {"workspace_bytes": 99} if attn else {}),
             (dict(txt=text(), d=drafts(), ws=ws, ctx=None), {"stream": types.SimpleNamespace(cuda_stream=321)})]
    if attn:
        forms.append((dict(txt=None, d=drafts(), ws=ws), {"workspace_bytes": 0}))
    if name == "rk_append_text_path":
        forms.append((dict(txt=text(), d=drafts(), kv=1 << 40, n=3), {}))
    if name == "rk_compress_quant":
        forms += [(dict(rw=rows(n_tokens_dev=tensor(B, dtype=torch.int32), strides=(7, 6, 5))), {}),
                  (dict(rw=rows(tok_idx=tensor(9, dtype=torch.int32), tok_off=1 << 33, n_tokens=9)), {"stream": 5})]
    for form, kw in forms:
        args = call(name, **form)
        assert record(name, args, kw, True) == record(name, args, kw, False)


@pytest.mark.parametrize("name", list(SIGNATURES))
def test_other_forms_go_to_ctypes(paths, name):
    _, bind = paths
    fast = getattr(bind, FAST[name])
    ws = torch.empty(10)
    forms = [dict(txt=text(), d=drafts(), ws=ws, kv=np.int64(4096)), dict(txt=text(), d=drafts(), ws=ws, kv=-16), dict(txt=text(), d=drafts(), ws=ws, kv="x")]
    if "attn" in name:
        forms += [dict(txt=text(), d=drafts(), ws=ws, scale="0.5"), dict(txt="text", d=drafts(), ws=ws), dict(txt=text(), d=drafts(), ws=4096)]
    if "tree" in name or "path" in name:
        forms += [dict(txt=text(), d=None, ws=ws), dict(txt=text(), d=drafts(OtherDrafts), ws=ws), dict(txt=text(), d=drafts(strides=[1, 2, 3]), ws=ws),
                  dict(txt=text(), d=drafts(n_tokens=1 << 40), ws=ws), dict(txt=text(), d=drafts(mask="m"), ws=ws)]
    if "path" in name:
        forms += [dict(txt=None, d=drafts()), dict(txt=text(), d=drafts(), n=1 << 40), dict(txt=text(), d=drafts(), n="3")]
    if "compress" in name:
        forms += [dict(rw="rows"), dict(rw=rows(strides=[1, 2, 3])), dict(rw=rows(n_tokens=1 << 31)), dict(rw=rows(tok_off="x"))]
    for form in forms:
        args = call(name, **{"n": 5, **form})
        assert fast(*args, None, *([None] if "attn" in name else [])) is None
    assert fast() is None


class Interrupted:
    def __init__(self):
        self.asked = 0

    def data_ptr(self):
        self.asked += 1
        if self.asked == 1:
            raise KeyboardInterrupt
        return 4096


@pytest.mark.parametrize("name", list(SIGNATURES))
def test_an_interrupt_is_not_swallowed(paths, name):
    record, _ = paths
    with pytest.raises(KeyboardInterrupt):
        record(name, call(name, txt=text(), d=drafts(), ws=torch.empty(10), kv=Interrupted(), n=5), {}, True)


def test_statuses():
    """Errors come out as from the ctypes path, with the library's text."""
    ctx = rk.rk_create(rk.RK_DEVICE_NONE)
    try:
        for n, status in ((T, rk.RK_ERR_NO_DEVICE), (0, rk.RK_ERR_INVALID_ARG)):
            texts = []
            for bind in (rk._bind, None):
                old, rk._bind = rk._bind, bind
                try:
                    with pytest.raises(rk.RotateKError) as e:
                        rk.rk_decode_attn_tree(*call("rk_decode_attn_tree", d=drafts(n_tokens=n), ws=1 << 20, ctx=ctx), workspace_bytes=1 << 30)
                finally:
                    rk._bind = old
                assert e.value.status == status
                texts.append(str(e.value))
            assert texts[0] == texts[1]
    finally:
        rk.rk_destroy(ctx)
