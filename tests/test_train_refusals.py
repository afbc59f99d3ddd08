"""What the training operators refuse, before anything reaches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2410_05589_b200 import binding as b

INVALID, UNSUPPORTED, CAPACITY = -1, -2, -3
FAKE = 1 << 20      # a 256-byte aligned address that no refused call may touch


@pytest.fixture(scope="module")
def lib():
    return b.load_library()


def attn_args(**kw):
    a = b.ps_group_attn_args()
    a.dtype, a.B, a.k_masks, a.n_heads, a.n_kv_heads, a.head_dim, a.scale = 1, 2, 4, 4, 2, 64, 0.125
    a.n_ctx, a.n_groups = b._iarr([3, 0]), b._iarr([2, 5])
    for f in ("q", "k", "v", "out", "lse", "dout", "dq", "dk", "dv"):
        setattr(a, f, FAKE)
    for f in ("ldq", "ldo", "lddo", "lddq"):
        setattr(a, f, 256)
    for f in ("ldk", "ldv", "lddk", "lddv"):
        setattr(a, f, 128)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def call_attn(lib, a, backward, ws=FAKE, nbytes=None):
    err = C.create_string_buffer(256)
    n = lib.ps_group_attn_workspace_bytes(C.byref(a), int(backward)) if a else 0
    fn = lib.ps_group_attn_backward if backward else lib.ps_group_attn
    rc = fn(C.byref(a) if a else None, ws, n if nbytes is None else nbytes, None, err, 256, None)
    return rc, err.value.decode()


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("field, value, want", [
    ("dtype", 2, INVALID), ("B", 0, INVALID), ("B", 129, INVALID), ("k_masks", -1, INVALID), ("k_masks", 16, INVALID),
    ("n_heads", 0, INVALID), ("n_heads", 5, INVALID), ("n_heads", 1026, INVALID), ("n_kv_heads", 0, INVALID),
    ("head_dim", 96, UNSUPPORTED), ("scale", float("nan"), INVALID), ("scale", float("inf"), INVALID),
    ("q", None, INVALID), ("k", None, INVALID), ("v", None, INVALID), ("out", None, INVALID), ("lse", None, INVALID),
    ("ldq", 255, INVALID), ("ldk", 127, INVALID), ("ldv", 0, INVALID), ("ldo", 8, INVALID)])
def test_attention_refuses(lib, field, value, want, backward):
    rc, text = call_attn(lib, attn_args(**{field: value}), backward, nbytes=1 << 40)
    assert rc == want and "ps_group_attn" in text


@pytest.mark.parametrize("field, value", [("dout", None), ("dq", None), ("dk", None), ("dv", None), ("lddo", 255),
                                          ("lddq", 1), ("lddk", 127), ("lddv", 2)])
def test_attention_backward_refuses(lib, field, value):
    assert call_attn(lib, attn_args(**{field: value}), True, nbytes=1 << 40)[0] == INVALID


def test_attention_refuses_sizes_and_workspaces(lib):
    a = attn_args()
    for what in ("n_ctx", "n_groups"):
        assert call_attn(lib, attn_args(**{what: b._iarr([1, -1])}), False, nbytes=1 << 40)[0] == INVALID
        assert call_attn(lib, attn_args(**{what: None}), False, nbytes=1 << 40)[0] == INVALID
        assert call_attn(lib, attn_args(**{what: b._iarr([1 << 29, 1 << 29])}), False, nbytes=1 << 40)[0] == INVALID
    assert call_attn(lib, None, False)[0] == INVALID and lib.ps_group_attn_workspace_bytes(None, 0) == 0
    for back in (False, True):
        n = lib.ps_group_attn_workspace_bytes(C.byref(a), int(back))
        assert n > 0
        assert call_attn(lib, a, back, nbytes=n - 1)[0] == CAPACITY
        assert call_attn(lib, a, back, ws=None)[0] == INVALID
        assert call_attn(lib, a, back, ws=FAKE + 16)[0] == INVALID
    # nothing to do: accepted without a device
    empty = attn_args(n_ctx=b._iarr([0, 0]), n_groups=b._iarr([0, 0]))
    assert call_attn(lib, empty, False)[0] == 0 and call_attn(lib, empty, True)[0] == 0


LOSS = dict(dtype=1, rows=4, hidden=64, vocab=100, x=FAKE, ldx=64, w=FAKE, labels=FAKE, loss=FAKE, lse=FAKE, dloss=FAKE,
            dx=FAKE, lddx=64, dw=FAKE, ws=FAKE, nbytes=1 << 40)


def call_loss(lib, backward, **kw):
    p = dict(LOSS, **kw)
    err = C.create_string_buffer(256)
    size = (p["dtype"], p["rows"], p["hidden"], p["vocab"])
    if backward:
        return lib.ps_lm_loss_backward(*size, p["x"], p["ldx"], p["w"], p["labels"], p["lse"], p["dloss"], p["dx"], p["lddx"],
                                       p["dw"], p["ws"], p["nbytes"], None, err, 256, None)
    return lib.ps_lm_loss(*size, p["x"], p["ldx"], p["w"], p["labels"], p["loss"], p["lse"], p["ws"], p["nbytes"], None, err, 256, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw, want", [
    (dict(dtype=2), INVALID), (dict(rows=-1), INVALID), (dict(rows=(1 << 20) + 1), INVALID), (dict(vocab=0), INVALID),
    (dict(vocab=(1 << 20) + 1), INVALID), (dict(hidden=0), INVALID), (dict(hidden=65544, ldx=65544), INVALID),
    (dict(hidden=60), UNSUPPORTED), (dict(w=FAKE + 8), UNSUPPORTED), (dict(x=None), INVALID), (dict(w=None), INVALID),
    (dict(labels=None), INVALID), (dict(lse=None), INVALID), (dict(ldx=63), INVALID), (dict(ws=None), INVALID),
    (dict(ws=FAKE + 128), INVALID), (dict(nbytes=1000), CAPACITY)])
def test_loss_refuses(lib, kw, want, backward):
    assert call_loss(lib, backward, **kw) == want


def test_loss_refuses_one_way(lib):
    assert call_loss(lib, False, loss=None) == INVALID
    assert call_loss(lib, True, dloss=None) == INVALID
    assert call_loss(lib, True, lddx=63) == INVALID
    assert call_loss(lib, True, dw=FAKE + 2) == UNSUPPORTED
    assert call_loss(lib, True, dx=None, dw=None) == 0 and call_loss(lib, False, rows=0) == 0
    assert lib.ps_lm_loss_workspace_bytes(1, 4, 60, 100, 0) == 0


EMBED = dict(dtype=1, rows=4, hidden=64, vocab=100, k=2, ids=FAKE, table=FAKE, masks=FAKE, out=FAKE, ldo=64, dout=FAKE, lddo=64,
             dt=FAKE, dm=FAKE, ws=FAKE, nbytes=1 << 40)


def call_embed(lib, backward, **kw):
    p = dict(EMBED, **kw)
    err = C.create_string_buffer(256)
    size = (p["dtype"], p["rows"], p["hidden"], p["vocab"], p["k"])
    if backward:
        return lib.ps_embed_rows_backward(*size, p["ids"], 1.0, p["dout"], p["lddo"], p["dt"], p["dm"], p["ws"], p["nbytes"], err, 256, None)
    return lib.ps_embed_rows(*size, p["ids"], p["table"], p["masks"], 1.0, p["out"], p["ldo"], err, 256, None)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw", [dict(dtype=-1), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(hidden=0), dict(hidden=65537),
                                dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(k=-1), dict(k=16), dict(ids=None)])
def test_embedding_refuses(lib, kw, backward):
    assert call_embed(lib, backward, **kw) == INVALID


def test_embedding_refuses_one_way(lib):
    for kw in (dict(table=None), dict(masks=None), dict(out=None), dict(ldo=63)):
        assert call_embed(lib, False, **kw) == INVALID
    for kw in (dict(dout=None), dict(lddo=63), dict(ws=None), dict(ws=FAKE + 4)):
        assert call_embed(lib, True, **kw) == INVALID
    assert call_embed(lib, True, nbytes=100) == CAPACITY
    assert call_embed(lib, True, dt=None, dm=None) == 0 and call_embed(lib, False, rows=0) == 0
    assert lib.ps_embed_rows_workspace_bytes(1, 4, 0, 100, 2) == 0


def test_binding_refuses_tensors_of_the_host():
    x = torch.zeros(4, 64)
    with pytest.raises(b.PsError):
        b.lm_loss(x, torch.zeros(100, 64), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(b.PsError):
        b.embed_rows(torch.zeros(4, dtype=torch.int32), x)
    with pytest.raises(b.PsError):
        b.embed_rows_backward(torch.zeros(4, dtype=torch.int32), x, 100)
    with pytest.raises(b.PsError):
        b.group_attention(torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), torch.zeros(1, 2, 64), [0], [1], 0)


def test_binding_reads_row_strides():
    t = torch.zeros(6, 3, 2, 64)
    assert b._rows(t[:, 0], 128, "k") == 384 and b._rows(t[:1, 0], 128, "k") == 128
    with pytest.raises(b.PsError):
        b._rows(t[:, :, 0], 128, "k")           # heads apart
    with pytest.raises(b.PsError):
        b._rows(t[:1].expand(6, 3, 2, 64), 384, "k")   # one row for all
    assert b._rows(torch.zeros(0, 128), 128, "k") == 128
