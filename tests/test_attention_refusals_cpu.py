"""What the attention entry points and the decoder's attention options refuse, on the host, before
anything is enqueued (no GPU needed)."""
import ctypes
import dataclasses
import math
import os

import pytest

from plain_decoder import Decoder

M = pytest.importorskip("paper_2505_00793_amd._lib")


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not os.path.exists(M.LIB_PATH):
        pytest.skip("libmfmg.so not built")
    M.lib()


OK = dict(heads=4, kv_heads=2, head_dim=64)


@pytest.mark.parametrize("bad", [
    dict(heads=0), dict(heads=3), dict(kv_heads=0), dict(kv_heads=8), dict(heads=2048), dict(head_dim=0),
    dict(head_dim=12), dict(head_dim=136), dict(precision=2), dict(scale=-1.0), dict(scale=float("nan")),
    dict(qk_norm=True, norm_eps=0.0), dict(rope_dims=3), dict(rope_dims=66), dict(rope_dims=-2),
    dict(rope_base=0.0), dict(rope_base=float("inf")), dict(rope_scaling=4), dict(rope_scaling=-1),
    dict(rope_scaling=1, rope_factor=0.5), dict(rope_scaling=2, rope_factor=2.0, rope_dims=2),
    dict(rope_scaling=3, rope_factor=2.0), dict(rope_scaling=3, rope_factor=2.0, rope_train_len=64.0,
                                                rope_slow=8.0, rope_fast=8.0),
    dict(rope_mscale=-1.0),
], ids=lambda b: "-".join(f"{k}{v}" for k, v in b.items()))
def test_bad_descriptions(bad):
    M.Attention(M.make_attn_desc(**OK))
    with pytest.raises(M.MfmgError) as e:
        M.Attention(M.make_attn_desc(**{**OK, **bad}))
    assert e.value.status == M.ERR_INVALID_ARGUMENT


def _status(name, *args):
    return getattr(M.lib(), name)(*args)


A, B = 1 << 20, 1 << 24   # made-up device addresses: every call below is refused before use


def _qkv(q=A, k=A, v=A, ldq=256, ldk=128, ldv=128):
    return ctypes.byref(M.mfmg_qkv(q, k, v, ldq, ldk, ldv))


def test_plan_refusals():
    n = ctypes.c_size_t(0)
    assert _status("mfmg_seq_plan_bytes", 100, 3, ctypes.byref(n)) == M.OK
    need = n.value
    for bad in ((-1, 3), (1 << 31, 3), (1 << 26, 3), (100, -1), (100, (1 << 20) + 1)):
        assert _status("mfmg_seq_plan_bytes", *bad, ctypes.byref(n)) == M.ERR_INVALID_ARGUMENT
    call = lambda cu=A, m=3, n=100, pos=None, plan=B, size=need: _status("mfmg_seq_plan", cu, m, n, pos, plan, size, None)
    assert call(cu=None) == M.ERR_INVALID_ARGUMENT
    assert call(cu=A + 2) == M.ERR_INVALID_ARGUMENT
    assert call(pos=A + 1) == M.ERR_INVALID_ARGUMENT
    assert call(plan=None) == M.ERR_INVALID_ARGUMENT
    assert call(plan=B + 16) == M.ERR_INVALID_ARGUMENT
    assert call(size=need - 1) == M.ERR_WORKSPACE
    assert call(n=-5) == M.ERR_INVALID_ARGUMENT


@pytest.mark.parametrize("norm", [False, True], ids=["rope", "norm"])
def test_rope_refusals(norm):
    op = M.Attention(M.make_attn_desc(**OK, qk_norm=norm, precision=1))
    W, n = 512, 64
    g = A if norm else None
    fwd = dict(plan=B, n=n, m=1, x=A, xd=None, ldx=W, gain=g, gaind=None, y=A, yd=None, ldy=W, stream=None)

    def f(**kw):
        return _status("mfmg_qk_rope_fwd", op._h, *{**fwd, **kw}.values())
    bad = [dict(plan=None), dict(plan=B + 8), dict(n=-1), dict(x=None), dict(y=None), dict(x=A + 4), dict(y=A + 8),
           dict(ldx=W - 4), dict(ldx=W + 1), dict(ldy=W + 4), dict(xd=A), dict(yd=A), dict(gaind=A),
           dict(gain=None if norm else A), dict(xd=A, yd=A, gaind=None if norm else A),
           dict(xd=A + 4, yd=A, gaind=g)]
    for kw in bad:
        assert f(**kw) == M.ERR_INVALID_ARGUMENT, kw
    need = op.mfmg_attn_ws_bytes(n)
    bwd = dict(plan=B, n=n, m=1, x=g, xd=None, ldx=W, gain=g, gaind=None, dy=A, dyd=None, lddy=W, dx=A, dxd=None,
               lddx=W, dgain=g, dgaind=None, ws=B, ws_bytes=need, stream=None)

    def b(**kw):
        return _status("mfmg_qk_rope_bwd", op._h, *{**bwd, **kw}.values())
    bad = [dict(plan=None), dict(dy=None), dict(dx=None), dict(dy=A + 2), dict(lddy=W - 8), dict(lddx=W + 2),
           dict(dyd=A), dict(dxd=A), dict(dyd=A, dxd=A, xd=A if not norm else None, gaind=g, dgaind=g),
           dict(x=A if not norm else None), dict(dgain=A if not norm else None), dict(dgaind=A),
           dict(ws=None), dict(ws=B + 128)]
    for kw in bad:
        assert b(**kw) == M.ERR_INVALID_ARGUMENT, kw
    assert b(ws_bytes=need - 1) == M.ERR_WORKSPACE


def test_attention_refusals():
    op = M.Attention(M.make_attn_desc(**OK, precision=1))
    n = 64
    fwd = dict(plan=B, n=n, m=1, x=_qkv(), xd=None, o=A, od=None, ldo=256, stats=A, stream=None)

    def f(**kw):
        return _status("mfmg_attn_fwd", op._h, *{**fwd, **kw}.values())
    bad = [dict(plan=None), dict(n=1 << 31), dict(x=None), dict(x=_qkv(q=None)), dict(x=_qkv(k=A + 2)),
           dict(x=_qkv(ldv=127)), dict(x=_qkv(ldq=260)), dict(o=None), dict(ldo=255), dict(stats=None),
           dict(stats=A + 2), dict(xd=_qkv()), dict(od=A), dict(xd=_qkv(v=None), od=A)]
    for kw in bad:
        assert f(**kw) == M.ERR_INVALID_ARGUMENT, kw
    need = op.mfmg_attn_ws_bytes(n)
    bwd = dict(plan=B, n=n, m=1, x=_qkv(), xd=None, o=A, od=None, ldo=256, stats=A, g=A, gd=None, ldg=256, dx=_qkv(),
               dxd=None, ws=B, ws_bytes=need, stream=None)

    def b(**kw):
        return _status("mfmg_attn_bwd", op._h, *{**bwd, **kw}.values())
    bad = [dict(x=None), dict(dx=None), dict(dx=_qkv(k=None)), dict(dx=_qkv(ldk=64)), dict(g=None), dict(ldg=200),
           dict(xd=_qkv()), dict(gd=A), dict(dxd=_qkv()), dict(xd=_qkv(), od=A, gd=A), dict(ws=None),
           dict(ws=B + 8), dict(stats=None)]
    for kw in bad:
        assert b(**kw) == M.ERR_INVALID_ARGUMENT, kw
    assert b(ws_bytes=need - 1) == M.ERR_WORKSPACE
    wide = M.Attention(M.make_attn_desc(heads=1024, head_dim=64))   # 2^30 rows of heads
    x = _qkv(ldq=65536, ldk=65536, ldv=65536)
    assert _status("mfmg_attn_fwd", wide._h, *{**fwd, "n": 1 << 20, "x": x, "ldo": 65536}.values()) == M.ERR_UNSUPPORTED
    assert _status("mfmg_attn_fwd", None, *fwd.values()) == M.ERR_INVALID_ARGUMENT


def test_binding_checks_tensors():
    """Types, shapes, strides and devices are checked before an address is taken."""
    torch = pytest.importorskip("torch")
    op = M.Attention(M.make_attn_desc(**OK, precision=1))
    plan = M.SeqPlan(torch.empty(1024, dtype=torch.uint8), 8, 1)
    q, k = torch.empty(8, 256, dtype=torch.bfloat16), torch.empty(8, 128, dtype=torch.bfloat16)
    with pytest.raises(M.MfmgError):   # on the CPU
        op.mfmg_attn_fwd(plan, q, k, k, q, torch.empty(2, 4, 8))
    with pytest.raises(M.MfmgError):
        op.mfmg_qk_rope_fwd(plan, torch.empty(8, 512), torch.empty(8, 512))   # y of another type
    with pytest.raises(M.MfmgError):
        M.mfmg_seq_plan(torch.zeros(2, dtype=torch.int64), 8)


PLAIN = Decoder(norm=0, K=4)


@pytest.mark.parametrize("bad", [
    dict(fused=0, K=2), dict(fused=0, norm=1), dict(fused=0, docs=((0, 60),)), dict(K=3), dict(K=-1), dict(norm=2),
    dict(rope=dict(rope_dims=3, rope_interleaved=1)), dict(rope=dict(rope_scaling=7)), dict(d=1024, K=1),
    dict(rope=dict(rope_scaling=1, rope_factor=0.0)), dict(norm=-1),
], ids=str)
def test_decoder_option_refusals(bad):
    with pytest.raises(M.MfmgError) as e:
        M.Problem(dataclasses.replace(PLAIN, **bad).desc())
    assert e.value.status == M.ERR_UNSUPPORTED
    M.Problem(dataclasses.replace(PLAIN, K=2).desc())


def test_decoder_sizes_with_options():
    """Parameters of grouped heads and gains; more documents than tokens are refused; a batch with
    documents needs their offsets; an MLP has no attention."""
    c = Decoder(K=2, norm=1)
    n = M.Problem(c.desc()).mfmg_query_sizes(2).n_theta
    assert n == sum(math.prod(s) for _, s in c.shapes())
    d = c.desc()
    d.docs = c.rows * c.S + 1
    with pytest.raises(M.MfmgError):
        M.Problem(d)
    d.docs = 2
    p = M.Problem(d)
    b = M.mfmg_batch(A, None, c.rows)
    s = M.lib().mfmg_inner_step(p.handle, A, None, A, ctypes.byref(b), 0, A, None, None, None, B, 1 << 40, None)
    assert s == M.ERR_INVALID_ARGUMENT and b"document" in M.lib().mfmg_last_error_message()
    m = M.make_desc(widths=(8, 4), rows=4, val_rows=4, qk_norm=1)
    with pytest.raises(M.MfmgError) as e:
        M.Problem(m)
    assert e.value.status == M.ERR_INVALID_ARGUMENT
