"""No-GPU checks of the stand-alone operators: bad arguments are refused on the host, before anything is launched."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def dare():
    from paper_2605_08134_b200 import build
    build.build()
    from paper_2605_08134_b200 import dare as d
    return d


def _with(cfg, **kw):
    c = type(cfg).from_buffer_copy(cfg)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


P, Q, R, S = 0x10000, 0x20000, 0x30000, 0x40000        # never dereferenced: every call here is refused (or has nothing to do)


def test_rope_table(dare):
    good = dare.RopeConfig(C.sizeof(dare.RopeConfig), 64, 1e4, 0, 4096, 2.0, 1.0, 32.0, 1.0)
    assert dare.dare_rope_table(None, P, 8) == dare.ERR_INVALID_ARG
    assert dare.dare_rope_table(good, None, 8) == dare.ERR_INVALID_ARG
    inf, nan = float("inf"), float("nan")
    for kw in (dict(struct_size=8), dict(scaling=5), dict(scaling=-1), dict(theta=0.0), dict(theta=nan), dict(theta=inf),
               dict(magnitude=nan), dict(scaling=1, factor=0.5), dict(scaling=1, factor=nan), dict(scaling=3, trained=0),
               dict(scaling=3, low=0.0), dict(scaling=3, low=4.0, high=4.0), dict(scaling=4, high=inf), dict(scaling=4, theta=0.5)):
        assert dare.dare_rope_table(_with(good, **kw), P, 8) == dare.ERR_INVALID_ARG, kw
    for kw in (dict(rotary_dim=0), dict(rotary_dim=63), dict(rotary_dim=258), dict(rotary_dim=2, scaling=2)):
        assert dare.dare_rope_table(_with(good, **kw), P, 8) == dare.ERR_SHAPE, kw
    assert dare.dare_rope_table(good, P, -1) == dare.ERR_SHAPE
    assert dare.dare_rope_table(good, P, (1 << 24) + 1) == dare.ERR_SHAPE
    assert dare.dare_rope_table(good, P + 4, 8) == dare.ERR_ALIGN
    assert dare.dare_rope_table(good, P, 0) == dare.OK


def test_rope(dare):
    good = dare.RopeApply(C.sizeof(dare.RopeApply), dare.BF16, 4, 2, 64, 64, 0, 0, 0, 128, 64, 128, 64, 100)
    call = lambda c, x=P, pos=None, t=Q, y=R: dare.dare_rope(c, x, pos, t, y)
    assert call(None) == dare.ERR_INVALID_ARG
    for kw in (dict(struct_size=0), dict(dtype=2), dict(layout=2), dict(transpose=2)):
        assert call(_with(good, **kw)) == dare.ERR_INVALID_ARG, kw
    for kw in (dict(tokens=-1), dict(tokens=(1 << 30) + 1), dict(heads=-1), dict(head_dim=0), dict(rotary_dim=0), dict(rotary_dim=7),
               dict(rotary_dim=66), dict(rotary_dim=258, head_dim=512), dict(table_positions=-1), dict(x_token=-1), dict(y_head=63),
               dict(y_token=63), dict(y_token=127), dict(y_token=64, y_head=255), dict(x_head=-64)):
        assert call(_with(good, **kw)) == dare.ERR_SHAPE, kw
    for kw in (dict(x=None), dict(t=None), dict(y=None)):
        assert call(good, **kw) == dare.ERR_INVALID_ARG, kw
    assert call(_with(good, x_head=128, x_token=512), y=P) == dare.ERR_INVALID_ARG           # in place with other strides
    for kw in (dict(x=P + 1), dict(y=R + 1), dict(t=Q + 4), dict(pos=S + 2)):
        assert call(good, **kw) == dare.ERR_ALIGN, kw
    assert call(_with(good, tokens=0), x=None) == dare.OK


def test_attention(dare):
    good = dare.AttentionConfig(C.sizeof(dare.AttentionConfig), dare.BF16, 2, 8, 2, 128, 1, 0.1, 16, 64, 1024, 128, 256, 128, 256, 128,
                                1024, 128)
    need = dare.dare_attention_workspace_bytes(good)
    assert need > 0
    W = 0x900000

    def call(c, q=P, k=Q, v=R, qb=S, kb=S + 64, kl=None, out=0x50000, lse=None, work=W, nbytes=need):
        return dare.dare_attention(c, q, k, v, qb, kb, kl, out, lse, work, nbytes)

    assert call(None) == dare.ERR_INVALID_ARG and dare.dare_attention_workspace_bytes(None) == 0
    inf, nan = float("inf"), float("nan")
    for kw in (dict(struct_size=4), dict(dtype=9), dict(causal=2), dict(scale=3e38), dict(scale=0.0), dict(scale=-1.0), dict(scale=nan), dict(scale=inf)):
        assert call(_with(good, **kw)) == dare.ERR_INVALID_ARG and dare.dare_attention_workspace_bytes(_with(good, **kw)) == 0, kw
    for kw in (dict(batch=0), dict(batch=65537), dict(n_heads=7), dict(n_heads=0), dict(n_kv_heads=0), dict(n_heads=2048), dict(head_dim=48),
               dict(q_rows=-1), dict(q_rows=(1 << 24) + 1), dict(k_rows=-1), dict(k_rows=(1 << 30) + 1), dict(k_token=-1), dict(v_head=1 << 38),
               dict(o_head=127), dict(o_token=127), dict(o_token=1023), dict(o_token=128, o_head=1024), dict(q_rows=1 << 24, n_heads=128)):
        assert call(_with(good, **kw)) == dare.ERR_SHAPE and dare.dare_attention_workspace_bytes(_with(good, **kw)) == 0, kw
    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(qb=None), dict(kb=None), dict(out=None), dict(work=None)):
        assert call(good, **kw) == dare.ERR_INVALID_ARG, kw
    for kw in (dict(q=P + 1), dict(k=Q + 1), dict(v=R + 1), dict(out=0x50001), dict(qb=S + 2), dict(kb=S + 2), dict(kl=S + 2),
               dict(lse=S + 2), dict(work=W + 8)):
        assert call(good, **kw) == dare.ERR_ALIGN, kw
    assert call(good, nbytes=need - 1) == dare.ERR_WORKSPACE
    assert call(_with(good, q_rows=0), q=None) == dare.OK


def test_linear(dare):
    good = dare.LinearConfig(C.sizeof(dare.LinearConfig), dare.BF16, 4, 64, 32, 0, 0, 64, 64, 32, 32)
    call = lambda c, x=P, w=Q, b=None, r=None, y=R: dare.dare_linear(c, x, w, b, r, y)
    assert call(None) == dare.ERR_INVALID_ARG
    for kw in (dict(struct_size=1), dict(dtype=3), dict(activation=5), dict(activation=-1), dict(reserved=1)):
        assert call(_with(good, **kw)) == dare.ERR_INVALID_ARG, kw
    for kw in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(in_features=0), dict(in_features=(1 << 20) + 1), dict(out_features=0),
               dict(out_features=(1 << 24) + 1), dict(rows=1 << 24, out_features=1 << 16), dict(x_row=-1), dict(w_row=1 << 38),
               dict(y_row=31), dict(resid_row=-1)):
        assert call(_with(good, **kw)) == dare.ERR_SHAPE, kw
    for kw in (dict(x=None), dict(w=None), dict(y=None)):
        assert call(good, **kw) == dare.ERR_INVALID_ARG, kw
    assert call(_with(good, resid_row=40), r=R) == dare.ERR_INVALID_ARG                     # resid is y with another stride
    for kw in (dict(x=P + 1), dict(w=Q + 1), dict(y=R + 1), dict(b=S + 2), dict(r=S + 1)):
        assert call(good, **kw) == dare.ERR_ALIGN, kw
    assert call(_with(good, rows=0), x=None) == dare.OK


def test_status_off_its_grid(dare):
    ap = dare.RopeApply(C.sizeof(dare.RopeApply), dare.BF16, 4, 2, 64, 64, 0, 0, 0, 128, 64, 128, 64, 16)
    assert dare.dare_rope(ap, P, None, Q, R, S + 2) == dare.ERR_ALIGN
    lc = dare.LinearConfig(C.sizeof(dare.LinearConfig), dare.BF16, 4, 64, 32, 0, 0, 64, 64, 32, 32)
    assert dare.dare_linear(lc, P, Q, None, None, R, S + 2) == dare.ERR_ALIGN
    ac = dare.AttentionConfig(C.sizeof(dare.AttentionConfig), dare.BF16, 2, 8, 2, 128, 1, 0.1, 16, 64, 1024, 128, 256, 128, 256, 128, 1024, 128)
    need = dare.dare_attention_workspace_bytes(ac)
    assert dare.dare_attention(ac, P, Q, R, S, S + 64, None, 0x50000, None, 0x900000, need, S + 2) == dare.ERR_ALIGN


def test_strides_past_any_memory(dare):
    """Products of a stride and a count have to stay inside 64 bits."""
    ap = dare.RopeApply(C.sizeof(dare.RopeApply), dare.BF16, 4, 8, 64, 64, 0, 0, 0, 128, 64, 512, 64, 16)
    for kw in (dict(y_token=1 << 62), dict(y_head=1 << 62), dict(x_token=1 << 62), dict(x_head=1 << 62), dict(y_token=1 << 38),
               dict(y_token=1 << 61, y_head=1 << 60)):
        assert dare.dare_rope(_with(ap, **kw), P, None, Q, R) == dare.ERR_SHAPE, kw
    lc = dare.LinearConfig(C.sizeof(dare.LinearConfig), dare.BF16, 4, 64, 32, 0, 0, 64, 64, 32, 32)
    for kw in (dict(y_row=1 << 62), dict(resid_row=1 << 62), dict(y_row=1 << 38), dict(resid_row=1 << 38)):
        assert dare.dare_linear(_with(lc, **kw), P, Q, None, S, R) == dare.ERR_SHAPE, kw
