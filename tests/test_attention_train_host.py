"""Refusals of the training attention and of the norm + rotation of queries and keys, before anything reaches a GPU: the C entry points on
addresses that are never read, and the binding on tensors of other shapes, types and devices."""
import ctypes as C

import pytest
import torch

OK, INVALID, SHAPE, UNSUPPORTED, ALIGNMENT, WORKSPACE = 0, 1, 2, 3, 4, 5
FAKE, ODD = C.c_void_p(0x1000), C.c_void_p(0x1004)


@pytest.fixture(scope="module")
def hq():
    from paper_2512_05746_b200 import build
    build.build()
    from paper_2512_05746_b200 import binding
    return binding


def fwd(hq, **change):
    a = dict(q=FAKE, ldq=128, k=FAKE, ldk=128, v=FAKE, ldv=128, Nb=2, Lq=64, Lk=64, heads=2, kv_heads=2, dh=64, scale=0.125, causal=0,
             q_lens=None, k_lens=None, out=FAKE, ldo=128, lse=FAKE, ws=FAKE, ws_bytes=1 << 30, status=None, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_attention_fwd(*a.values())


def bwd(hq, **change):
    a = dict(q=FAKE, ldq=128, k=FAKE, ldk=128, v=FAKE, ldv=128, out=FAKE, ldo=128, lse=FAKE, dout=FAKE, lddo=128, Nb=2, Lq=64, Lk=64, heads=2,
             kv_heads=2, dh=64, scale=0.125, causal=0, q_lens=None, k_lens=None, dq=FAKE, lddq=128, dk=FAKE, lddk=128, dv=FAKE, lddv=128,
             ws=FAKE, ws_bytes=1 << 30, status=None, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_attention_bwd(*a.values())


@pytest.mark.parametrize("call", [fwd, bwd])
@pytest.mark.parametrize("change,want", [
    (dict(Nb=0), OK), (dict(Nb=-1), SHAPE), (dict(Lq=0), SHAPE), (dict(Lk=0), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(heads=3), SHAPE), (dict(dh=0), SHAPE), (dict(dh=60), UNSUPPORTED), (dict(dh=136, ldq=512), UNSUPPORTED), (dict(Nb=65536), UNSUPPORTED),
    (dict(Lq=(1 << 24) + 1), UNSUPPORTED), (dict(scale=0.0), INVALID), (dict(scale=-1.0), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
    (dict(lse=None), INVALID), (dict(q=ODD), ALIGNMENT), (dict(v=ODD), ALIGNMENT), (dict(ldq=120), SHAPE), (dict(ldk=127), SHAPE),
    (dict(ldk=132), ALIGNMENT), (dict(ldo=130), ALIGNMENT), (dict(ldv=1 << 33), UNSUPPORTED)])
def test_attention_refuses(hq, call, change, want):
    assert call(hq, **change) == want


@pytest.mark.parametrize("change,want", [
    (dict(dout=None), INVALID), (dict(dq=None), INVALID), (dict(dk=ODD), ALIGNMENT), (dict(dv=FAKE, lddv=64), SHAPE), (dict(lddo=136, dout=ODD), ALIGNMENT),
    (dict(ws=None), INVALID), (dict(ws=ODD), ALIGNMENT), (dict(ws_bytes=4 * 1024 - 1), WORKSPACE)])
def test_attention_gradient_refuses(hq, change, want):
    assert bwd(hq, **change) == want


def test_workspace_sizes(hq):
    assert hq.hq_attention_bwd_workspace_size(2, 64, 64, 2, 2, 64) >= 4 * 1024
    assert hq.hq_attention_bwd_workspace_size(2, 129, 64, 2, 2, 64) >= 2 * 4 * 1024
    with pytest.raises(hq.HqError):
        hq.hq_attention_bwd_workspace_size(2, 64, 64, 3, 2, 64)
    with pytest.raises(hq.HqError):
        hq.hq_attention_fwd_workspace_size(2, 64, 64, 2, 2, 132)
    assert hq.hq_qk_norm_rope_bwd_workspace_size(10, 4, 2, 64) >= 2 * 64 * 4
    with pytest.raises(hq.HqError):
        hq.hq_qk_norm_rope_bwd_workspace_size(10, 4, 2, 60)
    out = C.c_size_t(0)
    assert hq.lib.hq_attention_fwd_workspace_size(1, 1, 1, 1, 1, 8, None) == INVALID
    assert hq.lib.hq_attention_bwd_workspace_size(0, 1, 1, 1, 1, 8, C.byref(out)) == OK


def rope(hq, **change):
    a = dict(q=FAKE, ldq=128, k=FAKE, ldk=128, dt=1, rows=4, heads=2, kv_heads=2, dh=64, gq=None, gk=None, eps=1e-6, cos=FAKE, sin=FAKE,
             npos=4, rot=64, pos=None, interleaved=0, qo=FAKE, ldqo=128, ko=FAKE, ldko=128, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_qk_norm_rope(*a.values())


def rope_bwd(hq, **change):
    a = dict(q=FAKE, ldq=128, k=FAKE, ldk=128, dt=1, rows=4, heads=2, kv_heads=2, dh=64, gq=FAKE, gk=FAKE, eps=1e-6, cos=FAKE, sin=FAKE,
             npos=4, rot=64, pos=None, interleaved=0, qo=FAKE, ldqo=128, ko=FAKE, ldko=128, dq=FAKE, lddq=128, dk=FAKE, lddk=128, dgq=FAKE,
             dgk=FAKE, ws=FAKE, ws_bytes=1 << 20, stream=None)
    assert not set(change) - set(a)
    a.update(change)
    return hq.lib.hq_qk_norm_rope_bwd(*a.values())


@pytest.mark.parametrize("call", [rope, rope_bwd])
@pytest.mark.parametrize("change,want", [
    (dict(rows=-1), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=-1), SHAPE), (dict(dh=0), SHAPE), (dict(rot=3), SHAPE), (dict(rot=66), SHAPE),
    (dict(npos=0), SHAPE), (dict(dh=60, rot=60), UNSUPPORTED), (dict(dh=256), UNSUPPORTED), (dict(dt=2), INVALID), (dict(cos=None), INVALID),
    (dict(sin=None), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID),
    (dict(ko=None), INVALID), (dict(q=ODD), ALIGNMENT), (dict(ldq=120), SHAPE), (dict(ldk=132), ALIGNMENT), (dict(ldqo=129), ALIGNMENT),
    (dict(dt=0, ldq=130), ALIGNMENT)])
def test_rope_refuses(hq, call, change, want):
    assert call(hq, **change) == want


def test_rope_without_rows_and_its_gradient_s_own(hq):
    assert rope(hq, rows=0) == OK
    for change, want in ((dict(dq=None), INVALID), (dict(ws=None), INVALID), (dict(ws_bytes=16), WORKSPACE), (dict(ws=C.c_void_p(0x1002)), ALIGNMENT),
                         (dict(lddk=64), SHAPE), (dict(kv_heads=0), INVALID)):
        assert rope_bwd(hq, **change) == want, change


def test_binding_refuses(hq):
    bf = torch.bfloat16
    q = torch.zeros((8, 128), dtype=bf)
    lse = torch.zeros((2, 2, 4))
    call = lambda q=q, k=q, v=q, Nb=2, H=2, G=2, out=q, lse=lse, **kw: hq.hq_attention_fwd(q, k, v, Nb, H, G, out, lse, **kw)  # noqa: E731
    for bad in (dict(Nb=3), dict(Nb=0), dict(H=3), dict(G=0), dict(G=1), dict(k=q.float()), dict(v=q[:, :64]), dict(out=q[:4]),
                dict(k=torch.zeros((128, 8), dtype=bf).t()), dict(q=q.half()), dict()):
        with pytest.raises(ValueError):
            call(**bad)                            # the last: everything fits, but the tensors are the host's
    x = torch.zeros((8, 128))
    cos = torch.zeros((8, 32))
    for bad in (dict(H=3), dict(k=None), dict(G=0), dict(sin=None), dict(gamma=torch.zeros(32)), dict(cos=cos.double()), dict(k=x.to(bf)),
                dict(pos=torch.zeros(8)), dict(pos=torch.zeros(7, dtype=torch.int32)), dict(q_out=x.to(bf)), dict()):
        a = dict(dict(k=x, H=2, G=2, gamma=None, cos=cos, sin=cos, q_out=x, pos=None), **bad)
        with pytest.raises(ValueError):
            hq.hq_qk_norm_rope(x, a["k"], a["H"], a["G"], a["gamma"], None, 1e-6, a["cos"], a["sin"], a["q_out"], x, positions=a["pos"])
    with pytest.raises(TypeError):
        h = x.half()
        hq.hq_qk_norm_rope(h, None, 2, 0, None, None, 1e-6, None, None, h, None)


def test_no_item_of_the_gradient_outlasts_a_wait(hq):
    """64 query heads on one key head, 2^22 queries: a tile of keys has 2^21 steps and comes in 16 shares at least, whose fp32 sums of
    dk and dv the workspace holds."""
    Lq, Lk, heads, dh = 1 << 22, 16384, 64, 128
    stats, shares = heads * Lq * 2 * 4, 16 * (Lk // 128) * 2 * (128 * dh * 4)
    assert hq.hq_attention_bwd_workspace_size(1, Lq, Lk, heads, 1, dh) >= stats + shares


@pytest.mark.parametrize("big", [(1 << 32) + 2, -(1 << 32) + 2, 1 << 31])
def test_counts_beyond_32_bits(hq, big):
    """A number of heads is not taken modulo 2^32, and neither is the tables' width."""
    bf = torch.bfloat16
    q, lse = torch.zeros((8, 128), dtype=bf), torch.zeros((2, 2, 4))
    ws = torch.zeros(1 << 16, dtype=torch.uint8)
    for H, G in ((big, 2), (2, big)):
        with pytest.raises(OverflowError):
            hq.hq_attention_fwd(q, q, q, 2, H, G, q, lse)
        with pytest.raises(OverflowError):
            hq.hq_attention_bwd(q, q, q, q, lse, q, 2, H, G, q, q, q, ws)
        with pytest.raises(OverflowError):
            hq.hq_qk_norm_rope(q, q, H, G, None, None, 1e-6, None, None, q, q)
        with pytest.raises(OverflowError):
            hq.hq_qk_norm_rope_bwd(q, q, H, G, None, None, 1e-6, None, None, q, q, q, q, None, None, None)


def test_tables_beyond_32_bits(hq):
    """2^31 + 32 columns are no rotation of 64 channels."""
    q, cos = torch.zeros((8, 128)), torch.empty((0, (1 << 31) + 32))
    with pytest.raises(OverflowError):
        hq.hq_qk_norm_rope(q, q, 2, 2, None, None, 1e-6, cos, cos, q, q)


def test_tiles_of_keys_come_in_shares_where_that_saves_time(hq):
    """The workspace holds the shares' sums (dk and dv of 128 keys in fp32 each) where a call makes shares, and else the statistics: 16 x
    1024 queries on 77 keys took 52 us whole and 68 in shares, 4 x 2027 causal, 4 heads of 64 61 and 79; one sample of 4096, 8 / 1 heads
    of 64 575 and 156, 2 x 4096 causal, 16 / 2 heads of 128 520 and 485 (unmasked 863 and 887, the same workspace)."""
    def shares(Nb, Lq, Lk, heads, kv_heads, dh):
        width, keys = 64 if dh <= 64 else 128, Nb * kv_heads * (-(-Lk // 128))
        stats = Nb * heads * (-(-Lq // 128)) * 1024 + 16
        return (hq.hq_attention_bwd_workspace_size(Nb, Lq, Lk, heads, kv_heads, dh) - stats) / (keys * 2 * 128 * width * 4)
    assert shares(16, 1024, 77, 8, 8, 64) == 0
    assert shares(4, 2027, 2027, 4, 4, 64) == 0
    assert shares(8, 1075, 77, 16, 16, 40) == 0
    assert shares(1, 4096, 4096, 8, 1, 64) >= 8
    assert shares(2, 4096, 77, 8, 8, 64) >= 4
    assert shares(2, 4096, 4096, 16, 2, 128) >= 2
