"""What the operators around a group rollout refuse, through the C interface and in Python, before
any HIP call."""
import ctypes
import math

import pytest
import torch

import paper_2608_17641_amd as rl
from paper_2608_17641_amd import _native as n

A = ctypes.c_void_p(0x10000)  # never dereferenced
ODD = ctypes.c_void_p(0x10001)


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("the pointers are made up: without a GPU a call that is not refused fails to launch")
    from paper_2608_17641_amd.build import build
    build(force=False)
    return n.load()


def test_token_logp(lib):
    def f(**kw):
        a = dict(x=A, t=A, lp=A, ent=None, M=2, V=3, ld=3, T=1.0, dtype=0, s=None)
        a.update(kw)
        return lib.rlcs_token_logp(*a.values())
    for kw in (dict(M=-1), dict(V=-1, ld=0), dict(ld=2), dict(T=0.0), dict(T=-1.0), dict(T=math.nan), dict(T=math.inf), dict(x=None),
               dict(t=None), dict(lp=None), dict(x=ODD), dict(t=ODD), dict(lp=ODD), dict(ent=ODD), dict(M=2 ** 31), dict(V=2 ** 30 + 1, ld=2 ** 31),
               dict(ld=2 ** 62), dict(T=1e-40)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert f(dtype=2) == n.RLCS_ERR_DTYPE
    assert f(M=0, x=None) == n.RLCS_OK and f(V=0, x=None) == n.RLCS_OK


def test_policy_loss(lib):
    def f(**kw):
        a = dict(x=A, t=A, old=A, adv=A, w=None, loss=A, g=ctypes.c_void_p(0x20000), lp=None, ent=None, M=2, V=3, ld=3, ldg=3, lo=0.2, hi=0.2, c=0.0,
                 T=1.0, dtype=0, s=None)
        a.update(kw)
        return lib.rlcs_policy_loss(*a.values())
    for kw in (dict(M=-1), dict(ld=2), dict(ldg=2), dict(lo=-0.1), dict(lo=1.5), dict(lo=math.nan), dict(hi=-1.0), dict(hi=math.nan), dict(c=math.inf),
               dict(c=math.nan), dict(T=0.0), dict(old=None), dict(adv=None), dict(loss=None), dict(t=None), dict(g=ODD), dict(w=ODD), dict(loss=ODD),
               dict(g=A, ld=4, ldg=3), dict(ldg=2 ** 62)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert f(dtype=-1) == n.RLCS_ERR_DTYPE
    assert f(M=0, x=None) == n.RLCS_OK


def test_sample(lib):
    def f(**kw):
        a = dict(x=A, e=A, T=None, k=None, p=None, mp=None, t=A, lp=None, M=2, V=3, ld=3, ldn=3, aT=1.0, ak=0, ap=1.0, amp=0.0, dtype=0, ws=None, wb=0,
                 s=None)
        a.update(kw)
        return lib.rlcs_sample(*a.values())
    for kw in (dict(M=-1), dict(V=2 ** 24 + 1, ld=2 ** 25, ldn=2 ** 25), dict(ld=2), dict(ldn=2), dict(aT=math.nan), dict(ap=math.nan), dict(amp=math.nan),
               dict(amp=1.5), dict(x=None), dict(t=None), dict(x=ODD), dict(e=ODD), dict(T=ODD), dict(k=ODD), dict(p=ODD), dict(mp=ODD), dict(t=ODD),
               dict(lp=ODD), dict(M=2 ** 31)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert f(dtype=2) == n.RLCS_ERR_DTYPE
    assert f(M=0, x=None) == n.RLCS_OK


def test_attn(lib):
    def f(**kw):
        a = dict(q=A, kp=A, vp=A, ks=A, vs=A, pl=None, sl=None, o=A, lse=None, N=1, G=2, Hq=4, Hkv=2, D=64, P=10, S=5, at=None, scale=0.1, dtype=1, ws=A,
                 wb=1 << 40, s=None)
        a.update(kw)
        return lib.rlcs_shared_prefix_attn(*a.values())
    EIGHT = ctypes.c_void_p(0x10008)
    for kw in (dict(N=-1), dict(S=-1), dict(D=260), dict(D=12), dict(Hq=5), dict(Hkv=0), dict(scale=math.nan), dict(scale=math.inf), dict(q=None),
               dict(o=None), dict(kp=None), dict(vs=None), dict(q=EIGHT), dict(kp=EIGHT), dict(o=EIGHT), dict(lse=ODD), dict(pl=ODD), dict(sl=ODD),
               dict(P=2 ** 30 + 1), dict(N=60000, G=60000), dict(G=65535, S=2 ** 30, Hq=65535, Hkv=65535, D=256)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    at = n.AttnLayout()
    for field, i, v in (("q", 0, 4), ("kp", 1, -64), ("vs", 3, 7), ("ks", 1, 2 ** 62)):
        at = n.AttnLayout()
        getattr(at, field)[i] = v
        assert f(at=ctypes.addressof(at)) == n.RLCS_ERR_INVALID_ARG, (field, v)
    assert f(dtype=3) == n.RLCS_ERR_DTYPE
    assert f(N=0, q=None) == n.RLCS_OK and f(G=0, q=None) == n.RLCS_OK


def test_python_refusals():
    x, t = torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="must be on a GPU"):
        rl.rlcs_token_logp(x, t)
    with pytest.raises(ValueError, match="must be on a GPU"):
        rl.rlcs_policy_loss(x, t, x[:, 0], x[:, 0], clip_low=0.2, clip_high=0.2)
    with pytest.raises(ValueError, match="must be on a GPU"):
        rl.rlcs_sample(x)
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        rl.rlcs_sample(x.double())
    with pytest.raises(ValueError, match="two dimensions"):
        rl.rlcs_token_logp(x[0], t)
    with pytest.raises(ValueError, match=r"\[N, G, Hq, D\]"):
        rl.rlcs_shared_prefix_attn(x, x, x)
    with pytest.raises(ValueError, match="must be on a GPU"):
        rl.rlcs_shared_prefix_attn(torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1, 8), torch.zeros(1, 1, 1, 8))


@pytest.mark.gpu
def test_python_refusals_on_device():
    x = torch.zeros(4, 8, device="cuda")
    t, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    p = dict(clip_low=0.2, clip_high=0.2)
    with pytest.raises(TypeError, match="tokens"):
        rl.rlcs_token_logp(x, t.long())
    with pytest.raises(ValueError, match="adv has shape"):
        rl.rlcs_policy_loss(x, t, f, f[:3], **p)
    with pytest.raises(TypeError, match="logp_old"):
        rl.rlcs_policy_loss(x, t, f.double(), f, **p)
    with pytest.raises(ValueError, match="dlogits"):
        rl.rlcs_policy_loss(x, t, f, f, dlogits=x.bfloat16(), **p)
    with pytest.raises(ValueError, match="do not overlap"):
        rl.rlcs_token_logp(x.t(), torch.zeros(8, dtype=torch.int32, device="cuda"))
    with pytest.raises(rl.RlcsError, match="INVALID_ARG"):
        rl.rlcs_policy_loss(x, t, f, f, clip_low=-1.0, clip_high=0.2)
    with pytest.raises(rl.RlcsError, match="INVALID_ARG"):
        rl.rlcs_token_logp(x, t, temperature=0.0)
    with pytest.raises(ValueError, match="noise"):
        rl.rlcs_sample(x, x.bfloat16())
    with pytest.raises(TypeError, match="top_k"):
        rl.rlcs_sample(x, top_k=f)
    with pytest.raises(ValueError, match="top_p"):
        rl.rlcs_sample(x, top_p=f[:2])
    q = torch.zeros(1, 2, 4, 64, device="cuda")
    kv, kv5 = torch.zeros(1, 5, 2, 64, device="cuda"), torch.zeros(1, 2, 3, 2, 64, device="cuda")
    with pytest.raises(ValueError, match="go together"):
        rl.rlcs_shared_prefix_attn(q, kv, kv, kv5)
    with pytest.raises(TypeError, match="vp has dtype"):
        rl.rlcs_shared_prefix_attn(q, kv, kv.bfloat16())
    with pytest.raises(ValueError, match="kp and vp"):
        rl.rlcs_shared_prefix_attn(q, kv, kv[:, :4])
    with pytest.raises(TypeError, match="prefix_len"):
        rl.rlcs_shared_prefix_attn(q, kv, kv, prefix_len=torch.zeros(1, dtype=torch.int64, device="cuda"))
    with pytest.raises(rl.RlcsError, match="WORKSPACE|INVALID_ARG"):
        rl.rlcs_shared_prefix_attn(q[..., :60], kv[..., :60], kv[..., :60])
