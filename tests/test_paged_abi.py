"""What the operators of speculative rollouts over a paged cache refuse, through the C interface and in Python,
before any HIP call."""
import ctypes
import math

import pytest
import torch

import paper_2608_17641_amd as rl
from paper_2608_17641_amd import _native as n

A = ctypes.c_void_p(0x10000)  # never dereferenced
B2 = ctypes.c_void_p(0x20000)
ODD = ctypes.c_void_p(0x10001)
EIGHT = ctypes.c_void_p(0x10008)


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("the pointers are made up: without a GPU a call that is not refused fails to launch")
    from paper_2608_17641_amd.build import build
    build(force=False)
    return n.load()


def test_paged_attn(lib):
    def f(**kw):
        a = dict(q=A, k=A, v=A, t=A, len=A, start=A, o=A, lse=None, n=6, B=3, W=4, ld=4, pages=9, page=16, Hq=4, Hkv=2, D=64, most=0, at=None, scale=0.1,
                 dtype=1, ws=A, wb=1 << 40, s=None)
        a.update(kw)
        return lib.rlcs_paged_attn(*a.values())
    for kw in (dict(n=-1), dict(B=-1), dict(W=-1), dict(pages=-1), dict(most=-1), dict(page=8), dict(page=24), dict(page=131072), dict(page=0), dict(D=12),
               dict(D=260), dict(D=264), dict(Hq=5), dict(Hkv=0), dict(scale=math.nan), dict(scale=math.inf), dict(q=None), dict(o=None), dict(k=None),
               dict(v=None), dict(t=None), dict(len=None), dict(q=EIGHT), dict(k=EIGHT), dict(v=EIGHT), dict(o=EIGHT), dict(lse=ODD), dict(t=ODD), dict(len=ODD),
               dict(start=ODD), dict(ld=3), dict(start=None, n=7), dict(W=2 ** 27, ld=2 ** 27), dict(n=2 ** 31), dict(n=2 ** 29), dict(ws=EIGHT),
               dict(ld=2 ** 61)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    for field, i, v in (("q", 0, 4), ("k_cache", 1, 1 << 24), ("k_cache", 0, -64), ("v_cache", 2, 7), ("v_cache", 0, 2 ** 60)):
        at = n.PagedLayout()
        getattr(at, field)[i] = v
        assert f(at=ctypes.addressof(at)) == n.RLCS_ERR_INVALID_ARG, (field, v)
    assert f(dtype=2) == n.RLCS_ERR_DTYPE
    need = lib.rlcs_workspace_size_paged(6, 3, 4, 2, 64, 0)
    assert need > 0 and f(ws=None) == f(wb=64) == n.RLCS_ERR_WORKSPACE
    assert f(n=0, q=None) == f(B=0, q=None) == f(Hq=0, q=None) == n.RLCS_OK
    size = lib.rlcs_workspace_size_paged
    assert size(-1, 3, 4, 2, 64, 0) == size(6, 3, 5, 2, 64, 0) == size(6, 3, 4, 2, 12, 0) == size(2 ** 40, 3, 4, 2, 64, 0) == 0


def test_paged_write(lib):
    def f(**kw):
        a = dict(k=A, v=A, kc=A, vc=A, t=A, len=A, start=A, n=6, B=3, W=4, ld=4, pages=9, page=16, Hkv=2, D=64, at=None, dtype=1, s=None)
        a.update(kw)
        return lib.rlcs_paged_write(*a.values())
    for kw in (dict(n=-1), dict(page=17), dict(D=4), dict(k=None), dict(v=None), dict(kc=None), dict(vc=None), dict(k=EIGHT), dict(v=EIGHT), dict(kc=EIGHT),
               dict(vc=EIGHT), dict(t=None), dict(len=None), dict(len=ODD), dict(ld=3), dict(start=None, n=7)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    for field, i, v in (("k_new", 0, 4), ("v_new", 1, -8), ("k_cache", 1, 3), ("v_cache", 1, 1 << 24)):
        at = n.PagedLayout()
        getattr(at, field)[i] = v
        assert f(at=ctypes.addressof(at)) == n.RLCS_ERR_INVALID_ARG, (field, v)
    assert f(dtype=-1) == n.RLCS_ERR_DTYPE
    assert f(n=0, k=None) == f(pages=0, kc=None) == n.RLCS_OK


def test_paged_write_to_overlapping_places(lib):
    for page, token, head in ((0, 128, 64), (2048, 64, 64), (1024, 128, 64), (2048, 128, 0), (64, 64 * 17, 64 * 9)):
        at = n.PagedLayout()
        at.k_new[:], at.v_new[:] = (128, 64), (128, 64)
        at.k_cache[:], at.v_cache[:] = (2048, 128, 64), (page, token, head)
        a = dict(k=A, v=A, kc=A, vc=A, t=A, len=A, start=A, n=6, B=3, W=4, ld=4, pages=9, page=16, Hkv=2, D=64, at=ctypes.addressof(at), dtype=1, s=None)
        assert lib.rlcs_paged_write(*a.values()) == n.RLCS_ERR_INVALID_ARG, (page, token, head)
        at.k_cache[:], at.v_cache[:] = at.v_cache[:], at.k_cache[:]
        assert lib.rlcs_paged_write(*a.values()) == n.RLCS_ERR_INVALID_ARG, (page, token, head)


def test_pages(lib):
    def fork(**kw):
        a = dict(t=A, len=A, refs=A, parent=A, to=B2, lo=B2, ro=B2, B=3, W=4, pages=9, page=16, ws=A, wb=1 << 30, s=None)
        a.update(kw)
        return lib.rlcs_pages_fork(*a.values())

    def resize(**kw):
        a = dict(t=A, len=A, refs=A, new=A, to=B2, lo=B2, ro=B2, moves=B2, B=3, W=4, pages=9, page=16, ws=A, wb=1 << 30, s=None)
        a.update(kw)
        return lib.rlcs_pages_resize(*a.values())

    def compact(**kw):
        a = dict(t=A, refs=A, to=B2, ro=B2, moves=B2, count=B2, B=3, W=4, pages=9, ws=A, wb=1 << 30, s=None)
        a.update(kw)
        return lib.rlcs_pages_compact(*a.values())

    for f in (fork, resize):
        for kw in (dict(B=-1), dict(W=-1), dict(pages=-1), dict(page=15), dict(page=8), dict(t=None), dict(len=None), dict(refs=None), dict(to=None), dict(lo=None),
                   dict(ro=None), dict(t=ODD), dict(len=ODD), dict(to=ODD), dict(W=2 ** 27), dict(B=2 ** 30, W=4), dict(pages=2 ** 30 + 1), dict(ws=EIGHT)):
            assert f(**kw) == n.RLCS_ERR_INVALID_ARG, (f.__name__, kw)
        assert f(ws=None) == f(wb=8) == n.RLCS_ERR_WORKSPACE
        assert f(B=0, t=None) == f(pages=0, t=None) == n.RLCS_OK
    assert fork(parent=None) == fork(parent=ODD) == fork(to=A) == fork(lo=A) == n.RLCS_ERR_INVALID_ARG
    assert resize(new=None) == resize(moves=None) == resize(moves=ODD) == n.RLCS_ERR_INVALID_ARG
    for kw in (dict(B=-1), dict(pages=-1), dict(refs=None), dict(ro=None), dict(count=None), dict(moves=None), dict(t=None), dict(to=None), dict(moves=ODD),
               dict(B=2 ** 20, W=2 ** 20)):
        assert compact(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert compact(ws=None) == n.RLCS_ERR_WORKSPACE and compact(pages=0, refs=None) == n.RLCS_OK
    assert lib.rlcs_workspace_size_pages(-1, 3) == 0 and lib.rlcs_workspace_size_pages(3, 1) > 0


def test_pages_copy(lib):
    def f(**kw):
        a = dict(c=A, m=A, n=3, layers=2, pages=4, ls=4096, ps=1024, size=1024, s=None)
        a.update(kw)
        return lib.rlcs_pages_copy(*a.values())
    for kw in (dict(n=-1), dict(layers=-1), dict(ps=-1), dict(ls=-1), dict(size=-1), dict(c=None), dict(m=None), dict(m=ODD), dict(ps=1000), dict(ls=3000), dict(ls=1024),
               dict(ps=2 ** 62), dict(layers=3, ls=2048, ps=4096), dict(n=2 ** 31), dict(pages=2 ** 30 + 1), dict(n=2 ** 30, size=2 ** 20, ps=2 ** 20, ls=2 ** 22)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert f(n=0, c=None) == f(size=0, c=None) == n.RLCS_OK


def test_verify(lib):
    def f(**kw):
        a = dict(t=A, d=A, x=A, u=A, e=A, nd=None, T=None, Td=None, tokens=A, count=A, logp=None, B=2, K=3, V=5, ts=20, tl=5, ds=15, dl=5, ne=5, aT=1.0, aTd=1.0,
                 dtype=0, ws=A, wb=1 << 30, s=None)
        a.update(kw)
        return lib.rlcs_verify_draft(*a.values())
    for kw in (dict(B=-1), dict(K=-1), dict(V=-1), dict(K=1025), dict(V=2 ** 24 + 1), dict(B=2 ** 30), dict(aT=math.nan), dict(aTd=math.nan), dict(t=None), dict(x=None),
               dict(u=None), dict(e=None), dict(tokens=None), dict(count=None), dict(t=ODD), dict(d=ODD), dict(x=ODD), dict(u=ODD), dict(e=ODD), dict(nd=ODD),
               dict(T=ODD), dict(Td=ODD), dict(tokens=ODD), dict(count=ODD), dict(logp=ODD), dict(ts=-1), dict(tl=2 ** 62), dict(dl=-5), dict(ne=2 ** 62), dict(ws=EIGHT)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert f(dtype=2) == n.RLCS_ERR_DTYPE and f(ws=None) == f(wb=8) == n.RLCS_ERR_WORKSPACE
    assert f(B=0, t=None) == f(V=0, t=None) == n.RLCS_OK
    assert lib.rlcs_workspace_size_verify(2, 1025, 5) == 0 and lib.rlcs_workspace_size_verify(2, 3, 5) > 0


def test_distill(lib):
    def f(**kw):
        a = dict(x=A, ids=A, top=A, w=None, loss=A, g=B2, M=2, V=5, K=3, ld=5, ldg=5, T=1.0, tail=0, dtype=0, s=None)
        a.update(kw)
        return lib.rlcs_distill_loss(*a.values())
    for kw in (dict(M=-1), dict(V=-1), dict(K=-1), dict(K=1025), dict(ld=4), dict(ldg=4), dict(T=0.0), dict(T=math.nan), dict(T=math.inf), dict(T=1e-40), dict(tail=2),
               dict(x=None), dict(ids=None), dict(top=None), dict(loss=None), dict(x=ODD), dict(ids=ODD), dict(top=ODD), dict(w=ODD), dict(loss=ODD), dict(g=ODD),
               dict(g=A, ld=6), dict(M=2 ** 31), dict(V=2 ** 30 + 1, ld=2 ** 31, ldg=2 ** 31), dict(ld=2 ** 62)):
        assert f(**kw) == n.RLCS_ERR_INVALID_ARG, kw
    assert f(dtype=7) == n.RLCS_ERR_DTYPE and f(M=0, x=None) == f(V=0, x=None) == n.RLCS_OK


def test_python_refusals():
    i = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    q, c = torch.zeros(2, 4, 64), torch.zeros(3, 16, 2, 64)
    with pytest.raises(ValueError, match="must be on a GPU"):
        rl.rlcs_paged_attn(q, c, c, i(2, 1), i(2))
    with pytest.raises(TypeError, match="float32 or bfloat16"):
        rl.rlcs_paged_attn(q.double(), c, c, i(2, 1), i(2))
    with pytest.raises(ValueError, match=r"\[tokens, heads, D\]"):
        rl.rlcs_paged_write(c, c, c, c, i(2, 1), i(2))
    for f in (lambda: rl.rlcs_pages_fork(i(2, 1), i(2), i(3), i(2), page=16), lambda: rl.rlcs_pages_resize(i(2, 1), i(2), i(3), i(2), page=16),
              lambda: rl.rlcs_pages_compact(i(2, 1), i(3)), lambda: rl.rlcs_pages_copy(c, i(2, 2)),
              lambda: rl.rlcs_verify_draft(q, q[:, 1:], i(2, 3), q[..., 0], q[:, 0]), lambda: rl.rlcs_distill_loss(q, i(2, 4, 3), q[..., :3])):
        with pytest.raises(ValueError, match="must be on a GPU"):
            f()
    with pytest.raises(ValueError, match=r"\[B, W\]"):
        rl.rlcs_pages_compact(i(2), i(3))


@pytest.mark.gpu
def test_python_refusals_on_device():
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    f = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    q, c = f(4, 4, 64), f(3, 16, 2, 64)
    t, n2 = i(2, 1), i(2)
    for match, kind, call in (
            ("v_cache has dtype", TypeError, lambda: rl.rlcs_paged_attn(q, c, c.bfloat16(), t, n2)),
            ("k_cache and v_cache", ValueError, lambda: rl.rlcs_paged_attn(q, c, c[:2], t, n2)),
            ("table must be", ValueError, lambda: rl.rlcs_paged_attn(q, c, c, t.long(), n2)),
            ("do not overlap", ValueError, lambda: rl.rlcs_paged_attn(q, c, c, i(5, 2).t(), n2)),
            ("length has dtype", TypeError, lambda: rl.rlcs_paged_attn(q, c, c, t, n2.float())),
            ("length must be", TypeError, lambda: rl.rlcs_paged_attn(q, c, c, t, None)),
            ("q_start has shape", ValueError, lambda: rl.rlcs_paged_attn(q, c, c, t, n2, n2)),
            ("q_start says", ValueError, lambda: rl.rlcs_paged_attn(q[:3], c, c, t, n2)),
            ("o has dtype", TypeError, lambda: rl.rlcs_paged_attn(q, c, c, t, n2, o=q.bfloat16())),
            ("INVALID_ARG|bad size", rl.RlcsError, lambda: rl.rlcs_paged_attn(q[:, :3], c, c, t, n2)),
            ("INVALID_ARG|bad size", rl.RlcsError, lambda: rl.rlcs_paged_attn(q, c[:, :12], c[:, :12], t, n2)),
            ("k and v have", ValueError, lambda: rl.rlcs_paged_write(q, q, c, c, t, n2)),
            ("v has dtype", TypeError, lambda: rl.rlcs_paged_write(q[:, :2], q[:, :2].bfloat16(), c, c, t, n2)),
            ("at least one page", ValueError, lambda: rl.rlcs_pages_compact(t, i(0))),
            ("a sequence and a column", ValueError, lambda: rl.rlcs_pages_fork(i(0, 3), i(0), i(4), i(0), page=16)),
            ("a sequence and a column", ValueError, lambda: rl.rlcs_pages_resize(i(2, 0), n2, i(4), n2, page=16)),
            ("parent has shape", ValueError, lambda: rl.rlcs_pages_fork(t, n2, i(4), i(3), page=16)),
            ("new_length has dtype", TypeError, lambda: rl.rlcs_pages_resize(t, n2, i(4), n2.long(), page=16)),
            ("moves has shape", ValueError, lambda: rl.rlcs_pages_resize(t, n2, i(4), n2, moves=i(3, 2), page=16)),
            ("INVALID_ARG|bad size", rl.RlcsError, lambda: rl.rlcs_pages_resize(t, n2, i(4), n2, page=20)),
            ("INVALID_ARG|bad size", rl.RlcsError, lambda: rl.rlcs_pages_fork(t, n2, i(4), n2, t, page=16)),
            (r"\[n, 2\]", ValueError, lambda: rl.rlcs_pages_copy(c, i(2, 3))),
            ("moves has dtype", TypeError, lambda: rl.rlcs_pages_copy(c, f(2, 2))),
            ("must be contiguous", ValueError, lambda: rl.rlcs_pages_copy(c[..., ::2], i(2, 2))),
            ("draft must be", ValueError, lambda: rl.rlcs_verify_draft(q, q, i(4, 3), f(4, 3), f(4, 64))),
            ("draft has dtype", TypeError, lambda: rl.rlcs_verify_draft(q, q[:, 1:].bfloat16(), i(4, 3), f(4, 3), f(4, 64))),
            ("noise must be", ValueError, lambda: rl.rlcs_verify_draft(q, None, i(4, 3), f(4, 3), f(4, 63))),
            ("u has shape", ValueError, lambda: rl.rlcs_verify_draft(q, None, i(4, 3), f(4, 2), f(4, 64))),
            ("temperature has shape", ValueError, lambda: rl.rlcs_verify_draft(q, None, i(4, 3), f(4, 3), f(4, 64), temperature=f(3))),
            ("INVALID_ARG|bad size", rl.RlcsError, lambda: rl.rlcs_verify_draft(q, None, i(4, 3), f(4, 3), f(4, 64), temperature=math.nan)),
            ("top_logp has shape", ValueError, lambda: rl.rlcs_distill_loss(q, i(4, 4, 3), f(4, 4, 2))),
            ("top_ids", ValueError, lambda: rl.rlcs_distill_loss(q, i(4, 3), f(4, 3))),
            ("dlogits must be", ValueError, lambda: rl.rlcs_distill_loss(q, i(4, 4, 3), f(4, 4, 3), dlogits=q.bfloat16())),
            ("INVALID_ARG|bad size", rl.RlcsError, lambda: rl.rlcs_distill_loss(q, i(4, 4, 3), f(4, 4, 3), temperature=0.0))):
        with pytest.raises(kind, match=match):
            call()
