"""Host-side refusals of the token operators' entry points, without a GPU: every bad argument is
turned down before anything is launched."""
import pytest


@pytest.fixture(scope="module")
def lib():
    from paper_2606_13426_gb300 import binding, buildlib
    try:
        buildlib.build()
    except RuntimeError as e:  # no nvcc on this machine
        pytest.skip(str(e))
    return binding.load()


def check(lib, fn, names, base, cases):
    """`fn` with the arguments `base` replaced one set at a time; each returns its code."""
    for kw, code in cases:
        a = dict(base)
        assert set(kw) <= set(a), kw
        a.update(kw)
        assert getattr(lib, fn)(*[a[n] for n in names]) == code, kw


def test_scores(lib):
    from paper_2606_13426_gb300 import binding as B
    names = "x stride N V dtype tok T k lp H m ls ids tlp st s".split()
    base = dict(x=0x1000, stride=100, N=2, V=100, dtype=B.SDV_BF16, tok=0x2000, T=1.0, k=4, lp=0x3000, H=0x4000, m=0x5000, ls=0x6000,
                ids=0x7000, tlp=0x8000, st=0, s=None)
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    check(lib, "sdv_token_scores", names, base, [
        (dict(x=0), bad), (dict(stride=99), bad), (dict(N=-1), bad), (dict(V=0), bad), (dict(V=(1 << 30) + 1, stride=1 << 31), bad),
        (dict(dtype=3), bad), (dict(T=0.0), bad), (dict(T=float("inf")), bad), (dict(T=float("nan")), bad), (dict(T=1e-39), bad),
        (dict(T=9e-10), bad), (dict(T=1.1e9), bad),
        (dict(k=-1), bad), (dict(k=33), bad), (dict(V=3, k=4), bad), (dict(ids=0), bad), (dict(tlp=0), bad), (dict(lp=0), bad),
        (dict(tok=0), bad), (dict(x=0x1001), align), (dict(x=0x1002, dtype=B.SDV_F32), align), (dict(H=0x4002), align),
        (dict(ids=0x7001), align), (dict(tok=0, lp=0, H=0, m=0, ls=0, k=0), bad),
        (dict(N=0, x=0), B.SDV_OK), (dict(N=0, dtype=5), bad)])


def test_gradients(lib):
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "x stride N V dtype tok T m ls H gl gh dx dstride s".split()
    base = dict(x=0x1000, stride=100, N=2, V=100, dtype=B.SDV_F32, tok=0x2000, T=1.0, m=0x3000, ls=0x4000, H=0x5000, gl=0x6000, gh=0x7000,
                dx=0x8000, dstride=100, s=None)
    check(lib, "sdv_token_scores_grad", names, base, [
        (dict(dx=0), bad), (dict(dstride=99), bad), (dict(m=0), bad), (dict(ls=0), bad), (dict(H=0), bad), (dict(gl=0, gh=0), bad),
        (dict(tok=0), bad), (dict(gl=0), bad), (dict(T=-1.0), bad), (dict(T=1e-12), bad), (dict(dx=0x8002), align), (dict(gh=0x7001), align),
        (dict(N=0, x=0), B.SDV_OK)])
    names = "x stride N V dtype tok T gl gh lp H m ls st dx dstride s".split()
    base.update(lp=0x9000, st=0)
    check(lib, "sdv_token_scores_train", names, base, [
        (dict(dx=0), bad), (dict(H=0), bad), (dict(m=0), bad), (dict(ls=0), bad), (dict(gl=0, gh=0), bad), (dict(tok=0), bad),
        (dict(lp=0), bad), (dict(dstride=1), bad), (dict(dx=0x8001), align), (dict(N=0, x=0), B.SDV_OK)])


def test_token_verify(lib):
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "q qb qr p pb pr tok B L V dtype T Td mode Leff seed coins race acc nxt lr st ws wsb s".split()
    wsb = B.sdv_token_verify_workspace_bytes(2, 3)
    assert wsb > 0 and wsb % 256 == 0
    assert B.sdv_token_verify_workspace_bytes(0, 3) == 0 and B.sdv_token_verify_workspace_bytes(2, 65) == 0
    base = dict(q=0x1000, qb=400, qr=100, p=0x2000, pb=300, pr=100, tok=0x3000, B=2, L=3, V=100, dtype=B.SDV_BF16, T=1.0, Td=1.0, mode=1,
                Leff=0, seed=1, coins=0, race=0, acc=0x4000, nxt=0x5000, lr=0, st=0, ws=0x6000, wsb=wsb, s=None)
    check(lib, "sdv_token_verify", names, base, [
        (dict(q=0), bad), (dict(p=0), bad), (dict(tok=0), bad), (dict(acc=0), bad), (dict(nxt=0), bad), (dict(B=0), bad), (dict(L=0), bad),
        (dict(L=65), bad), (dict(V=0), bad), (dict(dtype=7), bad), (dict(T=0.0), bad), (dict(Td=float("nan")), bad), (dict(mode=2), bad),
        (dict(T=1e-10), bad), (dict(Td=1e10), bad),
        (dict(qr=99), bad), (dict(pr=99), bad), (dict(qb=-1), bad), (dict(q=0x1001), align), (dict(p=0x2001), align),
        (dict(tok=0x3002), align), (dict(race=0x7001), align), (dict(ws=0), B.SDV_ENOWORKSPACE), (dict(wsb=wsb - 1), B.SDV_ENOWORKSPACE),
        (dict(ws=0x6010), align)])


CACHE = dict(kc=0x10000, vc=0x20000, ks=0x30000, vs=0x40000, pages=8, tab=0x50000, M=4, n=0x60000, cnt=0, st=0)


def test_cache_append(lib):
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "k v sb st_ sh dtype B W H D block kc vc ks vs pages tab M n cnt st s".split()
    base = dict(CACHE, k=0x1000, v=0x2000, sb=256, st_=128, sh=64, dtype=B.SDV_F32, B=2, W=2, H=2, D=64, block=16, s=None)
    check(lib, "sdv_cache_append", names, base, [
        (dict(k=0), bad), (dict(v=0), bad), (dict(n=0), bad), (dict(kc=0), bad), (dict(vc=0), bad), (dict(ks=0), bad), (dict(vs=0), bad),
        (dict(tab=0), bad), (dict(B=0), bad), (dict(W=0), bad), (dict(H=0), bad), (dict(D=96), bad), (dict(D=256), bad),
        (dict(block=8), bad), (dict(block=24), bad), (dict(block=144), bad), (dict(pages=0), bad), (dict(M=0), bad), (dict(sb=-1), bad),
        (dict(dtype=4), bad), (dict(kc=0x10008), align), (dict(vc=0x20001), align), (dict(ks=0x30002), align), (dict(k=0x1002), align),
        (dict(n=0x60001), align), (dict(M=1 << 28, block=16), bad)])


def test_cache_attend(lib):
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "q sb st_ sh dtype B W Hq H D block kc vc ks vs pages tab M n cnt scale span out lse st ws wsb s".split()
    wsb = B.sdv_attend_workspace_bytes(2, 2, 4, 2, 64)
    assert wsb > 0 and B.sdv_attend_workspace_bytes(2, 2, 3, 2, 64) == 0 and B.sdv_attend_workspace_bytes(2, 2, 4, 2, 80) == 0
    base = dict(CACHE, q=0x1000, sb=512, st_=256, sh=64, dtype=B.SDV_BF16, B=2, W=2, Hq=4, H=2, D=64, block=16, scale=0.1, span=0,
                out=0x2000, lse=0x3000, ws=0x100000, wsb=wsb, s=None)
    check(lib, "sdv_cache_attend", names, base, [
        (dict(q=0), bad), (dict(out=0), bad), (dict(n=0), bad), (dict(dtype=B.SDV_F32), bad), (dict(Hq=3), bad), (dict(Hq=1), bad),
        (dict(H=0), bad), (dict(W=0), bad), (dict(B=0), bad), (dict(D=32), bad), (dict(block=12), bad), (dict(span=-1), bad),
        (dict(scale=float("nan")), bad), (dict(scale=float("inf")), bad), (dict(st_=-1), bad), (dict(q=0x1001), align),
        (dict(M=(1 << 26) + 1), bad), (dict(M=(1 << 23) + 1, block=128), bad),
        (dict(out=0x2001), align), (dict(lse=0x3002), align), (dict(kc=0x10004), align), (dict(ws=0), B.SDV_ENOWORKSPACE),
        (dict(wsb=wsb - 1), B.SDV_ENOWORKSPACE), (dict(ws=0x100080), align)])


def test_api_refuses_host_tensors():
    """The torch-facing helpers take CUDA tensors only; nothing is computed on the CPU."""
    import torch
    from paper_2606_13426_gb300 import api
    x = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        api.token_scores(x)
    with pytest.raises(ValueError):
        api.token_scores_train(x, None, None, torch.zeros(2))
    with pytest.raises(ValueError):
        api.token_verify(torch.zeros(1, 2, 8), torch.zeros(1, 1, 8), torch.zeros(1, 1, dtype=torch.int32))
    with pytest.raises(ValueError):
        api.cache_append(api.make_token_cache(2, 1, 16, 64, "cpu"), torch.zeros(1, 1, 1, 64), torch.zeros(1, 1, 1, 64),
                         torch.zeros(1, 1, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))


def test_attend_workspace_follows_the_device(monkeypatch):
    """Sizes are remembered per device, whose SMs they depend on, and not without end."""
    import torch
    from paper_2606_13426_gb300 import api
    current = [0]
    asked = []

    def size(*sizes):                                       # a device of 152 SMs and one of 160
        asked.append(sizes)
        return 1000 * (152, 160)[current[0]]
    monkeypatch.setattr(api.B, "sdv_attend_workspace_bytes", size)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    api._attend_workspace.cache_clear()
    try:
        for _ in range(2):
            for current[0] in (0, 1):
                assert api._attend_workspace(torch.cuda.current_device(), 2, 2, 4, 2, 64) == 1000 * (152, 160)[current[0]]
        assert len(asked) == 2
        for n in range(5000):
            api._attend_workspace(0, n, 2, 4, 2, 64)
        assert api._attend_workspace.cache_info().currsize <= 1024
    finally:
        api._attend_workspace.cache_clear()


def test_binding_functions_hand_their_arguments_on(lib):
    """The binding's function of each entry point: arguments in the header's order, refusals as SDVError."""
    from paper_2606_13426_gb300 import binding as B
    ok = dict(
        sdv_token_scores=[0x1000, 100, 0, 100, B.SDV_F32, 0x2000, 1.0, 0, 0x3000, 0, 0, 0, 0, 0, 0, 0],
        sdv_token_scores_grad=[0x1000, 100, 0, 100, B.SDV_F32, 0x2000, 1.0, 0x3000, 0x4000, 0, 0x5000, 0, 0x6000, 100, 0],
        sdv_token_scores_train=[0x1000, 100, 0, 100, B.SDV_F32, 0x2000, 1.0, 0x3000, 0, 0x4000, 0x5000, 0x6000, 0x7000, 0, 0x8000, 100, 0])
    for name, args in ok.items():                           # no rows: nothing is launched
        assert getattr(B, name)(*args) == B.SDV_OK
    wrong = dict(
        {k: v[:3] + [0] + v[4:] for k, v in ok.items()},    # V = 0
        sdv_token_verify=[0x1000, 400, 100, 0x2000, 300, 100, 0x3000, 2, 3, 100, B.SDV_BF16, 1.0, 1.0, 2, 0, 1, 0, 0, 0x4000, 0x5000, 0, 0, 0x6000,
                          1 << 20, 0],                      # mode 2
        sdv_cache_append=[0x1000, 0x2000, 256, 128, 64, B.SDV_F32, 2, 2, 2, 96, 16, 0x10000, 0x20000, 0x30000, 0x40000, 8, 0x50000, 4, 0x60000, 0, 0,
                          0],                               # D = 96
        sdv_cache_attend=[0x1000, 512, 256, 64, B.SDV_BF16, 2, 2, 3, 2, 64, 16, 0x10000, 0x20000, 0x30000, 0x40000, 8, 0x50000, 4, 0x60000, 0, 0.1, 0,
                          0x2000, 0x3000, 0, 0x100000, 1 << 30, 0])   # 3 query heads on 2
    for name, args in wrong.items():
        with pytest.raises(B.SDVError) as e:
            getattr(B, name)(*args)
        assert e.value.code == B.SDV_EINVAL, name
