"""Host-side refusals of the tree operators' entry points, without a GPU: every bad argument is turned down
before anything is launched."""
import pytest

from test_abi_tokens_cpu import CACHE, check, lib  # noqa: F401


def test_cache_append_rotary(lib):  # noqa: F811
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = ("k v sb st_ sh q qb qt qh qo ob ot oh dtype B W Hq H D block freqs rot halves pos kc vc ks vs pages tab M n cnt st s").split()
    base = dict(CACHE, k=0x1000, v=0x2000, sb=256, st_=128, sh=64, q=0x3000, qb=512, qt=256, qh=64, qo=0x4000, ob=512, ot=256, oh=64,
                dtype=B.SDV_F32, B=2, W=2, Hq=4, H=2, D=64, block=16, freqs=0x5000, rot=64, halves=1, pos=0, s=None)
    check(lib, "sdv_cache_append_rotary", names, base, [
        (dict(k=0), bad), (dict(v=0), bad), (dict(n=0), bad), (dict(kc=0), bad), (dict(tab=0), bad), (dict(freqs=0), bad), (dict(B=0), bad),
        (dict(W=0), bad), (dict(H=0), bad), (dict(D=96), bad), (dict(block=24), bad), (dict(pages=0), bad), (dict(sb=-1), bad),
        (dict(dtype=3), bad), (dict(rot=0), bad), (dict(rot=63), bad), (dict(rot=66), bad), (dict(rot=-2), bad), (dict(halves=2), bad),
        (dict(q=0), bad), (dict(qo=0), bad), (dict(Hq=0), bad), (dict(Hq=(1 << 20) + 1), bad), (dict(qt=-1), bad), (dict(oh=-1), bad),
        (dict(qo=0x3000, ot=128), bad), (dict(k=0x1002), align), (dict(q=0x3001), align), (dict(qo=0x4002), align),
        (dict(freqs=0x5004), align), (dict(pos=0x6002), align), (dict(kc=0x10008), align), (dict(st=0x7001), align),
        (dict(W=1 << 30, B=1 << 20), bad), (dict(M=1 << 28), bad)])


def test_tree_attend(lib):  # noqa: F811
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "q sb st_ sh dtype B W Hq H D block kc vc ks vs pages tab M n par cnt scale out lse st ws wsb s".split()
    wsb = B.sdv_tree_attend_workspace_bytes(2, 2, 4, 2, 64)
    assert wsb > 0 and wsb >= 256
    for sizes in ((0, 2, 4, 2, 64), (2, 65, 4, 2, 64), (2, 0, 4, 2, 64), (2, 2, 3, 2, 64), (2, 2, 4, 2, 80)):
        assert B.sdv_tree_attend_workspace_bytes(*sizes) == 0
    base = dict(CACHE, q=0x1000, sb=512, st_=256, sh=64, dtype=B.SDV_BF16, B=2, W=2, Hq=4, H=2, D=64, block=16, par=0x70000, scale=0.1,
                out=0x2000, lse=0x3000, ws=0x100000, wsb=wsb, s=None)
    check(lib, "sdv_tree_attend", names, base, [
        (dict(q=0), bad), (dict(out=0), bad), (dict(n=0), bad), (dict(par=0), bad), (dict(dtype=B.SDV_F32), bad), (dict(Hq=3), bad),
        (dict(H=0), bad), (dict(W=0), bad), (dict(W=65), bad), (dict(B=0), bad), (dict(D=32), bad), (dict(block=12), bad),
        (dict(scale=float("nan")), bad), (dict(scale=float("-inf")), bad), (dict(st_=-1), bad), (dict(q=0x1001), align),
        (dict(par=0x70002), align), (dict(cnt=0x70001), align), (dict(out=0x2001), align), (dict(lse=0x3002), align),
        (dict(ws=0), B.SDV_ENOWORKSPACE), (dict(wsb=wsb - 1), B.SDV_ENOWORKSPACE), (dict(ws=0x100080), align)])


def test_tree_verify(lib):  # noqa: F811
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "q qb qr p pb pr tok par B W V dtype T Td cnt seed coins race acc path nxt lr st s".split()
    base = dict(q=0x1000, qb=400, qr=100, p=0x2000, pb=400, pr=100, tok=0x3000, par=0x3100, B=2, W=4, V=100, dtype=B.SDV_BF16, T=1.0, Td=1.0,
                cnt=0, seed=1, coins=0, race=0, acc=0x4000, path=0x4100, nxt=0x5000, lr=0, st=0, s=None)
    check(lib, "sdv_tree_verify", names, base, [
        (dict(q=0), bad), (dict(tok=0), bad), (dict(par=0), bad), (dict(acc=0), bad), (dict(path=0), bad), (dict(nxt=0), bad), (dict(B=0), bad),
        (dict(B=(1 << 20) + 1), bad), (dict(W=0), bad), (dict(W=65), bad), (dict(V=0), bad), (dict(V=(1 << 30) + 1, qr=1 << 31, pr=1 << 31), bad),
        (dict(dtype=7), bad), (dict(T=0.0), bad), (dict(Td=float("nan")), bad), (dict(T=1e-10), bad), (dict(Td=1e10), bad), (dict(qr=99), bad),
        (dict(pr=99), bad), (dict(qb=-1), bad), (dict(pb=-1), bad), (dict(q=0x1001), align), (dict(p=0x2001), align), (dict(tok=0x3002), align),
        (dict(path=0x4101), align), (dict(race=0x7001), align), (dict(st=0x7002), align)])


def test_cache_keep(lib):  # noqa: F811
    from paper_2606_13426_gb300 import binding as B
    bad, align = B.SDV_EINVAL, B.SDV_EALIGN
    names = "path B W H D block kc vc ks vs pages tab M n st s".split()
    base = dict(CACHE, path=0x1000, B=2, W=2, H=2, D=64, block=16, s=None)
    check(lib, "sdv_cache_keep", names, base, [
        (dict(path=0), bad), (dict(n=0), bad), (dict(B=0), bad), (dict(W=0), bad), (dict(W=65), bad), (dict(H=0), bad), (dict(D=96), bad),
        (dict(block=8), bad), (dict(kc=0), bad), (dict(vc=0), bad), (dict(ks=0), bad), (dict(vs=0), bad), (dict(tab=0), bad), (dict(pages=0), bad),
        (dict(M=0), bad), (dict(B=1 << 20, H=1 << 15), bad), (dict(path=0x1001), align), (dict(n=0x60001), align), (dict(st=0x7001), align),
        (dict(vc=0x20001), align)])


def test_api_refuses_host_tensors():
    """The torch-facing helpers take CUDA tensors only; nothing is computed on the CPU."""
    import torch
    from paper_2606_13426_gb300 import api
    c = api.make_token_cache(2, 1, 16, 64, "cpu")
    i32 = torch.zeros(1, 1, dtype=torch.int32)
    one = torch.zeros(1, dtype=torch.int32)
    k = torch.zeros(1, 1, 1, 64)
    for call in (lambda: api.cache_append_rotary(c, k, k, i32, one, api.rotary_freqs(64, device="cpu")),
                 lambda: api.tree_attend(k.bfloat16(), c, i32, one, i32),
                 lambda: api.tree_verify(torch.zeros(1, 1, 8), torch.zeros(1, 1, 8), i32, i32),
                 lambda: api.cache_keep(c, i32, i32, one)):
        with pytest.raises(ValueError):
            call()


def test_rotary_freqs():
    import math
    import torch
    from paper_2606_13426_gb300 import api
    f = api.rotary_freqs(8, 100.0, device="cpu")
    assert f.dtype is torch.float64 and all(math.isclose(float(f[i]), 100.0 ** (-2 * i / 8), rel_tol=1e-14) for i in range(4))


def test_binding_functions_hand_their_arguments_on(lib):  # noqa: F811
    """The binding's function of each entry point: arguments in the header's order, refusals as SDVError."""
    from paper_2606_13426_gb300 import binding as B
    cache = [0x10000, 0x20000, 0x30000, 0x40000, 8, 0x50000, 4, 0x60000]
    wrong = dict(
        sdv_cache_append_rotary=[0x1000, 0x2000, 256, 128, 64, 0, 0, 0, 0, 0, 0, 0, 0, B.SDV_F32, 2, 2, 0, 2, 96, 16, 0x5000, 64, 1, 0] + cache
        + [0, 0, 0],                                        # D = 96
        sdv_tree_attend=[0x1000, 512, 256, 64, B.SDV_BF16, 2, 2, 3, 2, 64, 16] + cache + [0x70000, 0, 0.1, 0x2000, 0x3000, 0, 0x100000, 1 << 30, 0],
        sdv_tree_verify=[0x1000, 400, 100, 0x2000, 400, 100, 0x3000, 0x3100, 2, 65, 100, B.SDV_BF16, 1.0, 1.0, 0, 1, 0, 0, 0x4000, 0x4100, 0x5000,
                         0, 0, 0],                          # 65 nodes
        sdv_cache_keep=[0x1000, 2, 65, 2, 64, 16] + cache + [0, 0])
    for name, args in wrong.items():
        with pytest.raises(B.SDVError) as e:
            getattr(B, name)(*args)
        assert e.value.code == B.SDV_EINVAL, name
        with pytest.raises(TypeError):
            getattr(B, name)(*args[:-1])
