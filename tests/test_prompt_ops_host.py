"""C-ABI checks of the operators that take prompts in that need no GPU:
refusals before anything touches the device, and what the binding passes on."""
import os

import pytest

from paper_2302_11665_amd import build, sim
from test_ops_host import BAD_CACHES, WRONG_CACHES, cache


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(build.SIM_LIB):
        pytest.skip("HIP library not built")
    from paper_2302_11665_amd import ops
    return ops.lib()


def test_norm_refusals(L):
    def call(x=0x10000, r=0x20000, t=0, n=4, k=64, xs=64, rs=64, gain=None, eps=1e-6, s=0x30000, ss=64, codes=0x40000,
             scale=0x50000, held=None):
        return L.as_norm_i8(x, r, t, n, k, xs, rs, gain, eps, s, ss, codes, scale, held, None)

    for kw in (dict(x=None), dict(codes=None), dict(scale=None), dict(t=2), dict(t=-1), dict(n=-1), dict(k=0),
               dict(xs=63), dict(rs=63), dict(ss=63), dict(eps=-1e-9), dict(eps=float("nan")), dict(eps=float("inf")),
               dict(codes=0x40008), dict(r=None), dict(s=None), dict(s=0x10002), dict(s=0x10000, ss=65, xs=64),
               dict(s=0x20080 - 2), dict(s=0x10000 - 64, ss=100, xs=100), dict(s=0x10000 + 63 * 2, ss=128, xs=128),
               dict(s=0x20000 + 128 + 2, ss=127, rs=127), dict(s=0x10001)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
        assert "norm_i8" in sim.as_last_error()
    assert call(k=131073, xs=131073, rs=131073, ss=131073) == sim.AS_E_LIMITS
    assert call(n=1 << 21) == sim.AS_E_LIMITS
    assert call(n=0, x=None, codes=None, s=None) == sim.AS_OK


def test_linear_codes_refusals(L):
    def call(c=0x100, cs=0x200, t=4, k=64, w=0x1000, ws=0x2000, n=32, y=0x3000, yt=0, ys=32):
        return L.as_linear_i8_codes(c, cs, t, k, w, ws, None, n, y, yt, ys, None)

    for kw in (dict(c=None), dict(cs=None), dict(w=None), dict(ws=None), dict(y=None), dict(yt=3), dict(yt=-1),
               dict(t=-1), dict(k=0), dict(n=0), dict(ys=31), dict(w=0x1001), dict(c=0x108)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
        assert "linear_i8_codes" in sim.as_last_error()
    assert call(k=131073) == sim.AS_E_LIMITS and call(t=1 << 21) == sim.AS_E_LIMITS
    assert call(n=1 << 25, ys=1 << 25) == sim.AS_E_LIMITS
    assert call(t=0, c=None, y=None) == sim.AS_OK


def test_prompt_refusals(L):
    def call(q=0x100000, k=0x200000, v=0x300000, t=0, n=10, hq=4, hk=2, dim=64, qs=256, ks=128, vs=128, off=0x400,
             seqs=2, scale=0.1, out=0x400000, ws=None, wb=0):
        return L.as_attention_prompt(q, k, v, t, n, hq, hk, dim, qs, ks, vs, off, seqs, scale, out, ws, wb, None)

    for kw in (dict(q=None), dict(k=None), dict(v=None), dict(off=None), dict(out=None), dict(t=2), dict(n=-1),
               dict(seqs=-1), dict(hq=3), dict(hq=0), dict(hk=0), dict(hk=-2), dict(qs=-256), dict(qs=252), dict(ks=4),
               dict(vs=129), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(scale=2.1e38), dict(q=0x100008), dict(k=0x200004), dict(v=0x300002), dict(out=0x400004),
               dict(out=0x100000), dict(out=0x200000 + 8), dict(out=0x300000 - 8), dict(out=0x100000 + 9 * 512 + 504)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
        assert "attention_prompt" in sim.as_last_error()
    for kw in (dict(dim=96), dict(dim=0), dict(n=(1 << 26) + 1, hq=1, hk=1), dict(seqs=(1 << 20) + 1), dict(hq=8192),
               dict(n=1 << 22, hq=1024, hk=1), dict(n=1 << 18, seqs=1 << 18, hq=128, hk=128)):
        assert call(**kw) == sim.AS_E_LIMITS, kw
    assert call(ks=(1 << 26) + 8) == sim.AS_E_LIMITS and call(vs=1 << 40) == sim.AS_E_LIMITS
    # few sequences need no scratch memory; many need the list of their blocks
    assert L.as_attention_prompt_workspace(10, 4, 2, 64) == 0
    need = L.as_attention_prompt_workspace(1000, 4, 2, 65)
    assert need >= (1000 * 2 // 128 + 65) * 16
    for kw in (dict(wb=0), dict(wb=need - 1, ws=0x1000), dict(wb=need), dict(wb=need, ws=0x1010)):
        assert call(n=1000, seqs=65, **kw) == sim.AS_E_INVALID_ARG, kw
    assert call(n=0, q=None) == sim.AS_OK and call(seqs=0, off=None) == sim.AS_OK


def test_long_prompts_of_few_heads_need_scratch_memory(L):
    need = L.as_attention_prompt_workspace(3000, 1, 1, 1)
    assert need > 24 * 128 * 130 * 4  # a part for every block of 128 rows at least

    def call(ws=None, wb=0):
        return L.as_attention_prompt(0x1000000, 0x2000000, 0x3000000, 0, 3000, 1, 1, 64, 64, 64, 64, 0x400, 1, 0.1,
                                     0x4000000, ws, wb, None)

    for kw in (dict(), dict(wb=need - 1, ws=0x1000), dict(wb=need), dict(wb=need, ws=0x1010)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
    # and no more than 512 MiB, whatever the sizes
    for tokens in (100, 1000, 5000, 20000, 100000, 1 << 20, 1 << 26):
        for heads in (1, 2, 4, 8, 16, 64):
            for seqs in (1, 2, 7, 64):
                assert 0 <= L.as_attention_prompt_workspace(tokens, heads, heads, seqs) <= 512 << 20


def test_pages_refusals(L):
    def reserve(stack=0x100, count=0x200, pages=8, table=0x300, seqs=2, mp=4, page=32, length=0x400, add=0x500, n=10,
                nc=0x600, nl=0x700, off=0x800, seq=0x900, slot=0xa00, ws=0x1000, wb=1 << 20):
        return L.as_pages_reserve(stack, count, pages, table, seqs, mp, page, length, add, n, nc, nl, off, seq, slot, ws,
                                  wb, None)

    def release(stack=0x100, count=0x200, pages=8, table=0x300, seqs=2, mp=4, page=32, length=0x400, which=0x500,
                nc=0x600, nl=0x700):
        return L.as_pages_release(stack, count, pages, table, seqs, mp, page, length, which, nc, nl, None)

    for name, f, more in (("pages_reserve", reserve, [dict(add=None), dict(off=None), dict(seq=None), dict(slot=None),
                                                      dict(n=-1), dict(ws=None), dict(ws=0x1010), dict(wb=0)]),
                          ("pages_release", release, [dict(which=None)])):
        for kw in more + [dict(stack=None), dict(count=None), dict(table=None), dict(length=None), dict(nc=None),
                          dict(nl=None), dict(pages=-1), dict(seqs=-1), dict(mp=-1)]:
            assert f(**kw) == sim.AS_E_INVALID_ARG, (name, kw)
            assert name in sim.as_last_error()
        for kw in (dict(page=48), dict(page=0), dict(page=8192), dict(page=-32), dict(mp=1 << 26),
                   dict(seqs=(1 << 20) + 1)):
            assert f(**kw) == sim.AS_E_LIMITS, (name, kw)
    assert reserve(n=(1 << 30) + 1) == sim.AS_E_LIMITS
    assert L.as_pages_reserve_workspace(0) == 0 and L.as_pages_reserve_workspace(100) >= 400


def test_packed_append_refusals(L):
    def call(c=None, k=0x100, v=0x200, t=0, n=4, ks=128, vs=128, seq=0x300, slot=0x400):
        return L.as_cache_append_packed(c or cache(), k, v, t, n, ks, vs, seq, slot, None, None, None, None)

    for kw in (dict(k=None), dict(v=None), dict(seq=None), dict(slot=None), dict(t=2), dict(n=-1)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
        assert "cache_append_packed" in sim.as_last_error()
    for n in ((1 << 28) + 1, 1 << 28):
        assert call(n=n) == sim.AS_E_LIMITS
    for kw in BAD_CACHES:
        assert call(c=cache(**kw)) == sim.AS_E_LIMITS, kw
    for kw in WRONG_CACHES:
        assert call(c=cache(**kw)) == sim.AS_E_INVALID_ARG, kw
    assert call(n=0, k=None) == sim.AS_OK and call(c=cache(n_seqs=0), k=None) == sim.AS_OK


@pytest.fixture
def calls(L, monkeypatch):
    """The operators' binding over tensors on the CPU, its calls recorded and not made."""
    from paper_2302_11665_amd import ops
    made = []
    monkeypatch.setattr(ops, "_need", lambda x, name, dtypes, dim=None, device=None, contiguous=True: x)
    monkeypatch.setattr(ops, "_call", lambda fn, device, *args: made.append((fn.__name__, args)))
    return made


def test_norm_does_not_read_overlapping_rows_as_if_they_lay_apart(calls):
    import torch
    from paper_2302_11665_amd import ops
    line = torch.randn(400).to(torch.bfloat16)
    for x in (line[:64].expand(8, 64), line[:64].view(1, 1, 64).expand(2, 4, 64), line.unfold(0, 64, 3)[:9]):
        ops.norm_i8(x, x)
        (_, args), = calls
        assert args[3] == x.numel() // 64 and args[5] >= 64 and args[6] >= 64
        assert args[0] != x.data_ptr() and args[1] != x.data_ptr()
        calls.clear()
    with pytest.raises(sim.SimError):
        ops.norm_i8(torch.zeros(4, 64), torch.zeros(4, 64), out=torch.zeros(1, 64).expand(4, 64))
    assert not calls
