"""C-ABI checks of the operators of a served model's step that need no GPU:
exports, struct layout, and refusals before anything touches the device."""
import ctypes
import os
import re

import pytest

from paper_2302_11665_amd import build, sim

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(build.SIM_LIB):
        pytest.skip("HIP library not built")
    from paper_2302_11665_amd import ops
    return ops.lib()


def cache(**over):
    from paper_2302_11665_amd import ops
    f = dict(n_pages=8, n_heads=2, dim=64, group=64, page=32, n_seqs=2, max_pages=4, reserved=0, k=0x1000, v=0x2000,
             k_par=0x3000, v_par=0x4000, pos=0x5000, acc=0x6000, page_table=0x7000)
    f.update(over)
    return ops.as_cache_t(**f)


def test_exports_every_declared_function(L):
    with open(os.path.join(ROOT, "include", "alpaserve_ops.h")) as f:
        src = re.sub(r"/\*.*?\*/", "", f.read(), flags=re.S)
    names = set(re.findall(r"\b(as_[a-z_0-9]+)\s*\(", src))
    assert {"as_linear_i8", "as_attention_kv4", "as_cache_append", "as_cache_evict"} <= names
    for n in names:
        assert hasattr(L, n), n


def test_struct_layout():
    from paper_2302_11665_amd import ops
    assert ctypes.sizeof(ops.as_cache_t) == 8 * 4 + 7 * 8
    assert ops.as_cache_t.k.offset == 32 and ops.as_cache_t.page_table.offset == 80


def test_linear_refusals(L):
    def call(x=0x100, xt=0, t=4, k=64, xs=64, w=0x1000, ws=0x2000, n=32, y=0x3000, yt=0, ys=32, work=0x4000, wb=1 << 20):
        return L.as_linear_i8(x, xt, t, k, xs, w, ws, None, n, y, yt, ys, work, wb, None)

    for kw in (dict(x=None), dict(w=None), dict(ws=None), dict(y=None), dict(xt=2), dict(xt=9), dict(yt=3),
               dict(yt=-1), dict(t=-1), dict(k=0), dict(n=0), dict(xs=63), dict(ys=31), dict(w=0x1001),
               dict(t=40, wb=0), dict(t=40, work=None), dict(t=40, work=0x4010)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
        assert "linear_i8" in sim.as_last_error()
    assert call(k=131073, xs=131073) == sim.AS_E_LIMITS
    assert call(t=1 << 21) == sim.AS_E_LIMITS
    assert call(n=1 << 25, ys=1 << 25) == sim.AS_E_LIMITS
    assert call(t=0, x=None, y=None, work=None, wb=0) == sim.AS_OK
    assert sim.as_last_error() == ""
    # a few tokens need no scratch memory, the tokens' codes and scales otherwise
    assert L.as_linear_i8_workspace(4, 64, 32) == 0
    assert L.as_linear_i8_workspace(40, 64, 32) >= 40 * 128 + 40 * 4


def test_quantize_refusals(L):
    def call(x=0x100, t=0, r=4, c=64, s=64, codes=0x1000, scale=0x2000):
        return L.as_quantize_i8(x, t, r, c, s, codes, scale, None)

    for kw in (dict(x=None), dict(codes=None), dict(scale=None), dict(t=5), dict(r=-1), dict(c=0), dict(s=63),
               dict(codes=0x1008)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
    assert call(c=131073, s=131073) == sim.AS_E_LIMITS
    assert call(r=0, x=None) == sim.AS_OK
    assert L.as_i8_bytes(17, 129) == 32 * 256 and L.as_i8_bytes(0, 5) == 0 and L.as_i8_bytes(1, 131073) == 0


BAD_CACHES = [dict(dim=96), dict(group=16), dict(group=128), dict(page=48), dict(page=0), dict(page=8192),
              dict(n_heads=0), dict(n_heads=2000), dict(max_pages=1 << 26)]
WRONG_CACHES = [dict(n_pages=-1), dict(n_seqs=-1), dict(max_pages=-1), dict(reserved=1), dict(k=None), dict(v=None),
                dict(k_par=None), dict(v_par=None), dict(page_table=None), dict(k=0x1004), dict(v_par=0x4002)]


def test_cache_refusals(L):
    calls = [lambda c: L.as_attention_kv4(c, 0x100, 0, 1, 4, 256, 256, 0x200, 0.1, 0x300, None, None, 0x400, 1 << 20,
                                          None),
             lambda c: L.as_cache_append(c, 0x100, 0x200, 0, 1, 128, 128, 128, 128, 0x300, None, None, None, None),
             lambda c: L.as_cache_evict(c, cache(), 0x100, 0x200, 8, 2, 0x300, 0x400, 1 << 20, None),
             lambda c: L.as_cache_evict(cache(), c, 0x100, 0x200, 8, 2, 0x300, 0x400, 1 << 20, None)]
    for f in calls:
        for kw in BAD_CACHES:
            assert f(cache(**kw)) == sim.AS_E_LIMITS, kw
        for kw in WRONG_CACHES:
            assert f(cache(**kw)) == sim.AS_E_INVALID_ARG, kw
        assert f(None) == sim.AS_E_INVALID_ARG
    for f in calls[2:]:
        assert f(cache(pos=None)) == sim.AS_E_INVALID_ARG
        assert f(cache(acc=None)) == sim.AS_E_INVALID_ARG


def test_attention_refusals(L):
    def call(c=None, q=0x100, t=0, nq=1, hq=4, qs=256, qt=256, n=0x200, scale=0.1, out=0x300, work=0x400, wb=1 << 20):
        return L.as_attention_kv4(c or cache(), q, t, nq, hq, qs, qt, n, scale, out, None, None, work, wb, None)

    for kw in (dict(q=None), dict(n=None), dict(out=None), dict(t=2), dict(nq=-1), dict(hq=3), dict(hq=0),
               dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=0x108),
               dict(qs=255), dict(qt=4)):
        assert call(**kw) == sim.AS_E_INVALID_ARG, kw
        assert "attention_kv4" in sim.as_last_error()
    assert call(hq=131072) == sim.AS_E_LIMITS and call(nq=70000) == sim.AS_E_LIMITS
    long = cache(max_pages=4096, n_pages=8192)
    need = L.as_attention_kv4_workspace(long, 1, 4, 1)
    assert need > 0 and call(c=long, wb=L.as_attention_kv4_workspace(long, 1, 4, 0) - 1) == sim.AS_E_INVALID_ARG
    assert call(nq=0, q=None) == sim.AS_OK and call(c=cache(n_seqs=0), q=None) == sim.AS_OK
    assert L.as_attention_kv4_workspace(None, 1, 4, 1) == 0


def test_append_and_evict_refusals(L):
    def app(k=0x100, v=0x200, t=0, n=1, start=0x300):
        return L.as_cache_append(cache(), k, v, t, n, 128, 128, 128, 128, start, None, None, None, None)

    for kw in (dict(k=None), dict(v=None), dict(start=None), dict(t=2), dict(n=-1)):
        assert app(**kw) == sim.AS_E_INVALID_ARG, kw
    assert app(n=1 << 25) == sim.AS_E_LIMITS
    assert app(n=0, k=None) == sim.AS_OK

    def ev(dst=None, n=0x100, total=0x200, keep=8, recent=2, out=0x300, work=0x400, wb=1 << 20):
        return L.as_cache_evict(cache(), dst or cache(), n, total, keep, recent, out, work, wb, None)

    for kw in (dict(n=None), dict(total=None), dict(out=None), dict(work=None), dict(wb=0), dict(work=0x410),
               dict(keep=0), dict(keep=129), dict(recent=-1), dict(recent=9), dict(dst=cache(dim=128)),
               dict(dst=cache(group=32)), dict(dst=cache(n_heads=1)), dict(dst=cache(n_seqs=1))):
        assert ev(**kw) == sim.AS_E_INVALID_ARG, kw
    assert L.as_cache_evict(cache(n_seqs=0), cache(n_seqs=0), None, None, 8, 2, None, None, 0, None) == sim.AS_OK


def test_profile_and_placement_problem():
    from paper_2302_11665_amd import served
    s = served.Shape(layers=10, hidden=64, heads=2, kv_heads=1, dim=64, inner=128, budget=32)
    p = served.profile(s, tokens=100, requests=3, block_bytes=1 << 20, cache_bytes=1 << 19, one=1e-3, many=2.4e-3,
                       batch=8)
    assert p.latency == pytest.approx(1.0) and p.slope == pytest.approx(0.2) and p.weight_mib == 25
    assert served.profile(s, 1, 0, 1, 0, 1e-3, 0.9e-3, 8).slope == 0.0
    gp = served.placement_problem([p, p], n_devices=4, device_mem_gb=1, rate=1.0, duration=10.0)
    assert [len(x["group_cfg"]) for x in gp.partitions] == [4, 2, 1]
    assert gp.stage_lat.shape == (2, 3, 4) and gp.stage_lat[0, 0, 0] == 1.0
    assert set(gp.model.tolist()) <= {0, 1} and (gp.weight_mib == 25).all()


@pytest.fixture
def calls(L, monkeypatch):
    """The operators' binding over tensors on the CPU, its calls recorded and not made."""
    from paper_2302_11665_amd import ops
    made = []

    def need(x, name, dtypes, dim=None, device=None, contiguous=True):
        return x

    monkeypatch.setattr(ops, "_need", need)
    monkeypatch.setattr(ops, "_call", lambda fn, device, *args: made.append((fn.__name__, args)))
    return made


def overlapping_rows():
    import torch
    line = torch.randn(400).to(torch.bfloat16)
    yield line[:64].expand(8, 64)                       # one row for all tokens
    yield line[:64].view(1, 1, 64).expand(2, 4, 64)     # the same, through a reshape
    yield line.unfold(0, 64, 3)[:9]                     # windows that share most of their values
    yield line[:1].expand(7, 1)                         # rows of one value


def test_linear_does_not_read_overlapping_rows_as_if_they_lay_apart(calls):
    import torch
    from paper_2302_11665_amd import ops
    for x in overlapping_rows():
        k = x.shape[-1]
        w = ops.PackedWeight(torch.zeros(ops.lib().as_i8_bytes(5, k), dtype=torch.int8), torch.zeros(5), 5, k)
        ops.linear_i8(x, w)
        ops.pack_weight(x.reshape(-1, k))
        for name, args in calls:
            rows, stride = args[2], args[4]
            assert rows == x.numel() // k > 1 and args[3] == k
            # the rows as they are passed: a copy, not x's memory with another stride
            assert stride >= k and args[0] != x.data_ptr(), (name, tuple(x.shape), x.stride(), stride)
        assert [name for name, _ in calls] == ["as_linear_i8", "as_quantize_i8"]
        calls.clear()


def test_linear_reads_rows_that_lie_apart_where_they_are(calls):
    import torch
    from paper_2302_11665_amd import ops
    big = torch.randn(6, 100).to(torch.bfloat16)
    w = ops.PackedWeight(torch.zeros(ops.lib().as_i8_bytes(5, 64), dtype=torch.int8), torch.zeros(5), 5, 64)
    for x, stride in ((big[:, 3:67], 100), (big[:, :64][::2], 200), (big[:1, :64], None), (big[0, :64], None)):
        ops.linear_i8(x, w)
        assert calls[-1][1][0] == x.data_ptr()
        assert calls[-1][1][4] == stride if stride else calls[-1][1][4] >= 64  # (of one row it does not matter)


def test_linear_refuses_an_output_with_overlapping_rows(calls):
    import torch
    from paper_2302_11665_amd import ops
    x = torch.randn(4, 64).to(torch.bfloat16)
    w = ops.PackedWeight(torch.zeros(ops.lib().as_i8_bytes(5, 64), dtype=torch.int8), torch.zeros(5), 5, 64)
    for out in (torch.zeros(1, 5).expand(4, 5), torch.zeros(40).unfold(0, 5, 2)[:4], torch.zeros(40).as_strided((4, 5), (4, 1))):
        with pytest.raises(sim.SimError):
            ops.linear_i8(x, w, out=out)
    assert not calls
    ops.linear_i8(x[:1], w, out=torch.zeros(9).as_strided((1, 5), (2, 1)))  # one row overlaps nothing
    assert calls[-1][1][11] == 5


def test_a_cache_keeps_the_arrays_that_its_calls_use():
    """A cache's calls take the addresses that it was made with: another array needs another cache."""
    from paper_2302_11665_amd import ops
    c = object.__new__(ops.Cache)
    for name in ("k", "v", "k_par", "v_par", "pos", "acc", "page_table"):
        with pytest.raises(AttributeError):
            setattr(c, name, None)


def test_evict_refuses_new_lengths_over_the_old_ones(L):
    """Workgroups of other heads still read the lengths and totals when the first one writes the new lengths."""
    for out in (0x100, 0x104, 0xfc, 0x200, 0x204):
        assert L.as_cache_evict(cache(), cache(), 0x100, 0x200, 8, 2, out, 0x400, 1 << 20, None) == sim.AS_E_INVALID_ARG
        assert "out_length" in sim.as_last_error()


def test_a_cache_without_room_to_grow_is_refused():
    """With no slack, a token behind a full table would be lost; with no budget, a cut keeps nothing."""
    from paper_2302_11665_amd import served
    f = dict(layers=1, hidden=64, heads=2, kv_heads=1, dim=64, inner=128, budget=64)
    for kw in (dict(slack=0), dict(slack=-1), dict(budget=0), dict(recent=-1)):
        with pytest.raises(ValueError):
            served.Shape(**{**f, **kw})
    served.Shape(**f, slack=1, recent=0)


def test_sizes_whose_launch_would_have_too_many_threads_are_refused(L):
    """A launch has fewer than 2^32 threads a dimension: 256 a row of codes, 256 for 32 tokens that a cut keeps."""
    assert L.as_quantize_i8(0x100, 0, 1 << 24, 64, 64, 0x1000, 0x2000, None) == sim.AS_E_LIMITS
    assert L.as_i8_bytes(1 << 24, 64) == 0 and L.as_i8_bytes((1 << 24) - 1, 64) == (1 << 24) * 128
    wide = cache(page=4096, max_pages=1 << 18)
    for keep in ((1 << 29) - 31, 1 << 29, 1 << 30):
        assert L.as_cache_evict(wide, wide, 0x100, 0x200, keep, 2, 0x300, 0x400, 1 << 62, None) == sim.AS_E_LIMITS


def test_attention_asks_for_scratch_memory_with_the_tensors_device_current(monkeypatch):
    """The size follows from the device's compute units: another device's would not do."""
    import contextlib
    import torch
    from paper_2302_11665_amd import ops
    current, seen = [5], []

    @contextlib.contextmanager
    def device(index):
        current.append(index)
        yield
        current.pop()

    class Lib:
        def as_attention_kv4_workspace(self, *args):
            seen.append(current[-1])
            return 512

        def as_attention_kv4(self, *args):
            seen.append(current[-1])
            return sim.AS_OK

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: current[-1], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(ops, "lib", Lib)
    c = object.__new__(ops.Cache)
    object.__setattr__(c, "_c", cache())
    object.__setattr__(c, "k", torch.zeros(1))
    ops.attention_kv4(torch.zeros(2, 1, 4, 64, dtype=torch.float16), c, torch.zeros(2, dtype=torch.int32))
    assert len(seen) == 2 and 5 not in seen


def test_attention_refuses_scales_beyond_fp32_once_times_log2_e(L):
    def call(scale):
        return L.as_attention_kv4(cache(), 0x100, 0, 1, 4, 256, 256, 0x200, scale, 0x300, None, None, None, 0, None)

    for scale in (2.4e38, 2.9e38, 3.4e38):
        assert call(scale) == sim.AS_E_INVALID_ARG and "scale" in sim.as_last_error()


def test_queries_of_one_sequence_or_token_at_any_stride(monkeypatch):
    """The stride of a dimension of one entry is never used, and torch leaves anything there."""
    import torch
    from paper_2302_11665_amd import ops
    passed = []

    class Lib:
        def as_attention_kv4_workspace(self, *args):
            return 0

        def as_attention_kv4(self, *args):
            pass

    monkeypatch.setattr(ops, "lib", Lib)
    monkeypatch.setattr(ops, "_on", lambda fn, device, *args: fn(*args), raising=False)
    monkeypatch.setattr(ops, "_call", lambda fn, device, *args: passed.append(args))
    line = torch.randn(4096).to(torch.bfloat16)
    for seqs, strides in ((1, (1003, 256, 64, 1)), (1, (1003, 77, 64, 1)), (2, (512, 77, 64, 1)), (1, (0, 0, 64, 1)),
                          (2, (0, 3, 64, 1))):
        c = object.__new__(ops.Cache)
        object.__setattr__(c, "_c", cache(n_seqs=seqs))
        object.__setattr__(c, "k", torch.zeros(1))
        q = line.as_strided((seqs, 1, 4, 64), strides)
        ops.attention_kv4(q, c, torch.zeros(seqs, dtype=torch.int32))
        _, at, _, queries, heads, q_seq, q_token = passed[-1][:7]
        assert (queries, heads) == (1, 4) and q_seq % 8 == 0 and q_token % 8 == 0 and at % 16 == 0
        assert at == q.data_ptr() and (seqs == 1 or q_seq == strides[0])  # where they are, not a copy


def test_an_empty_cache_has_the_sizes_that_were_asked_for(L):
    """Sizes that the storage cannot hold are refused, not rounded to others."""
    import torch
    from paper_2302_11665_amd import ops
    table = torch.zeros(1, 1, dtype=torch.int32)
    for kw in (dict(dim=128, group=48), dict(dim=130), dict(dim=64, group=50), dict(dim=64, group=0), dict(dim=64, page=48),
               dict(dim=64, group=128), dict(dim=65, group=33)):
        with pytest.raises(sim.SimError, match="(?s)channels|slots"):
            ops.Cache.empty(1, 1, page_table=table, device="cpu", **kw)


def test_counts_that_do_not_fit_32_bits_are_refused(calls):
    """ctypes would pass their lowest bits."""
    import torch
    from paper_2302_11665_amd import ops
    c = object.__new__(ops.Cache)
    object.__setattr__(c, "_c", cache())
    object.__setattr__(c, "k", torch.zeros(1))
    n = torch.zeros(2, dtype=torch.int32)
    for keep, recent in ((2 ** 32 + 8, 2), (8, 2 ** 32 + 2), (8, -2 ** 32 + 2), (2 ** 31, 0)):
        with pytest.raises(sim.SimError):
            ops.cache_evict(c, c, n, n, keep=keep, recent=recent)
    assert not calls
    ops.cache_evict(c, c, n, n, keep=8, recent=2)
    assert calls[-1][1][4:6] == (8, 2)
