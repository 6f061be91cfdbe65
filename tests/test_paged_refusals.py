"""What the calls of the paged cache refuse, on the host, before anything is launched (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2411_09909_amd import binding

P = ctypes.c_void_p(0x1000)  # never dereferenced: validation fails first
ODD = ctypes.c_void_p(0x1002)


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def fmt(scale=binding.FP8_E5M2, asym=True, group=32):
    return binding.make_format(scale, asym, group)


def pool(pages=16, page=64, kv=8, dim=128, reserved=0, at=0x1000):
    return binding.AmxPagedPool(pages, page, kv, dim, reserved, at, at, at, at)


BAD_POOLS = [(dict(pages=0), -1), (dict(pages=-3), -1), (dict(kv=0), -1), (dict(kv=1025), -1), (dict(dim=0), -1), (dict(dim=96), -2),
             (dict(dim=256), -2), (dict(page=48), -2), (dict(page=8), -2), (dict(page=2048), -2), (dict(page=-64), -1),
             (dict(pages=(1 << 24) + 1), -1), (dict(reserved=1), -1), (dict(at=None), -1), (dict(at=0x1008), -1)]
BAD_FORMATS = [(fmt(group=16), -2), (fmt(group=64), -2), (fmt(group=-1), -2), (fmt(group=0), -1), (fmt(scale=7), -1), (fmt(scale=-1), -1)]


def test_sizes(lib):
    f, p = fmt(), pool(at=None)  # the pointers are not looked at
    assert lib.amxfp4_paged_codes_bytes(ctypes.byref(f), ctypes.byref(p)) == 16 * 8 * 64 * 64
    assert lib.amxfp4_paged_scales_bytes(ctypes.byref(f), ctypes.byref(p)) == 16 * 8 * 4 * 64 * 2
    assert lib.amxfp4_paged_scales_bytes(ctypes.byref(fmt(asym=False)), ctypes.byref(p)) == 16 * 8 * 4 * 64
    big = pool(pages=1 << 20, page=1024, kv=128, at=None)
    assert lib.amxfp4_paged_codes_bytes(ctypes.byref(f), ctypes.byref(big)) == (1 << 30) * 128 * 64
    for kw, _ in BAD_POOLS[:-2]:
        assert lib.amxfp4_paged_codes_bytes(ctypes.byref(f), ctypes.byref(pool(**kw))) == 0
    assert lib.amxfp4_paged_codes_bytes(None, ctypes.byref(p)) == 0 and lib.amxfp4_paged_codes_bytes(ctypes.byref(f), None) == 0
    w = lib.amxfp4_paged_attention_workspace_bytes
    assert w(ctypes.byref(f), ctypes.byref(p), 4, 12, 4, 0) == 0        # 12 query heads, 8 of keys
    assert w(ctypes.byref(f), ctypes.byref(p), 0, 16, 4, 0) == 0
    assert w(ctypes.byref(f), ctypes.byref(p), 4, 16, 4097, 0) == 0


def test_plan(lib):
    def call(seqs=4, rows=8, page=64, pages=16, width=4, at=(P,) * 10):
        return lib.amxfp4_paged_plan(at[0], at[1], seqs, rows, page, pages, width, *at[2:], None)
    apart = [ctypes.c_void_p(0x1000 * (i + 1)) for i in range(10)]
    for i in range(10):
        assert call(at=apart[:i] + [None] + apart[i + 1:]) == -1
        assert call(at=apart[:i] + [ODD] + apart[i + 1:]) == -1
    for kw in (dict(seqs=0), dict(seqs=4097), dict(rows=0), dict(rows=(1 << 30) + 1), dict(pages=0), dict(width=0), dict(page=0),
               dict(pages=(1 << 24) + 1), dict(width=(1 << 24) + 1)):
        assert call(at=apart, **kw) == -1, kw
    for page in (8, 24, 2048):
        assert call(at=apart, page=page) == -2
    # lens_out is lens, state_out is state: reading and writing would have no order
    assert call(at=apart[:5] + [apart[0]] + apart[6:]) == -1 and b"buffers of their own" in lib.amxfp4_last_error()
    assert call(at=apart[:9] + [apart[2]]) == -1


@pytest.mark.parametrize("which", ["write", "read", "attention"])
def test_formats_and_pools(lib, which):
    def call(f, p):
        if which == "write":
            return lib.amxfp4_paged_write(f, p, P, 4, 48 * 128, 32, P, P, 10000.0, P, None)
        if which == "read":
            return lib.amxfp4_paged_read(f, p, P, 4, 1, P, P, None)
        return lib.amxfp4_paged_attention(f, p, P, 4, 32, P, 4, 4, P, P, P, 0.1, 0, P, P, 1 << 40, None)
    good = pool()
    for f, status in BAD_FORMATS:
        assert call(ctypes.byref(f), ctypes.byref(good)) == status
    for kw, status in BAD_POOLS:
        assert call(ctypes.byref(fmt()), ctypes.byref(pool(**kw))) == status, kw
    assert call(None, ctypes.byref(good)) == -1 and call(ctypes.byref(fmt()), None) == -1


def test_write(lib):
    f, p = fmt(), pool()

    def call(src=P, rows=4, ld=48 * 128, heads=32, slots=P, positions=P, theta=10000.0, q=P):
        return lib.amxfp4_paged_write(ctypes.byref(f), ctypes.byref(p), src, rows, ld, heads, slots, positions, theta, q, None)
    for kw in (dict(src=None), dict(slots=None), dict(positions=None), dict(q=None), dict(rows=0), dict(rows=(1 << 24) + 1), dict(heads=0),
               dict(heads=1025), dict(ld=48 * 128 - 4), dict(ld=48 * 128 + 2), dict(theta=1.0), dict(theta=float("nan")),
               dict(theta=float("inf")), dict(src=ctypes.c_void_p(0x1004)), dict(q=ctypes.c_void_p(0x1008)), dict(slots=ODD),
               dict(positions=ODD)):
        assert call(**kw) == -1, kw


def test_read(lib):
    f, p = fmt(), pool()

    def call(slots=P, rows=4, dtype=1, k=P, v=P):
        return lib.amxfp4_paged_read(ctypes.byref(f), ctypes.byref(p), slots, rows, dtype, k, v, None)
    for kw in (dict(slots=None), dict(k=None), dict(v=None), dict(rows=0), dict(rows=(1 << 24) + 1), dict(dtype=2), dict(dtype=-1),
               dict(k=ctypes.c_void_p(0x1008)), dict(v=ctypes.c_void_p(0x1008)), dict(slots=ODD)):
        assert call(**kw) == -1, kw


def test_attention(lib):
    f, p = fmt(), pool()

    def call(q=P, rows=4, heads=32, table=P, seqs=4, width=4, lens=P, starts=P, positions=P, scale=0.1, keys=0, out=P, ws=P, size=1 << 40):
        return lib.amxfp4_paged_attention(ctypes.byref(f), ctypes.byref(p), q, rows, heads, table, seqs, width, lens, starts, positions,
                                          scale, keys, out, ws, size, None)
    for kw in (dict(q=None), dict(table=None), dict(lens=None), dict(starts=None), dict(positions=None), dict(out=None), dict(rows=0),
               dict(rows=(1 << 24) + 1), dict(heads=12), dict(heads=0), dict(rows=1 << 24, heads=136), dict(heads=2048), dict(seqs=0), dict(seqs=4097), dict(width=0),
               dict(width=(1 << 24) + 1), dict(keys=-1), dict(keys=(1 << 30) + 1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(q=ctypes.c_void_p(0x1008)), dict(out=ctypes.c_void_p(0x1008)),
               dict(table=ODD), dict(lens=ODD), dict(starts=ODD), dict(positions=ODD)):
        assert call(**kw) == -1, kw


def test_binding_refuses_host_tensors_and_wrong_ones(lib):
    f = fmt()
    kc, ks = torch.zeros(4, 2, 16, 64, dtype=torch.uint8), torch.zeros(4, 2, 4, 16, 2, dtype=torch.uint8)
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: binding.paged_read(f, (kc, ks, kc, ks), i),
                 lambda: binding.paged_write(f, torch.zeros(4, 8 * 128), (kc, ks, kc, ks), i, i, 4, 10000.0),
                 lambda: binding.paged_plan(i, i, i[:, None], i, i, 16, rows=4),
                 lambda: binding.paged_attention(f, torch.zeros(4, 4, 128, dtype=torch.bfloat16), (kc, ks, kc, ks), i[:, None], i, i, i, 0.1)):
        with pytest.raises(binding.AmxError, match="device memory only"):
            call()
