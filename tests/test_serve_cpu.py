"""Refusals of the 8-bit serving operators: every bad argument that the host
can see is turned away before a device is touched (no GPU needed)."""
import ctypes
import os
import random

import pytest


@pytest.fixture(scope="module")
def vla():
    from paper_2606_08094_amd import vla
    if not os.path.exists(vla.LIB_PATH):
        pytest.skip("libvla.so not built")
    return vla


def status(vla, code):
    return vla.STATUS[code]


@pytest.mark.parametrize("change,want", [
    (dict(elem=2), "VLA_E_ARG"), (dict(elem=-1), "VLA_E_ARG"),
    (dict(M=-1), "VLA_E_SHAPE"), (dict(K=-8), "VLA_E_SHAPE"),
    (dict(ldx=63), "VLA_E_SHAPE"), (dict(ldq=63), "VLA_E_SHAPE"),
    (dict(x=None), "VLA_E_ARG"), (dict(q=None), "VLA_E_ARG"), (dict(r=None), "VLA_E_ARG"),
    (dict(x=8), "VLA_E_ARG"), (dict(q=17), "VLA_E_ARG"), (dict(r=4), "VLA_E_ARG"),
    (dict(M=1 << 30), "VLA_E_UNSUPPORTED"),
    (dict(M=0), "VLA_OK"), (dict(M=0, x=None, q=None, r=None), "VLA_OK"),
])
def test_quantize_tokens_refusals(vla, change, want):
    a = dict(elem=1, x=16, M=2, K=64, ldx=64, q=16, ldq=64, r=16)
    a.update(change)
    got = vla.lib().vla_quantize_tokens(a["elem"], a["x"], a["M"], a["K"], a["ldx"], a["q"], a["ldq"], a["r"], None)
    assert status(vla, got) == want, vla.lib().vla_last_error()


@pytest.mark.parametrize("change,want", [
    (dict(elem=3), "VLA_E_ARG"),
    (dict(M=-1), "VLA_E_SHAPE"), (dict(N=-1), "VLA_E_SHAPE"), (dict(K=-16), "VLA_E_SHAPE"),
    (dict(K=40, ldq=48, ldw=48), "VLA_E_SHAPE"), (dict(ldq=72), "VLA_E_SHAPE"), (dict(ldw=72), "VLA_E_SHAPE"),
    (dict(ldq=48), "VLA_E_SHAPE"), (dict(ldw=48), "VLA_E_SHAPE"), (dict(ldy=31), "VLA_E_SHAPE"),
    (dict(K=131072, ldq=131072, ldw=131072), "VLA_E_SHAPE"),
    (dict(q=None), "VLA_E_ARG"), (dict(w=None), "VLA_E_ARG"), (dict(r=None), "VLA_E_ARG"),
    (dict(w_scale=None), "VLA_E_ARG"), (dict(y=None), "VLA_E_ARG"),
    (dict(q=8), "VLA_E_ARG"), (dict(w=8), "VLA_E_ARG"), (dict(bias=20), "VLA_E_ARG"), (dict(y=2), "VLA_E_ARG"),
    (dict(M=1 << 24, N=1 << 24, ldy=1 << 24), "VLA_E_UNSUPPORTED"),
    (dict(M=0), "VLA_OK"), (dict(N=0), "VLA_OK"),
])
def test_int8_gemm_refusals(vla, change, want):
    a = dict(q=16, ldq=64, r=16, w=16, ldw=64, w_scale=16, bias=None, M=2, N=32, K=64, elem=1, y=16, ldy=32)
    a.update(change)
    got = vla.lib().vla_int8_gemm(a["q"], a["ldq"], a["r"], a["w"], a["ldw"], a["w_scale"], a["bias"], a["M"], a["N"],
                                  a["K"], a["elem"], a["y"], a["ldy"], None)
    assert status(vla, got) == want, vla.lib().vla_last_error()


PAGES = dict(type=2, n_pages=4, page_size=32, n_kv_heads=2, head_dim=128, k=16, v=16, k_scale=16, v_scale=16)
BATCH = dict(n_requests=2, max_pages=2, n_tokens=3, max_len=60, page_table=16, kv_len=16, q_start=16)

BAD_SIZES = [
    (dict(type=4), {}, "VLA_E_ARG"), (dict(type=-1), {}, "VLA_E_ARG"),
    (dict(n_pages=0), {}, "VLA_E_SHAPE"), (dict(n_kv_heads=0), {}, "VLA_E_SHAPE"),
    (dict(n_kv_heads=257), {}, "VLA_E_UNSUPPORTED"),
    (dict(page_size=8), {}, "VLA_E_SHAPE"), (dict(page_size=48), {}, "VLA_E_SHAPE"), (dict(page_size=2048), {}, "VLA_E_SHAPE"),
    (dict(head_dim=96), {}, "VLA_E_UNSUPPORTED"), (dict(type=0, head_dim=512), {}, "VLA_E_UNSUPPORTED"),
    ({}, dict(n_requests=-1), "VLA_E_SHAPE"), ({}, dict(n_requests=65537), "VLA_E_UNSUPPORTED"),
    ({}, dict(max_pages=0), "VLA_E_SHAPE"), ({}, dict(max_pages=1 << 26), "VLA_E_SHAPE"),
    ({}, dict(n_tokens=-1), "VLA_E_SHAPE"), ({}, dict(n_tokens=(1 << 24) + 1), "VLA_E_UNSUPPORTED"),
    ({}, dict(max_len=-1), "VLA_E_SHAPE"),
]
BAD_BUFFERS = [
    (dict(k=None), {}), (dict(v=None), {}), (dict(k=8), {}), (dict(k_scale=None), {}), (dict(v_scale=None), {}),
    (dict(v_scale=4), {}), ({}, dict(page_table=None)), ({}, dict(kv_len=None)), ({}, dict(kv_len=18)),
    ({}, dict(page_table=17)),
]


def structs(vla, pages, batch):
    return vla.VlaKvPages(**{**PAGES, **pages}), vla.VlaKvBatch(**{**BATCH, **batch})


@pytest.mark.parametrize("pages,batch,want", BAD_SIZES)
def test_bad_pool_and_batch_sizes_are_refused_by_every_call(vla, pages, batch, want):
    p, b = structs(vla, pages, batch)
    L = vla.lib()
    f32 = p.type == 0
    elem = 0 if f32 else 1
    assert status(vla, L.vla_kv_pages_write(p, b, elem, 16, 16, 256, 128, None)) == want
    assert status(vla, L.vla_kv_pages_read(p, b, 8, elem, 16, 16, None)) == want
    assert L.vla_paged_attention_workspace(p, b, p.n_kv_heads) == ctypes.c_size_t(-1).value
    assert status(vla, L.vla_paged_attention(p, b, p.n_kv_heads, elem, 16, 1 << 17, 16, 1 << 17, 1.0, 0, 0, None, None, 0,
                                             None)) == want


@pytest.mark.parametrize("pages,batch", BAD_BUFFERS)
def test_bad_buffers_are_refused_by_every_call(vla, pages, batch):
    p, b = structs(vla, pages, batch)
    L = vla.lib()
    assert status(vla, L.vla_kv_pages_write(p, b, 1, 16, 16, 256, 128, None)) == "VLA_E_ARG"
    assert status(vla, L.vla_kv_pages_read(p, b, 8, 1, 16, 16, None)) == "VLA_E_ARG"
    assert status(vla, L.vla_paged_attention(p, b, 2, 1, 16, 256, 16, 256, 1.0, 0, 0, None, 16, 1 << 40, None)) == "VLA_E_ARG"


def test_null_structs_are_refused(vla):
    p, b = structs(vla, {}, {})
    L = vla.lib()
    for pp, bb in ((None, b), (p, None)):
        assert status(vla, L.vla_kv_pages_write(pp, bb, 1, 16, 16, 256, 128, None)) == "VLA_E_ARG"
        assert status(vla, L.vla_kv_pages_read(pp, bb, 8, 1, 16, 16, None)) == "VLA_E_ARG"
        assert status(vla, L.vla_paged_attention(pp, bb, 2, 1, 16, 256, 16, 256, 1.0, 0, 0, None, 16, 1 << 40, None)) == "VLA_E_ARG"
        assert L.vla_paged_attention_workspace(pp, bb, 2) == ctypes.c_size_t(-1).value


@pytest.mark.parametrize("change,want", [
    (dict(elem=2), "VLA_E_ARG"), (dict(k=None), "VLA_E_ARG"), (dict(v=8), "VLA_E_ARG"),
    (dict(ts=-256), "VLA_E_SHAPE"), (dict(ts=260), "VLA_E_SHAPE"), (dict(hs=4), "VLA_E_SHAPE"), (dict(hs=-128), "VLA_E_SHAPE"),
    (dict(q_start=None), "VLA_E_ARG"), (dict(q_start=2), "VLA_E_ARG"),
    (dict(n_tokens=0), "VLA_OK"), (dict(n_requests=0), "VLA_OK"),
])
def test_kv_pages_write_refusals(vla, change, want):
    a = dict(elem=1, k=16, v=16, ts=256, hs=128)
    a.update({k: v for k, v in change.items() if k in a})
    p, b = structs(vla, {}, {k: v for k, v in change.items() if k not in a})
    got = vla.lib().vla_kv_pages_write(p, b, a["elem"], a["k"], a["v"], a["ts"], a["hs"], None)
    assert status(vla, got) == want, vla.lib().vla_last_error()


@pytest.mark.parametrize("change,want", [
    (dict(elem=2), "VLA_E_ARG"), (dict(rows=-1), "VLA_E_SHAPE"), (dict(k=None), "VLA_E_ARG"), (dict(v=8), "VLA_E_ARG"),
    (dict(rows=1 << 30, n_requests=65536), "VLA_E_UNSUPPORTED"),
    (dict(rows=0), "VLA_OK"), (dict(n_requests=0), "VLA_OK"),
])
def test_kv_pages_read_refusals(vla, change, want):
    a = dict(elem=1, k=16, v=16, rows=4)
    a.update({k: v for k, v in change.items() if k in a})
    p, b = structs(vla, {}, {k: v for k, v in change.items() if k not in a})
    got = vla.lib().vla_kv_pages_read(p, b, a["rows"], a["elem"], a["k"], a["v"], None)
    assert status(vla, got) == want, vla.lib().vla_last_error()


@pytest.mark.parametrize("change,want", [
    (dict(heads=3), "VLA_E_SHAPE"), (dict(heads=0), "VLA_E_SHAPE"), (dict(heads=34, ldq=34 * 128, ldo=34 * 128), "VLA_E_UNSUPPORTED"),
    (dict(elem=0), "VLA_E_UNSUPPORTED"), (dict(elem=5), "VLA_E_ARG"),
    (dict(ldq=511), "VLA_E_SHAPE"), (dict(ldo=384), "VLA_E_SHAPE"), (dict(ldq=516), "VLA_E_SHAPE"),
    (dict(scale=float("inf")), "VLA_E_ARG"), (dict(scale=float("nan")), "VLA_E_ARG"),
    (dict(causal=2), "VLA_E_ARG"), (dict(window=-1), "VLA_E_SHAPE"),
    (dict(q=None), "VLA_E_ARG"), (dict(o=24), "VLA_E_ARG"), (dict(lse=4), "VLA_E_ARG"), (dict(q_start=None), "VLA_E_ARG"),
    (dict(n_tokens=1 << 24, heads=32, ldq=4096, ldo=4096), "VLA_E_UNSUPPORTED"),
    (dict(n_tokens=0), "VLA_OK"), (dict(n_requests=0), "VLA_OK"),
])
def test_paged_attention_refusals(vla, change, want):
    a = dict(heads=4, elem=1, q=16, ldq=512, o=16, ldo=512, scale=0.1, causal=1, window=0, lse=None)
    a.update({k: v for k, v in change.items() if k in a})
    p, b = structs(vla, {}, {k: v for k, v in change.items() if k not in a})
    got = vla.lib().vla_paged_attention(p, b, a["heads"], a["elem"], a["q"], a["ldq"], a["o"], a["ldo"], a["scale"],
                                        a["causal"], a["window"], a["lse"], 16, 1 << 45, None)
    assert status(vla, got) == want, vla.lib().vla_last_error()


def test_paged_attention_workspace_is_checked(vla):
    p, b = structs(vla, {}, dict(max_len=64 * 1024, max_pages=4096))
    L = vla.lib()
    need = L.vla_paged_attention_workspace(p, b, 4)
    assert 0 < need < 1 << 30
    call = lambda w, n: status(vla, L.vla_paged_attention(p, b, 4, 1, 16, 512, 16, 512, 0.1, 1, 0, None, w, n, None))  # noqa: E731
    assert call(16, need - 1) == "VLA_E_SHAPE"
    assert call(None, need) == "VLA_E_ARG"
    assert call(24, need) == "VLA_E_ARG"


def test_workspace_covers_every_window(vla):
    """The bound is asked for without a window: the work of a call with one may
    not need more (it is refused otherwise, with a NULL query after that check)."""
    L = vla.lib()
    for n_requests, n_tokens, max_len in ((1, 1, 100000), (64, 64, 8192), (3, 4096, 10000), (1, 17, 300)):
        p, b = structs(vla, {}, dict(n_requests=n_requests, n_tokens=n_tokens, max_len=max_len, max_pages=1 << 14))
        need = L.vla_paged_attention_workspace(p, b, 4)
        for window in (0, 1, 31, 1000, 50000, 2 ** 31 - 1):
            got = L.vla_paged_attention(p, b, 4, 1, None, 512, 16, 512, 0.1, 1, window, None, 16, need, None)
            assert status(vla, got) == "VLA_E_ARG" and b"q and o" in L.vla_last_error()


def test_workspace_covers_every_window_over_the_sizes(vla):
    L, rng = vla.lib(), random.Random(5)
    for _ in range(3000):
        kind, hd, G, R = rng.randrange(4), rng.choice([64, 128, 256]), rng.choice([1, 2, 5, 8]), rng.choice([1, 3, 8])
        B = int(2 ** rng.uniform(0, 7))
        p, b = structs(vla, dict(type=kind, head_dim=hd, n_kv_heads=G, k_scale=16, v_scale=16),
                       dict(n_requests=B, n_tokens=int(B * 2 ** rng.uniform(0, 10)), max_len=int(2 ** rng.uniform(0, 16)), max_pages=1 << 12))
        need = L.vla_paged_attention_workspace(p, b, G * R)
        window, ld, elem = int(2 ** rng.uniform(0, 17)), G * R * hd, 0 if kind == 0 else 1
        got = L.vla_paged_attention(p, b, G * R, elem, None, ld, 16, ld, 0.1, 1, window, None, 16, need, None)
        assert status(vla, got) == "VLA_E_ARG" and b"q and o" in L.vla_last_error(), (kind, hd, G, R, B, window)


def test_binding_turns_host_tensors_away(vla):
    """A host tensor's address would be read by a kernel: refused before the call."""
    import torch
    x = torch.zeros(2, 64)
    with pytest.raises(vla.VlaError, match="device memory"):
        vla.KVPages("f32", 1, 16, 1, 64, x, x)
    with pytest.raises(vla.VlaError, match="device memory"):
        vla.KVBatch(1, 1, 1, 1, x, 16, 16)
    for f, args in ((vla.quantize_tokens, (0, x, 2, 64, 64, 16, 64, 16)),
                    (vla.int8_gemm, (16, 64, 16, 16, 64, 16, x, 2, 2, 64, 0, 16, 2))):
        with pytest.raises(vla.VlaError, match="device memory"):
            f(*args)


def test_binding_reports_what_the_library_refuses(vla):
    p = vla.KVPages("i8", 4, 48, 2, 128, 16, 16, 16, 16)
    b = vla.KVBatch(2, 2, 3, 60, 16, 16, 16)
    with pytest.raises(vla.VlaError, match="power of two"):
        vla.paged_attention_workspace(p, b, 2)
    with pytest.raises(KeyError):
        vla.KVPages("fp4", 4, 32, 2, 128, 16, 16)
