"""The 8-bit serving operators (quantize_tokens, int8_gemm, the paged K/V cache
and its attention) against their definitions in 64 bits, at the sizes and masks
where they can go wrong, and a run of them together as a server makes it."""
import numpy as np
import pytest

import serve_ref as ref
import workloads as wl

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def torch():
    import torch as t
    if not t.cuda.is_available():
        pytest.skip("no GPU")
    return t


@pytest.fixture(scope="module")
def vla():
    from paper_2606_08094_amd import vla
    return vla


def dev(torch, arr, elem=None):
    """numpy -> device, as bf16 when elem is "bf16"."""
    t = torch.from_numpy(np.ascontiguousarray(arr)).cuda()
    return t.to(torch.bfloat16) if elem == "bf16" else t


def host(t):
    return t.float().cpu().numpy()


# ---- quantize_tokens ----------------------------------------------------------

@pytest.mark.parametrize("elem", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,pad_x,pad_q", [
    (1, 0, 0, 0), (1, 1, 0, 0), (3, 7, 1, 2), (1, 16, 0, 0), (5, 64, 8, 16), (50, 720, 0, 0), (7, 1023, 1, 1), (2, 2048, 0, 0),
    (3, 2056, 0, 8), (4, 2560, 0, 0), (2, 6912, 8, 0), (1, 16384, 0, 0), (2, 16392, 0, 0), (2, 40000, 0, 0), (257, 64, 0, 0),
    (1027, 200, 0, 0), (1025, 1032, 0, 8), (1030, 2056, 8, 0), (1025, 4104, 0, 0),      # a wave per row
])
def test_quantize_tokens(torch, vla, elem, M, K, pad_x, pad_q):
    rng = np.random.default_rng(M * 1000 + K)
    x = ref.rounded(rng.standard_normal((M, K + pad_x)).astype(np.float32), elem)
    if M > 2 and K > 4:
        x[0] = 0.0                                         # a row of zeros
        x[1, :K] = x[1, :K] * np.float32(1e-7)              # below the least maximum
        x[2, :K:2] = x[2, 0] / 2                            # codes that end in a half
    want, r = ref.quantise(ref.rounded(x, elem)[:, :K], "i8")   # what the device gets
    q = torch.full((M, K + pad_q), 77, dtype=torch.int8, device="cuda")
    rr = torch.full((M,), NAN, device="cuda")
    vla.quantize_tokens(vla.ELEMS[elem], dev(torch, x, elem), M, K, K + pad_x, q, K + pad_q, rr)
    assert np.array_equal(host(rr), r)
    assert np.array_equal(q[:, :K].cpu().numpy(), want)
    assert bool((q[:, K:] == 77).all())                    # the columns behind the row


def test_quantize_tokens_marks_rows_that_are_not_finite(torch, vla):
    for K in (64, 100):                                    # both alignments of a row
        x = np.ones((5, K), np.float32)
        x[1, 3], x[2, K - 1], x[3, 0] = np.nan, np.inf, -np.inf
        for elem in ("f32", "bf16"):
            q = torch.full((5, K), 9, dtype=torch.int8, device="cuda")
            r = torch.zeros(5, device="cuda")
            vla.quantize_tokens(vla.ELEMS[elem], dev(torch, x, elem), 5, K, K, q, K, r)
            assert np.array_equal(np.isnan(host(r)), [False, True, True, True, False])
            assert np.array_equal(q.cpu().numpy(), np.array([127, 0, 0, 0, 127], np.int8)[:, None] * np.ones((1, K), np.int8))


# ---- int8_gemm ------------------------------------------------------------------

GEMM = [  # M, N, K, extra pitch of q, w, y
    (1, 1, 16, 0, 0, 0), (1, 5, 48, 16, 0, 3), (3, 16, 64, 0, 16, 0), (16, 17, 80, 0, 0, 0), (17, 100, 128, 16, 16, 4),
    (1, 2560, 2560, 0, 0, 0), (8, 720, 2048, 0, 0, 0), (31, 33, 720, 0, 0, 1), (50, 1601, 1024, 0, 0, 0), (64, 128, 6912, 0, 0, 0),
    (65, 257, 144, 0, 0, 0), (128, 256, 256, 0, 0, 0), (129, 255, 272, 0, 0, 0), (241, 1601, 720, 0, 0, 0), (256, 256, 64, 0, 0, 8),
    (257, 513, 1040, 16, 32, 0), (400, 720, 960, 0, 0, 0), (816, 512, 2048, 0, 0, 0), (2, 3, 0, 0, 0, 0), (300, 70, 0, 0, 0, 0),
    (1000, 96, 4096, 0, 0, 0), (37, 2000, 131056, 0, 0, 0), (700, 1300, 16, 0, 0, 0),
    (20, 300, 1040, 0, 0, 0), (33, 70, 4096, 16, 0, 1), (3, 8200, 2048, 0, 0, 0), (17, 8199, 3008, 0, 0, 0),   # few tokens
    (816, 2050, 528, 0, 0, 0), (1100, 1500, 2048, 0, 16, 0), (1000, 3000, 1040, 0, 0, 0), (1030, 2100, 528, 0, 0, 4),   # and
    (2049, 2050, 256, 0, 0, 0), (2100, 2100, 80, 0, 0, 0), (1500, 4100, 144, 16, 0, 0), (4100, 4100, 272, 0, 0, 0),     # tiles
]


@pytest.mark.parametrize("elem", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K,px,pw,py", GEMM)
def test_int8_gemm(torch, vla, elem, M, N, K, px, pw, py):
    g = torch.Generator(device="cuda").manual_seed(M + 7 * N + 31 * K)
    q = torch.randint(-128, 128, (M, K + px), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (N, K + pw), generator=g, device="cuda", dtype=torch.int8)
    r = torch.rand(M, generator=g, device="cuda") + 0.5
    ws = (torch.rand(N, generator=g, device="cuda") + 0.5) / 1000
    bias = torch.randn(N, generator=g, device="cuda") if (M + N) % 2 else None
    y = torch.full((M, N + py), 7.5, dtype=torch.float32 if elem == "f32" else torch.bfloat16, device="cuda")
    vla.int8_gemm(q, K + px, r, w, K + pw, ws, bias, M, N, K, vla.ELEMS[elem], y, N + py)
    # int8 products of up to 131056 terms are exact in float64
    acc = q[:, :K].double() @ w[:, :K].double().t().contiguous()
    prod = acc * ws.double() * r.double()[:, None] / 127
    want = prod + (bias.double() if bias is not None else 0)
    # float(sum), scale * r, / 127 and the product: four roundings, the bias one more
    tol = 4.01 * ref.U * prod.abs() + 1.01 * ref.U * want.abs()
    if elem == "bf16":
        tol = tol + 1.01 * ref.UB * want.abs()
    err = (y[:, :N].double() - want).abs()
    assert bool((err <= tol).all()), float((err - tol).max())
    assert bool((y[:, N:] == 7.5).all())


def test_int8_gemm_extreme_codes(torch, vla):
    """Every code -128: the largest sum there is, 128 * 128 * 131056 < 2^31."""
    K = 131056
    q = torch.full((2, K), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(2, device="cuda")
    y = torch.zeros(2, 2, device="cuda")
    vla.int8_gemm(q, K, one * 127, q, K, one, None, 2, 2, K, 0, y, 2)
    assert bool((y.double() / (128.0 * 128 * K) - 1).abs().max() <= 4 * ref.U)


def test_int8_gemm_nan_rows_stay_rows(torch, vla):
    for M in (5, 200):
        q = torch.ones(M, 64, dtype=torch.int8, device="cuda")
        r = torch.ones(M, device="cuda")
        r[2] = NAN
        y = torch.zeros(M, 32, device="cuda")
        vla.int8_gemm(q, 64, r, q[:1].expand(32, 64).contiguous(), 64, torch.ones(32, device="cuda"), None, M, 32, 64, 0, y, 32)
        nan = torch.isnan(y)
        assert bool(nan[2].all()) and int(nan.sum()) == 32


# ---- the paged cache --------------------------------------------------------------

class Paged:
    """A pool whose pages are dealt at random to requests of the given lengths,
    every row that no request has (and every row at first) filled with bits
    that read as NaN, with the rows that the requests have on the host."""

    def __init__(self, torch, vla, kind, hd, G, page, lens, news, seed=0, first=0, pad=0, spare=2, extra_pages=0):
        rng = np.random.default_rng(seed)
        self.kind, self.hd, self.G, self.page, self.lens, self.news = kind, hd, G, page, lens, news
        need = [-(-max(n, 0) // page) for n in lens]
        self.n_pages = sum(need) + spare
        self.max_pages = max(need + [1]) + extra_pages
        order = rng.permutation(self.n_pages)
        self.table = rng.integers(-5, 2 ** 31 - 1, (len(lens), self.max_pages)).astype(np.int32)  # entries past the end: anything
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, G, page, hd)
        dt = dict(f32=torch.float32, bf16=torch.bfloat16, i8=torch.int8, e4m3=torch.float8_e4m3fn)[kind]
        self.k, self.v = (torch.full(shape, 0x7F if kind == "e4m3" else 0, dtype=torch.uint8 if kind == "e4m3" else dt, device="cuda")
                          for _ in range(2))
        self.ks = self.vs = None
        if kind == "e4m3":
            self.k, self.v = self.k.view(dt), self.v.view(dt)
        elif kind != "i8":
            self.k.fill_(NAN), self.v.fill_(NAN)
        if kind in ref.TOP:
            self.ks, self.vs = (torch.full(shape[:3], NAN, device="cuda") for _ in range(2))
        self.pages = vla.KVPages(kind, self.n_pages, page, G, hd, self.k, self.v, self.ks, self.vs)
        self.starts = np.cumsum([first] + list(news)).astype(np.int32)
        self.T = int(self.starts[-1]) + pad
        self.elem = "f32" if kind == "f32" else "bf16"
        self.torch, self.vla, self.rng = torch, vla, rng
        # rows as float32 values that elem holds
        self.rows = [[ref.rounded(rng.standard_normal((max(n, 0), G, hd)).astype(np.float32), self.elem) for _ in range(2)] for n in lens]

    def batch(self, max_len=None, starts=None, lens=None, T=None):
        t = self.torch
        starts = self.starts if starts is None else starts
        lens = self.lens if lens is None else lens
        self.table_d, self.lens_d, self.starts_d = (t.from_numpy(np.asarray(x, np.int32).copy()).cuda() for x in (self.table, lens, starts))
        return self.vla.KVBatch(len(lens), self.max_pages, self.T if T is None else T, max(list(lens) + [0]) if max_len is None else max_len,
                                self.table_d, self.lens_d, self.starts_d)

    def fill(self):
        """Write every row of every request in one call."""
        lens = [max(n, 0) for n in self.lens]
        starts = np.cumsum([0] + lens)
        T = int(starts[-1])
        if T == 0:
            return
        both = [dev(self.torch, np.concatenate([r[i] for r in self.rows]), self.elem) for i in range(2)]
        b = self.batch(starts=starts, lens=lens, T=T)
        self.vla.kv_pages_write(self.pages, b, self.vla.ELEMS[self.elem], both[0], both[1], self.G * self.hd, self.hd)
        self.torch.cuda.synchronize()

    def values(self, b, which):
        """The rows of request b as the pages hold them, float64 [L][G][hd]."""
        x = self.rows[b][which]
        if self.kind not in ref.TOP:
            return x.astype(np.float64)
        code, r = ref.quantise(x, self.kind)
        return ref.code_values(code, self.kind) * (r / ref.TOP[self.kind]).astype(np.float64)[..., None]


CACHE = [  # hd, G, page, lengths
    (64, 1, 16, [1]), (64, 5, 16, [0, 17, 1, 33]), (128, 1, 32, [31, 32, 33]), (128, 2, 64, [200, 0, 5]), (256, 1, 256, [300, 7]),
    (64, 8, 128, [129, 1, 0]), (128, 5, 1024, [1025, 3]), (256, 3, 16, [50, 50, 50]),
]


@pytest.mark.parametrize("source", ["f32", "bf16"])
@pytest.mark.parametrize("kind", ["f32", "bf16", "i8", "e4m3"])
@pytest.mark.parametrize("hd,G,page,lens", CACHE)
def test_write_and_read_back(torch, vla, kind, source, hd, G, page, lens):
    """Codes, scales and values bit for bit; rows and pages of nobody untouched;
    rows behind a request's last untouched in the output."""
    P = Paged(torch, vla, kind, hd, G, page, lens, lens, seed=hd + G)
    P.elem = source
    P.rows = [[ref.rounded(P.rng.standard_normal((n, G, hd)).astype(np.float32), source) for _ in range(2)] for n in lens]
    before = [t.clone().view(torch.uint8) for t in (P.k, P.v)]
    P.fill()
    owned = np.zeros((P.n_pages, page), bool)
    for b, n in enumerate(lens):
        for j in range(n):
            owned[P.table[b, j // page], j % page] = True
    rest = torch.from_numpy(~owned).cuda()
    for t, old in ((P.k, before[0]), (P.v, before[1])):
        u, o = t.view(torch.uint8).transpose(1, 2), old.transpose(1, 2)
        assert torch.equal(u[rest], o[rest])
    if kind in ref.TOP:
        assert all(bool(torch.isnan(t.transpose(1, 2)[rest]).all()) for t in (P.ks, P.vs))
    for elem in ("f32", "bf16"):
        rows = max(lens) + 2
        out = [torch.full((len(lens), G, rows, hd), 3.25, dtype=torch.float32 if elem == "f32" else torch.bfloat16, device="cuda")
               for _ in range(2)]
        vla.kv_pages_read(P.pages, P.batch(), rows, vla.ELEMS[elem], out[0], out[1])
        for which in range(2):
            got = host(out[which])
            for b, n in enumerate(lens):
                x = P.rows[b][which]
                if kind in ref.TOP:
                    code, r = ref.quantise(x, kind)
                    val = ref.code_values(code, kind).astype(np.float32) * (r / ref.TOP[kind])[..., None]
                else:
                    val = ref.rounded(x, kind)
                assert np.array_equal(got[b, :, :n], ref.rounded(val, elem).transpose(1, 0, 2)), (elem, which, b)
                assert (got[b, :, n:] == 3.25).all()
        few = torch.full((len(lens), G, 1, hd), 3.25, dtype=out[0].dtype, device="cuda")   # fewer rows than there are
        vla.kv_pages_read(P.pages, P.batch(), 1, vla.ELEMS[elem], few, few.clone())
        assert np.array_equal(host(few), host(out[0][:, :, :1]))


@pytest.mark.parametrize("kind,source", [("i8", "bf16"), ("e4m3", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("hd,G,page,lens", [(64, 4, 256, [3001, 1, 0, 1100]), (64, 4, 64, [9000, 17, 7500]), (128, 2, 16, [1, 8300])])
def test_write_and_read_back_many_rows(torch, vla, kind, source, hd, G, page, lens):
    """As many rows as are written several to a wave."""
    test_write_and_read_back(torch, vla, kind, source, hd, G, page, lens)


def test_write_ties_zeros_and_rows_that_are_not_finite(torch, vla):
    lens = [6]
    for kind in ("i8", "e4m3"):
        P = Paged(torch, vla, kind, 64, 1, 16, lens, lens)
        k = P.rows[0][0]
        k[0] = 0
        k[1] = 1e-9
        k[2, :, ::2] = np.abs(k[2]).max() / 2
        k[3, 0, 5], k[4, 0, 0], k[5, 0, 63] = np.nan, np.inf, -np.inf
        P.fill()
        k = k.astype(np.float32)
        k[1] = ref.rounded(k[1], P.elem)             # what the device gets
        out = [torch.zeros(1, 1, 6, 64, device="cuda") for _ in range(2)]
        vla.kv_pages_read(P.pages, P.batch(), 6, 0, out[0], out[1])
        code, r = ref.quantise(k, kind)
        want = ref.code_values(code, kind).astype(np.float32) * (r / ref.TOP[kind])[..., None]
        assert np.array_equal(host(out[0])[0, 0], want[:, 0], equal_nan=True)
        assert np.isnan(want[3:]).all() and np.isfinite(want[:3]).all()
        # the finite rows of V next to them are what they were
        assert np.isfinite(host(out[1])).all()


def test_write_appends_leaves_the_rest_and_skips_what_has_no_page(torch, vla):
    """Tokens given inside a fused projection's rows; padding before and behind;
    a request without new tokens; a page id outside the pool; a row before the
    first and one past the page table."""
    G, hd, page = 2, 64, 16
    lens, news = [40, 20, 33, 2, 30], [3, 0, 2, 4, 1]
    P = Paged(torch, vla, "bf16", hd, G, page, lens, news, first=2, pad=3)
    P.table[2, 2] = P.n_pages                       # row 32 of request 2: outside the pool
    lens2 = list(lens)
    lens2[4] = P.max_pages * page + 1               # its new token is past the page table
    fused = torch.randn(P.T, 3 * G * hd, device="cuda").to(torch.bfloat16)
    b = P.batch(lens=lens2)
    old = [P.k.clone(), P.v.clone()]
    vla.kv_pages_write(P.pages, b, 1, fused[:, G * hd:], fused[:, 2 * G * hd:], 3 * G * hd, hd)
    for which, (t, o) in enumerate(((P.k, old[0]), (P.v, old[1]))):
        want = o.clone()
        for r, n in enumerate(news):
            for i in range(n):
                j, tok = lens2[r] - n + i, int(P.starts[r]) + i
                if 0 <= j < P.max_pages * page and 0 <= P.table[r, j // page] < P.n_pages:
                    want[int(P.table[r, j // page]), :, j % page] = fused[tok].view(3, G, hd)[1 + which]
        assert torch.equal(t.view(torch.int16), want.view(torch.int16))


def test_read_marks_rows_without_a_page(torch, vla):
    P = Paged(torch, vla, "i8", 64, 1, 16, [40], [0])
    P.fill()
    P.table[0, 1] = -1
    out = [torch.zeros(1, 1, 60, 64, device="cuda") for _ in range(2)]
    vla.kv_pages_read(P.pages, P.batch(lens=[P.max_pages * 16 + 5]), 60, 0, out[0], out[1])
    for o in out:
        nan = np.isnan(host(o))[0, 0]
        assert nan[16:32].all() and nan[48:53].all() and not nan[:16].any() and not nan[32:40].any()
        assert not nan[53:].any()                   # behind the last row: as it was


# ---- paged attention ---------------------------------------------------------------

def check_attention(torch, vla, P, R, causal, window, max_len=None, starts=None, lens=None, ldq_extra=0, in_place=False,
                    with_lse=True, scale=None, heads=None):
    """Run paged_attention on P's filled pool and compare every new token with the definition."""
    G, hd = P.G, P.hd
    H = G * R
    lens = P.lens if lens is None else lens
    scale = hd ** -0.5 if scale is None else scale
    f32 = P.kind == "f32"
    dt = torch.float32 if f32 else torch.bfloat16
    q = ref.rounded(P.rng.standard_normal((P.T, H * hd + ldq_extra)).astype(np.float32), P.elem)
    qd = dev(torch, q, P.elem)
    o = qd if in_place else torch.full((P.T, H * hd), 5.5, dtype=dt, device="cuda")
    lse = torch.full((P.T, H), 5.5, device="cuda") if with_lse else None
    batch = P.batch(max_len=max_len, lens=lens)
    n = vla.paged_attention_workspace(P.pages, batch, H)
    ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")   # NaN bits
    vla.paged_attention(P.pages, batch, H, 0 if f32 else 1, qd, H * hd + ldq_extra, o, H * hd + (ldq_extra if in_place else 0), scale,
                        causal=causal, window=window, lse=lse, workspace=ws if n else None, workspace_bytes=n)
    torch.cuda.synchronize()
    got = o.double().cpu().numpy()
    got_lse = lse.double().cpu().numpy() if with_lse else None
    mine = np.zeros(P.T, bool)
    worst = 0.0
    for b, L in enumerate(lens):
        L = max(L, 0)
        s0, s1 = int(P.starts[b]), int(P.starts[b + 1])
        if s0 == s1:
            continue
        mine[s0:s1] = True
        pos = L - (s1 - s0) + np.arange(s1 - s0)
        k, v = P.values(b, 0)[:L], P.values(b, 1)[:L]
        for h in heads or range(H):
            want, wl_, mag, big = ref.attention(q[s0:s1, h * hd:(h + 1) * hd].astype(np.float64), k[:, h // R], v[:, h // R],
                                                pos, scale, causal, window)
            # scores: hd products and a few roundings of scale and code scale; a score off by d moves p by d,
            # exp2 two steps; sums of L terms; bf16 inputs of the second product and the output one rounding each
            d = (hd + 8) * ref.U * big[:, None]
            low = 0.0 if f32 else ref.UB
            tol = (2 * d + 1.01 * low + (L + 24) * ref.U) * mag + (1.01 * low + 2 * ref.U) * np.abs(want) + 1e-30
            with np.errstate(invalid="ignore"):
                err = np.abs(got[s0:s1, h * hd:(h + 1) * hd] - want)
            nan = np.isnan(want)
            assert np.array_equal(np.isnan(got[s0:s1, h * hd:(h + 1) * hd]), nan), (b, h)
            ok = nan | (got[s0:s1, h * hd:(h + 1) * hd] == want) | (err <= tol)
            assert ok.all(), (b, h, np.nanmax(err), np.nanmax(err / tol))
            worst = max(worst, float(np.nanmax(np.where(nan, 0, err / tol), initial=0)))
            if with_lse:
                with np.errstate(invalid="ignore"):
                    e = np.abs(got_lse[s0:s1, h] - wl_)
                t = d[:, 0] + (L + 24) * ref.U + 4 * ref.U * np.abs(wl_)
                assert ((got_lse[s0:s1, h] == wl_) | (e <= t) | (np.isnan(wl_) & np.isnan(got_lse[s0:s1, h]))).all(), (b, h)
    rest = torch.from_numpy(~mine).cuda()
    if not in_place:
        assert bool((o[rest] == 5.5).all())
    else:
        assert np.array_equal(host(o)[~mine], q[~mine])
    if with_lse:
        assert bool((lse[rest] == 5.5).all())
    return worst


SHAPES = [  # hd, G, R, page, lengths, new tokens
    (64, 1, 1, 16, [1], [1]),
    (64, 2, 3, 16, [17, 1, 40], [1, 1, 1]),
    (128, 1, 8, 32, [33, 64, 5, 200], [1, 2, 5, 20]),
    (256, 1, 8, 64, [130, 66], [50, 50]),
    (128, 2, 4, 128, [700, 129, 0, 31], [1, 1, 0, 1]),
    (64, 5, 2, 16, [300, 9], [37, 9]),
    (64, 1, 16, 256, [257, 600], [3, 70]),
    (256, 2, 1, 16, [95, 500, 33], [33, 1, 33]),
    (128, 1, 5, 64, [1500], [130]),
]


@pytest.mark.parametrize("kind", ["bf16", "i8", "e4m3", "f32"])
@pytest.mark.parametrize("causal,window", [(False, 0), (True, 0), (True, 24), (False, 17)])
@pytest.mark.parametrize("hd,G,R,page,lens,news", SHAPES)
def test_paged_attention(torch, vla, kind, causal, window, hd, G, R, page, lens, news):
    P = Paged(torch, vla, kind, hd, G, page, lens, news, seed=hd + R, pad=2)
    P.fill()
    check_attention(torch, vla, P, R, causal, window)


@pytest.mark.parametrize("kind", ["bf16", "i8", "e4m3", "f32"])
def test_paged_attention_rows_that_see_nothing(torch, vla, kind):
    """No cached row at all, more new tokens than rows, a negative length, a
    window of one: o = 0 and lse = -infinity where nothing is seen."""
    P = Paged(torch, vla, kind, 64, 1, 16, [0, 3, 20, -7], [2, 9, 20, 1], first=1, pad=1)
    P.fill()
    for causal, window in ((True, 0), (False, 0), (True, 1), (False, 1)):
        check_attention(torch, vla, P, 3, causal, window)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
@pytest.mark.parametrize("max_len", [0, 1, 100, 1 << 20, 1 << 30])
def test_paged_attention_does_not_depend_on_the_length_hint(torch, vla, kind, max_len):
    P = Paged(torch, vla, kind, 64, 1, 32, [900, 40, 1], [1, 1, 1], extra_pages=2000)
    P.fill()
    check_attention(torch, vla, P, 4, True, 0, max_len=max_len)
    check_attention(torch, vla, P, 4, True, 200, max_len=max_len)


@pytest.mark.parametrize("kind", ["bf16", "i8", "f32"])
def test_paged_attention_many_requests(torch, vla, kind):
    """More requests than lanes, some without new tokens, at the start and the end too."""
    rng = np.random.default_rng(3)
    news = [int(n) for n in rng.integers(0, 4, 150)]
    news[0] = news[63] = news[64] = news[149] = 0
    lens = [n + int(x) for n, x in zip(news, rng.integers(0, 50, 150))]
    P = Paged(torch, vla, kind, 64, 1, 16, lens, news, pad=5)
    P.fill()
    check_attention(torch, vla, P, 2, True, 0)


@pytest.mark.parametrize("kind", ["bf16", "i8", "e4m3"])
@pytest.mark.parametrize("hd,G,R,lens,news", [
    (64, 4, 16, [900, 100, 2100], [800, 90, 1300]),        # tiles for several rounds of the chip
    (128, 8, 1, [3000, 40, 5000, 1], [1, 1, 1, 1]),        # one token each, the keys in many splits
    (256, 1, 8, [4000, 500], [1, 3]),
    (128, 1, 4, [9000], [40]),                             # one round of tiles, the keys in many splits
    (64, 5, 8, [4000, 700, 2500, 1, 900, 3100], [21, 3, 12, 1, 20, 7]),     # few rows each, more than a round of splits
])
def test_paged_attention_at_size(torch, vla, kind, hd, G, R, lens, news):
    """The shapes whose work is spread in other ways; some heads of each."""
    P = Paged(torch, vla, kind, hd, G, 64, lens, news, seed=11, pad=1)
    P.fill()
    check_attention(torch, vla, P, R, True, 0, heads=[0, G * R - 1])
    check_attention(torch, vla, P, R, True, 700, heads=[G * R // 2])


@pytest.mark.parametrize("kind,hd", [("bf16", 128), ("f32", 64), ("i8", 256)])
def test_paged_attention_pitch_in_place_and_without_lse(torch, vla, kind, hd):
    P = Paged(torch, vla, kind, hd, 2, 16, [70, 20], [20, 3], pad=1)
    P.fill()
    check_attention(torch, vla, P, 2, True, 0, ldq_extra=64, with_lse=False)
    check_attention(torch, vla, P, 2, True, 0, in_place=True)
    check_attention(torch, vla, P, 2, True, 0, ldq_extra=8, in_place=True, with_lse=False)
    long = Paged(torch, vla, kind, hd, 1, 16, [3000], [1])
    long.fill()
    check_attention(torch, vla, long, 4, True, 0, in_place=True)     # in place with the keys split


@pytest.mark.parametrize("kind", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("n", [12, 90])
def test_paged_attention_hidden_rows_have_no_influence(torch, vla, kind, n):
    """NaN and infinities in K and V rows of the chunk: the tokens before them
    (causal) and those whose window has passed them are what they would be
    without; the others are what the definition gives."""
    L, hd = n + 21, 64
    P = Paged(torch, vla, kind, hd, 1, 16, [L], [n])
    P.fill()

    def put(t, j, c, value):
        page, row = int(P.table[0, j // 16]), j % 16
        if kind == "e4m3":
            t.view(torch.uint8)[page, 0, row, c] = 0x7F
        else:
            t[page, 0, row, c] = value

    bad = {"k": [], "v": []}
    for j, c, value in ((25, 3, NAN), (28, 9, float("inf")), (28, 40, float("-inf")), (n + 10, 63, NAN)):
        put(P.v, j, c, value)
        bad["v"].append((j, c, NAN if kind == "e4m3" else value))
    put(P.k, n + 15, 7, NAN)
    bad["k"].append((n + 15, 7, NAN))
    true = P.values

    def values(b, which):
        x = true(b, which).copy()
        for j, c, value in bad["v" if which else "k"]:
            x[j, 0, c] = value
        return x

    P.values = values
    check_attention(torch, vla, P, 3, True, 0)
    check_attention(torch, vla, P, 3, True, 8)
    check_attention(torch, vla, P, 1, False, 8)


@pytest.mark.parametrize("kind", ["bf16", "i8"])
def test_paged_attention_pages_outside_the_pool(torch, vla, kind):
    """Tokens that see a row of such a page are NaN, the others are not; all
    tokens of a request longer than its page table are NaN."""
    for n in (30, 120):
        lens = [n + 20, n + 40]
        P = Paged(torch, vla, kind, 64, 1, 16, lens, [n, n])
        P.fill()
        P.table[0, 2] = -1 if n == 30 else P.n_pages           # rows 32 .. 47 of request 0
        true = P.values
        P.values = lambda b, w, true=true: np.where((np.arange(lens[b]) // 16 == 2)[:, None, None] & (b == 0), NAN, true(b, w))
        check_attention(torch, vla, P, 2, True, 0)
        check_attention(torch, vla, P, 2, True, 10)
        # a request with one row more than its page table has: all NaN, the other one finite again
        P.table[0, 2] = P.table[1, 2]

        def values(b, w, true=true):
            if b == 1:
                return np.full((P.max_pages * 16 + 1, 1, 64), NAN)
            x, m = true(0, w).copy(), min(lens[0], 48) - 32
            x[32:32 + m] = true(1, w)[32:32 + m]         # the page that both read
            return x

        P.values = values
        check_attention(torch, vla, P, 2, True, 0, lens=[lens[0], P.max_pages * 16 + 1])


@pytest.mark.parametrize("kind", ["bf16", "i8", "e4m3"])
def test_paged_attention_large_scores(torch, vla, kind):
    """Scores of a few hundred, both signs: the running maximum moves far."""
    P = Paged(torch, vla, kind, 128, 1, 32, [500], [40])
    for x in P.rows[0]:
        x *= 4
    P.fill()
    check_attention(torch, vla, P, 4, True, 0, scale=1.0)
    check_attention(torch, vla, P, 4, False, 0, scale=-1.0)
    check_attention(torch, vla, P, 4, False, 0, scale=0.0)


def test_offsets_past_32_bits(torch, vla):
    """A pool of more than 2^31 elements and 2^32 bytes: pages at its far end."""
    G, hd, page = 8, 256, 1024
    n_pages = 2 ** 32 // (G * hd * page * 2) + 2 + 1024         # > 2^31 elements, > 4 GiB of bf16
    k = torch.zeros(n_pages, G, page, hd, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    pages = vla.KVPages("bf16", n_pages, page, G, hd, k, v)
    T = 40
    x = torch.randn(2, T, G, hd, device="cuda").to(torch.bfloat16)
    table = torch.tensor([[n_pages - 1]], dtype=torch.int32, device="cuda")
    batch = vla.KVBatch(1, 1, T, T, table, torch.tensor([T], dtype=torch.int32, device="cuda"),
                        torch.tensor([0, T], dtype=torch.int32, device="cuda"))
    vla.kv_pages_write(pages, batch, 1, x[0], x[1], G * hd, hd)
    assert torch.equal(k[-1, :, :T].transpose(0, 1), x[0]) and torch.equal(v[-1, :, :T].transpose(0, 1), x[1])
    assert not bool(k[:-1].any())
    out = [torch.zeros(1, G, T, hd, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    vla.kv_pages_read(pages, batch, T, 1, out[0], out[1])
    assert torch.equal(out[0][0].transpose(0, 1), x[0]) and torch.equal(out[1][0].transpose(0, 1), x[1])
    q = torch.zeros(T, G * hd, dtype=torch.bfloat16, device="cuda")
    o = torch.zeros_like(q)
    n = vla.paged_attention_workspace(pages, batch, G)
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    vla.paged_attention(pages, batch, G, 1, q, G * hd, o, G * hd, 1.0, workspace=ws, workspace_bytes=n)
    want = x[1].double().mean(0).view(1, -1).expand(T, -1)       # equal scores: the mean
    tol = (2.02 * ref.UB + 64 * ref.U) * x[1].double().abs().mean(0).view(1, -1) + 2 * ref.UB * want.abs()
    assert bool(((o.double() - want).abs() <= tol).all())


# ---- together -----------------------------------------------------------------------

def test_dense_cache_through_pages_gives_the_same_chunk(torch, vla):
    """A prefix cache built for the action expert, kept in bf16 pages and read
    back, gives vla_denoise the same bytes: the chunk is the same bit for bit."""
    from vla_testlib import Pipeline
    cfg = wl.SMOLVLA_BF16.with_(n_layers=2, n_steps=2)
    inp = wl.make_batch(cfg, 1)
    pipe = Pipeline(cfg, wl.make_weights(cfg), inp)
    try:
        pipe.build_cache()
        tau = wl.uniform_schedule(2)
        want = pipe.denoise(tau).clone()
        Lc, G, P, hd = cfg.n_cache_layers, cfg.n_kv_heads, cfg.prefix_len, cfg.head_dim
        dense = pipe.cache.view(torch.bfloat16).view(Lc, 2, G, P, hd)
        saved = dense.clone()
        page = 32
        per = -(-P // page)
        k = torch.zeros(Lc * per, G, page, hd, dtype=torch.bfloat16, device="cuda")
        v = torch.zeros_like(k)
        pages = vla.KVPages("bf16", Lc * per, page, G, hd, k, v)
        lens = torch.tensor([P], dtype=torch.int32, device="cuda")
        starts = torch.tensor([0, P], dtype=torch.int32, device="cuda")
        table = torch.arange(Lc * per, dtype=torch.int32, device="cuda").flip(0).view(Lc, per).contiguous()
        for l in range(Lc):
            b = vla.KVBatch(1, per, P, P, table[l], lens, starts)
            vla.kv_pages_write(pages, b, 1, dense[l, 0], dense[l, 1], hd, P * hd)
        dense.zero_()
        for l in range(Lc):
            b = vla.KVBatch(1, per, 0, P, table[l], lens)
            vla.kv_pages_read(pages, b, P, 1, dense[l, 0], dense[l, 1])
        assert torch.equal(dense.view(torch.int16), saved.view(torch.int16))
        assert torch.equal(pipe.denoise(tau), want)
    finally:
        pipe.close()


class Layer:
    """An attention layer as a server runs it: int8 projections, an 8-bit paged
    cache, requests of different lengths."""

    def __init__(self, torch, vla, kind="i8", d=512, G=2, R=4, hd=128, page=32, lens=(70, 200, 33), news=(5, 1, 33), seed=5):
        self.torch, self.vla, self.d, self.G, self.H, self.hd = torch, vla, d, G, G * R, hd
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.P = Paged(torch, vla, kind, hd, G, page, list(lens), list(news), seed=seed, pad=2)
        self.P.fill()
        self.batch = self.P.batch()
        T, H = self.P.T, self.H
        self.n_qkv = (H + 2 * G) * hd
        self.wqkv = torch.randint(-127, 128, (self.n_qkv, d), generator=g, device="cuda", dtype=torch.int8)
        self.wo = torch.randint(-127, 128, (d, H * hd), generator=g, device="cuda", dtype=torch.int8)
        self.sqkv = (torch.rand(self.n_qkv, generator=g, device="cuda") + 0.5) / (73 * d ** 0.5)
        self.so = (torch.rand(d, generator=g, device="cuda") + 0.5) / (73 * (H * hd) ** 0.5)
        self.x = torch.randn(T, d, generator=g, device="cuda").to(torch.bfloat16)
        self.q8 = torch.zeros(T, max(d, H * hd), dtype=torch.int8, device="cuda")
        self.r = torch.zeros(T, device="cuda")
        self.qkv = torch.zeros(T, self.n_qkv, dtype=torch.bfloat16, device="cuda")
        self.o = torch.zeros(T, H * hd, dtype=torch.bfloat16, device="cuda")
        self.y = torch.zeros(T, d, dtype=torch.bfloat16, device="cuda")
        self.ws_bytes = vla.paged_attention_workspace(self.P.pages, self.batch, H)
        self.ws = torch.empty(max(self.ws_bytes, 16), dtype=torch.uint8, device="cuda")

    def run(self, stream=None):
        v, T, d, H, G, hd, n = self.vla, self.P.T, self.d, self.H, self.G, self.hd, self.n_qkv
        ld = self.q8.shape[1]
        v.quantize_tokens(1, self.x, T, d, d, self.q8, ld, self.r, stream)
        v.int8_gemm(self.q8, ld, self.r, self.wqkv, d, self.sqkv, None, T, n, d, 1, self.qkv, n, stream)
        v.kv_pages_write(self.P.pages, self.batch, 1, self.qkv[:, H * hd:], self.qkv[:, (H + G) * hd:], n, hd, stream)
        v.paged_attention(self.P.pages, self.batch, H, 1, self.qkv, n, self.o, H * hd, hd ** -0.5, causal=True, workspace=self.ws,
                          workspace_bytes=self.ws_bytes, stream=stream)
        v.quantize_tokens(1, self.o, T, H * hd, H * hd, self.q8, ld, self.r, stream)
        v.int8_gemm(self.q8, ld, self.r, self.wo, H * hd, self.so, None, T, d, H * hd, 1, self.y, d, stream)
        return self.y


@pytest.mark.parametrize("kind", ["i8", "e4m3", "bf16"])
def test_attention_layer_in_8_bits(torch, vla, kind):
    """Every step against its definition on the inputs that the step itself
    had, and the whole layer against 64 bits from its input alone, where an
    activation may land on the next code (one step of 127 of a row's maximum)."""
    lay = Layer(torch, vla, kind)
    y = host(lay.run())
    P, H, G, hd, d = lay.P, lay.H, lay.G, lay.hd, lay.d
    x = host(lay.x)

    def linear(x, w, s):
        code, r = ref.quantise(x, "i8")
        return (code.astype(np.float64) @ w.cpu().numpy().astype(np.float64).T) * (r.astype(np.float64)[:, None] / 127) * host(s).astype(np.float64)

    qkv = linear(x, lay.wqkv, lay.sqkv)
    got = host(lay.qkv).astype(np.float64)
    assert (np.abs(got - qkv) <= (1.01 * ref.UB + 5 * ref.U) * np.abs(qkv)).all()
    # the attention on the projection's own output
    o = np.zeros((P.T, H * hd))
    mags = np.zeros_like(o)
    for b in range(len(P.lens)):
        s0, s1, L = int(P.starts[b]), int(P.starts[b + 1]), P.lens[b]
        for g in range(G):
            rows = []
            for which in range(2):
                new = got[s0:s1, (H + which * G + g) * hd:(H + which * G + g + 1) * hd].astype(np.float32)
                vals = P.values(b, which)[:, g].copy()
                if kind in ref.TOP:
                    code, r = ref.quantise(new, kind)
                    new = ref.code_values(code, kind) * (r / ref.TOP[kind]).astype(np.float64)[:, None]
                vals[L - (s1 - s0):] = new
                rows.append(vals)
            for h in range(g * (H // G), (g + 1) * (H // G)):
                o[s0:s1, h * hd:(h + 1) * hd], _, mags[s0:s1, h * hd:(h + 1) * hd], _ = ref.attention(
                    got[s0:s1, h * hd:(h + 1) * hd], rows[0], rows[1], L - (s1 - s0) + np.arange(s1 - s0), hd ** -0.5, True, 0)
    live = slice(0, int(P.starts[-1]))
    got_o = host(lay.o).astype(np.float64)
    assert (np.abs(got_o - o)[live] <= (1.5 * ref.UB) * mags[live] + 1.1 * ref.UB * np.abs(o[live])).all()
    want = linear(got_o.astype(np.float32), lay.wo, lay.so)
    assert (np.abs(y - want)[live] <= (1.01 * ref.UB + 5 * ref.U) * np.abs(want[live])).all()


@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_captured_layer_sees_new_lengths_and_inputs(torch, vla, kind):
    """The layer captured once and replayed, with other inputs, lengths and page
    tables written into its tensors between the replays and eager work around
    them: each replay is what an eager run gives, bit for bit."""
    lay = Layer(torch, vla, kind, lens=(70, 200, 40), news=(5, 1, 33))
    lay.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            lay.run()
    torch.cuda.synchronize()
    for i, (lens, news) in enumerate([((70, 200, 40), (5, 1, 33)), ((60, 199, 33), (33, 5, 1)), ((39, 1, 34), (39, 0, 0)), ((5, 80, 6), (5, 28, 6))]):
        lay.x.normal_()
        lay.P.lens_d.copy_(torch.tensor(lens, dtype=torch.int32))
        lay.P.starts_d.copy_(torch.tensor(np.cumsum((0,) + news), dtype=torch.int32))
        lay.P.table_d[0, 0], lay.P.table_d[1, 0] = lay.P.table_d[1, 0].clone(), lay.P.table_d[0, 0].clone()
        before = [t.clone() for t in (lay.P.k, lay.P.v)]
        scales = [t.clone() for t in (lay.P.ks, lay.P.vs)] if lay.P.ks is not None else []
        lay.y.zero_(), lay.o.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (lay.y, lay.o, lay.P.k, lay.P.v)]
        lay.P.k.copy_(before[0]), lay.P.v.copy_(before[1])
        for t, old in zip((lay.P.ks, lay.P.vs), scales):
            t.copy_(old)
        lay.y.zero_(), lay.o.zero_()
        lay.run()
        torch.cuda.synchronize()
        for a, b in zip(got, (lay.y, lay.o, lay.P.k, lay.P.v)):
            assert torch.equal(a.view(torch.int8), b.view(torch.int8)), i


def test_layers_on_two_streams(torch, vla):
    """Two layers side by side, a workspace each, many times: what each gives alone."""
    lays = [Layer(torch, vla, "i8", lens=(3000, 50), news=(1, 1), seed=1), Layer(torch, vla, "bf16", lens=(800, 2000), news=(20, 3), seed=2)]
    want = [lay.run().clone() for lay in lays]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in lays]
    for _ in range(20):
        for lay, s in zip(lays, streams):
            with torch.cuda.stream(s):
                lay.y.zero_()
                lay.run(s)
    torch.cuda.synchronize()
    for lay, w in zip(lays, want):
        assert torch.equal(lay.y, w)


def test_results_do_not_change_from_run_to_run(torch, vla):
    lay = Layer(torch, vla, "e4m3", lens=(4000, 700, 50), news=(1, 40, 3))
    first = [t.clone() for t in (lay.run(), lay.o)]
    for _ in range(5):
        lay.run()
        assert torch.equal(lay.y, first[0]) and torch.equal(lay.o, first[1])
