"""Every form of the linear layers' kernels (QASR_LINEAR names one), bit for bit against the definition: remainders of rows,
channels and codes, all stages of their rings, weights past the cache or through it, one matrix and groups.

The launch chooses a form by a model of its time, so a size alone does not say which kernel it tests."""
import pytest
import torch

import paper_2103_16827_amd as Q

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.float16, torch.bfloat16]
FILL = 77
# rows and channels of a tile, in the order of linear.hip's tables
FORMS = [(16, 16), (16, 32), (16, 64), (32, 32), (32, 64), (64, 64), (64, 128), (128, 128), (128, 256), (256, 256)]
ROW_FORMS = [(16, 16), (16, 32), (32, 32), (64, 64), (64, 128), (128, 256)]
SHORT_ROW_FORMS = 3                  # those that take fewer than 16 codes


def draw(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    codes = lambda *s: torch.randint(-128, 128, s, generator=g, device="cuda", dtype=torch.int32).to(torch.int8)
    scales = lambda *s: (torch.rand(*s, generator=g, device="cuda") * 0.02 + 0.001) * (1 - 2 * (torch.rand(*s, generator=g, device="cuda") < 0.2).float())
    return g, codes, scales


def strided(host, stride, shift):
    """The matrix with rows `stride` apart in a buffer that begins `shift` elements into its allocation."""
    raw = torch.full((shift + host.shape[0] * stride + 64,), FILL, dtype=host.dtype, device="cuda")
    view = raw.as_strided(host.shape, (stride, 1), shift)
    view.copy_(host)
    return view


def bits(t):
    return t.contiguous().view(torch.int32 if t.dtype == torch.float32 else torch.int16)


def definition(x, xs, w, ws, bias, dtype):
    acc = (x.double() @ w.double().t().contiguous()).float()
    return (acc * xs[:, None] * ws + (0.0 if bias is None else bias)).to(dtype)


def layer(dtype, M, N, K, bias, pad, shift, ypad, seed):
    g, codes, scales = draw(seed)
    x, w, xs, ws = codes(M, K), codes(N, K), scales(M), scales(N)
    b = torch.randn(N, generator=g, device="cuda") * 20 if bias else None
    y = torch.full((M * (N + ypad) + 64,), float(FILL), dtype=dtype, device="cuda")
    want = y.clone()
    want.as_strided((M, N), (N + ypad, 1), 0).copy_(definition(x, xs, w, ws, b, dtype))
    Q.linear_int8(strided(x, K + pad, shift), xs, strided(w, K + pad, shift), ws, b, y.as_strided((M, N), (N + ypad, 1), 0))
    assert torch.equal(bits(y), bits(want)), f"{M} x {N} x {K}, pad {pad}, shift {shift}, ypad {ypad}"


def experts(dtype, sizes, N, K, bias, pad, shift, seed):
    """Groups of these sizes behind two rows of none and before three, rows by an index with unknown ones among them."""
    g, codes, scales = draw(seed)
    E, T, M = len(sizes), 50, sum(sizes) + 5
    x, xs, w, ws = codes(T, K), scales(T), codes(E, N, K), scales(E, N)
    b = torch.randn(E, N, generator=g, device="cuda") if bias else None
    index = torch.randint(0, T, (M,), generator=g, device="cuda", dtype=torch.int32)
    index[5::11] = -1
    index[7::13] = T
    there = (index >= 0) & (index < T)
    i = index.long() * there
    y = torch.full((M, N), float(FILL), dtype=dtype, device="cuda")
    want, lo, offsets = y.clone(), 2, [2]
    for e, n in enumerate(sizes):
        hi = lo + n
        if n:
            want[lo:hi] = definition(x[i[lo:hi]] * there[lo:hi, None], xs[i[lo:hi]] * there[lo:hi], w[e], ws[e], None if b is None else b[e], dtype)
        lo = hi
        offsets.append(lo)
    wv = strided(w.reshape(E * N, K), K + pad, shift).as_strided((E, N, K), (N * (K + pad), K + pad, 1), shift)
    Q.experts_int8(strided(x, K + pad, shift), xs, torch.tensor(offsets, dtype=torch.int32, device="cuda"), index, wv, ws, b, y)
    assert torch.equal(bits(y), bits(want)), f"groups {sizes} x {N} x {K}, pad {pad}, shift {shift}"


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("once", [1, 2])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_forms(form, once, dtype, tuning_env):
    """Rows on 16-byte boundaries; K of one step, of whole steps and of a last one with 16 or 112 codes, fewer and more than a ring holds."""
    BM, BN = FORMS[form]
    print(f"[case] form {BM} x {BN} once {once} {dtype}", flush=True)
    tuning_env("QASR_LINEAR", f"{form + 1},{once}")
    for j, K in enumerate([16, 112, 128, 256, 272, 368, 640, 1136, 1152]):
        layer(dtype, 2 * BM + 5, 2 * BN, K, j % 2 == 0, 0, 0, 0, 10 * form + j)                  # whole lines of y
        layer(dtype, BM + BM // 2 + 1, BN + BN // 2 + 7, K, j % 2 == 1, 16, 16, j % 3, 10 * form + j)
    layer(dtype, BM, BN, 512, True, 0, 0, 0, form)
    layer(dtype, 1, 3, 144, True, 0, 0, 5, form)
    for j, K in enumerate([16, 272, 368, 1152]):
        experts(dtype, [BM + 3, 0, 1, 2 * BM, 0, BM // 2 + 1, 17], BN + 12, K, j % 2 == 0, 16 * (j % 2), 0, 20 * form + j)
    experts(dtype, [0] * 60 + [3, BM, 0, 0, 5, 0, BM + 1], 2 * BN, 400, True, 0, 0, form)         # more groups than lanes


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", range(len(ROW_FORMS)))
def test_forms_of_any_alignment(form, dtype, tuning_env):
    BM, BN = ROW_FORMS[form]
    print(f"[case] rows {BM} x {BN} {dtype}", flush=True)
    tuning_env("QASR_LINEAR", str(form + 1))
    short = [1, 5, 15] if form < SHORT_ROW_FORMS else []
    for j, K in enumerate(short + [17, 31, 127, 129, 143, 255, 257, 1003]):
        layer(dtype, 2 * BM + 5, 2 * BN, K, j % 2 == 0, 0, 0, 0, 10 * form + j)
        layer(dtype, BM + BM // 2 + 1, BN + BN // 2 + 7, K, j % 2 == 1, 3, 1, j % 3, 10 * form + j)
    for K in (16, 128, 400):                                       # rows that begin off a boundary
        layer(dtype, BM + 3, BN + 5, K, True, 0, 3, 0, form)
    for j, K in enumerate(short + [16, 129, 520, 1003]):
        experts(dtype, [BM + 3, 0, 1, 2 * BM, 0, BM // 2 + 1, 17], BN + 12, K, j % 2 == 0, 5 * (j % 2), 1, 20 * form + j)
    experts(dtype, [0] * 60 + [3, BM, 0, 0, 5, 0, BM + 1], 2 * BN, 401, True, 0, 0, form)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 33, 16), (1, 8200, 2048), (2, 16, 4096), (3, 40, 80), (5, 300, 1008), (8, 77, 1024), (13, 20, 624), (16, 130, 512), (16, 64, 16)])
def test_floats_in_one_launch(M, N, K, dtype):
    """Up to 16 float tokens and 8192 elements are quantised by the layer's workgroups: the same bits as the two calls, and as the definition."""
    print(f"[case] floats in one launch {M} x {N} x {K} {dtype}", flush=True)
    g, codes, scales = draw(M + N + K)
    x = (torch.randn(M, K, generator=g, device="cuda") * torch.rand(M, 1, generator=g, device="cuda") * 9)
    x[M // 2, K // 2] = float("inf")
    if M > 2:
        x[0] = 0.0
        x[1] = float("nan")
        x[M - 1, ::3] = float("-inf")
        x[M - 1, 1] = float("nan")
    if M > 4:
        x[3] = float("inf")
        x[4] = x[4] * 1e-30
    x = x.to(dtype)
    w, ws, b = codes(N, K), scales(N), torch.randn(N, generator=g, device="cuda")
    for pad, wpad, bias, ydt in ((0, 0, b, torch.float32), (16 // x.element_size(), 16, None, torch.bfloat16), (48, 0, b, torch.float16)):
        xv, wv = strided(x, K + pad, 16), strided(w, K + wpad, 32)
        work = torch.full((Q.linear_workspace_bytes(M, K),), FILL, dtype=torch.int8, device="cuda")
        one, two = torch.empty(M, N, dtype=ydt, device="cuda"), torch.empty(M, N, dtype=ydt, device="cuda")
        Q.linear_int8_dynamic(xv, wv, ws, bias, one, work)
        q, S = torch.empty(M, K, dtype=torch.int8, device="cuda"), torch.empty(M, device="cuda")
        Q.quantize_tokens(xv, q, S)
        Q.linear_int8(q, S, wv, ws, bias, two)
        assert bool((work == FILL).all()), "the layer took two launches"
        assert torch.equal(bits(one), bits(two)), f"pad {pad}, {ydt}"
        assert torch.equal(bits(two), bits(definition(q, S, w, ws, bias, ydt))), f"pad {pad}, {ydt}, of codes"
