"""Language-model operators: every call that their documentation refuses is refused before any HIP call (CPU only)."""
import ctypes

import pytest
import torch

import paper_2103_16827_amd as Q

f = ctypes.c_void_p
A, B, C, D, E, F, G = (f(n << 24) for n in range(1, 8))     # addresses far apart
OK, NULL, SHAPE, PARAM, ALIAS, WORKSPACE = 0, -1, -2, -3, -5, -6


def desc(M=4, N=8, K=32, y_type=Q.F32, xs=0, ws=0, ys=0, reserved=0):
    return Q.LinearDesc(M, N, K, y_type, xs, ws, ys, reserved)


def linear(d, x=A, xs=B, w=C, ws=D, bias=E, y=F):
    return Q.lib().qasr_linear_int8(ctypes.byref(d) if d is not None else None, x, xs, w, ws, bias, y, None)


def dynamic(d, x=A, kind=Q.F32, w=C, ws=D, bias=E, y=F, work=G, nbytes=None):
    nbytes = Q.linear_workspace_bytes(d.M, d.K) if nbytes is None else nbytes
    return Q.lib().qasr_linear_int8_dynamic(ctypes.byref(d), x, kind, w, ws, bias, y, work, nbytes, None)


def experts(l=None, E_=3, rows=4, wes=0, x=A, xs=B, offsets=f(100 << 24), index=f(101 << 24), w=C, ws=D, bias=E, y=F, d=True):
    l = desc() if l is None else l
    e = Q.ExpertsDesc(l, E_, rows, wes)
    return Q.lib().qasr_experts_int8(ctypes.byref(e) if d else None, x, xs, offsets, index, w, ws, bias, y, None)


def quantize(x=A, kind=Q.F32, M=4, K=32, xs=0, q=B, qs=0, scale=C):
    return Q.lib().qasr_quantize_tokens(x, kind, M, K, xs, q, qs, scale, None)


def logprobs(x=A, kind=Q.F32, rows=4, V=100, xs=0, tokens=B, n=1, lp=C, ent=D, top=5, ids=E, tlp=F, work=G, nbytes=1 << 22):
    return Q.lib().qasr_token_logprobs(x, kind, rows, V, xs, tokens, n, lp, ent, top, ids, tlp, work, nbytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=131072), SHAPE), (dict(xs=31), SHAPE), (dict(ws=31), SHAPE),
    (dict(ys=7), SHAPE), (dict(xs=-32), SHAPE), (dict(ws=1 << 60), SHAPE), (dict(y_type=3), PARAM), (dict(y_type=-1), PARAM), (dict(reserved=1), PARAM)])
def test_linear_descriptors(kw, status):
    d = desc(**kw)
    assert linear(d) == status
    assert dynamic(d, nbytes=1 << 20) == status
    assert experts(d) == status


@pytest.mark.parametrize("kw", [dict(M=(1 << 30) + 1), dict(N=(1 << 30) + 1), dict(N=(1 << 31) - 1, K=1), dict(M=(1 << 31) - 1, K=1), dict(M=1 << 20, N=1 << 20)])
def test_linear_sides(kw):
    d = desc(**kw)
    assert linear(d) == SHAPE
    assert dynamic(d, nbytes=1 << 20) == SHAPE
    assert experts(d, rows=(1 << 31) - 1) == SHAPE


def test_more_tiles_than_a_launch_counts():
    assert experts(desc(M=100, N=1 << 29), 64) == SHAPE      # (a tile more for every group)
    assert quantize(K=(1 << 30) + 1) == SHAPE
    assert quantize(K=(1 << 31) - 1) == SHAPE


def test_no_rows_are_no_work():
    d = desc(M=0)
    assert linear(d, None, None, None, None, None, None) == OK
    assert dynamic(d, None, Q.F16, None, None, None, None, None, 0) == OK
    assert experts(d, 1, 1, 0, None, None, None, None, None, None, None, None) == OK
    assert quantize(None, Q.F32, 0, 5, 0, None, 0, None) == OK
    assert logprobs(None, rows=0, tokens=None, lp=None, ent=None, ids=None, tlp=None, work=None, nbytes=0) == OK
    assert logprobs(None, tokens=None, n=0, lp=None, ent=None, top=0, ids=None, tlp=None, work=None, nbytes=0) == OK   # nothing asked for


def test_linear_pointers():
    assert linear(None) == NULL
    for k in ("x", "xs", "w", "ws", "y"):
        assert linear(desc(), **{k: None}) == NULL, k
    for k in ("xs", "ws", "bias", "y"):
        assert linear(desc(), **{k: f((9 << 24) + 2)}) == PARAM, k
    assert linear(desc(y_type=Q.BF16), y=f((9 << 24) + 1)) == PARAM
    inside = lambda p, n: f(p.value + n)
    assert linear(desc(), x=inside(F, 4 * 4 * 8 - 1)) == ALIAS       # the last byte of y
    assert linear(desc(), w=inside(F, -(8 * 32 - 1))) == ALIAS       # y begins on w's last byte
    assert linear(desc(), xs=inside(F, 12)) == ALIAS
    assert linear(desc(), ws=inside(F, 12)) == ALIAS
    assert linear(desc(), bias=inside(F, 12)) == ALIAS
    assert linear(desc(ys=1 << 20), x=inside(F, 4 * 3 * (1 << 20))) == ALIAS     # y's last row


def test_dynamic_workspace():
    d = desc()
    assert Q.linear_workspace_bytes(4, 32) == 256 + 256
    assert Q.linear_workspace_bytes(100, 33) == 4864 + 512
    assert Q.linear_workspace_bytes(0, 33) == 0 and Q.linear_workspace_bytes(-1, 33) == 0 and Q.linear_workspace_bytes(1, 131072) == 0
    assert Q.linear_workspace_bytes((1 << 31) - 1, 131071) == ((1 << 31) - 1) * 131072 + (1 << 33)
    assert dynamic(d, kind=5) == PARAM
    assert dynamic(d, x=f((9 << 24) + 2)) == PARAM
    for k in ("x", "w", "ws", "y"):
        assert dynamic(d, **{k: None}) == NULL, k
    assert dynamic(d, work=None) == WORKSPACE
    assert dynamic(d, work=f((7 << 24) + 128)) == WORKSPACE
    assert dynamic(d, nbytes=511) == WORKSPACE
    for k in ("x", "w", "ws", "bias", "y"):
        assert dynamic(d, **{k: f((7 << 24) + 508)}) == ALIAS, k
    assert dynamic(d, x=F) == ALIAS


@pytest.mark.parametrize("kw,status", [
    (dict(d=False), NULL), (dict(E_=0), SHAPE), (dict(E_=4097), SHAPE), (dict(rows=0), SHAPE), (dict(wes=255), SHAPE), (dict(wes=-1), SHAPE),
    (dict(index=None, rows=3), SHAPE), (dict(x=None), NULL), (dict(xs=None), NULL), (dict(offsets=None), NULL), (dict(w=None), NULL),
    (dict(ws=None), NULL), (dict(y=None), NULL), (dict(offsets=f((9 << 24) + 2)), PARAM), (dict(index=f((9 << 24) + 2)), PARAM),
    (dict(offsets=F), ALIAS), (dict(index=F), ALIAS), (dict(x=F), ALIAS), (dict(w=f(F.value - 3 * 256 + 1)), ALIAS), (dict(ws=F), ALIAS),
    (dict(bias=f(F.value - 92)), ALIAS), (dict(xs=F), ALIAS)])
def test_experts_arguments(kw, status):
    assert experts(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(kind=3), PARAM), (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(xs=31), SHAPE), (dict(qs=31), SHAPE), (dict(x=None), NULL),
    (dict(q=None), NULL), (dict(scale=None), NULL), (dict(x=f((9 << 24) + 2)), PARAM), (dict(scale=f((9 << 24) + 2)), PARAM),
    (dict(q=f(A.value + 511)), ALIAS), (dict(scale=f(A.value + 508)), ALIAS), (dict(scale=f(B.value + 124)), ALIAS)])
def test_quantiser_arguments(kw, status):
    assert quantize(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(kind=3), PARAM), (dict(rows=-1), SHAPE), (dict(V=0), SHAPE), (dict(xs=99), SHAPE), (dict(n=-1), SHAPE), (dict(top=-1), SHAPE),
    (dict(top=65), SHAPE), (dict(V=4), SHAPE), (dict(x=None), NULL), (dict(tokens=None), NULL), (dict(lp=None), NULL), (dict(ids=None), NULL),
    (dict(tlp=None), NULL), (dict(x=f((9 << 24) + 2)), PARAM), (dict(ent=f((9 << 24) + 1)), PARAM), (dict(tokens=f((9 << 24) + 2)), PARAM),
    (dict(ids=f((9 << 24) + 2)), PARAM), (dict(lp=f(A.value + 1596)), ALIAS), (dict(ent=B), ALIAS), (dict(ids=f(F.value + 76)), ALIAS),
    (dict(tlp=C), ALIAS)])
def test_logprob_arguments(kw, status):
    assert logprobs(**kw) == status


def test_logprob_workspace():
    assert Q.logprobs_workspace_bytes(-1, 10, 0) == 0 and Q.logprobs_workspace_bytes(1, 0, 0) == 0 and Q.logprobs_workspace_bytes(1, 10, 11) == 0
    for rows, V in ((1, 1 << 18), (3, 1 << 20), (1, (1 << 31) - 1)):
        need = Q.logprobs_workspace_bytes(rows, V, 20)
        if need:
            assert logprobs(rows=rows, V=V, x=f(1 << 40), top=20, nbytes=need - 1) == WORKSPACE
            assert logprobs(rows=rows, V=V, x=f(1 << 40), top=20, nbytes=need, work=None) == WORKSPACE
            assert logprobs(rows=rows, V=V, x=f(1 << 40), top=20, nbytes=need, work=f(G.value + 64)) == WORKSPACE
            assert logprobs(rows=rows, V=V, x=f(1 << 40), top=20, nbytes=need, work=D) == ALIAS


def test_binding_holds_tensors_against_the_call():
    """What the library cannot see of a tensor (types, shapes, strides, where it lives) is refused by the binding."""
    i8, f32 = lambda *s: torch.zeros(*s, dtype=torch.int8), lambda *s: torch.zeros(*s)
    x, xs, w, ws, y = i8(4, 32), f32(4), i8(8, 32), f32(8), f32(4, 8)
    bad = [(x.float(), xs, w, ws, None, y), (x.t().contiguous().t(), xs, w, ws, None, y), (x, f32(5), w, ws, None, y),
           (x, xs, i8(8, 31), ws, None, y), (x, xs, w, f32(4), None, y), (x, xs, w, ws, f32(7), y), (x, xs, w, ws, None, f32(4, 9)),
           (x, xs, w, ws, None, y.double()), (x[:1].expand(4, 32), xs, w, ws, None, y), (x, xs, w, f32(16)[::2], None, y),
           (x, xs, w, ws, None, y)]                                   # (the last one: in host memory)
    for args in bad:
        with pytest.raises(ValueError):
            Q.linear_int8(*args)
    with pytest.raises(ValueError):
        Q.linear_int8_dynamic(x, w, ws, None, y, i8(512))
    with pytest.raises(ValueError):
        Q.quantize_tokens(f32(4, 32), i8(4, 31), f32(4))
    off, idx, we, wse = torch.zeros(4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), i8(3, 8, 32), f32(3, 8)
    for args in [(x, xs, off.long(), idx, we, wse, None, y), (x, xs, off[:3], idx, we, wse, None, y), (x, xs, off, torch.zeros(5, dtype=torch.int32), we, wse, None, y),
                 (x, xs, off, idx, w, wse, None, y), (x, xs, off, idx, we, ws, None, y), (x, xs, off, idx, we[:1].expand(3, 8, 32), wse, None, y),
                 (x, xs, off, idx, we, wse, ws, y), (x, xs, off, idx, we, wse, None, y)]:
        with pytest.raises(ValueError):
            Q.experts_int8(*args)
    lg, tok = f32(4, 100), torch.zeros(4, 1, dtype=torch.int32)
    for args in [(lg, tok), (lg, tok.long(), f32(4, 1)), (lg, tok, f32(4, 2)), (lg, None, None, f32(4, 1)), (lg, None, None, None, tok),
                 (lg, None, None, None, tok, f32(4, 2)), (lg[:, ::2], tok, f32(4, 1)), (lg, tok, f32(4, 1))]:
        with pytest.raises(ValueError):
            Q.token_logprobs(*args)


@pytest.mark.parametrize("work", [torch.zeros(1, dtype=torch.int8).expand(1 << 16), torch.zeros(1 << 17, dtype=torch.int8)[::2],
                                  torch.zeros(1, 64).expand(1024, 64), torch.zeros(64, 1024).t()], ids=["one byte", "every other byte", "one row", "transposed"])
def test_binding_refuses_workspaces_with_less_room_than_elements(work):
    """A workspace that repeats its elements has fewer bytes than it counts; the gaps of one that skips some are another's."""
    x, w, ws, y = torch.zeros(4, 32), torch.zeros(8, 32, dtype=torch.int8), torch.zeros(8), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="workspace"):
        Q.linear_int8_dynamic(x, w, ws, None, y, work)
    with pytest.raises(ValueError, match="workspace"):
        Q.token_logprobs(torch.zeros(4, 100), entropy=torch.zeros(4), workspace=work)


@pytest.mark.parametrize("rows,V,top", [(1 << 40, (1 << 31) - 1, 64), (1 << 40, (1 << 18) + 1, 0), ((1 << 27) + 1, (1 << 31) - 1, 1), ((1 << 40) + 1, 1, 0)])
def test_logprob_workspace_of_refused_sizes(rows, V, top):
    """Logits whose addresses the call refuses have no workspace either (pieces of the first would pass 64 bits)."""
    assert logprobs(x=f(1 << 50), rows=rows, V=V, top=top) == SHAPE
    assert Q.logprobs_workspace_bytes(rows, V, top) == 0


def test_logprob_workspace_of_the_most_logits():
    """2^58 logits: pieces of at most 8 x 64 x 13 loads of 16 bytes, one of 12 bytes and `top` keys of 8 for each."""
    rows, V, top = 1 << 27, (1 << 31) - 1, 64
    pieces = -(-V * 4 // (8 * 64 * 13 * 16))
    need = Q.logprobs_workspace_bytes(rows, V, top)
    assert rows * pieces * (12 + 8 * top) <= need <= rows * 2 * pieces * (16 + 8 * top) + 256


def test_binding_refuses_what_is_no_matrix():
    """A tensor of too few or too many dimensions is a ValueError as well, in every place."""
    i8, i32, f32 = (lambda *s, d=d: torch.zeros(*s, dtype=d) for d in (torch.int8, torch.int32, torch.float32))
    x, xs, w, ws, y = i8(4, 32), f32(4), i8(8, 32), f32(8), f32(4, 8)
    off, idx, we, wse, work, lg = i32(4), i32(4), i8(3, 8, 32), f32(3, 8), i8(512), f32(4, 100)
    for call, args in [(Q.quantize_tokens, (f32(4), i8(4), xs)), (Q.quantize_tokens, (f32(()), i8(()), xs)), (Q.linear_int8, (i8(()), xs, w, ws, None, y)),
                       (Q.linear_int8, (x, xs, i8(()), ws, None, y)), (Q.linear_int8, (x, xs, i8(8), ws, None, y)), (Q.linear_int8, (x, xs, w, ws, None, f32(()))),
                       (Q.linear_int8_dynamic, (f32(4, 32), i8(()), ws, None, y, work)), (Q.linear_int8_dynamic, (f32(4, 32), i8(8, 32, 1), ws, None, y, work)),
                       (Q.experts_int8, (x, xs, off, idx, we, wse, None, f32(()))), (Q.experts_int8, (x, xs, off, idx, we, wse, None, f32(4))),
                       (Q.experts_int8, (x, xs, off, i32(()), we, wse, None, y)), (Q.experts_int8, (x, xs, off, i32(4, 1), we, wse, None, y)),
                       (Q.experts_int8, (x, xs, off, idx, i8(3), wse, None, y)), (Q.experts_int8, (x, xs, off, idx, i8(3, 8, 32, 1), wse, None, y)),
                       (Q.token_logprobs, (lg, i32(4), f32(4))), (Q.token_logprobs, (lg, i32(()), f32(()))), (Q.token_logprobs, (lg, i32(4, 1, 1), f32(4, 1, 1))),
                       (Q.token_logprobs, (lg, None, None, None, i32(4), f32(4))), (Q.token_logprobs, (lg, None, None, None, i32(()), f32(()))),
                       (Q.token_logprobs, (f32(100), None, None, f32(1)))]:
        with pytest.raises(ValueError):
            call(*args)
