"""Rotary positions against float64, their gradients, and the call in front of the INT8 attention."""
import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2603_02170_amd import binding
from paper_2603_02170_amd.autograd import sage_attention, sage_rotary

pytestmark = pytest.mark.gpu

HALF = 2.0 ** -8      # half a step of bf16
# (sine and cosine are within a few 2^-24 and the angle within 2^-25 turns: 2^-20 of the channel pair's magnitude covers them, and two FP32 roundings)
SLACK = 2.0 ** -20


def _np(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


def _freq(half):
    return (10000.0 ** (-torch.arange(half, dtype=torch.float64) / half)).float()


def _close(got, want, x):
    pair = np.abs(x).max(-1, keepdims=True)
    err = np.abs(_np(got) - want)
    assert (err <= HALF * np.abs(want) + SLACK * 2 * pair + 1e-38).all(), float(err.max())


@pytest.mark.parametrize("T,Hq,Hk,d,rot,sections,adjacent,far", [
    (1, 1, 1, 64, 64, None, False, 10), (33, 8, 2, 128, 128, None, False, 1 << 20), (7, 3, 3, 64, 32, None, True, 5000),
    (257, 4, 1, 128, 128, [16, 24, 24], False, 4000), (50, 2, 2, 80, 48, [4, 20], False, 300), (19, 5, 5, 128, 64, [0, 31, 1, 0], True, 1 << 28),
    (3000, 9, 3, 64, 64, [8, 12, 12], False, 1 << 17), (2, 70, 1, 512, 512, [1, 85, 85, 85], True, 99), (64, 2, 1, 16, 16, None, False, 70),
])
@pytest.mark.parametrize("wide", [torch.int32, torch.int64])
def test_rotary_against_float64(T, Hq, Hk, d, rot, sections, adjacent, far, wide):
    g = torch.Generator().manual_seed(T + d)
    axes = len(sections) if sections else 1
    pos = torch.randint(-5, far, (axes, T), generator=g)
    qkv = torch.randn((T, Hq + Hk + 1, d), generator=g).to(torch.bfloat16).cuda()
    Q, K = qkv[:, :Hq], qkv[:, Hq:Hq + Hk]
    f = _freq(rot // 2)
    p = pos.to(wide).cuda()
    Qo, Ko = sage_rotary(Q, K, p if sections else p[0], f.cuda(), sections=sections, adjacent=adjacent)
    sec = sections or [rot // 2]
    for got, x in ((Qo, Q), (Ko, K)):
        assert got.is_contiguous() and got.shape == x.shape
        _close(got, ref.rotary(_np(x), pos.numpy(), f.numpy(), sec, adjacent), _np(x))
        assert torch.equal(got[..., rot:], x[..., rot:])
    only, none = sage_rotary(Q, None, p, f.cuda(), sections=sections, adjacent=adjacent)
    assert none is None and torch.equal(only, Qo)
    Qi, _ = sage_rotary(Q, K, p, f.cuda(), sections=sections, adjacent=adjacent, inverse=True)
    _close(Qi, ref.rotary(_np(Q), pos.numpy(), f.numpy(), sec, adjacent, inverse=True), _np(Q))


def test_layouts_and_positions_of_batches():
    g = torch.Generator().manual_seed(1)
    B, N, Hq, Hk, d = 3, 21, 4, 2, 64
    f = _freq(32).cuda()
    Q, K = (torch.randn((B, N, h, d), generator=g).to(torch.bfloat16).cuda() for h in (Hq, Hk))
    pos = torch.randint(0, 1000, (2, B, N), generator=g, dtype=torch.int32).cuda()
    one, three = sage_rotary(Q, K, pos, f, sections=[10, 22])
    flat = sage_rotary(Q.flatten(0, 1), K.flatten(0, 1), pos.flatten(1), f, sections=[10, 22])
    assert torch.equal(one.flatten(0, 1), flat[0]) and torch.equal(three.flatten(0, 1), flat[1])
    heads = sage_rotary(Q.transpose(1, 2), K.transpose(1, 2).contiguous(), pos, f, sections=[10, 22], token_major=False)
    assert torch.equal(heads[0], one.transpose(1, 2)) and torch.equal(heads[1], three.transpose(1, 2)) and heads[0].is_contiguous()
    shared = sage_rotary(Q, K, pos[:, 0], f, sections=[10, 22])       # every batch at the same positions
    assert torch.equal(shared[0], sage_rotary(Q, K, pos[:, :1].expand(2, B, N), f, sections=[10, 22])[0])
    assert torch.equal(sage_rotary(Q, K, pos[0, 0], f)[0], sage_rotary(Q, K, pos[0, :1].expand(B, N), f)[0])
    # rows that do not begin on 16 bytes, channels that are not adjacent, a tensor of one row
    odd = torch.empty((B, N, Hq, d + 3), dtype=torch.bfloat16, device="cuda")[..., 3:]
    odd.copy_(Q)
    assert torch.equal(sage_rotary(odd, K, pos, f, sections=[10, 22])[0], one)
    assert torch.equal(sage_rotary(Q[:1, :1], K[:1, :1], pos[:, :1, :1], f, sections=[10, 22])[0], one[:1, :1])
    wide = torch.empty((B, N, Hq, 2 * d), dtype=torch.bfloat16, device="cuda")[..., ::2]
    wide.copy_(Q)
    assert torch.equal(sage_rotary(wide, K, pos, f, sections=[10, 22])[0], one)
    empty = sage_rotary(Q[:, :0], K[:, :0], pos[:, :, :0], f, sections=[10, 22])
    assert empty[0].shape == (B, 0, Hq, d)


def test_gradients_by_the_formula_and_by_differences():
    g = torch.Generator().manual_seed(2)
    T, d = 45, 64
    pos = torch.randint(0, 1 << 18, (3, T), generator=g, dtype=torch.int32).cuda()
    f = _freq(32).cuda()
    Q, K = (torch.randn((T, h, d), generator=g).to(torch.bfloat16).cuda().requires_grad_() for h in (4, 2))
    dQ, dK = (torch.randn((T, h, d), generator=g).to(torch.bfloat16).cuda() for h in (4, 2))
    out = sage_rotary(Q, K, pos, f, sections=[8, 12, 12])
    gq, gk = torch.autograd.grad(out, [Q, K], [dQ, dK])
    for got, x in ((gq, dQ), (gk, dK)):
        _close(got, ref.rotary(_np(x), pos.cpu().numpy(), f.cpu().numpy(), [8, 12, 12], False, inverse=True), _np(x))
    # differences of <dQ, rotary(Q)> in float64, which the turn, being linear, has exactly
    want = np.zeros(d)
    for c in range(d):
        e = np.zeros((T, 1, d))
        e[7, 0, c] = 1.0
        turned = ref.rotary(e, pos.cpu().numpy(), f.cpu().numpy(), [8, 12, 12], False)
        want[c] = (turned[:, 0] * _np(dQ)[:, 0]).sum()
    assert np.abs(_np(gq)[7, 0] - want).max() <= 2 * HALF * np.abs(_np(dQ)[7, 0]).max()
    # one of the outputs alone, and an expanded gradient
    out = sage_rotary(Q, K, pos, f, sections=[8, 12, 12])
    (only,) = torch.autograd.grad(out[1], [K], [dK], retain_graph=True)
    assert torch.equal(only, gk)
    (summed,) = torch.autograd.grad(out[0].sum(), [Q])
    _close(summed, ref.rotary(np.ones((T, 4, d)), pos.cpu().numpy(), f.cpu().numpy(), [8, 12, 12], False, inverse=True), np.ones((T, 4, d)))
    # shared input, gradient of a gradient
    out = sage_rotary(Q, Q, pos, f, sections=[8, 12, 12])
    (both,) = torch.autograd.grad(out, [Q], [dQ, dQ], create_graph=True)
    # (two bf16 gradients summed in bf16)
    assert (both.float() - 2 * gq.float()).abs().max() <= 2 * HALF * 2 * gq.float().abs().max()
    leaf = dQ.clone().requires_grad_()
    out, _ = sage_rotary(Q, None, pos, f, sections=[8, 12, 12])
    (first,) = torch.autograd.grad(out, [Q], [leaf], create_graph=True)
    (second,) = torch.autograd.grad(first, [leaf], [dQ])
    assert torch.equal(second, sage_rotary(dQ, None, pos, f, sections=[8, 12, 12])[0])


def test_positions_changed_in_place_before_the_backward_are_noticed():
    Q = torch.randn(4, 1, 64, device="cuda").to(torch.bfloat16).requires_grad_()
    pos = torch.arange(4, device="cuda")
    out, _ = sage_rotary(Q, None, pos, _freq(32).cuda())
    pos += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


@pytest.mark.parametrize("token_major", [False, True])
def test_in_front_of_the_attention(token_major):
    """What a model's block does in training: the gradients are those of the two calls one after the other."""
    g = torch.Generator().manual_seed(3)
    shape = (2, 192, 3, 64) if token_major else (2, 3, 192, 64)
    Q, K, V, dO = (torch.randn(shape, generator=g).to(torch.bfloat16).cuda() for _ in range(4))
    pos, f = torch.arange(192, device="cuda"), _freq(32).cuda()
    q, k, v = (t.clone().requires_grad_() for t in (Q, K, V))
    qr, kr = sage_rotary(q, k, pos, f, token_major=token_major)
    sage_attention(qr, kr, v, token_major=token_major).backward(dO)
    q2, k2 = (t.detach().requires_grad_() for t in sage_rotary(Q, K, pos, f, token_major=token_major))
    v2 = V.clone().requires_grad_()
    sage_attention(q2, k2, v2, token_major=token_major).backward(dO)
    back = sage_rotary(q2.grad, k2.grad, pos, f, token_major=token_major, inverse=True)
    assert torch.equal(q.grad, back[0]) and torch.equal(k.grad, back[1]) and torch.equal(v.grad, v2.grad)


def test_captured_and_replayed():
    g = torch.Generator().manual_seed(4)
    Q, K, dQ = (torch.randn((40, 2, 128), generator=g).to(torch.bfloat16).cuda() for _ in range(3))
    Q.requires_grad_()
    pos, f = torch.arange(40, device="cuda", dtype=torch.int32), _freq(64).cuda()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = sage_rotary(Q, K, pos, f)
        torch.autograd.grad(out[0], [Q], [dQ])
        del out            # (an eager graph of the same leaf that lives on would tie the capture to its stream)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sage_rotary(Q, K, pos, f)
        (grad,) = torch.autograd.grad(out[0], [Q], [dQ])
    for step in range(3):
        with torch.no_grad():
            pos += 100
            Q.mul_(0.5)
        graph.replay()
        torch.cuda.synchronize()
        eager = sage_rotary(Q, K, pos, f)
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])
        assert torch.equal(grad, sage_rotary(dQ, None, pos, f, inverse=True)[0])


def test_outputs_in_the_place_of_the_inputs():
    """The C call allows it."""
    import ctypes

    class P(ctypes.Structure):
        _fields_ = [(n, ctypes.c_int32) for n in ("B", "N", "Hq", "Hk", "d", "rotary_dim", "axes")] + [("sections", ctypes.c_int32 * 4)] + \
            [(n, ctypes.c_int32) for n in ("adjacent", "inverse", "positions64")] + [(n, ctypes.c_int64 * 3) for n in ("q", "k", "qo", "ko")]

    Q, K = (torch.randn(30, h, 64, device="cuda").to(torch.bfloat16) for h in (3, 1))
    pos, f = torch.arange(30, device="cuda", dtype=torch.int32), _freq(16).cuda()
    want = sage_rotary(Q, K, pos, f)
    q, k = (0, 192, 64), (0, 64, 64)
    p = P(1, 30, 3, 1, 64, 32, 1, (16, 0, 0, 0), 0, 0, 0, q, k, q, k)
    lib = binding.load_library()
    vp = ctypes.c_void_p
    rc = lib.sagebwd_rotary(vp(Q.data_ptr()), vp(K.data_ptr()), vp(Q.data_ptr()), vp(K.data_ptr()), vp(pos.data_ptr()), vp(f.data_ptr()),
                            ctypes.byref(p), vp(torch.cuda.current_stream().cuda_stream))
    assert rc == 0 and torch.equal(Q, want[0]) and torch.equal(K, want[1])


def test_frequencies_that_want_a_gradient_are_refused():
    Q = torch.randn(3, 2, 64, device="cuda").to(torch.bfloat16)
    pos, freq = torch.arange(3, device="cuda", dtype=torch.int32), torch.rand(32, device="cuda", requires_grad=True)
    with pytest.raises(NotImplementedError):
        sage_rotary(Q, None, pos, freq)
    with torch.no_grad():
        a = sage_rotary(Q, None, pos, freq)[0]
    assert torch.equal(a, sage_rotary(Q, None, pos, freq.detach())[0])
