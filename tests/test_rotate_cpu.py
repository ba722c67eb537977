"""Norms and rotation without a GPU: the oracle's own pins, and what the library refuses before anything is enqueued."""
import ctypes

import pytest
import torch

from oracle import rotate_torch as ref
from paper_2309_12307_b200 import binding as s2a


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("eps", [None, 1e-3])
def test_oracle_gradients_are_those_of_differences(interleaved, eps):
    g = torch.Generator().manual_seed(0)
    x, dy = (torch.randn(3, 2, 8, generator=g, dtype=torch.float64) for _ in range(2))
    w = 1 + 0.3 * torch.randn(8, generator=g, dtype=torch.float64) if eps is not None else None
    positions, radians = torch.tensor([5, -3, 100_000]), [1.0, 0.1, 0.01]

    def f(x, w):
        return float((ref.rotate(x, positions, radians, interleaved, w, eps) * dy).sum())

    dx, dw = ref.rotate_bwd(x, dy, positions, radians, interleaved, w, eps)
    h = 1e-6
    for i in range(x.numel()):
        step = torch.zeros(x.numel(), dtype=torch.float64)
        step[i] = h
        step = step.view_as(x)
        assert abs((f(x + step, w) - f(x - step, w)) / (2 * h) - float(dx.flatten()[i])) < 1e-7
    for i in range(8 if w is not None else 0):
        step = torch.zeros(8, dtype=torch.float64)
        step[i] = h
        assert abs((f(x, w + step) - f(x, w - step)) / (2 * h) - float(dw[i])) < 1e-7


def test_oracle_keeps_sizes_of_pairs_and_adds_angles():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(4, 1, 12, generator=g, dtype=torch.float64)
    p, radians = torch.tensor([0, 1, 7, -20]), [0.3, 2.0]
    y = ref.rotate(x, p, radians)
    assert torch.equal(y[0], x[0]) and torch.equal(y[..., 4:], x[..., 4:])
    assert torch.allclose(y[..., 0] ** 2 + y[..., 2] ** 2, x[..., 0] ** 2 + x[..., 2] ** 2)
    assert torch.allclose(ref.rotate(y, 3 - p, radians), ref.rotate(x, torch.full((4,), 3), radians))
    neighbours = ref.rotate(x[..., [0, 2, 1, 3] + list(range(4, 12))], p, radians, interleaved=True)
    assert torch.allclose(neighbours[..., [0, 2, 1, 3]], y[..., :4])


def test_frequencies():
    with pytest.raises(ValueError, match="even"):
        s2a.rotary_turns(3, device="cpu")
    with pytest.raises(ValueError, match="base"):
        s2a.rotary_turns(4, base=0.0, device="cpu")
    assert s2a.rotary_turns(4, base=4.0, device="cpu").tolist() == [round(2**64 / 6.283185307179586), round(2**64 * 0.5 / 6.283185307179586)]


class Rotation(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("positions", ctypes.c_void_p)] + [(n, ctypes.c_int) for n in ("n_positions", "r", "interleaved", "norm", "weight_type")] + \
               [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_float)]


def test_the_library_refuses_without_a_device():
    from test_paged_cpu import Batch, Cache

    lib = s2a.load()
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 255) & ~255  # never dereferenced on these paths

    def call(rotation=(), q=a, q_out=a, dq=a, q_stride=256, T=5, H=4, Hkv=2, d=64, workspace=a, no_rotation=False):
        r = Rotation(**{**dict(turns=a, positions=a, n_positions=5, r=64, interleaved=0, norm=1, weight_type=0, q_weight=a, k_weight=a, eps=1e-5), **dict(rotation)})
        r = None if no_rotation else ctypes.byref(r)
        c = Cache(k=a, v=a, k_exp=a, v_exp=a, type=1, pages=4, Hkv=Hkv, page_size=16, d=d)
        b = Batch(table=a, starts=a, lengths=a, width=2, B=3, T=T)
        return (lib.s2a_rotate(q, q_stride, a, 128, q_out, 256, a, 128, r, T, H, Hkv, d, None),
                lib.s2a_rotate_bwd(a, 256, a, 128, q, q_stride, a, 128, dq, a, a if r and rotation and dict(rotation).get("norm") == 0 else None, None, r, T, H, Hkv, d, workspace, 0, None),
                lib.s2a_rotate_write(q, q_stride, a, 128, a, 128, q_out, r, ctypes.byref(c), ctypes.byref(b), H, None))

    invalid, unsupported = s2a.S2A_ERR_INVALID_ARG, s2a.S2A_ERR_UNSUPPORTED
    for change in (dict(turns=None), dict(turns=a + 4), dict(positions=a + 2), dict(n_positions=0), dict(r=-16), dict(r=80), dict(interleaved=2), dict(norm=2),
                   dict(norm=0), dict(weight_type=2), dict(q_weight=a + 8), dict(k_weight=a + 2), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert call(rotation=change) == (invalid,) * 3, change
    assert call(rotation=dict(r=24)) == (unsupported,) * 3
    for change in (dict(q=None), dict(q=a + 8), dict(q_stride=252), dict(q_stride=248), dict(T=0), dict(H=0), dict(no_rotation=True)):
        assert call(**change) == (invalid,) * 3, change
    for change in (dict(d=96, rotation=dict(r=0)), dict(T=1 << 28), dict(q_stride=(1 << 28) + 8)):
        assert call(**change) == (unsupported,) * 3, change
    assert call(q_out=a + 4)[::2] == (invalid,) * 2 and call(dq=None)[1] == invalid
    assert call(workspace=a + 16)[1] == invalid and call(workspace=None)[1] == invalid
    assert call(rotation=dict(positions=None, n_positions=0))[:2] == (invalid,) * 2
    assert lib.s2a_rotate_bwd_workspace_bytes(96) == 0


@pytest.mark.parametrize("H,Hkv,d", [((1 << 22) + 1, 2, 64), (1 << 25, 2, 64), ((1 << 21) + 1, 2, 128), (4, (1 << 22) + 1, 64)])
def test_a_tokens_heads_lie_within_a_limit(H, Hkv, d):
    """2^28 values, of a single token too, whose stride is not looked at: the place of a head in a token is an int."""
    from test_paged_cpu import Batch, Cache

    lib = s2a.load()
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 255) & ~255  # never dereferenced on these paths
    r = ctypes.byref(Rotation(turns=a, positions=a, n_positions=1, r=64, norm=1, q_weight=a, k_weight=a, eps=1e-5))
    c = Cache(k=a, v=a, k_exp=a, v_exp=a, type=1, pages=4, Hkv=Hkv, page_size=16, d=d)
    b = Batch(table=a, starts=a, lengths=a, width=2, B=1, T=1)
    for status in (lib.s2a_rotate(a, 0, a, 0, a, 0, a, 0, r, 1, H, Hkv, d, None),
                   lib.s2a_rotate_bwd(a, 0, a, 0, a, 0, a, 0, a, a, a, None, r, 1, H, Hkv, d, a, 0, None),
                   lib.s2a_rotate_write(a, 0, a, 0, a, 0, a, r, ctypes.byref(c), ctypes.byref(b), H, None)):
        assert status == s2a.S2A_ERR_UNSUPPORTED
