"""Rotary positions on the GPU against the definition in float64, within the roundings: both layouts, parts of
the head, several axes, far and negative positions, slices, gradients."""
import numpy as np
import pytest
import torch

from paper_2607_01701_amd import rotary, rotary_apply, rotary_frequencies

from gpu_util import log

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def turned(x, positions, freqs, layout, sections, mscale, sign=1.0):
    """float64 result and its bound: the sum of two products in 32 bits (sine and cosine off by 2^-22, two
    roundings) and one rounding to bf16."""
    x = x.double().cpu().numpy()
    axis = np.repeat(np.arange(len(sections)), sections)
    angle = positions.cpu().numpy().reshape(len(sections), -1)[axis].T.astype(np.longdouble) * freqs
    angle = np.asarray(np.mod(angle, np.longdouble("6.28318530717958647692528676655900577")),
                       dtype=np.float64)
    n = len(freqs)
    a, b = (slice(0, n), slice(n, 2 * n)) if layout == "half" else (slice(0, 2 * n, 2), slice(1, 2 * n, 2))
    c, s = np.cos(angle)[:, None] * mscale, sign * np.sin(angle)[:, None] * mscale
    y, bound = x.copy(), np.zeros_like(x)
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    bound[..., a] = bound[..., b] = 2.0 ** -21 * abs(mscale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    bound[..., :2 * n] += 2.0 ** -8 * np.abs(y[..., :2 * n])
    return y, bound


def check(got, ref, bound, what):
    e = np.abs(got.double().cpu().numpy() - ref)
    worst = float((e / (bound + 1e-30)).max()) if e.size else 0.0
    log(f"{what}: {worst:.3f} of the bound; untouched exact: {bool((e[bound == 0] == 0).all())}")
    assert worst <= 1.0 and (e[bound == 0] == 0).all()


CASES = [  # tokens, H, Hk, D, sections, first position
    (1, 40, 8, 128, (64,), 1_000_003), (77, 30, 10, 64, (18,), 0), (300, 2, 2, 128, (16, 24, 24), 0),
    (129, 3, 1, 128, (1,), -5), (64, 5, 5, 64, (32,), 2 ** 31 - 64), (33, 6, 2, 128, (31,), -2 ** 31),
    (200, 4, 4, 64, (0, 13, 3), 7), (1000, 24, 8, 128, (32,), 100_000), (65, 12, 12, 128, (60,), 0),
]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("T,H,Hk,D,sections,start", CASES)
def test_values_and_gradients(T, H, Hk, D, sections, start, layout):
    log(f"case {T} {H}/{Hk}x{D} {sections} from {start} {layout}")
    g = torch.Generator().manual_seed(T + H)
    mk = lambda h: torch.randn((T, h, D), generator=g).bfloat16().cuda()  # noqa: E731
    q, k, dq, dk = mk(H), mk(Hk), mk(H), mk(Hk)
    r = np.random.default_rng(T)
    pos = np.stack([np.arange(start, start + T, dtype=np.int64).astype(np.int32)] +
                   [r.integers(-2 ** 31, 2 ** 31, T).astype(np.int32) for _ in sections[1:]])
    pos = torch.from_numpy(pos).cuda()
    freqs, _ = rotary_frequencies(sections)
    q.requires_grad_(True)
    k.requires_grad_(True)
    qr, kr = rotary(q, k, pos, freqs, layout, sections, 1.25)
    gq, gk = torch.autograd.grad((qr, kr), (q, k), (dq, dk))
    torch.cuda.synchronize()
    for got, x, sign in ((qr, q, 1.0), (kr, k, 1.0), (gq, dq, -1.0), (gk, dk, -1.0)):
        check(got.detach(), *turned(x.detach(), pos, freqs, layout, sections, 1.25, sign), "value" if sign > 0 else "gradient")


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_slices_single_tensors_and_outputs(layout):
    log("case slices")
    T, H, Hk, D = 50, 6, 2, 128
    qkv = torch.randn(T, H + 2 * Hk, D, generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    q, k = qkv[:, :H], qkv[:, H:H + Hk]
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    freqs, _ = rotary_frequencies(64)
    both = rotary_apply(q, k, pos, freqs, layout)
    whole = rotary_apply(q.contiguous(), k.contiguous(), pos, freqs, layout)
    buf = torch.full((2, T, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    only_q = rotary_apply(q, None, pos, freqs, layout, q_out=buf[0])
    only_k = rotary_apply(None, k, pos, freqs, layout)
    torch.cuda.synchronize()
    assert torch.equal(both[0], whole[0]) and torch.equal(both[1], whole[1])
    assert torch.equal(only_q[0], both[0]) and only_q[1] is None and torch.equal(only_k[1], both[1])
    assert (buf[1] == 7.0).all()  # rows behind the last are left as they were
    back = rotary_apply(*both, pos, freqs, layout, inverse=True)
    assert (back[0].float() - q.float()).abs().max() <= 2 ** -7 * 1.5 * q.float().abs().max()
    empty = rotary_apply(q[:0], k[:0], pos[:0], freqs, layout)
    assert empty[0].shape == (0, H, D)


def test_only_one_output_has_a_gradient():
    log("case one gradient")
    q = torch.randn(9, 4, 64).bfloat16().cuda().requires_grad_(True)
    k = torch.randn(9, 2, 64).bfloat16().cuda().requires_grad_(True)
    pos = torch.arange(9, dtype=torch.int32, device="cuda")
    freqs, _ = rotary_frequencies(20)
    qr, kr = rotary(q, k, pos, freqs)
    kr.float().sum().backward()
    torch.cuda.synchronize()
    assert q.grad is None or (q.grad == 0).all()
    check(k.grad, *turned(torch.ones_like(k).detach(), pos, freqs, "half", (20,), 1.0, -1.0), "gradient")
