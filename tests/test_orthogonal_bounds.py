"""What the bound on orthogonalised updates lets through, by the iteration in pairs of 16-bit floats on the host, with and without mistakes."""
import pytest

torch = pytest.importorskip("torch")
from test_gpu_orthogonal import _as_32_bits, _want  # noqa: E402
import paper_1910_04940_amd as bl  # noqa: E402


def _pair(x, scale, single=False):
    """(hi, lo) of scale * x, as 64-bit numbers."""
    hi = (x * scale).half().double()
    return hi / scale, torch.zeros_like(hi) if single else ((x * scale - hi).half().double()) / scale


def _product(p, q, lost=None):
    (ph, pl), (qh, ql) = p, q
    terms = {"hi hi": (ph, qh), "hi lo": (ph, ql), "lo hi": (pl, qh)}
    return sum(a @ b.mT for name, (a, b) in terms.items() if name != lost)


def _in_pairs(m, mistake=None):
    x = m.double()
    tall = x.shape[0] > x.shape[1]
    x = x.mT.contiguous() if tall else x
    x = x / (torch.linalg.matrix_norm(x) + 1e-7)
    eye = torch.eye(len(x), dtype=torch.float64)
    for a, b, c in bl.BLINK_STEPS:
        pair = _pair(x, 2.0 ** 14, mistake == "single X")
        gram = _pair(_product(pair, pair, "hi lo" if mistake == "lost in A" else None), 2.0 ** 14, mistake == "single A")
        square = _product(gram, gram, "lo hi" if mistake == "lost in A A" else None)
        poly = _pair(a * eye + b * (gram[0] + gram[1]) + c * square, 2.0 ** 13, mistake == "single B")
        turned = tuple(v.mT.contiguous() for v in pair)
        if mistake == "lo of another column":
            turned = (turned[0], turned[1].roll(1, 1))
        x = _product(poly, turned, "hi lo" if mistake == "lost in B X" else None)
    return x.mT if tall else x


@pytest.mark.parametrize("shape", [(64, 64), (22, 2025), (389, 1003), (130, 65)])
@pytest.mark.parametrize("mistake", [None, "single X", "single A", "single B", "lost in A", "lost in A A", "lost in B X", "lo of another column"])
def test_pairs_pass_and_mistakes_do_not(shape, mistake):
    m = 1e-3 * torch.randn(*shape, generator=torch.Generator().manual_seed(3))
    want = _want(m)
    assert _as_32_bits(_in_pairs(m, mistake) - want, m, want) == (mistake is None)
