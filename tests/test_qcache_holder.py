"""What the holder of the 8-bit cache passes on of a tensor's layout: no GPU is needed."""
import pytest

from paper_2609_03494_b200 import binding as B

torch = pytest.importorskip("torch")


class Batch:
    def __init__(self, n_rows):
        self.n_rows, self.device = n_rows, torch.device("cpu")


def holder():
    c = B.QCache.__new__(B.QCache)
    c.torch, c.device, c.head_dim, c._checked = torch, torch.device("cpu"), 64, {}
    c._types = {torch.bfloat16: B.GP_TYPE_BF16, torch.float16: B.GP_TYPE_F16, torch.float32: B.GP_TYPE_F32}
    return c


def test_the_distance_between_rows_is_passed_on():
    q = torch.zeros(3, 10 * 64, dtype=torch.bfloat16)[:, 64:5 * 64].view(3, 4, 64)
    assert holder()._rows("q", q, Batch(3), 4) == 640


@pytest.mark.parametrize("width", [4 * 64 + 4, 4 * 64 + 1, 8 * 64])
def test_a_single_row_has_no_distance_to_another(width):
    """A slice of one row of a wider tensor: its stride is that tensor's width, which may be no multiple of 8."""
    q = torch.zeros(2, width, dtype=torch.bfloat16)[:, :4 * 64].view(2, 4, 64)[:1]
    assert q.stride(0) == width
    assert holder()._rows("q", q, Batch(1), 4) == 4 * 64


def test_tensors_that_want_a_gradient_are_refused():
    c = holder()
    c.n_kv_heads = 2
    t = lambda heads, grad=False: torch.zeros(3, heads, 64, dtype=torch.bfloat16, requires_grad=grad)  # noqa: E731
    w = torch.ones(64, requires_grad=True)
    for kw in (dict(k=t(2, True)), dict(v=t(2, True)), dict(q=t(4, True)), dict(q=t(4), q_weight=w), dict(k_weight=w)):
        with pytest.raises(ValueError, match="no backward"):
            c.append(Batch(3), **{"k": t(2), "v": t(2), **kw})
    for call in (c.attention, lambda b, q: c.select(b, q, 4)):
        with pytest.raises(ValueError, match="no backward"):
            call(Batch(3), t(4, True))
    with torch.no_grad():
        c._no_grad(t(2, True), None, w)                   # (the same tensors where no gradients are recorded)


def test_the_status_word_can_be_asked_for():
    c = holder()
    c.tensors = (None, None, None, torch.tensor([4], dtype=torch.int32))
    assert c.status_bits() == 4
    c.tensors = (None, None, None, None)
    with pytest.raises(ValueError):
        c.status_bits()
