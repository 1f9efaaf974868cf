"""An output or workspace that the allocator refuses raises torch's own error from the classes, as from the rest of the binding, and the
next call works."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture
def refusing():
    """The allocator as it is once the process has what it may have: nothing is taken from the device."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()

    class Limit:
        def __enter__(self):
            torch.cuda.set_per_process_memory_fraction(1e-4)

        def __exit__(self, *error):
            torch.cuda.set_per_process_memory_fraction(1.0)
    return Limit()


def test_out_of_memory(refusing):
    from paper_2607_19378_b200 import hyenand as hn
    x = torch.zeros((1, 64, 1 << 20), device="cuda")
    rng = torch.zeros(2, dtype=torch.int64, device="cuda")
    rec, blk = hn.Recurrence(1 << 20, 1, 64), hn.Block((1 << 20,), 1, 64, p=0.1)
    _, _, marks = rec.forward(x, x, x, x, marks=True)
    r, _, stats = blk.forward(x, x, rng=rng, stats=True)
    del r
    wide = torch.zeros((1 << 13, 1 << 13), device="cuda")
    one = hn.Recurrence(1, 1 << 13, 1 << 13)
    calls = [lambda: rec.forward(x, x, x, x), lambda: rec.backward(x, x, x, x, marks, x), lambda: one.step(wide, wide, wide, wide, wide),
             lambda: blk.forward(x, x, rng=rng), lambda: blk.backward(x, x, stats, rng=rng, dr=x), lambda: hn.Dropout(0.1)(x, rng)]
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for call in calls:
        with refusing, pytest.raises(torch.OutOfMemoryError):
            call()
    for call in calls:
        call()
    torch.cuda.synchronize()
