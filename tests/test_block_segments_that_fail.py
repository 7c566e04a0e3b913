"""A segment that fails after buffers have been written to: the one before it has no backward any more, as what that needs is gone.  Without a GPU: the
entry points are replaced by ones that do nothing, or fail."""
import pytest

torch = pytest.importorskip("torch")

from paper_2603_09237_amd import attention, memory  # noqa: E402


class Quiet:
    """The binding's functions; `fails`: the one that raises."""
    fails = None

    def __getattr__(self, name):
        import paper_2603_09237_amd.binding as real
        if name.endswith("_bytes"):
            return lambda *a: 512
        if not callable(getattr(real, name)) or isinstance(getattr(real, name), type):
            return getattr(real, name)

        def call(*a, **k):
            if name == self.fails:
                raise real.MorlaxError(real.ERR_UNSUPPORTED, name)
        return call


@pytest.fixture
def quiet(monkeypatch):
    q = Quiet()
    monkeypatch.setattr(memory, "binding", q)
    monkeypatch.setattr(attention, "binding", q)
    return q


def attention_block():
    b = attention.AttentionBlock(3, 8, heads=4, kv_heads=2, head_dim=4, buckets=3, window=6, rank=2, device="cpu", dtype=torch.float32)

    def segment(T, N, index=None):
        x = torch.zeros(T, N, 8)
        return b.segment(x, x.clone(), torch.zeros(N, dtype=torch.int32) if index is None else index, None, b.new_state(N), train=True)

    return b, segment, lambda T, N: b.backward(torch.zeros(T, N, 8), torch.zeros(T, N, 8))


def memory_block():
    b = memory.MemoryBlock(3, 8, heads=2, head_dim=4, state=4, rank=2, device="cpu", dtype=torch.float32)

    def segment(T, N, index=None):
        return b.segment(torch.zeros(T, N, 8), torch.zeros(N, dtype=torch.int32) if index is None else index, None, b.new_state(N), train=True)

    return b, segment, lambda T, N: b.backward(torch.zeros(T, N, 8))


BLOCKS = pytest.mark.parametrize("make,fails", [(attention_block, "attn_fwd"), (memory_block, "scan_fwd")])


@BLOCKS
def test_an_index_of_another_length(quiet, make, fails):
    """The buffer of the rows' indices has the failed segment's size: the old segment's backward would read behind it."""
    b, segment, backward = make()
    segment(16, 9)
    backward(16, 9)
    with pytest.raises(RuntimeError):
        segment(2, 3, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(RuntimeError, match="train=True"):
        backward(16, 9)
    segment(16, 9)
    backward(16, 9)


@BLOCKS
def test_an_entry_point_that_refuses(quiet, make, fails):
    b, segment, backward = make()
    segment(4, 5)
    quiet.fails = fails
    with pytest.raises(RuntimeError):
        segment(4, 5)
    quiet.fails = None
    with pytest.raises(RuntimeError, match="train=True"):
        backward(4, 5)


@BLOCKS
def test_arguments_that_are_refused_first_change_nothing(quiet, make, fails):
    b, segment, backward = make()
    segment(4, 5)
    state = b.new_state(6)
    x = torch.zeros(4, 5, 8)
    with pytest.raises(ValueError):
        b.segment(*([x, x] if make is attention_block else [x]), torch.zeros(5, dtype=torch.int32), None, state)
    backward(4, 5)
