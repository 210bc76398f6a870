"""What the Python calls of a policy update refuse before the library sees it, on the CPU: a stand-in for the library takes whatever gets through."""
import pytest
import torch

from paper_2506_24119_amd import binding as sb


class Library:
    """Makes optimisers out of nothing and notes the gradients that it is given."""

    def __init__(self):
        self.made, self.given, self.checked = 0, [], []

    def spiral_adamw_create(self, arr, n, mem, nbytes, stream, out):
        self.made += 1
        out._obj.value = self.made
        return 0

    def spiral_adamw_check_grads(self, opt, arr, n):
        self.checked.append(list(arr))
        return 0

    def spiral_adamw_set_grads(self, opt, arr, stream):
        self.given.append(list(arr))
        return 0

    def spiral_adamw_free(self, opt):
        pass


@pytest.fixture
def lib(monkeypatch):
    lib = Library()
    monkeypatch.setattr(sb, "load_library", lambda: lib)
    return lib


def tensors():
    a, b = torch.zeros(300, dtype=torch.bfloat16), torch.zeros(6, 50)
    recs = [sb.spiral_adamw_tensor(a, a.clone(), torch.zeros(300), torch.zeros(300)), sb.spiral_adamw_tensor(b, b.clone(), torch.zeros(300), torch.zeros(300))]
    return recs, a, b


def test_exchanged_gradients_are_of_the_records_number_size_and_type(lib):
    recs, a, b = tensors()
    opt = sb.spiral_adamw_create(recs, torch.zeros(4096, dtype=torch.uint8), stream=0)
    for bad in ([], [a], [a, b, b], [a[:299], b], [a, b[:5]], [a, torch.zeros(301)], [a.float(), b], [a.half(), b], [a, b.bfloat16()], [a, torch.zeros(50, 6).t()],
                [torch.zeros(600, dtype=torch.bfloat16)[::2], b], [b, a]):
        with pytest.raises(ValueError):
            sb.spiral_adamw_set_grads(opt, bad, stream=0)
    with pytest.raises(TypeError):
        sb.spiral_adamw_set_grads(opt, [a, b.double()], stream=0)
    assert not lib.given
    sb.spiral_adamw_set_grads(opt, [a, b], stream=0)
    sb.spiral_adamw_set_grads(opt, [a, b.view(-1)], stream=0)
    assert lib.given == lib.checked[-2:] == [[a.data_ptr(), b.data_ptr()]] * 2


def test_optimisers_have_their_own_records_until_they_are_freed(lib):
    recs, a, b = tensors()
    mem = torch.zeros(4096, dtype=torch.uint8)
    one, two = sb.spiral_adamw_create(recs, mem, stream=0), sb.spiral_adamw_create(recs[:1], mem, stream=0)
    sb.spiral_adamw_set_grads(two, [a], stream=0)
    sb.spiral_adamw_set_grads(one, [a, b], stream=0)
    with pytest.raises(ValueError):
        sb.spiral_adamw_set_grads(one, [a], stream=0)
    sb.spiral_adamw_free(one)
    for gone in (one, 77, None):
        with pytest.raises(ValueError):
            sb.spiral_adamw_set_grads(gone, [a, b], stream=0)
    sb.spiral_adamw_set_grads(two, [a], stream=0)
    assert len(lib.given) == 3


def test_no_optimiser_without_memory(lib):
    """The size of no memory is 0, which the library refuses by name."""
    recs, _, _ = tensors()
    seen = []
    lib.spiral_adamw_create = lambda arr, n, mem, nbytes, stream, out: seen.append((mem, nbytes)) or sb.SPIRAL_ERR_INVALID_ARG
    lib.spiral_last_error = lambda: b"adamw_create: memory is null"
    with pytest.raises(sb.SpiralError):
        sb.spiral_adamw_create(recs, None, stream=0)
    assert seen == [(None, 0)]


def test_the_check_of_gradients_needs_an_object():
    assert sb.load_library().spiral_adamw_check_grads(None, None, 1) == sb.SPIRAL_ERR_NOT_LOADED
    assert "null object" in sb.spiral_last_error()
