"""What goes wrong in a call around the paged cache and how it is told: reasons that belong to the call, errors that pass through the extension."""
import pytest
import torch

from paper_2002_12798_amd import binding as B
from paper_2002_12798_amd import device
from tests.test_cache_args import AT, _rope, _rows


def test_a_refusal_made_in_python_has_no_other_calls_reason():
    """The library's last reason stays on the thread; an error that the library has not been asked about must not name it."""
    with pytest.raises(B.AmapError) as e:
        B.amap_rotary(_rows(head=4096), _rows(5 * AT, head=4096), 10, 4096, _rope(), AT, 0)
    assert "2048" in str(e.value)
    for what in ("amap_rotary", "amap_cache_append", "amap_cache_attend", "amap_cache_assign"):
        said = str(device._refused(what, "x is not contiguous along its last dimension", B.AMAP_E_UNSUPPORTED))
        assert said.startswith(what + ": x is not contiguous") and "2048" not in said


@pytest.mark.gpu
def test_that_refusal_for_a_tensor():
    with pytest.raises(B.AmapError):
        B.amap_rotary(_rows(head=4096), _rows(5 * AT, head=4096), 10, 4096, _rope(), AT, 0)
    x = torch.zeros((4, 2, 64, 2), dtype=torch.float16, device="cuda")[..., 0]
    with pytest.raises(B.AmapError) as e:
        device.rotary(x, device.Rope(torch.ones(32, device="cuda")), torch.zeros(4, dtype=torch.int32, device="cuda"))
    assert e.value.status == B.AMAP_E_UNSUPPORTED and "not contiguous" in str(e.value) and "2048" not in str(e.value)


@pytest.mark.gpu
def test_an_interrupt_passes_through_the_extension():
    """Raised while it asks an object for its handle: an interrupt and an exit go on to the caller, any other error leaves the call to the way through ctypes."""
    class Cache:
        def __init__(self, error):
            self.error, self.asked = error, 0

        @property
        def _cache_at(self):
            self.asked += 1
            raise self.error

    x, slot = torch.zeros((1, 1, 8), device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    table, n = torch.zeros((1, 1), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for call in (lambda c: device._native.append(c, x, x, slot, None, None, None, None, None), lambda c: device._native.attend(c, x.half(), table, n, None, 0, None, None, None, None)):
        for error in (KeyboardInterrupt, SystemExit):
            cache = Cache(error())
            with pytest.raises(error):
                call(cache)
            assert cache.asked == 1
        cache = Cache(ValueError())
        assert call(cache) is None and cache.asked == 1
