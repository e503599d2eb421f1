"""What holds device addresses for later calls keeps the tensors that they are of: an address of a tensor that has been freed may be
another one's by the time of the call."""
import gc
import weakref

import pytest

from paper_2505_06901_b200 import binding as B


class Tensor:
    """What the binding asks of a CUDA tensor."""
    is_cuda = True

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return id(self)


def tensors(n):
    return [Tensor() for _ in range(n)]


MAKERS = {
    "paged_cache": (4, lambda t: B.paged_cache(*t, 4, 2, 16)),
    "paged_batch": (4, lambda t: B.paged_batch(t[0], 4, *t[1:], 2, 3, 2, 60, 4)),
    "decompress_items": (6, lambda t: B.decompress_items([(t[0], t[1], 5, t[2]), (t[3], t[4], 6, t[5])])),
    "gemv_items": (8, lambda t: B.gemv_items([(t[4 * i], t[4 * i + 1], 32, 128, t[4 * i + 2], t[4 * i + 3]) for i in range(2)])),
}


@pytest.mark.parametrize("name", MAKERS)
def test_temporaries_live_as_long_as_what_holds_their_addresses(name):
    n, make = MAKERS[name]
    parts = tensors(n)
    refs = [weakref.ref(t) for t in parts]
    held = make(parts)
    del parts
    gc.collect()
    assert all(r() is not None for r in refs)
    del held
    gc.collect()
    assert all(r() is None for r in refs)


def test_addresses_given_as_numbers_stay_possible():
    cache = B.paged_cache(64, 128, 192, 256, 4, 2, 16)
    batch = B.paged_batch(0, 0, 64, 128, 192, 2, 3, 2, 60, 4)
    assert (cache.d_k_meta, cache.d_v_blocks, cache.page_size) == (64, 256, 16)
    assert not batch.d_block_tables and batch.d_kv_tiles == 192 and batch.max_tiles == 4
