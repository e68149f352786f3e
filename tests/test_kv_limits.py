"""The sizes up to which the paged cache's kernels count in 32 bits (CPU only: addresses are made up)."""
import pytest

from tests.test_kv_refusals import A, CAPACITY, CUDA, F, parts  # noqa: F401

MOST = 2 ** 31 - 1024


@pytest.mark.parametrize("name,most", [("table_stride", MOST // 64), ("n_tokens", MOST), ("n_seqs", MOST)])
@pytest.mark.parametrize("max_new", [4, 400])
def test_sizes_that_a_tile_past_the_end_would_take_out_of_32_bits(F, name, most, max_new):  # noqa: F811
    """Tiles and key blocks end up to a few hundred tokens past the last one."""
    L = F.lib()
    rest = [4, A[5], 512, 0.0, A[6], A[7], 512, A[8], A[9], A[10], None]
    for value, code in ((most, CUDA), (most + 1, CAPACITY), (2 ** 31 - 1, CAPACITY)):
        c, b = parts(F, max_new=max_new, **{name: value})
        assert L.fl_k_kv_attention(c, b, *rest) == code, value
        if code == CAPACITY:
            assert L.fl_k_kv_append(c, b, 4, None, 0, A[6], 256, A[7], 256, None, 0, 0, 0, None, None, None, 0, A[11],
                                    None) == code
