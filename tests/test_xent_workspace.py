"""The cross entropy's workspace at the sizes the header allows, on the host: x's rows and the gradient's sums beside a
bounded piece of the vocabulary."""
import pytest

import paper_2005_04680_amd as pk

MB = 1 << 20


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("dim", [4, 64, 128, 132, 300, 2048, 16384])
def test_a_piece_of_the_vocabulary_is_bounded(dim, backward, f32):
    padded = -(-dim // 64) * 64  # of x's rows, more than enough
    for rows in (1, 64, 65, 256, 257, 512, 4096, 8192, 65536, 1 << 20):
        for vocab in (1, 1000, 32001, 131072, 1 << 20, 2 ** 31 - 1):
            got = pk.embbag_xent_workspace_bytes(rows, vocab, dim, pk.EMBBAG_F32 if f32 else pk.EMBBAG_BF16, backward)
            if rows * vocab > 1 << 40:
                assert got == 0
                continue
            # x in BF16 (FP32: three terms, twice for few rows), 64 bytes of a row, FP32 sums of grad_x.
            of_rows = (rows + 31) * (padded * (12 if f32 else 2) + 64 + (dim * 4 if backward else 0))
            # 512 MB each of the sums' parts and of the table's terms; of D and its second term, of kept scores and of
            # the gradients' parts; 256 columns at least.
            piece = (1024 + (2048 if backward else 0)) * MB + 256 * rows * (12 if backward else 0)
            assert 0 < got <= of_rows + piece, (rows, vocab)
