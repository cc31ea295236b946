"""The matrix that the training example's rank rule is evaluated at (host only)."""
import pytest


def test_reference_shape():
    tb = pytest.importorskip("paper_2511_10333_amd.train_block")
    ref = tb.reference_shape
    assert ref([(512, 256), (512, 256), (256, 512), (256,), (4, 256)]) == (512, 256)        # 4 x 256 is sent as it stands at rank 4
    assert ref([(640, 192), (192, 640), (16, 192), (192,)]) == (640, 192)                   # 16 x 192 is at rank 64
    assert ref([(4096, 1024), (1024, 500), (1, 1024)]) == (1024, 500)
    assert ref([(65, 4096), (2048, 130)]) == (2048, 130)                                    # (65 + 4096) 64 > 65 * 4096
    assert ref([(96, 64), (7,)]) == (128, 128)                                              # nothing is compressed at rank 64
