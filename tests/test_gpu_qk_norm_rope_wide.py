"""emb_qk_norm_rope where a token has more rows (heads of queries, keys and values) than an item holds (12 KB: 48 of 128, 24 of
256): its rows are cut into runs, which may end within the queries, the keys or the values."""
import pytest

from tests.test_gpu_qk_norm_rope import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,H,Hk,d", [
    (1, 32, 32, 128), (5, 32, 32, 128), (700, 32, 32, 128), (40, 64, 8, 128), (3, 41, 4, 128), (17, 48, 1, 128), (9, 16, 16, 256), (300, 32, 4, 256),
    (2, 1, 25, 256), (6, 128, 128, 64), (4, 4096, 64, 8), (2, 64, 2048, 16), (1, 4096, 4096, 8)])
@pytest.mark.parametrize("packed", [False, True])
def test_tokens_wider_than_an_item(cuda_device, T, H, Hk, d, packed):
    _run(T, H, Hk, d, packed=packed, seed=T + H)


@pytest.mark.parametrize("kw", [dict(norm=""), dict(norm="q"), dict(norm="k"), dict(rot=64), dict(rot=0), dict(axes=3), dict(drop=(0, 3, 8)),
                                dict(pos0=1 << 20), dict(page=64, axes=4, rot=120)])
def test_forms(cuda_device, kw):
    _run(11, 40, 20, 128, packed=True, seed=5, **kw)
