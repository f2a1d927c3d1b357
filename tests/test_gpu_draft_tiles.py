"""The tile items of drafted trees: several row tiles and pieces under head counts that do not divide 8, and batches without pieces to join."""
import pytest

from paper_2601_07667_amd import asl
from test_gpu_draft import _tree_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(gpu_device):
    c = asl.Asl(2, 1, 1)
    c.asl_paged_reserve(4096, 1 << 17, 256)
    yield c
    assert c.asl_device_fault() == 0, "a test left the fault word set"
    c.close()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("Hk", [1, 2, 3, 4, 5, 6, 7])
def test_tree_row_tiles_of_any_number_of_heads(ctx, gpu_device, Hk, d):
    """420 and 91 rows of a KV head, in as many pieces as 47 and 10 tiles of keys give: whole and partial turns of splits."""
    _tree_case(ctx, gpu_device, [3000, 640], [60, 13], 7 * Hk, Hk, d, 64, "bf16", seed=Hk, what="Hk %d" % Hk, max_kv=1 << 20)


@pytest.mark.parametrize("d,ps", [(128, 16), (128, 64), (64, 16), (72, 64), (96, 16)])
@pytest.mark.parametrize("G,Hk", [(8, 4), (5, 6), (4, 8)])
def test_tree_batches_without_pieces(ctx, gpu_device, G, Hk, d, ps):
    """More than 192 tiles of rows and no more than 8192 keys by what is stated: every item has its whole span.  Drafts of one to three tiles of
    rows, contexts from none on, sequences with fewer keys than nodes, with none, and without nodes."""
    n_q = [40, 1, 17, 33, 0, 64, 25, 9, 40, 2, 31, 32, 16, 38, 5, 40, 26, 12, 3, 40, 7, 29, 21, 1, 36, 11]
    lens = [2300, 900, 0, 20, 50, 64, 25 + 64, 2048, 1, 3, 700, 32 + 128, 16 + 31, 1500, 5, 40 + 63, 90, 12 + 32, 333, 1000, 7 + 95, 1290, 21 + 1, 1, 36 + 256, 400]
    _tree_case(ctx, gpu_device, lens, n_q, G * Hk, Hk, d, ps, "bf16", seed=d + G, what="whole", max_kv=2500)
