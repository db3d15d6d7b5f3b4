"""GPU tests of calls on pools of very many pages, or of very many rows."""
import pytest

from paper_2606_24033_amd import blockgtq as bg
from paper_2606_24033_amd import synth
from tests.test_gpu_cache_readers import D, Packed, i32

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def _require_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    bg.lib()


@pytest.fixture(scope="module")
def rotations():
    return synth.rotations(7)


def test_rows_read_back_from_two_million_pages(rotations):
    """A row of each page: no fewer than a workgroup could take of each page's head."""
    few = Packed(rotations, 3, batch=6, kv=1, cap=64, k_budget=64, v_bits=1, kind="uniform")
    pages = (1 << 21) + 5
    cfg = bg.Config(n_layers=1, batch=pages, n_kv_heads=1, group=few.cfg.group, capacity=64, k_budget=64, v_bits=1)
    pool = bg.Cache(cfg)
    at = torch.tensor([pages - 1, 3, pages - 70000, 1 << 20, 7, (1 << 21) - 1], device="cuda")
    for n in ("k_codes", "k_norms", "v_codes", "v_norms"):
        getattr(pool, n)[:, at] = getattr(few.cache, n)
    place = [63, 0, 17, 32, 31, 5]
    pos = torch.zeros(pages, dtype=torch.int32, device="cuda")
    pos[at] = i32(place)
    k, v = bg.blockgtq_dequantize_rows(cfg, few.layout, 0, pool, pos, 1, out_dtype=torch.bfloat16)
    k1, v1 = bg.blockgtq_dequantize_rows(few.cfg, few.layout, 0, few.cache, i32(place), 1, out_dtype=torch.bfloat16)
    assert torch.equal(k[at], k1) and torch.equal(v[at], v1)
    empty = torch.ones(pages, dtype=torch.bool, device="cuda")
    empty[at] = False
    assert k.shape == (pages, 1, 1, D) and not k[empty].any() and not v[empty].any()
