"""The decode loop's own state (paper_2607_02119_amd/cached_decode.py): what it reports, and how
large its steps may be."""
import pytest

torch = pytest.importorskip("torch")
mcd = pytest.importorskip("paper_2607_02119_amd.mcd", reason="libmcd.so not built")

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="no GPU")]


def test_status_of_a_workspace_that_was_replaced():
    """A bit that a step set before the workspace grew is still reported, once."""
    from paper_2607_02119_amd.cached_decode import CachedDecode
    loop = CachedDecode(rows=4, bound=100, keep=70, recent=20, Hq=4, Hkv=2, D=64, K=3, V=64,
                        V_text=128, seed=3)
    before = loop.workspace
    before[0] = mcd.MCD_DEV_BAD_PAGE
    loop.step()
    assert loop.workspace is not before
    assert loop.status() == mcd.MCD_DEV_BAD_PAGE
    assert loop.status() == 0


def test_more_prompt_tokens_than_a_small_loop_has():
    """800 rows plan up to 6400 tokens in a step."""
    from paper_2607_02119_amd.cached_decode import CachedDecode
    loop = CachedDecode(rows=800, bound=64, keep=40, recent=8, Hq=1, Hkv=1, D=64, K=2, V=32,
                        V_text=64, seed=1)
    seen = []
    loop.step(check=lambda self, b, context, q, out: seen.append(int(b["row_tokens"].sum())))
    assert seen[0] > 4096 and loop.status() == 0
