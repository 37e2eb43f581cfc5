"""bf16 attention over prompts and pages keeps 16 significant bits of every softmax weight, in tiles of 32 rows and in wide ones: a
token's error does not depend on the batch that it comes in."""
import pytest

from tests import paged_bounds as B
from tests.paged_cases import Paged
from tests.test_gpu_prefill_attention import _case, _run

pytestmark = pytest.mark.gpu

PROMPTS = [
    (128, 32, 8, [520] * 6), (64, 32, 8, [520] * 6), (128, 16, 2, [2100]), (64, 16, 2, [2100]), (128, 8, 2, [260, 17]), (64, 8, 2, [260, 17]),
]
PAGES = [
    (128, 32, 8, 16, [2600, 700, 1], [1540, 1, 1]), (64, 32, 8, 16, [2600, 700, 1], [1540, 1, 1]),
    (128, 32, 4, 32, [5000, 4000], [2000, 1]), (64, 32, 4, 32, [5000, 4000], [2000, 1]),
    (128, 8, 2, 64, [6000], [400]), (64, 8, 2, 64, [6000], [400]),
    (128, 8, 2, 16, [3000, 40], [1, 1]), (64, 8, 2, 16, [3000, 40], [3, 1]),
]


@pytest.mark.parametrize("d,hq,hkv,lens", PROMPTS)
def test_prompts(d, hq, hkv, lens):
    (q, k, v), cu = _case(sum(lens) + d, "bf16", d, hq, hkv, lens)
    out, _ = _run("bf16", q, k, v, cu, max(lens), d ** -0.5, "tokens")
    worst = B.two_term_error(out, B.prompts(q, k, v, cu, d ** -0.5), d, d ** -0.5)
    assert worst <= 1.0, f"error {worst:.3g} of its bound"


@pytest.mark.parametrize("d,hq,hkv,page,lens,new", PAGES)
def test_pages(d, hq, hkv, page, lens, new):
    from paper_2508_11661_amd import samkv as S
    x = Paged(sum(lens) + d, "bf16", d, hq, hkv, page, lens, new)
    out, _ = x.attend(S, "tokens")
    worst = B.two_term_error(out, B.pages(x), d, x.scale)
    assert worst <= 1.0, f"error {worst:.3g} of its bound"
