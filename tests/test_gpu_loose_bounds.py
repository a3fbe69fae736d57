"""Bounds of the lengths that are far above them, as a captured graph has: selection, attention over chosen pages and over a whole cache in 4 bits give what the lengths say.
Tolerances: those of the tests whose checks these are."""
import pytest

from paper_2605_13473_amd import binding as ob
from tests.test_gpu_page_select import bounds_of, check_attention, check_choice, make
from tests.test_gpu_paged_mx import DECODE, call, compare, make_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,slack", [(4, 1), (4, 7), (9, 50), (20, 2000), (4, 100000)])
@pytest.mark.parametrize("form", [dict(io="bf16"), dict(io="f32"), dict(io="bf16", mx=True), dict(io="f32", mx=True)], ids=str)
def test_selected_pages(form, n, slack):
    """Uneven rows, a bound of the lengths up to some hundred times the longest: on both sides of the rule for who makes the scores, with and without room in the table."""
    for lengths, Hq, Hk, K, page in (([300, 0, 17, 129], 8, 2, 128, 8), ([(97 * b) % 260 for b in range(19)], 6, 3, 64, 8), ([5, 700, 64, 701], 4, 1, 256, 4)):
        x = make(lengths, Hq, Hk, K, page, **form)
        chosen, tokens = check_choice(x, bounds_of(x), n, max_length=x["longest"] + page * slack)
        check_attention(x, chosen, tokens)
        check_attention(x, chosen, tokens, max_length=n * page + page * slack)


def test_the_rule_of_the_scores_has_both_sides_here():
    """The workspace is that of the keys, which a launch of their own makes: none where a row's workgroup does."""
    ask = lambda B, Hk, K, length: ob.osdn_page_select_workspace_bytes(ob.make_select_params(B, Hk, Hk, K, True, length, pages=4), 8) > 0
    assert [ask(4, 2, 128, 300 + 8 * s) for s in (1, 7, 50, 2000, 100000)] == [False, False, False, True, True]


@pytest.mark.parametrize("times", [2, 30, 1000])
@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(v) for v in c.values())[:80])
def test_a_whole_cache_in_4_bits(case, times):
    x = make_decode(**case)
    compare(x, *call(x, max_length=max(1, x["longest"]) * times + 3))
