"""Head sizes above 64 and up to 96: of keys, the last 32 channels of two tokens lie together, so each kernel takes them apart."""
import pytest

from paper_2207_10741_amd import binding as B
from tests import test_gpu_attention as small, test_gpu_attention_long as long

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dim,dtype", [(65, B.BF16), (72, B.F16), (95, B.BF16), (96, B.F16), (97, B.BF16)])
def test_cache_of_head_sizes_about_96(dim, dtype):
    small.test_appends_of_all_sizes_and_read_back(dim, dtype)


@pytest.mark.parametrize("lengths,news,heads,group,dim,dtype,causal", [
    ([1, 0, 17, 48, 65, 129], [1] * 6, 2, 4, 96, B.BF16, True),
    ([1, 0, 17, 48, 65, 129], [1] * 6, 2, 3, 66, B.F16, True),
    ([700, 1, 64], [1] * 3, 1, 17, 96, B.F16, True),
    ([200, 65], [3, 2], 2, 7, 88, B.BF16, True),
    ([150], [150], 2, 2, 96, B.BF16, True),
    ([150], [150], 1, 3, 81, B.F16, False),
    ([97, 0, 64, 31], [40, 2, 64, 50], 1, 4, 90, B.BF16, True),
])
def test_attention_of_head_sizes_about_96(lengths, news, heads, group, dim, dtype, causal):
    small.test_attention_over_the_cache(lengths, news, heads, group, dim, dtype, causal)


@pytest.mark.parametrize("length,new,heads,group,dim,dtype,causal", [
    (9000, 1, 1, 8, 96, B.BF16, True),
    (40000, 1, 1, 4, 72, B.F16, True),
    (9000, 3, 1, 8, 96, B.F16, True),
    (3000, 100, 1, 1, 80, B.BF16, True),
    (2100, 2100, 16, 4, 96, B.BF16, True),
])
def test_long_calls_of_head_sizes_about_96(length, new, heads, group, dim, dtype, causal):
    long.test_rows_of_long_calls(length, new, heads, group, dim, dtype, causal)


@pytest.mark.parametrize("which", ["k", "v", "kv"])
@pytest.mark.parametrize("news", [5, 140])
def test_nan_of_tokens_that_lie_beside_others(which, news):
    small.test_what_is_not_attended_to_has_no_influence(which, news, 96)


@pytest.mark.parametrize("lengths,news,heads,group,dim,dtype,first,last,top", [
    ([640, 0, 64, 65, 1500], [1] * 5, 2, 4, 96, B.BF16, 1, 2, 3),
    ([700, 449], [30, 449], 2, 3, 72, B.F16, 1, 1, 2),
    ([5000], [3], 1, 4, 95, B.BF16, 1, 2, 60),
])
def test_selection_of_head_sizes_about_96(lengths, news, heads, group, dim, dtype, first, last, top):
    small.test_selected_blocks_and_attention_over_them(lengths, news, heads, group, dim, dtype, first, last, top)


@pytest.mark.parametrize("group,dim,dtype,top", [(4, 96, B.BF16, 5), (2, 70, B.F16, 9)])
def test_neighbouring_tokens_of_head_sizes_about_96(group, dim, dtype, top):
    long.test_neighbouring_tokens_together(group, dim, dtype, top)


@pytest.mark.parametrize("heads,group,dim,dtype", [(2, 4, 96, B.BF16), (1, 18, 72, B.F16)])
def test_lists_of_head_sizes_about_96(heads, group, dim, dtype):
    long.test_lists_of_a_piece_of_a_prompt(heads, group, dim, dtype)


@pytest.mark.parametrize("length,new,heads,group,dim,dtype,causal", [
    (2100, 2100, 16, 4, 64, B.BF16, True),
    (2100, 2050, 16, 4, 40, B.F16, False),
    (2100, 2050, 16, 4, 72, B.F16, False),
])
def test_many_rows_of_small_heads(length, new, heads, group, dim, dtype, causal):
    long.test_rows_of_long_calls(length, new, heads, group, dim, dtype, causal)
