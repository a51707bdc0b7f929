"""Arguments of the rollout step's calls that would lead past the caller's memory are refused (CPU: nothing is launched)."""
import pytest
import torch

import paper_2609_14636_amd as P

BF = torch.bfloat16


def i32(n):
    return torch.zeros(n, dtype=torch.int32)


@pytest.mark.parametrize("case", ["expanded", "overlapping"])
def test_page_table_rows_closer_than_their_length(case):
    """Rows of one table row expand()ed, or of overlapping views, are not max_pages apart."""
    table = i32(4).view(1, 4).expand(3, -1) if case == "expanded" else i32(8).as_strided((3, 4), (2, 1))
    x, k = torch.zeros(4, 16, 2, 64, dtype=BF), torch.zeros(2, 2, 64, dtype=BF)
    with pytest.raises(P.StrideError) as e:
        P.stride_kv_append(P.KVCache(x, torch.zeros_like(x), table), k, k, i32(2), i32(2), stream=0)
    assert e.value.status == 1


def test_page_table_of_one_row_may_have_any_stride():
    for table in (i32(4).view(1, 4).expand(1, -1), i32(4).as_strided((1, 4), (1, 1)), i32(4).as_strided((1, 4), (0, 1))):
        cache = P.KVCache(torch.zeros(4, 16, 2, 64, dtype=BF), torch.zeros(4, 16, 2, 64, dtype=BF), table)
        assert cache._c.table_ld >= 4


@pytest.mark.parametrize("what", ["logits", "noise"])
def test_sampling_from_views_narrower_than_the_vocabulary(what):
    """Columns of a wider buffer: its row stride passes the vocabulary, the view's own columns do not, and its last
    row would be read past its end."""
    x = dict(logits=torch.zeros(2, 208), noise=torch.zeros(2, 208))
    x[what] = x[what][:, 104:]
    buf = torch.zeros(512, dtype=torch.uint8)
    ws = buf[(-buf.data_ptr()) % 256:][:256]
    with pytest.raises(P.StrideError) as e:
        P.stride_sample(150, x["logits"], x["noise"], torch.ones(2), None, None, None, i32(2), None, ws, stream=0)
    assert e.value.status == 1 and "150" in str(e.value)
