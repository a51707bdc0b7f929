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


def aligned(nbytes):
    buf = torch.zeros(nbytes + 256, dtype=torch.uint8)
    off = (-buf.data_ptr()) % 256
    return buf[off:off + nbytes]


def test_counts_that_pass_32_bits_within_a_tile():
    """The last keys of a sequence and the last rows of a call are counted in whole tiles, up to 255 further."""
    x = torch.zeros(4, 1, 2, 64, dtype=BF)
    k = torch.zeros(2, 2, 64, dtype=BF)
    for pages, code in ((2 ** 31 - 1, 2), (2 ** 31 - 255, 2), (2 ** 31 - 256, None)):
        c = P.KVCache(x, x.clone(), i32(2).view(2, 1))
        c._c.max_pages = c._c.table_ld = pages
        # a key that is not 16-byte aligned is refused after the cache has been checked
        bad = torch.zeros(257, dtype=BF)[1:].view(2, 2, 64)
        with pytest.raises(P.StrideError) as e:
            P.stride_kv_append(c, bad, k, i32(2), i32(2), stream=0)
        assert e.value.status == 2 and ("max_pages" in str(e.value)) == (code is not None), str(e.value)
    c = P.KVCache(x, x.clone(), i32(2).view(2, 1))
    for n, heads in ((2 ** 25 - 1, 64), (2 ** 30 - 127, 2)):
        q = torch.zeros(1, heads, 64, dtype=BF).expand(n, -1, -1)
        with pytest.raises(P.StrideError) as e:
            P.stride_tree_attention(c, q, i32(3), i32(2), None, 0.1, q, None, None, aligned(256), stream=0)
        assert e.value.status == 2 and "2^31 - 256" in str(e.value)


def test_workspace_sizes_of_refused_calls_are_0():
    x = torch.zeros(4, 16, 2, 64, dtype=BF)
    c = P.KVCache(x, x.clone(), i32(4).view(2, 2))
    assert P.stride_attention_workspace_size(c, 3, 4) > 0
    assert P.stride_attention_workspace_size(c, 2 ** 30, 4) == 0 and P.stride_attention_workspace_size(c, -1, 4) == 0
    for field, value in (("head_dim", 80), ("page_size", 24), ("dtype", 7), ("max_pages", 2 ** 30), ("n_pages", -1),
                         ("n_pages", 0), ("n_seqs", 0)):
        c = P.KVCache(x, x.clone(), i32(4).view(2, 2))
        setattr(c._c, field, value)
        assert P.stride_attention_workspace_size(c, 3, 4) == 0, field
    c = P.KVCache(x, x.clone(), i32(4).view(2, 2))
    c._c.k = c._c.v = c._c.page_table = None  # only sizes are read
    assert P.stride_attention_workspace_size(c, 3, 4) > 0
    assert P.stride_sample_workspace_size(2, 2 ** 30) > 0 and P.stride_sample_workspace_size(2, 2 ** 30 + 1) == 0
    assert P.stride_sample_workspace_size(-1, 100) == 0


def test_query_outputs_without_queries():
    x, k = torch.zeros(4, 16, 2, 64, dtype=BF), torch.zeros(2, 2, 64, dtype=BF)
    with pytest.raises(ValueError):
        P.stride_kv_append(P.KVCache(x, x.clone(), i32(4).view(2, 2)), k, k, i32(2), i32(2), q_out=k.clone(), stream=0)
