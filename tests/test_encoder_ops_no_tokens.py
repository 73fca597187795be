"""attention_run and attention_select on a batch without tokens, through the C ABI on the CPU: nothing to do for either."""
import paper_2211_07715_amd as sl
from test_encoder_ops_host import ATTN, P, attn, select


def test_no_tokens_is_nothing_to_do():
    for change in (dict(m_tokens=0), dict(m_tokens=0, x=0, seq_start=0), dict(m_tokens=0, n_seq=7, max_len=4096)):
        assert attn(**change) == 0
        assert attn(**change, blocks=P) == 0
        assert select(**change) == 0
        assert select(blocks=0, workspace=0, size=0, **change) == 0


def test_what_is_wrong_is_refused_all_the_same():
    assert select(m_tokens=0, query_block=5) == select(m_tokens=0, top_k=0) == select(m_tokens=0, head_dim=7) == -2
    assert select(m_tokens=0, max_len=262145) == -5
    assert sl.load().attention_select_workspace(sl._ATTN_ARGS.pack(*{**ATTN, "m_tokens": 0}.values())) > 0
