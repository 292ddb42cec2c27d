"""The serving-step entry points refuse a call whose launch would have 2^32 work-items or more in a dimension, which HIP does
not take, before any device work.  Host only: the addresses are never read."""
import paper_2607_04031_amd as tl
from tests.test_host_serve import addr, append, cache, status


def test_append():
    # 64 query heads over 8, head size 128: a workgroup a row's queries, an eighth of one its values, a sixteenth its keys
    for n in (1 << 24, 14128182):
        assert status(append, cache=cache(), n=n) == tl.TL_EUNSUPPORTED, n
    assert status(append, cache=cache(), n=1 << 24, K=None, V=None, slots=None) == tl.TL_EUNSUPPORTED
    assert status(append, cache=cache(kv_heads=1024), n=1 << 20, Q=None, q_heads=0, Q_out=None, ldk=1 << 17, ldv=1 << 17) == tl.TL_EUNSUPPORTED


def test_read():
    assert status(tl.tl_kv_read, cache=cache(), slots=addr(7), n=1 << 27, K_out=addr(8), V_out=addr(9), stream=0) == tl.TL_EUNSUPPORTED


def test_keep():
    assert status(tl.tl_kv_keep, cache=cache(), page_table=addr(7), max_pages=4, starts=addr(8), path=addr(9), max_path=6, counts=addr(10),
                  num_seqs=1 << 21, stream=0) == tl.TL_EUNSUPPORTED


def test_attn():
    assert status(tl.tl_attn, Q=addr(4), ldq=64 * 128, cache=cache(), page_table=addr(7), max_pages=4, lens=addr(8), q_offsets=addr(9), mask=None,
                  mask_words=0, num_seqs=1 << 21, total_q=1 << 21, max_q=1, max_len=200, q_heads=64, scale=0.1, O=addr(11),
                  stream=0) == tl.TL_EUNSUPPORTED


def test_verify():
    def verify(**kw):
        d = dict(logits=addr(0), logits_dtype=tl.TL_OUT_BF16, vocab=1000, node_offsets=addr(1), parents=addr(2), tokens=addr(3), num_seqs=4,
                 total_nodes=20, max_nodes=8, draft=addr(4), draft_dtype=tl.TL_OUT_F32, temperature=addr(5), uniform=addr(6), noise=addr(7),
                 path=addr(8), counts=addr(9), next_token=addr(10), stream=0)
        d.update(kw)
        tl.tl_verify(**d)
    assert status(verify, total_nodes=1 << 24) == tl.TL_EUNSUPPORTED
    assert status(verify, num_seqs=1 << 22) == tl.TL_EUNSUPPORTED


def test_attn_scale():
    """The kernels take scores in units of log2(e): a scale that overflows there has no finite scores."""
    for scale in (2.36e38, 3.4e38):
        assert status(tl.tl_attn, Q=addr(4), ldq=64 * 128, cache=cache(), page_table=addr(7), max_pages=4, lens=addr(8), q_offsets=addr(9),
                      mask=None, mask_words=0, num_seqs=3, total_q=12, max_q=6, max_len=200, q_heads=64, scale=scale, O=addr(11),
                      stream=0) == tl.TL_EUNSUPPORTED, scale
