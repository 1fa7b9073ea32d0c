"""The paged 8-bit cache behind the library's own draft trees (kv8_flow)."""
import pytest

import kv8_flow
from paper_2601_19278_b200 import runner
from paper_2601_19278_b200 import synthetic as syn

pytestmark = pytest.mark.gpu

C1 = syn.WORKLOADS["C1"]


@pytest.mark.parametrize("fmt,page_tokens,hkv,heads,dim", [("e4m3", 16, 2, 4, 64), ("int8", 64, 1, 5, 128), ("e4m3", 32, 2, 10, 128), ("int8", 16, 2, 2, 64)])
@pytest.mark.parametrize("over", [dict(), dict(batch=3, K=6, tree_budget=60), dict(batch=2, K=8, tree_budget=31)], ids=["C1", "b3_60", "b2_31"])
def test_trees_and_paths_of_the_library_go_through_attention_and_append(over, fmt, page_tokens, hkv, heads, dim):
    w = syn.small_variant(C1, **over)
    ses = runner.DraftSession(w, syn.make_weights(w), syn.make_ngram_rows(w.vocab, min(w.ngram_rows, 20000), w.ngram_mode))
    ses.load_inputs(syn.make_step_inputs(w))
    ses.step()
    ses.tree()
    assert kv8_flow.run(ses, fmt, page_tokens, hkv, heads, dim, [37, 150, 16][:w.batch], seed=heads) > 0
    ses.close()
