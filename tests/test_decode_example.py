"""The example that runs attention and sparse FFN together: what its sequences see after forks, rejected tokens and a compaction is what
sequences of the same tokens see that were never touched by any of them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_sequences_after_forks_truncation_and_compaction_equal_fresh_ones():
    from examples.decode import Decoder, main
    got = main(steps=5, dense=True)
    assert got["pages"] < got["pages_before"] and got["moved"] > 0
    table, refs = got["model"].kv.table.cpu(), got["model"].kv.refs.cpu()
    used = got["model"].kv.state()["used_pages"]
    assert set(table[table >= 0].tolist()) == set(range(used)) and (refs[:used] > 0).all() and (refs[used:] == 0).all()
    for slot, tokens in got["sequences"].items():
        fresh = Decoder(dense=True)
        for at in range(0, len(tokens), 11):               # in pieces of another size, in another slot
            logits = fresh.step([tokens[at:at + 11] if s == 5 else [] for s in range(fresh.seqs)])[5][-1]
        scale = logits.abs().max()
        # two layers of fp16 activations: a few roundings of 2^-11 each, and the sums in another order
        assert (logits - got["logits"][slot]).abs().max() <= 2e-2 * scale, slot
