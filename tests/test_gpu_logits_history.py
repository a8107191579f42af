"""Adjusted logits of rows whose histories grow: entries outside the vocabulary are skipped, so a
row keeps one array of tokens, filled with -1 behind the history, and its tokens are put there as
they come, also between the replays of a graph."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab,n", [(1003, 3), (32000, 1)])
def test_a_history_grows_in_place(vocab, n):
    import torch
    import paper_2606_29565_amd as spp
    g = torch.Generator(device="cuda").manual_seed(vocab)
    room, prompt = 400, 30
    src = torch.empty(n, vocab, device="cuda").normal_(0, 2, generator=g)
    history = torch.full((n, room), -1, dtype=torch.int32, device="cuda")
    history[:, :prompt] = torch.randint(0, vocab, (n, prompt), generator=g, device="cuda").int()
    out, ref, rep = (torch.empty_like(src) for _ in range(3))

    def rows(dst, tokens):
        return [spp.AdjustRow(src[i], dst[i], tokens=tokens[i], n_prompt=prompt, repetition=1.3, frequency=0.2,
                              presence=0.1) for i in range(n)]

    held, replayed = spp.LogitsAdjust(vocab, rows(out, history)), spp.LogitsAdjust(vocab, rows(rep, history))
    replayed()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        summ = replayed()
    for step in range(5):
        got = held()
        graph.replay()
        want = spp.LogitsAdjust(vocab, rows(ref, history[:, :prompt + step].contiguous()))()
        torch.cuda.synchronize()
        assert torch.equal(out, ref) and torch.equal(rep, ref)
        for name in ("argmax", "top1", "top2", "lse", "flags"):
            assert torch.equal(getattr(got, name), getattr(want, name)), name
            assert torch.equal(getattr(summ, name), getattr(want, name)), name
        history[:, prompt + step] = got.argmax                  # (on the device: no new object)
