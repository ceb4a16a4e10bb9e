"""Generation with trees of drafts and over a bounded cache, end to end on the GPU."""

import numpy as np
import pytest
import torch

from test_gpu_serving_example import plain

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def serving():
    from paper_2609_15039_gb300 import serving, spl
    assert torch.cuda.is_available(), "GPU tests need CUDA"
    spl.lib()
    return serving


@pytest.mark.parametrize("branches", [[], [1], [3, 2, 1], [2, 2, 2, 2]], ids=str)
def test_a_tree_gives_each_branchs_logits(serving, branches):
    """The logits of a tree's nodes against those of the tokens on the way to each, in 64 bits (the tolerance is that of
    test_gpu_serving_example: the cache's binary16 through two layers)."""
    target, _, pages = serving.synthetic(2, seqs=2, max_len=320)
    tree = serving.Tree(branches)
    g = np.random.default_rng(3)
    prompts = [g.integers(0, 1024, n).tolist() for n in (150, 63)]
    target.forward(torch.tensor(sum(prompts, []), device="cuda"), pages.grow([150, 63]))
    nodes = g.integers(0, 1024, (2, tree.nodes))
    got = target.forward(torch.as_tensor(nodes.reshape(-1)).cuda(), pages.grow([tree.nodes] * 2), tree.rows(tree.levels, 2))
    got = got.cpu().numpy().reshape(2, tree.nodes, -1)
    for b in range(2):
        for i in range(tree.nodes):
            way, at = [], i
            while at >= 0:
                way, at = [int(nodes[b, at])] + way, tree.parents[at]
            assert np.max(np.abs(got[b, i] - plain(target, prompts[b] + way)[-1])) < 1e-2
    from paper_2609_15039_gb300 import spl
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("branches", [[1, 1], [3, 2, 1]], ids=str)
def test_the_caches_hold_what_was_generated(serving, branches):
    """After rounds of drafts, accepted or not, both decoders' next logits are those of the tokens that were generated."""
    target, draft, pages = serving.synthetic(2, seqs=3, max_len=300, formats=("f16", "f16"))
    total = len(pages.free)
    prompts = [list(range(b, b + n)) for b, n in enumerate((62, 1, 100))]
    out, history = serving.generate_tree(target, draft, pages, prompts, branches, rounds=8)
    assert [len(o) for o in out] == [1 + sum(h[b] + 1 for h in history) for b in range(3)]
    lens = [len(p) + len(o) - 1 for p, o in zip(prompts, out)]  # the last token is pending
    assert pages.lens == lens and len(pages.free) == total - sum(-(-n // 64) for n in lens)
    batch = pages.grow([1] * 3)
    last = torch.tensor([o[-1] for o in out], device="cuda")
    for decoder in (target, draft):
        got = decoder.forward(last, batch).cpu().numpy()
        for b in range(3):
            assert np.max(np.abs(got[b] - plain(decoder, prompts[b] + out[b])[-1])) < 1e-2
    from paper_2609_15039_gb300 import spl
    assert spl.spl_get_device_status() == spl.SPL_OK


def test_a_decoder_that_drafts_itself_is_accepted(serving):
    """Drafts by the target's own logits, three a node: most rounds accept some (a sharp distribution's three largest)."""
    target, _, pages = serving.synthetic(1, seqs=4, max_len=400, formats=("f16", "f16"))
    prompts = [list(range(b, b + n)) for b, n in enumerate((64, 1, 37, 100))]
    _, history = serving.generate_tree(target, _, pages, prompts, [3, 3], rounds=6)
    assert sum(map(sum, history)) > 0


def test_a_bound_that_is_never_reached_changes_nothing(serving):
    target, _, pages = serving.synthetic(2, seqs=2, max_len=300)
    prompts = [list(range(20)), list(range(5, 100))]
    out = serving.generate_bounded(target, pages, prompts, 12, keep=200, recent=10)
    assert pages.lens == [len(p) + 11 for p in prompts]
    for b, p in enumerate(prompts):
        logits = plain(target, p + out[b][:-1])
        # each token was drawn from the distribution of those before it: none is out of its reach
        for i, t in enumerate(out[b]):
            assert logits[len(p) - 1 + i].max() - logits[len(p) - 1 + i][t] < 25
    # every row of a layer gives a weight of 1 a query head, spread over the tokens that it sees
    for score in target.scores:
        j = torch.tensor([(int(pages.table[b, i // 64]), i % 64) for b in range(2) for i in range(pages.lens[b])], device="cuda")
        total = score[j[:, 0], :, j[:, 1]].double().sum().item()
        assert abs(total - 8 * sum(pages.lens)) < 1e-3 * total


def test_a_bounded_cache_stays_bounded(serving):
    """A cache of 64 tokens and a page: lengths stay inside, pages are given back, the step after an eviction attends to
    what was kept."""
    target, _, pages = serving.synthetic(2, seqs=3, max_len=256, page_size=16)
    total = len(pages.free)
    out = serving.generate_bounded(target, pages, [list(range(n)) for n in (200, 3, 70)], 60, keep=64, recent=16)
    assert [len(o) for o in out] == [60] * 3
    assert max(pages.lens) <= 64 + 16 and len(pages.free) == total - sum(-(-n // 16) for n in pages.lens)
    from paper_2609_15039_gb300 import spl
    assert spl.spl_get_device_status() == spl.SPL_OK


@pytest.mark.parametrize("more,said", [(["--tree", "3,2,1"], "a round accepted"), (["--keep", "40"], "in the cache")])
def test_the_command(serving, capsys, more, said):
    assert serving.main(["--sequences", "3", "--layers", "2", "--rounds", "20", "--prompt", "33", "--eps", "4"] + more) == 0
    line = capsys.readouterr().out
    assert "status SPL_OK" in line and said in line


@pytest.mark.parametrize("tree", [False, True])
def test_tokens_that_are_not_weighed_start_from_nothing(serving, tree):
    """What their slots' last owners gathered is not theirs: a step after them weighs them as if they had been new to the pool."""
    got = []
    for stale in (0.0, 1000.0):
        target, _, pages = serving.synthetic(2, seqs=2, max_len=320)
        target.scores = [torch.full(tuple(c.k.shape[:3]), stale, device="cuda") for c in target.caches]
        g = np.random.default_rng(1)
        draw = lambda n: torch.as_tensor(g.integers(0, 1024, n)).cuda()  # noqa: E731
        target.forward(draw(193), pages.grow([63, 130]), weigh=True)
        target.forward(draw(20), pages.grow([10, 10]), serving.Tree([1] * 9).rows(10, 2) if tree else None)
        target.forward(draw(2), pages.grow([1, 1]), weigh=True)
        j = torch.tensor([(int(pages.table[b, i // 64]), i % 64) for b in range(2) for i in range(pages.lens[b])]).cuda()
        got.append([score[j[:, 0], :, j[:, 1]] for score in target.scores])
        # every row that is weighed gives a weight of 1 a query head
        for score in got[-1]:
            assert abs(score.double().sum().item() - 8 * 195) < 1e-3 * 8 * 195
    assert all(torch.equal(a, b) for a, b in zip(*got))
    from paper_2609_15039_gb300 import spl
    assert spl.spl_get_device_status() == spl.SPL_OK
