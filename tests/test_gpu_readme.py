"""The README's beam search, run as it stands there: its beams stay unlike, and its pages hold."""
import os
import re

import pytest
import torch

import paper_2302_01318_b200 as sps

pytestmark = pytest.mark.gpu


def test_the_example_of_a_beam_search_finds_beams_that_differ():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
    blocks = re.findall(r"```python\n(.*?)```", open(path).read(), re.S)
    at = next(i for i, b in enumerate(blocks) if "sps_beam_select" in b)
    names = {"torch": torch, "sps": sps}
    exec(blocks[at - 1], names)
    made, step = blocks[at].split("\n\n", 1)
    exec(made, names)
    texts = [[] for _ in range(8)]

    def forward(table, want, tokens):                          # logits that follow from a beam's text, as a model's do
        rows = []
        for i, t in enumerate(texts):
            seed = i // 4
            for x in t:
                seed = (seed * 40503 + x + 1) % 2 ** 31
            rows.append(torch.randn(32000, generator=torch.Generator().manual_seed(seed)))
        return torch.stack(rows).view(2, 4, 32000).cuda()

    names["forward"] = forward
    for n in range(1, 4):
        exec(step, names)
        texts = [texts[p] + [t] for p, t in zip(names["parents"].view(-1).tolist(), names["tokens"].view(-1).tolist())]
        assert all(len({tuple(t) for t in texts[i:i + 4]}) == 4 for i in (0, 4))
        assert torch.isfinite(names["scores"]).all() and names["table"].lens.tolist() == [n] * 8
        assert int(names["pool"].status) == 0 and int(names["pool"].refs.sum()) == 8
