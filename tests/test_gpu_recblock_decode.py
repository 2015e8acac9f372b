"""What the example of recurrent layers asks of the operators when it decodes, and when it trains."""

import pytest
import torch

from tests.test_gpu_recblock_together import example  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("decoding", [True, False])
def test_hidden_values_are_kept_for_a_backward_alone(example, monkeypatch, decoding):  # noqa: F811
    print(f"\n[gpu case] what is kept, decoding {decoding}", flush=True)
    kept = []
    for name in ("gdr2_gatedff_fwd", "gdr2_gatedrec_fwd"):
        real = getattr(example.g2, name)
        monkeypatch.setattr(example.g2, name, lambda *a, real=real, **kw: kept.append(kw.get("save", False)) or real(*a, **kw))
    torch.manual_seed(4)
    model = example.Model().to("cuda")
    tokens = torch.randint(0, 32, (2, 40), device="cuda")
    if decoding:
        logits = example.decode(model, tokens, 30)
        assert logits.shape[:2] == tokens.shape and bool(torch.isfinite(logits).all())
        # two layers: the prompt's recurrence and feed-forward, and ten tokens' feed-forwards
        assert kept == [False] * (2 * (2 + 10))
    else:
        model(tokens)[0].sum().backward()
        assert kept == [True] * 4
