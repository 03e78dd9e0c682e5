"""GPT-2 (two layers of GPT-2 Small's width, random init) with its blocks on the
training-step operators: loss and gradients of a packed batch against the same
model run document by document on torch's operators, and end-to-end steps of
the command line."""
import json

import pytest

torch = pytest.importorskip("torch")
pytest.importorskip("transformers")

pytestmark = pytest.mark.gpu


def _model(dev):
    from transformers import GPT2Config, GPT2LMHeadModel
    torch.manual_seed(7)
    cfg = GPT2Config(n_layer=2, n_embd=768, n_head=12, n_positions=256, vocab_size=1003, attn_pdrop=0.0,
                     resid_pdrop=0.0, embd_pdrop=0.0)
    return GPT2LMHeadModel(cfg).to(dev)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_packed_model_matches_documents(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_36692_amd import e2e_gpt2 as E
    dev = torch.device("cuda:0")
    lens = [200, 1, 37, 130, 256]
    gen = torch.Generator().manual_seed(3)
    tokens = torch.randint(0, 1003, (1, sum(lens)), generator=gen).to(dev)

    ref = _model(dev)
    at, total, count = 0, 0.0, sum(n - 1 for n in lens)
    for n in lens:
        x = tokens[:, at:at + n]
        at += n
        if n > 1:
            (ref(x, labels=x).loss * ((n - 1) / count)).backward()
            with torch.no_grad():
                total += ref(x, labels=x).loss.item() * (n - 1) / count

    model = _model(dev)
    packing = E.Packing(dev)
    E.use_train_ops(model, packing, dtype)
    pos, start = packing.set(lens)
    with torch.autocast("cuda", torch.bfloat16, enabled=dtype == torch.bfloat16):
        loss = model(tokens, position_ids=pos, labels=tokens.masked_fill(start, -100)).loss
    loss.backward()
    # fp32: the forward pass differs by rounding alone, the gradients by the
    # 8-bit codes: steps of at most amax / 63, an error of at most 1/126 of a
    # group's largest value, with random signs over the tokens.  bf16: 2^-8 a
    # rounding, several of them in a row in each of the two blocks.
    assert abs(loss.item() - total) <= (1e-5 if dtype == torch.float32 else 2e-2) * total
    bound = 2e-2 if dtype == torch.float32 else 6e-2
    for (name, p), (_, q) in zip(model.named_parameters(), ref.named_parameters()):
        assert p.grad is not None and p.grad.dtype == torch.float32, name
        err = ((p.grad - q.grad).norm() / q.grad.norm()).item()
        print(f"{name}: {err:.2e}")
        assert err <= bound, (name, err)


@pytest.mark.parametrize("optimizer,dtype", [("normpre-g", "fp32"), ("normpre-l", "bf16")])
def test_command_line_steps(optimizer, dtype, capsys):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_36692_amd import e2e_gpt2 as E
    E.main(["--optimizer", optimizer, "--train-ops", "--dtype", dtype, "--batch", "2", "--seq", "256", "--documents",
            "5", "--steps", "2", "--warmup", "1"])
    out = json.loads(capsys.readouterr().out.strip().splitlines()[-1])
    assert out["optimizer"] == optimizer and dtype in out["metric"]
    # Random tokens over 50257 words: log 50257 = 10.8 at the start.
    assert 9.0 < out["final_loss"] < 13.0
    assert 0.0 < out["descent_alignment_last_step"] <= 1.0
