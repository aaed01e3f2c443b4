"""Sampled stairs passes and generations through a context: tokens drawn from the pass's own scores as the 64-bit definition draws them, kept by the
walk, committed to the sequence, and the same output for every draft length."""
import numpy as np
import pytest
import torch

from paper_2407_19947_b200 import workloads as wl
from tests import operator_util as ou

pytestmark = pytest.mark.gpu


def engine(wdtype=wl.WDTYPE_BF16, requests=2, k_max=6, draft=True, seed=13):
    from paper_2407_19947_b200 import build, stairs
    build.build()
    shape = wl.family_b(2, 256, 8, 2, 64, 512, 4096, 256, wdtype)
    src = wl.WeightSource(shape, seed, "numpy", norm_jitter=0.1, std=0.05)
    dsrc = wl.WeightSource(shape.replace(n_layers=1), seed, "numpy", norm_jitter=0.1, std=0.05, share_globals_with=src, share_layers_with=src) if draft else None
    return stairs, shape, stairs.Stairs(src, dsrc, max_requests=requests, max_seq_len=160, k_max=k_max, kv_page_tokens=16)


@pytest.mark.parametrize("wdtype", [wl.WDTYPE_BF16, wl.WDTYPE_F32], ids=["bf16", "fp32"])
@pytest.mark.parametrize("ks", [[6, 2], [0, 5], [0, 0]])
def test_validate_sampled_draws_walks_and_commits(wdtype, ks):
    st, shape, eng = engine(wdtype)
    prompts = [list(wl.zipf_tokens(30, shape.vocab, 1)), list(wl.zipf_tokens(17, shape.vocab, 2))]
    for r, p in enumerate(prompts):
        eng.prefill(r, p)
    rng = np.random.default_rng(3)
    settings = [(0.9, 40, 0.95, 0.0), (1.2, 0, 0.8, 0.01)]
    kw = dict(zip(("temperature", "top_k", "top_p", "min_p"), zip(*settings)))
    rows = sum(ks) + 2
    u = torch.from_numpy(rng.random(rows, dtype=np.float32)).cuda()
    drafts = torch.from_numpy(rng.integers(0, shape.vocab, size=(2, 6)).astype(np.int32)).cuda()
    # drafts that the drawn tokens meet for a while: the drawn token of a row depends on the drafts before it alone
    for r in range(max(ks)):
        tt, _, _ = eng.validate_sampled([0, 1], ks, drafts, u, **kw)
        if r < 3:
            drafts[0, r] = tt[0, r]
        drafts[1, r] = tt[1, r] + (1 if r == 2 else 0)
    before = [eng.sequence(r) for r in (0, 1)]
    tt, al, logits = eng.validate_sampled([0, 1], ks, drafts, u, commit=False, **kw)
    eng.sync()
    assert [eng.sequence(r) for r in (0, 1)] == before
    tt2, al2, logits2 = eng.validate_sampled([0, 1], ks, drafts, u, commit=True, **kw)
    assert torch.equal(tt, tt2) and torch.equal(al, al2) and torch.equal(logits, logits2)
    x, un, row = logits.double().cpu().numpy(), u.cpu().numpy(), 0
    for i, k in enumerate(ks):
        want = [ou.sample_ref(x[row + r], un[row + r], *settings[i]) for r in range(k + 1)]
        assert tt[i, : k + 1].tolist() == want
        d = drafts[i, :k].tolist()
        a = next((r for r in range(k) if d[r] != want[r]), k)
        assert int(al[i]) == a
        assert eng.sequence(i) == before[i] + d[:a] + [want[a]]
        row += k + 1
    eng.close()


def test_generate_sampled_is_the_same_for_every_draft_length():
    st, shape, eng = engine(requests=1)
    prompt = list(wl.zipf_tokens(25, shape.vocab, 4))
    n = 40
    u = torch.rand(n, generator=torch.Generator().manual_seed(5)).cuda()
    kw = dict(temperature=0.7, top_k=30, top_p=0.9)
    ref, stats = eng.generate_sampled(0, prompt, 0, n, u, **kw)
    assert len(ref) == n and stats["iterations"] == n
    assert eng.sequence(0) == prompt + ref
    # token by token through validate_sampled
    eng.prefill(0, prompt)
    for i in range(n):
        tt, _, _ = eng.validate_sampled([0], [0], None, u[i: i + 1].contiguous(), commit=True, **kw)
    assert eng.sequence(0) == prompt + ref
    for k in (1, 3, 6):
        out, stats = eng.generate_sampled(0, prompt, k, n, u, **kw)
        assert out == ref and stats["emitted"] == stats["iterations"] + stats["accepted"]
    other, _ = eng.generate_sampled(0, prompt, 3, n, (u + 0.37) % 1.0, **kw)
    assert other != ref
    # greedy settings: the greedy generation
    greedy, _ = eng.generate(0, prompt, 2, n)
    out, _ = eng.generate_sampled(0, prompt, 2, n, u, temperature=0)
    assert out == greedy
    # stops at the end token
    eos = ref[7]
    out, _ = eng.generate_sampled(0, prompt, 3, n, u, eos=eos, **kw)
    assert out[: ref.index(eos) + 1] == ref[: ref.index(eos) + 1] and eos in out
    eng.close()


def test_sampled_calls_refuse_before_they_enqueue():
    st, shape, eng = engine(requests=1)
    eng.prefill(0, list(wl.zipf_tokens(10, shape.vocab, 1)))
    eng.sync()
    u = torch.rand(8, device="cuda")
    d = torch.zeros((1, 6), dtype=torch.int32, device="cuda")
    launches, seq = eng.launch_count(), eng.sequence(0)
    for kw in (dict(temperature=-1.0), dict(top_k=-1), dict(top_p=0.0), dict(min_p=2.0)):
        with pytest.raises(st.StairsError) as e:
            eng.validate_sampled([0], [2], d, u, commit=True, **kw)
        assert e.value.code == 1 and "stairs_validate_sampled" in str(e.value)
        with pytest.raises(st.StairsError):
            eng.generate_sampled(0, [1, 2, 3], 1, 4, u, **kw)
    for bad in (lambda: eng.validate_sampled([0], [7], d, u), lambda: eng.validate_sampled([1], [2], d, u), lambda: eng.validate_sampled([0, 0], [0, 0], d, u)):
        with pytest.raises((st.StairsError, ValueError)):
            bad()
    for bad in (lambda: eng.validate_sampled([0], [2], d, u[:2]), lambda: eng.validate_sampled([0], [2], d, u.double()), lambda: eng.validate_sampled([0], [2], d.cpu(), u),
                lambda: eng.validate_sampled([0], [2], d.long(), u), lambda: eng.generate_sampled(0, [1, 2], 0, 9, u)):
        with pytest.raises(ValueError):
            bad()
    assert eng.launch_count() == launches and eng.sequence(0) == seq
    eng.close()
