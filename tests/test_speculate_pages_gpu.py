"""The decoding loop over a pool whose pages lie anywhere."""
import pytest

torch = pytest.importorskip("torch")

from paper_2502_15572_b200 import speculate
from tests.test_speculate_room_gpu import check_text

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("quantised,page,n,L", [(False, 16, 3, 4), (True, 32, 2, 6), (False, 16, 0, 0)])
def test_pages_that_lie_anywhere(quantised, page, n, L):
    """The pool shuffled behind the prompts: used pages, free ones and the table's entries in any order."""
    model, count = speculate.Decoder(seed=5), 40
    gen = torch.Generator().manual_seed(6)
    prompts = [torch.randint(model.vocab, (m,), generator=gen).tolist() for m in (1, 40, 70)]
    store = None
    if n:
        plain, _ = speculate.Speculator(model, prompts, count, quantised=quantised).run(count)
        store = speculate.make_datastore(model, [p + t for p, t in zip(prompts, plain)], L + 1)
    spec = speculate.Speculator(model, prompts, count + L, store, n, L, page_size=page, quantised=quantised)
    pages = spec.refs.shape[0]
    to = torch.randperm(pages, generator=gen).cuda()          # page p becomes page to[p]
    for t in (spec.cache.k_pages, spec.cache.v_pages, spec.cache.k_exps, spec.cache.v_exps):
        if t is not None:
            t.copy_(t[:, to.argsort()])
    spec.refs.copy_(spec.refs[to.argsort()])
    spec.table.copy_(torch.where(spec.table >= 0, to[spec.table.clamp(min=0).long()].int(), spec.table))
    texts, steps = spec.run(count)
    assert n == 0 or steps < count - 1, "no draft was ever accepted"
    for prompt, text in zip(prompts, texts):
        check_text(model, quantised, prompt, text)
    rows = [[e for e in row if e >= 0] for row in spec.table.tolist()]
    assert any(sorted(row) != row for row in rows)
