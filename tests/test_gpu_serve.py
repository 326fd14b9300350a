"""The serving loop over documents and a paged cache: requests come, ask, answer and end; its last step against binary64."""
import pytest

from paper_2510_20878_amd import serve

pytestmark = pytest.mark.gpu

# Relative size of the output's error, two norms: the weights of either attention and the output are rounded to BF16, each off by half a
# step (2^-8) at most: twice that, with binary32 arithmetic in between, and cancellation in the output against sums of |v|
# (random signs) by a factor of a few: 2^-8 * 2 * 4.
LIMIT = 2.0 ** -5


@pytest.mark.parametrize("steps", [1, 4, 27, 32])
def test_serving_loop(steps):
    _, error = serve.serve(n_requests=6, n_steps=steps, n_layers=2, doc_tokens=100, n_docs=12, per_request=3, check=True)
    assert error < LIMIT, error


def test_serving_loop_other_shape():
    _, error = serve.serve(n_requests=3, n_steps=9, n_layers=1, kv_heads=2, q_heads=14, doc_tokens=64, n_docs=6, per_request=2,
                           question=(200, 5), answer=6, page_tokens=12, check=True)
    assert error < LIMIT, error


@pytest.mark.parametrize("steps,live", [(6, False), (7, True), (12, False), (20, True)])
def test_serving_loop_of_one_request_that_ends(steps, live):
    """Steps 0 to 4 answer, step 5 has no rows, steps 6 to 10 answer the next one's question, and so on."""
    _, error = serve.serve(n_requests=1, n_steps=steps, n_layers=1, doc_tokens=64, n_docs=4, per_request=2, question=(9,), answer=5,
                           check=True)
    assert error < LIMIT if live else error is None, error
