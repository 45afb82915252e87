"""Trees whose drafts are all the tokens that a row leaves possible."""

import numpy as np
import pytest

from test_gpu_verify import upload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seqs,vocab", [(4, 2), (4, 5000), (300, 9000)])
def test_the_last_possible_token_comes(gpu, seqs, vocab):
    """Row 0 holds two tokens, of 1 and of 8.6 x 2^-23, both drafted. The number of the
    first lies past its probability, 1 - 2^-24 > 1 - 1.03e-6. Of what is left, the second
    has all, and any number below 1 accepts it: the sum 1 + 8.6 x 2^-23 may round in
    binary32, to 1 + 9 x 2^-23 then, and 0.99 of what that leaves is more than the token
    has. It comes all the same, as the accepted draft or as the token that follows."""
    a = dict(logits=np.full((3 * seqs, vocab), -np.inf, np.float32),
             tokens=np.tile(np.array([0, 0, 1]), seqs), offsets=np.arange(0, 3 * seqs + 1, 3),
             max_accept=1, uniforms=np.tile(np.float32([0.5, 1 - 2.0 ** -24, 0.99]), seqs),
             draft=None, parents=np.tile(np.int32([-1, 0, 0]), seqs))
    a["logits"][:, 0] = 0.0
    a["logits"][0::3, 1] = np.log(8.6 * 2.0 ** -23)
    counts, following, paths = (t.tolist() for t in gpu.verify_drafts(**upload((a, "f32", 0))))
    for count, token, path in zip(counts, following, paths):
        assert token >= 0
        assert (path == [0, 2] and token == 0) if count else (path == [0, -1] and token == 1)
