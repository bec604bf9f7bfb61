"""How far rows of attention over many keys are off, measured by what a block of lost or doubled keys would do to them.

An element's worst case (``_paged.attention_bound``) adds every rounding up with one sign; over tens of thousands of keys that is more than
128 of them weigh.  Row by row and head by head, the norm of the error over that of the last rounding alone tells: with n keys of like weight,
values of both signs and D channels the last rounding has a norm of some 2^-9.3 |O|, and 128 lost keys change O by sqrt(128 / n) |O|, 18
times as much at n = 131071.  What the kernel may add: two bf16 terms of a probability (items of up to 128 rows) next to nothing, one term (more
rows) an independent error of the last rounding's size, sqrt(2) on average, with a spread of a tenth over a row of 64 channels.
"""
import torch

TWO_TERMS, ONE_TERM = 1.2, 3.0

# (requests (rows, keys), query heads, key heads, head dimension, page): every row sees 500 keys or more
LONG = [([(1, 70000)], 64, 8, 128, 64), ([(61, 30000)], 16, 2, 128, 64), ([(300, 20000)], 8, 1, 64, 128),
        ([(1, 40000), (1, 600), (600, 3000), (1, 9000)], 16, 4, 128, 16), ([(2, 131071)], 4, 1, 64, 48), ([(1, 131071)], 8, 1, 64, 16),
        ([(1, 50000)], 4, 4, 128, 48), ([(12, 60000)], 8, 2, 64, 16), ([(30, 25000), (1, 3000)], 8, 2, 128, 48)]


def limit(r, Hq, Hkv):
    return ONE_TERM if r * (Hq // Hkv) > 128 else TWO_TERMS


def row_errors(O, want, D):
    """[rows, heads]: the norm of O - want over that of the rounding of want to bf16."""
    err, own = ((x.double() - want).view(want.shape[0], -1, D).norm(dim=-1) for x in (O, want.to(torch.bfloat16)))
    return err / own
