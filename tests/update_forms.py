"""Batches that bring attention's launches into each of their forms, shared by the test that checks the
forms on the host and the tests that run them."""

# name: lengths, query heads, key heads, head size, bf16, keys shared out by the waves, dK/dV in parts
FORMS = {
    "rollouts 128": ([1300, 900, 0, 601, 701], 32, 8, 128, True, False, False),
    "rollouts 128, in parts": ([1300, 850], 32, 8, 128, True, False, True),
    "rollouts 64": ([1000, 900, 950, 871], 32, 16, 64, True, False, False),
    "rollouts 64, in parts": ([1300, 700, 1001], 32, 8, 64, True, False, True),
    "rollouts 32": ([900, 901, 33, 1100, 1200, 1001, 1003, 997, 899], 32, 32, 32, True, False, False),
    "float 128": ([1003, 897, 33, 1100, 1200, 1001, 1003, 997, 899], 32, 32, 128, False, False, False),
    "float 64, in parts": ([1300, 700, 1001], 32, 8, 64, False, False, True),
    "float 32": ([900, 901, 33, 1100, 1200, 1001, 1003, 997, 899], 32, 32, 32, False, False, False),
    "many, keys shared, 32": ([160 + (7 * i) % 23 for i in range(66)], 1, 1, 32, True, True, True),
    "many, keys shared, 64": ([150 + (7 * i) % 41 for i in range(70)], 3, 1, 64, True, True, False),
    "many, keys shared, 128": ([500 + (7 * i) % 53 for i in range(65)], 1, 1, 128, True, True, False),
    "many, keys shared, float 32": ([160 + (7 * i) % 23 for i in range(66)], 1, 1, 32, False, True, True),
    "many, keys shared, float 64": ([500 + (7 * i) % 53 for i in range(65)], 1, 1, 64, False, True, True),
    "many, ordinary": ([150 + (7 * i) % 41 for i in range(130)], 8, 2, 64, True, False, False),
}
