"""Calls of the 8-bit products and of the mixture-of-experts layer that between
them take every kernel the rules reach, tiles with a whole and with a split sum and
with operands as they are and copied, every way of the choice with one table and
with one for each rank.  Sizes are the cheapest of a search over the rules.

INT8: call, ranks, rows, in, out, elements between rows, workspace.
MOE: ranks, tokens, in, hidden, experts of a rank, top, types of x, weights and
result, elements between rows of the weights, logits of each rank's own."""

INT8 = [(c[0], *map(int, c[1:])) for c in map(str.split, """\
linear 1 1 43 1 16 0
linear 1 1 48 1 0 0
linear 1 1 64 1 1 0
linear 1 1 1024 1 16 0
linear 1 1 1071 1 16 1
linear 1 1 1104 1 1 0
linear 1 1 2048 1 1 0
linear 1 1 2048 1 16 1
linear 1 1 2048 8462 1 1
linear 1 1 2629 1 1 1
linear 1 1 4096 1 0 1
linear 1 1 4096 1 1 1
linear 1 1 6119 1 0 0
linear 1 17 40 2 0 0
linear 1 17 48 1 0 1
linear 1 17 1024 1 1 1
linear 1 17 1024 1 16 0
linear 1 17 2048 1 1 1
linear 1 17 2048 1 16 0
linear 1 17 4096 1 1 0
linear 1 17 4096 1 16 0
linear 1 33 45 1 1 1
linear 1 33 48 1 0 1
linear 1 33 883 1 0 1
linear 1 33 942 2 0 1
linear 1 33 1792 1 16 1
linear 1 33 16384 2 1 1
linear 1 533 64 7243 16 1
linear 1 695 2105 1546 16 1
linear 1 1175 64 7077 0 1
linear 2 1 48 4795 0 1
linear 2 33 1024 8421 0 1
linear 2 49 1040 8175 1 1
linear 3 33 1024 7113 1 1
linear 3 49 61 5592 0 0
linear 3 49 2048 6152 0 1
linear 3 77 64 8287 0 1
linear 3 701 16384 65 0 1
linear 8 17 1088 2337 16 1
linear 8 17 2560 2007 1 1
linear 8 33 2048 2444 0 0
linear 8 33 2162 1991 16 1
linear 8 49 1024 2036 0 1
linear 8 980 8192 65 0 1
linear 33 1 42 243 0 1
linear 33 1 1024 226 1 1
linear 33 1 1024 240 0 1
linear 33 1 2048 238 0 1
linear 33 17 53 464 1 0
linear 33 17 64 505 0 1
linear 33 17 1168 479 1 1
linear 33 17 2048 479 16 1
linear 33 33 42 543 0 1
linear 33 33 64 453 0 1
linear 33 33 2048 1 0 1
linear 33 49 48 482 0 1
linear 33 49 2048 521 1 1
linear 33 105 4096 65 1 1
linear 33 452 48 1 16 1
linear 33 718 64 78 1 0
gated 1 1 41 1 1 0
gated 1 1 48 1 0 0
gated 1 1 64 1 1 1
gated 1 1 1024 1 0 1
gated 1 1 1024 1 1 0
gated 1 1 1484 1 16 1
gated 1 1 2048 1 0 1
gated 1 1 2048 1 1 1
gated 1 1 2048 8756 16 1
gated 1 1 2107 1 16 0
gated 1 1 4096 1 0 1
gated 1 1 4096 1 1 1
gated 1 1 4494 1 0 1
gated 1 17 45 1 0 0
gated 1 17 48 1 16 1
gated 1 17 48 8610 1 1
gated 1 17 1024 1 16 1
gated 1 17 1024 8343 0 1
gated 1 17 1037 1 1 0
gated 1 17 2048 1 0 1
gated 1 17 2064 1 1 1
gated 1 17 4096 1 0 1
gated 1 17 4096 1 1 0
gated 1 33 48 1 1 0
gated 1 33 48 2 16 1
gated 1 33 52 8505 16 1
gated 1 33 822 2 0 1
gated 1 33 919 1 1 1
gated 1 33 1744 1 0 1
gated 1 33 2048 8220 0 1
gated 1 33 2117 8393 1 1
gated 1 33 16384 2 1 1
gated 1 49 42 8778 16 1
gated 1 49 2048 8833 0 1
gated 1 71 8192 2096 0 1
gated 1 1155 48 1776 16 1
gated 1 1158 1678 603 16 1
gated 1 2146 577 2447 1 1
gated 2 1 2048 4289 1 1
gated 2 17 2048 4574 1 0
gated 2 49 48 4466 0 1
gated 2 86 67 6479 16 1
gated 3 1 48 2899 16 1
gated 3 144 48 6551 16 1
gated 3 1086 5480 33 0 1
gated 8 1 1024 1118 0 1
gated 8 17 1039 1145 0 0
gated 8 17 2048 1067 0 1
gated 8 49 1024 1019 16 1
gated 8 72 64 1672 0 0
gated 33 1 44 230 1 1
gated 33 1 1328 252 1 1
gated 33 17 64 233 0 1
gated 33 33 48 231 16 1
gated 33 33 1024 227 0 0
gated 33 33 1024 233 1 1
gated 33 33 2048 1 0 1
gated 33 59 2048 247 1 0
gated 33 64 1024 232 1 0
gated 33 712 48 1 0 1
""".splitlines())]

MOE = [(*map(int, c[:6]), *c[6:9], *map(int, c[9:]))
       for c in map(str.split, """\
1 1 16 11 2 1 bfloat16 bfloat16 bfloat16 0 0
1 1 30 186 1 1 bfloat16 bfloat16 bfloat16 0 1
1 1 32 16 1 1 float16 float16 float16 0 1
1 1 32 67 1 1 float16 float16 float16 0 1
1 1 32 80 1 1 bfloat16 int8 bfloat16 1 1
1 1 32 128 1 1 bfloat16 bfloat16 bfloat16 0 0
1 1 48 160 1 1 bfloat16 int8 bfloat16 0 0
1 1 64 147 1 1 float16 int8 float16 0 1
1 1 2048 29 1 1 bfloat16 int8 bfloat16 0 1
1 2 16 16 1 1 float32 float32 float32 0 0
1 2 28 16 1 1 bfloat16 int8 float32 0 0
1 2 29 16 1 1 float16 int8 float16 0 1
1 2 32 16 1 1 bfloat16 bfloat16 float32 0 1
1 7 2191 9 12 4 float16 int8 float16 0 0
1 8 16 9 2 1 float16 float16 float32 1 0
1 8 2496 8 12 3 float16 float16 float16 0 1
1 9 22 16 3 2 bfloat16 int8 bfloat16 0 1
1 9 25 8 2 2 float16 float16 float16 0 1
1 9 28 16 2 1 float16 int8 float32 0 0
1 9 32 19 2 1 bfloat16 bfloat16 float32 0 0
1 9 48 11 1 1 float16 int8 float32 0 1
1 9 48 16 1 1 float16 float16 float32 0 0
1 9 64 9 1 1 bfloat16 bfloat16 bfloat16 1 0
1 9 64 16 1 1 bfloat16 int8 bfloat16 0 1
1 9 2048 8 2 1 bfloat16 int8 float32 0 1
1 9 8192 8 4 3 float32 float32 float32 0 0
1 9 8192 1024 3 3 bfloat16 bfloat16 float32 0 0
1 16 16 32 8 1 float32 float32 float32 0 0
1 16 18 48 1 1 float16 float16 float16 1 1
1 16 20 32 2 1 bfloat16 int8 float32 0 0
1 16 24 16 4 1 bfloat16 bfloat16 bfloat16 0 1
1 16 32 14 2 1 bfloat16 int8 float32 0 1
1 16 32 16 1 1 bfloat16 bfloat16 bfloat16 0 1
1 16 32 16 1 1 float16 int8 float16 1 1
1 16 32 16 2 1 float16 int8 float32 1 1
1 16 34 18 2 1 float16 float16 float16 0 1
1 16 2048 10 12 8 bfloat16 int8 bfloat16 0 1
1 16 2048 16 12 8 float32 float32 float32 0 0
1 17 16 16 2 1 float16 int8 float16 0 1
1 17 32 12 3 1 float16 float16 float32 0 0
1 17 64 16 1 1 bfloat16 bfloat16 float32 0 1
1 17 720 8 32 3 bfloat16 int8 float32 0 1
1 17 2688 8 12 8 bfloat16 bfloat16 bfloat16 0 0
1 17 7146 8 4 3 bfloat16 bfloat16 float32 0 1
1 17 8192 9 3 2 bfloat16 bfloat16 bfloat16 0 1
1 17 8192 16 3 2 float16 float16 float32 0 1
1 26 64 11 1 1 float16 float16 float32 0 1
1 30 48 16 1 1 float32 float32 float32 0 1
1 40 32 10 1 1 bfloat16 bfloat16 float32 0 0
1 40 32 10 1 1 bfloat16 int8 float32 0 0
1 40 80 12 1 1 float16 int8 float32 0 0
1 40 512 9 1 1 float32 float32 float32 0 1
1 40 1024 8 1 1 float16 float16 float32 0 0
1 40 2048 11 12 4 float16 int8 float16 0 0
1 40 4096 16 1 1 float16 int8 float32 0 0
1 40 8192 16 3 1 float16 int8 float32 0 0
1 83 2048 9 1 1 bfloat16 int8 bfloat16 0 1
1 128 224 512 100 8 float32 float32 float32 0 0
1 128 239 1024 100 8 float16 float16 float32 0 0
1 128 330 2048 64 1 bfloat16 int8 float32 0 0
2 1 24 80 1 1 float16 int8 float16 0 1
2 8 4096 9 3 1 float32 float32 float32 0 1
2 9 28 16 1 1 float16 float16 float16 0 1
2 9 1808 8 4 1 float16 float16 float32 0 1
2 9 2272 8 2 1 bfloat16 int8 bfloat16 0 1
2 10 1088 11 3 1 bfloat16 bfloat16 bfloat16 0 0
2 16 2320 9 1 1 bfloat16 bfloat16 bfloat16 0 0
2 16 4096 2048 3 4 float16 int8 float16 0 1
2 17 26 16 1 1 bfloat16 bfloat16 float32 0 1
2 17 2112 11 3 1 float16 int8 float16 0 1
2 40 976 1024 12 8 bfloat16 bfloat16 bfloat16 0 1
3 1 8192 16 1 3 float16 int8 float16 0 0
3 2 4096 8 2 4 bfloat16 bfloat16 bfloat16 0 1
3 8 1024 9 8 3 bfloat16 bfloat16 float32 0 1
3 8 3040 8 3 1 bfloat16 bfloat16 float32 0 0
3 9 1024 8 8 8 float16 float16 float32 0 1
3 9 1024 16 8 3 bfloat16 int8 float32 0 0
3 9 2048 14 1 1 float16 int8 float16 0 1
3 9 3111 8 3 1 bfloat16 int8 bfloat16 0 0
3 16 8192 16 1 2 bfloat16 int8 float32 0 1
3 17 8192 11 1 2 float16 float16 float16 0 1
3 17 8192 13 1 2 float16 float16 float32 0 1
3 40 8192 9 1 2 bfloat16 bfloat16 float32 0 0
3 73 80 1024 64 3 float16 float16 float16 0 1
3 128 71 512 64 4 float32 float32 float32 0 0
3 128 221 1024 32 8 float16 float16 float16 0 1
3 128 454 2048 16 4 bfloat16 int8 bfloat16 0 1
4 1 21 112 1 3 float16 float16 float16 0 1
4 1 8192 9 1 4 float16 int8 float32 0 1
4 8 713 16 8 4 bfloat16 int8 bfloat16 0 0
4 8 3168 9 2 2 float16 float16 float16 0 1
4 16 512 10 2 1 float32 float32 float32 0 1
4 16 718 16 8 3 float16 int8 float32 0 0
4 16 2151 9 3 8 float32 float32 float32 0 1
4 16 8912 8 1 4 float16 float16 float16 0 0
4 17 2048 8 3 1 bfloat16 bfloat16 bfloat16 1 1
4 128 22 4096 100 4 float16 int8 float32 0 0
4 128 32 1024 100 8 float16 float16 float32 0 1
4 128 32 2048 100 4 bfloat16 int8 bfloat16 0 0
4 128 32 2368 100 3 float16 int8 float16 0 1
35 1 16 12 1 2 float32 float32 float32 1 1
35 2 20 11 1 1 float16 int8 float32 0 0
35 9 17 19 1 2 bfloat16 int8 bfloat16 0 0
35 16 25 16 1 8 float32 float32 float32 0 1
35 40 748 9 1 1 float16 float16 float32 0 1
35 119 32 16 1 1 float32 float32 float32 0 0
35 128 16 1024 12 4 bfloat16 bfloat16 float32 0 1
35 128 24 1040 12 4 bfloat16 bfloat16 bfloat16 0 1
""".splitlines())]
